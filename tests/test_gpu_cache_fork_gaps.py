"""Children of requests that have lost pages: an entry that is no page has none in the child either, also where the
child's tokens end in it."""
import random

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ra():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_02584_amd import rotate_attn as m
    m.lib()
    return m


def _i32(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("gap", [-1, -2 ** 31, 40, 2 ** 31 - 1])
def test_a_child_that_ends_in_a_lost_page_takes_none(ra, gap, apart):
    """Lengths around the gap's blocks (2 and 3 of 6); pages, stack and holders by hand."""
    page, pages = 16, 40
    p = ra.make_cache_params(1, 1, 64, page_size=page, num_pages=pages, max_blocks=6)
    row = [9, 4, gap, gap, 7, 1]
    lens = [32, 33, 47, 48, 50, 64, 65, 90, 0, 16]
    n = len(lens)
    table = np.full((n + 1, 6), -5, np.int32)
    table[0] = row
    seq = [90] + [0] * n
    refs = np.zeros(pages, np.int32)
    stack = [30, 31, 32, 33, 34] + [0] * (pages - 5)
    t = dict(seq_lens=_i32(seq), block_table=_i32(table), page_refs=_i32(refs), free_pages=_i32(stack), free_count=_i32([5]))
    cache = torch.randint(0, 256, (pages, ra.cache_layout(p)["page_bytes"]), dtype=torch.uint8, device="cuda")
    before = cache.clone()
    ws, status = ra.cache_pages_workspace(p, n + 1), _i32([-9] * 4)
    ws.fill_(0x5A)
    out, kw = t, {}
    if apart:
        out = {k: torch.full_like(v, -77) for k, v in t.items()}
        kw = dict(zip(("seq_out", "table_out", "refs_out", "free_out", "count_out"), out.values()))
    ra.cache_fork(p, _i32([0] * n), _i32(range(1, n + 1)), *t.values(), cache, ws, status, lens=_i32(lens), **kw)
    torch.cuda.synchronize()
    # tokens of 65 and 90 end in pages 7 and 1: the only copies, from the top
    want, held, top, copies, shared = table.copy(), refs.copy(), 5, {}, 0
    for c, L in enumerate(lens, 1):
        for j in range(L // page):
            want[c, j] = row[j]
            if 0 <= row[j] < pages:
                held[row[j]] += 1
                shared += 1
        if L % page:
            want[c, L // page] = -1
            if 0 <= row[L // page] < pages:
                top -= 1
                want[c, L // page] = stack[top]
                copies[stack[top]] = row[L // page]
    assert status.tolist() == [0, 2, shared, 90] and top == 3
    assert out["seq_lens"].tolist() == [90] + lens
    assert np.array_equal(out["block_table"].cpu().numpy(), want)
    assert np.array_equal(out["page_refs"].cpu().numpy(), held)
    assert out["free_pages"].tolist() == stack and out["free_count"].item() == top
    for id in range(pages):
        assert torch.equal(cache[id], before[copies.get(id, id)]), id


def test_no_free_page_is_needed_for_a_lost_one(ra):
    p = ra.make_cache_params(1, 1, 64, page_size=16, num_pages=4, max_blocks=3)
    t = [_i32([40, 0]), _i32([[2, 1, -1], [-1] * 3]), _i32([0] * 4), _i32([0] * 4), _i32([0])]
    cache = torch.zeros(4, ra.cache_layout(p)["page_bytes"], dtype=torch.uint8, device="cuda")
    ws, status = ra.cache_pages_workspace(p, 2), _i32([9] * 4)
    ra.cache_fork(p, _i32([0]), _i32([1]), *t, cache, ws, status)
    assert status.tolist() == [0, 0, 2, 40] and t[1].tolist() == [[2, 1, -1], [2, 1, -1]] and t[4].item() == 0


def test_a_child_sees_what_its_parent_saw(ra):
    """A request runs on under a window and loses pages, children begin inside its gap and in its window, and the pages
    that the stack would have given them hold another request's keys: no query of theirs sees these."""
    page, window, sinks, D = 16, 40, 5, 64
    p = ra.make_cache_params(2, 1, D, page_size=page, num_pages=30, max_blocks=20, window=window, out_dtype=ra.FP32)
    R, T = 4, 300
    st = ra.alloc_cache(p, R)
    tables = [st[k] for k in ("seq_lens", "block_table", "page_refs", "free_pages", "free_count")]
    wp, status = ra.cache_pages_workspace(p, R), _i32([0] * 4)
    ws = ra.cache_workspace(p, R, T, T)
    q_start, positions, slots = _i32([0] * (R + 1)), _i32([0] * T), _i32([0] * T)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(T, 4, D, generator=g, device="cuda").to(torch.bfloat16)

    def step(new):
        ra.cache_plan(p, st["seq_lens"], _i32(new), st["block_table"], st["free_pages"], st["free_count"], q_start, positions,
                      slots, status)
        assert status[0].item() == 0
        ra.cache_append(p, x[:, 2:3], x[:, 3:], slots, st["cache"])

    step([200, 0, 0, 90])
    ra.cache_trim(p, *tables, st["cache"], wp, status, keep=_i32([-1, -1, -1, 0]), sinks=sinks)   # 3 ends, its pages go back
    ra.cache_fork(p, _i32([0, 0]), _i32([1, 2]), *tables, st["cache"], wp, status, lens=_i32([56, 199]))
    assert status[0].item() == 0
    # the last 6 and 7 tokens of the children as queries: once with their pages, once with all pages else full of NaN
    start, lens = _i32([0, 0, 6, 13, 13]), st["seq_lens"]
    out = []
    for spoil in (False, True):
        cache = st["cache"].clone()
        if spoil:
            held = {i for row, n in zip(st["block_table"].tolist()[:1], (200,)) for i in row[:-(-n // page)] if i >= 0}
            held.add(st["block_table"][2, 199 // page].item())
            for i in range(30):
                if i not in held:
                    cache[i].view(torch.float32)[:] = float("nan")
        o, lse = torch.full((T, 2, D), 5.0, device="cuda"), torch.full((T, 2), 5.0, device="cuda")
        ra.cache_attn_sinks(p, sinks, x[:, :2], cache, st["block_table"], start, lens, 10, o, ws, lse=lse)
        torch.cuda.synchronize()
        out.append((o[:13].clone(), lse[:13].clone()))
    assert torch.isfinite(out[0][0]).all() and torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


def test_random_gaps(ra):
    """Many parents with lost pages, random lengths: no page is taken without bytes to copy into it."""
    rng = random.Random(4)
    R, page, blocks, pages = 60, 16, 9, 700
    p = ra.make_cache_params(1, 1, 64, page_size=page, num_pages=pages, max_blocks=blocks)
    order = list(range(pages))
    rng.shuffle(order)
    seq = [rng.randint(1, blocks * page) if r < 20 else 0 for r in range(R)]
    table = [[order.pop() if j * page < seq[r] and rng.random() < 0.6 else -1 for j in range(blocks)] for r in range(R)]
    stack = order + [-7] * (pages - len(order))
    t = [_i32(seq), _i32(table), _i32([0] * pages), _i32(stack), _i32([len(order)])]
    words = ra.cache_layout(p)["page_bytes"]
    cache = torch.arange(pages, device="cuda", dtype=torch.int32)[:, None].repeat(1, words // 4).contiguous().view(torch.uint8)
    ws, status = ra.cache_pages_workspace(p, R), _i32([9] * 4)
    parents = [rng.randrange(20) for _ in range(40)]
    lens = [rng.randint(0, seq[a]) for a in parents]
    ra.cache_fork(p, _i32(parents), _i32(range(20, 60)), *t, cache, ws, status, lens=_i32(lens))
    torch.cuda.synchronize()
    got, content = t[1].tolist(), cache.view(torch.int32)[:, 0].tolist()
    top = len(order)
    for i, (a, L) in enumerate(zip(parents, lens)):
        row = got[20 + i]
        assert row[:L // page] == table[a][:L // page]
        if L % page:
            last = table[a][L // page]
            if last >= 0:
                top -= 1
                assert row[L // page] == stack[top] and content[stack[top]] == last
            else:
                assert row[L // page] == -1
    assert t[4].item() == top and status.tolist()[:2] == [0, len(order) - top]
