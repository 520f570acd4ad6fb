"""Fork, trim and compact of the paged KV cache against plain Python (tests/cache_pages_ref.py): whole numbers and
bytes, which have to be equal."""
import random

import numpy as np
import pytest

import cache_pages_ref as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ra():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_02584_amd import rotate_attn as m
    m.lib()
    return m


def _i32(x, device="cuda"):
    return torch.tensor(np.asarray(x, np.int32), device=device)


class Cache:
    """A state in plain Python and on the device."""

    def __init__(self, ra, rng, R, page, max_blocks, pages, Hkv=1, D=64, lens=None, share=0.0, window=0, spare=None):
        self.ra, self.page, self.blocks, self.pages = ra, page, max_blocks, pages
        self.p = ra.make_cache_params(Hkv, Hkv, D, page_size=page, num_pages=pages, max_blocks=max_blocks, window=window)
        size = ra.cache_layout(self.p)["page_bytes"]
        lens = [rng.randint(0, max_blocks * page) for _ in range(R)] if lens is None else lens
        order = list(range(pages))
        rng.shuffle(order)
        table, held = [], [0] * pages
        for r in range(R):
            row = []
            for j in range(ref.up(lens[r], page)):
                # full blocks of another request that is at least as long may be shared
                if j < lens[r] // page and table and rng.random() < share and len(table[0]) > j and j < lens[0] // page and table[0][j] >= 0:
                    id = table[0][j]
                else:
                    id = order.pop()
                held[id] += 1
                row.append(id)
            table.append(row + [-1] * (max_blocks - len(row)))
        stack = [i for i in order if not held[i]]
        self.state = dict(seq=list(lens), table=table, refs=[max(0, h - 1) for h in held], free=stack + [-7] * (pages - len(stack)),
                          count=len(stack), cache=list(range(pages)))
        self.bytes = np.random.default_rng(rng.randrange(1 << 30)).integers(0, 256, (pages, size), dtype=np.uint8)
        self.cache = torch.from_numpy(self.bytes).cuda()
        self.ws = ra.cache_pages_workspace(self.p, R)
        self.ws.fill_(0x5A)
        self.status = _i32([-9] * 4)
        self.upload()

    def upload(self):
        s = self.state
        self.t = dict(seq_lens=_i32(s["seq"]), block_table=_i32(s["table"]).view(len(s["seq"]), self.blocks),
                      page_refs=_i32(s["refs"]), free_pages=_i32(s["free"]), free_count=_i32([s["count"]]))
        self.cache.copy_(torch.from_numpy(self.bytes[s["cache"]]))

    def call(self, name, *args, apart=False, **kw):
        """The operator in place, or (apart) into arrays of their own, and the tables it leaves."""
        out = self.t
        if apart:
            out = {k: torch.full_like(v, -77) for k, v in self.t.items()}
            kw.update(seq_out=out["seq_lens"], table_out=out["block_table"], refs_out=out["page_refs"],
                      free_out=out["free_pages"], count_out=out["free_count"])
        before = {k: v.clone() for k, v in self.t.items()}
        t = self.t
        getattr(self.ra, name)(self.p, *args, t["seq_lens"], t["block_table"], t["page_refs"], t["free_pages"], t["free_count"],
                               self.cache, self.ws, self.status, **kw)
        torch.cuda.synchronize()
        if apart:
            for k, v in before.items():
                assert torch.equal(v, t[k]), f"{k} was an input"
        return out

    def check(self, out, want, status):
        got = {k: v.cpu().numpy() for k, v in out.items()}
        s = self.status.cpu().tolist()
        if isinstance(status, int):
            assert s[0] == status
        else:
            assert s == status
        assert got["seq_lens"].tolist() == want["seq"]
        assert got["block_table"].tolist() == want["table"]
        assert got["page_refs"].tolist() == want["refs"]
        assert got["free_pages"].tolist() == want["free"]
        assert got["free_count"].tolist() == [want["count"]]
        assert np.array_equal(self.cache.cpu().numpy(), self.bytes[want["cache"]])


def _sound(c, state):
    s = dict(state, free=list(state["free"]))
    ref.valid(s, c.page)


SHAPES = [  # R, page, max_blocks, pages, Hkv, D
    (1, 16, 3, 9, 1, 64), (5, 64, 4, 40, 2, 128), (37, 16, 9, 420, 3, 64), (300, 32, 5, 2200, 1, 128), (4, 256, 2, 14, 5, 64),
    (1500, 16, 4, 9000, 1, 64),
]


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("R,page,blocks,pages,Hkv,D", SHAPES)
def test_fork(ra, R, page, blocks, pages, Hkv, D, apart):
    rng = random.Random(R * page + apart)
    lens = [0 if rng.random() < 0.5 else rng.choice([1, page - 1, page, page + 1, rng.randint(0, blocks * page), blocks * page])
            for _ in range(R)]
    c = Cache(ra, rng, R, page, blocks, pages, Hkv, D, lens=lens, share=0.3)
    _sound(c, c.state)
    children = [r for r in range(R) if lens[r] == 0]
    rng.shuffle(children)
    children = children[:rng.randint(min(1, len(children)), len(children))]
    parents = [rng.randrange(R) for _ in children]       # empty ones among them, and children of the same call
    cut = None if apart else [rng.randint(0, lens[a]) for a in parents]
    want, status = ref.fork(c.state, page, blocks, parents, children, cut)
    out = c.call("cache_fork", _i32(parents), _i32(children), apart=apart, lens=None if cut is None else _i32(cut))
    c.check(out, want, status)
    _sound(c, want)


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("window,sinks", [(0, -1), (40, 0), (1, 5), (17, 200), (100000, 3)])
@pytest.mark.parametrize("R,page,blocks,pages,Hkv,D", SHAPES)
def test_trim(ra, R, page, blocks, pages, Hkv, D, window, sinks, apart):
    rng = random.Random(R * page + window + apart)
    c = Cache(ra, rng, R, page, blocks, pages, Hkv, D, share=0.5, window=window)
    _sound(c, c.state)
    lens = c.state["seq"]
    keep = [rng.choice([-1, -2 ** 31, 0, n, rng.randint(0, n), max(0, n - rng.randint(0, 9)), n // page * page]) for n in lens]
    want, status = ref.trim(c.state, page, blocks, window, keep, sinks)
    out = c.call("cache_trim", apart=apart, keep=_i32(keep), sinks=sinks)
    c.check(out, want, status)
    _sound(c, want)
    # and once more, what is kept now: nothing goes but pages behind the window that are gone already
    c.state = want
    c.upload()
    want, status = ref.trim(want, page, blocks, window, None, sinks)
    c.check(c.call("cache_trim", sinks=sinks), want, status)
    assert status[1:3] == [0, 0]


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("R,page,blocks,pages,Hkv,D", SHAPES)
def test_compact(ra, R, page, blocks, pages, Hkv, D, apart):
    rng = random.Random(R * page + apart)
    c = Cache(ra, rng, R, page, blocks, pages, Hkv, D, share=0.4)
    # entries behind a request's length are nobody's
    for n, row in zip(c.state["seq"], c.state["table"]):
        if ref.up(n, page) < blocks:
            row[-1] = rng.randrange(pages)
    c.upload()
    want, status = ref.compact(c.state, page, blocks)
    out = c.call("cache_compact", apart=apart)
    c.check(out, want, status)
    _sound(c, dict(want, table=[row[:ref.up(n, page)] for n, row in zip(want["seq"], want["table"])]))
    c.state = want
    c.upload()
    want, status = ref.compact(want, page, blocks)
    c.check(c.call("cache_compact"), want, status)
    assert status[1] == 0


def test_compact_of_nothing_and_of_everything(ra):
    rng = random.Random(5)
    for lens, pages in (([0, 0], 7), ([32, 16], 3), ([0], 1)):
        c = Cache(ra, rng, len(lens), 16, 4, pages, lens=lens)
        want, status = ref.compact(c.state, 16, 4)
        c.check(c.call("cache_compact"), want, status)
        assert status[1] == 0


def test_refused_calls_change_nothing(ra):
    """One impossible value each; everything stays as it is, in arrays of their own too."""
    rng = random.Random(3)
    lens = [0, 40, 0, 33, 0, 64]

    def state():
        return Cache(ra, rng, 6, 16, 4, 20, lens=list(lens), share=0.5)

    for apart in (False, True):
        for parents, children, cut, seq, count, bit in [
                ([1], [3], None, None, None, 1), ([1, 3], [2, 2], None, None, None, 1), ([6], [2], None, None, None, 1),
                ([1], [-1], None, None, None, 1), ([1], [2], [41], None, None, 1), ([1], [2], [-1], None, None, 1),
                ([1], [2], None, (1, 65), None, 1), ([1], [2], None, (1, -5), None, 1), ([1, 3], [2, 4], None, None, 1, 4),
                ([1], [2], None, None, -1, 8), ([1], [2], None, None, 21, 8), ([1], [2], None, None, 0, 4)]:
            c = state()
            if seq:
                c.state["seq"][seq[0]] = seq[1]
            if count is not None:
                c.state["count"] = count
            c.upload()
            out = c.call("cache_fork", _i32(parents), _i32(children), apart=apart, lens=None if cut is None else _i32(cut))
            c.check(out, c.state, bit)
        for keep, seq, count, bit in [([-1, 41, -1, -1, -1, -1], None, None, 1), (None, (3, 65), None, 1), (None, (3, -1), None, 1),
                                      (None, None, -4, 8), (None, None, 21, 8)]:
            c = state()
            if seq:
                c.state["seq"][seq[0]] = seq[1]
            if count is not None:
                c.state["count"] = count
            c.upload()
            c.check(c.call("cache_trim", apart=apart, keep=None if keep is None else _i32(keep)), c.state, bit)
        c = state()
        c.state["refs"][c.state["table"][1][1]] = 1      # held by another table, say: a copy is due, and no page left
        c.state["count"] = 0
        c.upload()
        c.check(c.call("cache_trim", apart=apart, keep=_i32([-1, 20, -1, -1, -1, -1])), c.state, 4)
        for edit, bit in ((("count", -1), 8), (("count", 21), 8), (("free", 20), 16), (("free", -1), 16), (("free", None), 16),
                          (("seq", 65), 1), (("seq", -1), 1)):
            c = state()
            if edit[0] == "count":
                c.state["count"] = edit[1]
            elif edit[0] == "seq":
                c.state["seq"][5] = edit[1]
            else:
                c.state["free"][1] = c.state["free"][0] if edit[1] is None else edit[1]
            c.upload()
            c.check(c.call("cache_compact", apart=apart), c.state, bit)


def test_damaged_entries_touch_nothing_outside(ra):
    """Entries and stack numbers that are no page: passed over, neighbours of the tables unharmed."""
    rng = random.Random(11)
    c = Cache(ra, rng, 4, 16, 4, 12, lens=[0, 40, 33, 64])
    wide = {k: torch.full((v.numel() + 64,), 123, dtype=torch.int32, device="cuda") for k, v in c.t.items()}
    c.state["table"][1][0], c.state["table"][1][2], c.state["table"][3][1] = 12, 2 ** 31 - 1, -2 ** 31
    c.state["free"][c.state["count"] - 1] = 99
    for name, args, kw in (("cache_fork", ([1], [0]), {}), ("cache_trim", (), dict(keep=_i32([-1, 7, 0, 20])))):
        c.upload()
        for k, v in c.t.items():
            wide[k].fill_(123)
            wide[k][32:32 + v.numel()] = v.flatten()
            c.t[k] = wide[k][32:32 + v.numel()].view(v.shape)
        getattr(ra, name)(c.p, *map(_i32, args), c.t["seq_lens"], c.t["block_table"], c.t["page_refs"], c.t["free_pages"],
                          c.t["free_count"], c.cache, c.ws, c.status, **kw)
        torch.cuda.synchronize()
        assert c.status[0].item() == 0
        for k, v in wide.items():
            assert (v[:32] == 123).all() and (v[32 + c.t[k].numel():] == 123).all(), (name, k)
        assert np.array_equal(c.cache.cpu().numpy(), c.bytes), name
        if name == "cache_fork":       # the page that was to hold the copy is none: the child has no entry there
            assert c.t["block_table"][0].tolist() == [12, c.state["table"][1][1], -1, -1] and c.t["seq_lens"][0].item() == 40
        else:
            assert c.t["block_table"].tolist()[1][1:] == [-1, -1, -1] and c.t["block_table"].tolist()[2] == [-1] * 4


def test_many_pages_cross_chunks_and_bit_rounds(ra):
    """More pages than one round of the compaction's bits (2^19), and giving back over many chunks of 2^12."""
    page, pages, blocks = 16, (1 << 19) + 70000, 1 << 14
    R = 16
    p = ra.make_cache_params(1, 1, 64, page_size=page, num_pages=pages, max_blocks=blocks)
    rng = np.random.default_rng(2)
    order = rng.permutation(pages).astype(np.int32)
    lens = np.array([blocks * page - 16 * rng.integers(0, 50) for _ in range(R)], np.int32)
    nb = lens // page
    table = np.full((R, blocks), -1, np.int32)
    at = 0
    for r in range(R):
        table[r, :nb[r]] = order[at:at + nb[r]]
        at += nb[r]
    used = at
    stack = np.concatenate([order[used:], order[:used]]).astype(np.int32)
    words = ra.cache_layout(p)["page_bytes"] // 4
    cache = torch.zeros(pages, words, dtype=torch.int32, device="cuda")
    cache[:, 0] = torch.arange(pages, device="cuda", dtype=torch.int32)
    cache[:, words - 1] = -cache[:, 0]
    tag = cache.view(torch.uint8)
    t = dict(seq_lens=_i32(lens), block_table=_i32(table), page_refs=_i32(np.zeros(pages)), free_pages=_i32(stack),
             free_count=_i32([pages - used]))
    ws, status = ra.cache_pages_workspace(p, R), _i32([0] * 4)
    ra.cache_compact(p, *t.values(), tag, ws, status)
    k = used
    st = status.cpu().tolist()
    assert st[0] == 0 and st[2] == k and st[1] == int((order[:used] >= k).sum())
    new = t["block_table"].cpu().numpy()
    live = np.concatenate([new[r, :nb[r]] for r in range(R)])
    assert np.array_equal(np.sort(live), np.arange(k))
    # every entry still names the same contents, and those from k on moved in ascending order
    assert np.array_equal(cache[:, 0].cpu().numpy()[live], order[:used])
    assert np.array_equal(cache[:, words - 1].cpu().numpy()[live], -order[:used])
    src = np.sort(order[:used][order[:used] >= k])
    dst = np.sort(order[used:][order[used:] < k])
    moved = dict(zip(src.tolist(), dst.tolist()))
    assert np.array_equal(live, [moved.get(int(x), int(x)) for x in order[:used]])
    assert np.array_equal(t["free_pages"].cpu().numpy()[:pages - used], np.arange(pages - 1, k - 1, -1))
    # every second request ends
    keep = np.where(np.arange(R) % 2, -1, 0)
    before = t["block_table"].cpu().numpy()
    ra.cache_trim(p, *t.values(), tag, ws, status, keep=_i32(keep))
    gone = np.sort(np.concatenate([before[r, :nb[r]] for r in range(0, R, 2)]))
    n = pages - used
    assert status.cpu().tolist()[:3] == [0, 0, len(gone)]
    assert t["free_count"].item() == n + len(gone)
    assert np.array_equal(t["free_pages"].cpu().numpy()[n:n + len(gone)], gone)
    assert (t["page_refs"] == 0).all()


def test_a_search_from_plan_to_the_end(ra):
    """A prompt is cached, forked, every continuation grows, one is rolled back, the others end, the cache is put in
    order: the values read back are those of the same tokens cached without any of it."""
    rng = np.random.default_rng(0)
    Hkv, D, page = 2, 64, 16
    p = ra.make_cache_params(4, Hkv, D, page_size=page, num_pages=40, max_blocks=8, out_dtype=ra.FP32)
    R, T = 4, 64
    st = ra.alloc_cache(p, R)
    tables = [st[k] for k in ("seq_lens", "block_table", "page_refs", "free_pages", "free_count")]
    ws, status = ra.cache_pages_workspace(p, R), _i32([0] * 4)
    q_start, positions, slots = _i32([0] * (R + 1)), _i32([0] * T), _i32([0] * T)
    tokens = {}

    def step(new):
        ra.cache_plan(p, st["seq_lens"], _i32(new), st["block_table"], st["free_pages"], st["free_count"], q_start, positions,
                      slots, status)
        assert status[0].item() == 0
        k, v = (torch.from_numpy(rng.standard_normal((T, Hkv, D))).to(torch.bfloat16).cuda() for _ in range(2))
        ra.cache_append(p, k, v, slots, st["cache"])
        t = 0
        for r in range(R):
            tokens.setdefault(r, []).extend((k[t + i], v[t + i]) for i in range(new[r]))
            t += new[r]

    step([37, 0, 0, 20])
    ra.cache_fork(p, _i32([0, 0]), _i32([1, 2]), *tables, st["cache"], ws, status)
    tokens[1], tokens[2] = list(tokens[0]), list(tokens[0])
    step([5, 20, 13, 1])
    ra.cache_fork(p, _i32([1]), _i32([0]), *tables, st["cache"], ws, status)      # 0 holds tokens: refused
    assert status[0].item() == 1
    ra.cache_trim(p, *tables, st["cache"], ws, status, keep=_i32([0, 33, 20, -1]))
    # 1 ends in its own third page; 2 in its second, which the prompt's 37 tokens fill and 0 and 1 hold
    assert status.cpu().tolist()[:2] == [0, 1]
    tokens[0], tokens[1], tokens[2] = [], tokens[1][:33], tokens[2][:20]
    step([3, 9, 12, 0])
    ra.cache_compact(p, *tables, st["cache"], ws, status)
    assert status[0].item() == 0
    seq, table, refs = st["seq_lens"].tolist(), st["block_table"].tolist(), st["page_refs"].tolist()
    count = st["free_count"].item()
    ref.valid(dict(seq=seq, table=table, refs=refs, free=st["free_pages"].tolist(), count=count), page)
    assert seq == [3, 42, 32, 21] and max(max(x) for x in table) < 40 - count
    other = ra.alloc_cache(p, R)
    for r in range(R):
        where = _i32([table[r][i // page] * page + i % page for i in range(seq[r])])
        kd, vd = (torch.stack([x[w] for x in tokens[r]]) for w in (0, 1))
        plain = torch.arange(seq[r], device="cuda", dtype=torch.int32)
        ra.cache_append(p, kd, vd, plain, other["cache"])
        got, want = [[torch.empty(seq[r], Hkv, D, device="cuda") for _ in range(2)] for _ in range(2)]
        ra.cache_read(p, st["cache"], where, *got)
        ra.cache_read(p, other["cache"], plain, *want)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), r


def test_captured_calls_follow_the_tables(ra):
    """Fork and trim in one graph, replayed on other tables, with eager work between the replays."""
    rng = random.Random(8)
    c = Cache(ra, rng, 6, 16, 4, 40, lens=[0, 40, 0, 33, 0, 64])
    parents, children, keep = _i32([1, 3]), _i32([2, 4]), _i32([-1] * 6)
    t = c.t
    args = lambda: (t["seq_lens"], t["block_table"], t["page_refs"], t["free_pages"], t["free_count"], c.cache, c.ws, c.status)

    def both():
        ra.cache_fork(c.p, parents, children, *args())
        ra.cache_trim(c.p, *args(), keep=keep)
        ra.cache_compact(c.p, *args())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            both()
    torch.cuda.synchronize()
    for i in range(5):
        d = Cache(ra, random.Random(20 + i), 6, 16, 4, 40, lens=[0, rng.randint(1, 64), 0, rng.randint(1, 64), 0, rng.randint(1, 64)])
        pairs = [[1, 3], [5, 5], [3, 3], [1, 5], [5, 1]][i]
        cut = [rng.randint(0, 20) for _ in range(6)]
        want, _ = ref.fork(d.state, 16, 4, pairs, [2, 4])
        cut = [min(x, n) for x, n in zip(cut, want["seq"])]
        want, _ = ref.trim(want, 16, 4, 0, cut)
        want, status = ref.compact(want, 16, 4)
        for k in t:
            t[k].copy_(d.t[k])
        c.cache.copy_(d.cache)
        c.bytes = d.bytes
        parents.copy_(_i32(pairs))
        keep.copy_(_i32(cut))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        c.check(t, want, status)
        _sound(c, want)


def test_another_stream(ra):
    rng = random.Random(9)
    c = Cache(ra, rng, 5, 64, 4, 40, 2, 128, lens=[0, 100, 0, 256, 31])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    c.call("cache_fork", _i32([3, 1]), _i32([0, 2]), stream=side.cuda_stream)
    want, status = ref.fork(c.state, 64, 4, [3, 1], [0, 2])
    c.check(c.t, want, status)


def test_nothing_to_do(ra):
    """No requests, no pairs, no pages free."""
    rng = random.Random(1)
    c = Cache(ra, rng, 3, 16, 2, 6, lens=[32, 32, 32])
    assert c.state["count"] == 0
    for apart in (False, True):
        for name, args in (("cache_fork", (_i32([]), _i32([]))), ("cache_trim", ()), ("cache_compact", ())):
            out = c.call(name, *args, apart=apart)
            c.check(out, c.state, [0, 0, {"cache_compact": 6}.get(name, 0), 0 if name == "cache_compact" else 32])
    p = ra.make_cache_params(1, 1, 64, page_size=16, num_pages=4, max_blocks=2)
    t = [torch.zeros(n, dtype=torch.int32, device="cuda") for n in ((0,), (0, 2), (4,), (4,), (1,))]
    t[3].copy_(_i32([3, 1, 0, 2]))
    t[4].fill_(4)
    cache, ws, status = torch.zeros(4, 16 * 72, dtype=torch.uint8, device="cuda"), ra.cache_pages_workspace(p, 0), _i32([9] * 4)
    ra.cache_fork(p, _i32([]), _i32([]), *t, cache, ws, status)
    assert status.tolist() == [0, 0, 0, 0]
    ra.cache_trim(p, *t, cache, ws, status)
    assert status.tolist() == [0, 0, 0, 0] and t[3].tolist() == [3, 1, 0, 2] and t[4].item() == 4
    ra.cache_compact(p, *t, cache, ws, status)
    assert status.tolist() == [0, 0, 0, 0] and t[3].tolist() == [3, 2, 1, 0]


def test_pages_past_32_bits(ra):
    """A cache of more than 4 GiB: its last pages are copied from and to where they are."""
    Hkv, D, page = 8, 128, 256
    pages = (5 << 30) // (Hkv * page * (D + 8))
    p = ra.make_cache_params(Hkv, Hkv, D, page_size=page, num_pages=pages, max_blocks=2)
    size = ra.cache_layout(p)["page_bytes"]
    cache = torch.zeros(pages, size, dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    last = torch.randint(0, 256, (2, size), generator=g, dtype=torch.uint8, device="cuda")
    cache[pages - 2:] = last
    stack = [pages - 3] + [0] * (pages - 1)
    t = dict(seq=_i32([300, 0]), table=_i32([[pages - 1, pages - 2], [-1, -1]]), refs=_i32(np.zeros(pages)),
             free=_i32(stack), count=_i32([1]))
    ws, status = ra.cache_pages_workspace(p, 2), _i32([0] * 4)
    ra.cache_fork(p, _i32([0]), _i32([1]), *t.values(), cache, ws, status)
    assert status.tolist() == [0, 1, 1, 300] and torch.equal(cache[pages - 3], last[0])
    ra.cache_trim(p, *t.values(), cache, ws, status, keep=_i32([0, -1]))
    assert status.tolist() == [0, 0, 1, 300]
    # the stack names every page but two that lie at the end: they move to the front
    free = np.arange(pages)
    free = free[(free != pages - 1) & (free != pages - 3)]
    t["free"].copy_(_i32(np.concatenate([free, [0, 0]])))
    t["count"].fill_(pages - 2)
    ra.cache_compact(p, *t.values(), cache, ws, status)
    assert status.tolist() == [0, 2, 2, 0] and t["table"].tolist() == [[-1, -1], [1, 0]]
    assert torch.equal(cache[0], last[0]) and torch.equal(cache[1], last[1])
