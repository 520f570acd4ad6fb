"""Fork, trim and compact refuse what they cannot do before any HIP call, in the library and in the binding (CPU only);
and the plain reference that the GPU is compared with keeps its own tables sound."""
import copy
import ctypes
import random

import pytest

import cache_pages_ref as ref


@pytest.fixture(scope="module")
def ra():
    import os
    from paper_2607_02584_amd import rotate_attn as m
    if not os.path.exists(m.LIB_PATH):
        pytest.skip("library not built")
    return m


def _tables(ra, **kw):
    at = dict(seq_lens=0x10000, block_table=0x20000, page_refs=0x30000, free_pages=0x40000, free_count=0x50000)
    at.update(kw)
    return ra.CacheTables(**at)


STATUS, CACHE, WS = 0x60000, 0x100000, 0x8000000


def _calls(ra, p, R=6, t=None, out=None, cache=CACHE, ws=WS, nws=1 << 40, status=STATUS, **kw):
    """Status of fork, trim and compact with these arguments (all refused: nothing here may be launched)."""
    L, r, P = ra.lib(), ctypes.byref(p), ctypes.c_void_p
    t = _tables(ra) if t is None else t
    rest = (t, out, P(cache), P(ws), nws, P(status), None)
    return (L.rotate_attn_cache_fork(r, R, kw.get("n", 2), P(kw.get("parents", 0x70000)), P(kw.get("children", 0x71000)),
                                     P(kw.get("lens", 0)), *rest),
            L.rotate_attn_cache_trim(r, R, P(kw.get("keep", 0)), kw.get("sinks", -1), *rest),
            L.rotate_attn_cache_compact(r, R, *rest))


def _p(ra, **kw):
    return ra.make_cache_params(8, 2, 128, **{**dict(page_size=16, num_pages=10, max_blocks=4), **kw})


def test_pointers_that_are_refused(ra):
    p = _p(ra)
    for name in ("seq_lens", "block_table", "page_refs", "free_pages", "free_count"):
        assert _calls(ra, p, t=_tables(ra, **{name: None})) == (-1, -1, -1)
        assert b"NULL" in ra.lib().rotate_attn_last_error()
        assert _calls(ra, p, out=_tables(ra, **{name: None})) == (-1, -1, -1)
    assert _calls(ra, p, cache=None) == (-1, -1, -1) and _calls(ra, p, status=None) == (-1, -1, -1)
    assert _calls(ra, p, cache=CACHE + 64) == (-1, -1, -1) and b"aligned" in ra.lib().rotate_attn_last_error()
    assert _calls(ra, p, ws=None) == (-3, -3, -3) and _calls(ra, p, ws=WS + 128) == (-3, -3, -3)
    n = ctypes.c_size_t()
    assert ra.lib().rotate_attn_cache_pages_workspace_size(ctypes.byref(p), 6, ctypes.byref(n)) == 0
    assert _calls(ra, p, nws=n.value - 1) == (-3, -3, -3)
    assert _calls(ra, p, R=-1) == (-1, -1, -1) and _calls(ra, p, R=65537)[1:] == (-2, -2)
    assert _calls(ra, _p(ra, page_size=48)) == (-2, -2, -2)
    L, r, P = ra.lib(), ctypes.byref(p), ctypes.c_void_p
    assert L.rotate_attn_cache_compact(r, 6, None, None, P(CACHE), P(WS), 1 << 40, P(STATUS), None) == -1
    for f in (-1, 7):
        assert _calls(ra, p, n=f, nws=0)[0] == -1
    for kw in ({"parents": 0}, {"children": 0}):
        assert _calls(ra, p, nws=0, **kw)[0] == -1
    assert L.rotate_attn_cache_pages_workspace_size(r, 1, None) == -1
    assert L.rotate_attn_cache_pages_workspace_size(r, 65537, ctypes.byref(n)) == -2
    assert L.rotate_attn_cache_pages_workspace_size(None, 1, ctypes.byref(n)) == -1


def test_tables_that_overlap_are_refused(ra):
    p, err = _p(ra), ra.lib().rotate_attn_last_error
    for t, out in ((_tables(ra, page_refs=0x40000), None), (_tables(ra, page_refs=0x40000 + 36), None),
                   (_tables(ra, block_table=0x10000 + 20), None), (_tables(ra, free_count=STATUS + 12), None),
                   (None, _tables(ra, page_refs=0x30004)), (None, _tables(ra, seq_lens=0x20000)),
                   (None, _tables(ra, block_table=0x20000 - 4 * 24 + 4)), (None, _tables(ra, free_pages=0x30000))):
        assert _calls(ra, p, t=t, out=out) == (-1, -1, -1) and b"overlap" in err()
    assert _calls(ra, p, t=_tables(ra, seq_lens=CACHE + 256)) == (-1, -1, -1) and b"overlap" in err()
    assert _calls(ra, p, ws=0x30000) == (-1, -1, -1) and b"overlap" in err()
    for kw in ({"parents": 0x10000}, {"children": 0x20010}, {"lens": 0x30008}):
        assert _calls(ra, p, nws=0, **kw)[0] == -1
    assert _calls(ra, p, keep=0x10000, nws=0)[1] == -1 and _calls(ra, p, keep=STATUS, nws=0)[1] == -1
    # tables side by side are fine (a workspace of no bytes is what refuses them)
    side = _tables(ra, seq_lens=0x10000, block_table=0x10000 + 24, page_refs=0x10000 + 120, free_pages=0x10000 + 160,
                   free_count=0x10000 + 200)
    assert _calls(ra, p, t=side, nws=0) == (-3, -3, -3)
    assert _calls(ra, p, out=_tables(ra), nws=0) == (-3, -3, -3)


def test_sinks_need_a_window(ra):
    p = _p(ra)
    L, P = ra.lib(), ctypes.c_void_p
    assert L.rotate_attn_cache_trim(ctypes.byref(p), 6, None, 0, _tables(ra), None, P(CACHE), P(WS), 0, P(STATUS), None) == -1
    assert b"window" in L.rotate_attn_last_error()


def test_binding_checks_tensors(ra):
    torch = pytest.importorskip("torch")
    p = _p(ra)
    i = lambda *n: torch.zeros(*n, dtype=torch.int32)
    cache = torch.zeros(10, 2 * 16 * 136, dtype=torch.uint8)
    ws = torch.zeros(512, dtype=torch.uint8)
    tables = [i(6), i(6, 4), i(10), i(10), i(1)]
    for call, args in ((ra.cache_fork, (i(2), i(2))), (ra.cache_trim, ()), (ra.cache_compact, ())):
        with pytest.raises(ValueError, match="device tensor"):
            call(p, *args, *tables, cache, ws, i(4))
        with pytest.raises(ValueError, match="shape"):
            call(p, *args, *tables, cache[:9], ws, i(4))


def _state(rng, R, page, blocks, pages):
    lens = [rng.randint(0, blocks * page) if rng.random() < 0.6 else 0 for _ in range(R)]
    order = list(range(pages))
    rng.shuffle(order)
    table = []
    for n in lens:
        row = [order.pop() for _ in range(ref.up(n, page))]
        table.append(row + [-1] * (blocks - len(row)))
    return dict(seq=lens, table=table, refs=[0] * pages, free=order + [-7] * (pages - len(order)), count=len(order),
                cache=list(range(pages)))


def _tokens(s, page):
    """What every request's cached tokens are: (contents, place) of each."""
    return [[None if row[i // page] < 0 else (s["cache"][row[i // page]], i % page) for i in range(n)]
            for n, row in zip(s["seq"], s["table"])]


@pytest.mark.parametrize("seed", range(40))
def test_the_reference_keeps_tables_sound_and_tokens_alike(seed):
    rng = random.Random(seed)
    page, blocks, pages, R = rng.choice([16, 32]), 5, 90, 8
    s = _state(rng, R, page, blocks, pages)
    ref.valid(s, page)
    for _ in range(12):
        before, tokens = copy.deepcopy(s), _tokens(s, page)
        op = rng.choice(["fork", "trim", "trim", "compact"])
        if op == "fork":
            free = [r for r in range(R) if s["seq"][r] == 0]
            children = rng.sample(free, rng.randint(0, len(free)))
            parents = [rng.randrange(R) for _ in children]
            s, status = ref.fork(s, page, blocks, parents, children)
            if not isinstance(status, int):
                for a, c in zip(parents, children):
                    tokens[c] = [] if a in children else list(tokens[a])
        elif op == "trim":
            keep = [rng.choice([-1, -1, 0, rng.randint(0, n)]) for n in s["seq"]]
            s, status = ref.trim(s, page, blocks, 0, keep)
            if not isinstance(status, int):
                tokens = [x if k < 0 else x[:k] for x, k in zip(tokens, keep)]
        else:
            s, status = ref.compact(s, page, blocks)
        if isinstance(status, int):
            assert s == before
        else:
            got = _tokens(s, page)
            assert [[t for t in x] for x in got] == tokens
        ref.valid(s, page)
