"""cache_attn_sinks and cache_attn_shared refuse what they cannot do before any HIP call, in the library and in the
binding (CPU only)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def ra():
    import os
    from paper_2607_02584_amd import rotate_attn as m
    if not os.path.exists(m.LIB_PATH):
        pytest.skip("library not built")
    return m


P = ctypes.c_void_p


def _p(ra, Hq=8, Hkv=2, D=128, **kw):
    return ra.make_cache_params(Hq, Hkv, D, **{**dict(page_size=16, num_pages=10, max_blocks=4), **kw})


OK, ODD = P(0x1000), P(0x1008)


def _sinks(ra, p, sinks=4, R=1, T=1, max_q=1, q=OK, qs=(128, 128), cache=OK, table=OK, start=OK, lens=OK, rope=None, rows=0,
           o=OK, ws=OK, nws=0):
    return ra.lib().rotate_attn_cache_attn_sinks(ctypes.byref(p), sinks, R, T, max_q, q, *qs, cache, table, start, lens, rope,
                                                 rows, o, None, ws, nws, None)


def _shared(ra, p, R=1, T=1, groups=1, q=OK, qs=(128, 128), cache=OK, table=OK, start=OK, lens=OK, pos=OK, gs=OK, pre=OK,
            rope=None, rows=0, o=OK, ws=OK, nws=0):
    return ra.lib().rotate_attn_cache_attn_shared(ctypes.byref(p), R, T, groups, q, *qs, cache, table, start, lens, pos, gs, pre,
                                                  rope, rows, o, None, ws, nws, None)


TENSORS = ({"q": None}, {"cache": None}, {"table": None}, {"start": None}, {"lens": None}, {"o": None}, {"q": ODD}, {"o": ODD},
           {"cache": P(0x1010)}, {"qs": (4, 128)}, {"qs": (128, -8)}, {"rope": OK}, {"rope": ODD, "rows": 9}, {"R": -1}, {"T": -1})


def test_sinks_arguments(ra):
    """(A workspace of no bytes refuses, with -3, what nothing else does.)"""
    p = _p(ra, window=20)
    assert _sinks(ra, p) == -3 and _sinks(ra, _p(ra)) == -3 and _sinks(ra, p, sinks=0) == -3 and _sinks(ra, p, sinks=1 << 30) == -3
    for kw in TENSORS + ({"sinks": -1}, {"max_q": -1}):
        assert _sinks(ra, p, **kw) == -1, kw
    assert _sinks(ra, p, sinks=(1 << 30) + 1) == -2 and b"sinks" in ra.lib().rotate_attn_last_error()
    assert _sinks(ra, _p(ra, causal=False)) == -2 and b"causal" in ra.lib().rotate_attn_last_error()
    assert _sinks(ra, _p(ra, D=96)) == -2
    for kw in ({"R": 0}, {"T": 0}, {"max_q": 0}):
        assert _sinks(ra, p, **kw) == 0
    need = ra.cache_workspace_size(p, 1, 1, 1)
    for kw in ({"ws": None, "nws": need}, {"ws": P(0x1080), "nws": need}, {"nws": need - 1}):
        assert _sinks(ra, p, **kw) == -3
    assert _sinks(ra, _p(ra, 1024, 1024, 64), R=16380) == -2


def test_shared_arguments(ra):
    p = _p(ra)
    assert _shared(ra, p) == -3 and _shared(ra, p, groups=0, gs=None, pre=None) == -3
    for kw in TENSORS + ({"pos": None}, {"gs": None}, {"pre": None}, {"groups": -1}, {"groups": 2}):
        assert _shared(ra, p, **kw) == -1, kw
    assert _shared(ra, _p(ra, causal=False)) == -2 and b"causal" in ra.lib().rotate_attn_last_error()
    assert _shared(ra, _p(ra, window=5)) == -2 and b"window" in ra.lib().rotate_attn_last_error()
    for kw in ({"R": 0, "groups": 0}, {"T": 0}):
        assert _shared(ra, p, **kw) == 0
    n = ctypes.c_size_t()
    size = ra.lib().rotate_attn_cache_shared_workspace_size
    assert size(ctypes.byref(p), 1, 1, 1, ctypes.byref(n)) == 0 and n.value % 256 == 0
    for kw in ({"ws": None, "nws": n.value}, {"ws": P(0x1080), "nws": n.value}, {"nws": n.value - 1}):
        assert _shared(ra, p, **kw) == -3
    assert size(ctypes.byref(p), 1, 1, 1, None) == -1 and size(None, 1, 1, 1, ctypes.byref(n)) == -1
    assert size(ctypes.byref(p), 2, 3, 1, ctypes.byref(n)) == -1 and size(ctypes.byref(p), 65537, 1, 1, ctypes.byref(n)) == -2


# 2^24 workgroups of a launch, of which 4096 are kept for cuts; a workgroup per token; 16 work-items per query head's row
@pytest.mark.parametrize("Hq,Hkv,R,groups,T,ok", [
    (64, 64, 65536, 65504, 1, False), (64, 64, 65536, 65503, 1, True), (8, 2, 65536, 65536, 1 << 22, True),
    (8, 2, 65536, 65536, (1 << 22) + 1, False), (32, 8, 1, 1, 1 << 21, True), (32, 8, 1, 1, (1 << 21) + 1, False),
    (1, 1, 1, 0, 1 << 22, True), (1024, 1024, 1, 1, 1 << 16, True),
])
def test_more_than_a_launch_holds_is_refused(ra, Hq, Hkv, R, groups, T, ok):
    p = _p(ra, Hq, Hkv, 64)
    n = ctypes.c_size_t()
    assert ra.lib().rotate_attn_cache_shared_workspace_size(ctypes.byref(p), R, groups, T, ctypes.byref(n)) == (0 if ok else -2)
    assert _shared(ra, p, R=R, groups=groups, T=T) == (-3 if ok else -2)


def test_binding_checks_tensors(ra):
    torch = pytest.importorskip("torch")
    p = _p(ra)
    i = lambda *n: torch.zeros(*n, dtype=torch.int32)
    q = torch.zeros(3, 8, 128, dtype=torch.bfloat16)
    cache, ws = torch.zeros(10, 2 * 16 * 136, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8)
    for bad in (cache, cache[:9], cache.int()):
        with pytest.raises(ValueError):
            ra.cache_attn_sinks(p, 4, q, bad, i(2, 4), i(3), i(2), 1, q, ws)
        with pytest.raises(ValueError):
            ra.cache_attn_shared(p, q, bad, i(2, 4), i(3), i(2), i(3), i(2), i(1), q, ws)
    with pytest.raises(ValueError, match="tensor"):
        ra._cache_tensor("x", "x", torch.int32, (2,), torch.device("cuda", 0))
    with pytest.raises(ValueError, match="device tensor"):
        ra._cache_tensor(i(2), "x", torch.int32, (2,), torch.device("cuda", 0))
    with pytest.raises(ValueError, match="shape"):
        ra._cache_tensor(i(3), "x", torch.int32, (2,), torch.device("cuda", 0))
