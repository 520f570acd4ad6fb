"""The paged KV cache's entry points refuse what they cannot do before any HIP
call, in the library and in the binding (CPU only)."""
import ctypes

import numpy as np
import pytest

import cache_ref as ref


@pytest.fixture(scope="module")
def ra():
    import os
    from paper_2607_02584_amd import rotate_attn as m
    if not os.path.exists(m.LIB_PATH):
        pytest.skip("library not built")
    return m


def _p(ra, **kw):
    base = dict(page_size=16, num_pages=10, max_blocks=4)
    base.update(kw)
    return ra.make_cache_params(8, 2, 128, **base)


@pytest.mark.parametrize("field,value,status", [
    ("D", 96, -2), ("D", 256, -2), ("Hq", 0, -1), ("Hkv", 0, -1), ("Hkv", 3, -1), ("Hq", 2048, -2),
    ("page_size", 8, -2), ("page_size", 48, -2), ("page_size", 512, -2), ("num_pages", 0, -1), ("max_blocks", 0, -1),
    ("num_pages", 1 << 27, -2), ("max_blocks", (1 << 26) + 1, -2), ("rotation", 1, -2), ("rotation", 2, -2),
    ("v_rotation", 2, -1), ("causal", 2, -1), ("window", -1, -1), ("sm_scale", -1.0, -1),
    ("sm_scale", float("nan"), -1), ("in_dtype", 2, -1), ("out_dtype", 3, -1),
])
def test_parameters_that_are_refused(ra, field, value, status):
    p = _p(ra)
    setattr(p, field, value)
    for call in (lambda: ra.cache_layout(p), lambda: ra.cache_workspace_size(p, 1, 1, 1)):
        with pytest.raises(ra.RAError) as e:
            call()
        assert e.value.status == status


def test_window_needs_causal(ra):
    with pytest.raises(ra.RAError) as e:
        ra.cache_layout(_p(ra, causal=False, window=4))
    assert e.value.status == -2


def test_layout(ra):
    L = ra.cache_layout(_p(ra))
    assert L == {"head_bytes": 16 * 136, "page_bytes": 2 * 16 * 136, "cache_bytes": 20 * 16 * 136, "v_codes": 1024,
                 "k_scales": 2048, "v_scales": 2112}
    # every code has its own place, and codes, scales and heads do not overlap
    for D in (64, 128):
        for page in (16, 256):
            t, d = np.meshgrid(np.arange(page), np.arange(D), indexing="ij")
            k, v = ref.k_byte(D, t, d) * 2 + d % 2, ref.v_byte(D, page, t, d) * 2 + d % 2
            assert sorted(k.ravel()) == list(range(page * D))
            assert sorted(v.ravel()) == list(range(page * D, 2 * page * D))


def test_sizes_that_are_refused(ra):
    p = _p(ra)
    n = ctypes.c_size_t()
    f = ra.lib().rotate_attn_cache_workspace_size
    assert f(ctypes.byref(p), -1, 1, 1, ctypes.byref(n)) == -1
    assert f(ctypes.byref(p), 1, -1, 1, ctypes.byref(n)) == -1
    assert f(ctypes.byref(p), 1, 1, -1, ctypes.byref(n)) == -1
    assert f(ctypes.byref(p), 65537, 1, 1, ctypes.byref(n)) == -2
    assert f(ctypes.byref(p), 1, (1 << 24) + 1, 1, ctypes.byref(n)) == -2
    assert f(ctypes.byref(p), 1, 1, 1, None) == -1
    assert f(None, 1, 1, 1, ctypes.byref(n)) == -1
    assert f(ctypes.byref(p), 65536, 1 << 24, 1 << 24, ctypes.byref(n)) == 0 and n.value > 0


def test_pointers_that_are_refused(ra):
    L, p = ra.lib(), _p(ra)
    P, r = ctypes.c_void_p, ctypes.byref(_p(ra))
    ok, odd = P(0x1000), P(0x1008)
    err = L.rotate_attn_last_error
    plan = [ok] * 12
    assert L.rotate_attn_cache_plan(None, 1, 1, *plan, None) == -1
    for i in (0, 1, 3, 4, 5, 6, 7, 8, 9, 10, 11):          # 2 (release) may be NULL
        a = list(plan)
        a[i] = None
        a[6] = P(0x2000) if i != 6 else None               # seq_out apart from new_lens
        assert L.rotate_attn_cache_plan(r, 1, 1, *a, None) == -1 and b"NULL" in err(), i
    a = list(plan)
    a[2] = None
    assert L.rotate_attn_cache_plan(r, 1, 1, *a, None) == -1 and b"new_lens" in err()
    assert L.rotate_attn_cache_plan(r, -1, 1, *plan, None) == -1
    assert L.rotate_attn_cache_plan(r, 70000, 1, *plan, None) == -2

    def append(T=1, k=ok, ks=(128, 128), v=ok, vs=(128, 128), slots=ok, pos=ok, rope=ok, rows=64, cache=ok):
        return L.rotate_attn_cache_append(r, T, k, *ks, v, *vs, slots, pos, rope, rows, cache, None)
    assert append(T=0, k=None) == 0
    assert append(T=-1) == -1
    for kw in ({"k": None}, {"v": None}, {"slots": None}, {"cache": None}):
        assert append(**kw) == -1 and b"NULL" in err()
    for kw in ({"k": odd}, {"v": odd}, {"rope": odd}, {"cache": P(0x1010)}):
        assert append(**kw) == -1 and b"aligned" in err()
    for kw in ({"ks": (12, 128)}, {"vs": (128, 4)}, {"ks": (-128, 128)}):
        assert append(**kw) == -1 and b"stride" in err()
    assert append(pos=None) == -1 and b"positions" in err()
    assert append(rows=0) == -1 and b"rope_rows" in err()

    def read(T=1, cache=ok, slots=ok, k=ok, v=ok):
        return L.rotate_attn_cache_read(r, T, cache, slots, k, v, None)
    assert read(T=0) == 0
    for kw in ({"cache": None}, {"slots": None}, {"k": None}, {"v": None}, {"k": odd}, {"v": odd}, {"T": -3}):
        assert read(**kw) == -1

    def attn(R=1, T=1, max_q=1, q=ok, qs=(128, 128), cache=ok, table=ok, start=ok, lens=ok, rope=None, rows=0, o=ok,
             ws=ok, nws=1 << 40):
        return L.rotate_attn_cache_attn(r, R, T, max_q, q, *qs, cache, table, start, lens, rope, rows, o, None, ws, nws, None)
    for kw in ({"R": 0}, {"T": 0}, {"max_q": 0}):
        assert attn(**kw) == 0
    for kw in ({"R": -1}, {"T": -1}, {"max_q": -1}, {"q": None}, {"cache": None}, {"table": None}, {"start": None},
               {"lens": None}, {"o": None}, {"q": odd}, {"o": odd}, {"qs": (4, 128)}, {"rope": ok}, {"rope": odd, "rows": 9}):
        assert attn(**kw) == -1, kw
    need = ra.cache_workspace_size(p, 1, 1, 1)
    for kw in ({"ws": None}, {"ws": P(0x1080)}, {"nws": need - 1}):
        assert attn(**kw) == -3, kw


def test_binding_checks_tensors(ra):
    torch = pytest.importorskip("torch")
    p = _p(ra)
    i = lambda n: torch.zeros(n, dtype=torch.int32)
    x = torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    cache = torch.zeros(10, 2 * 16 * 136, dtype=torch.uint8)
    with pytest.raises(ValueError, match="device tensor"):
        ra.cache_append(p, x, x, i(3), cache)
    with pytest.raises(ValueError, match="shape"):
        ra.cache_append(p, x, x, i(3), cache[:9])
    with pytest.raises(ValueError, match="uint8"):
        ra.cache_read(p, cache.int(), i(3), x, x)
    with pytest.raises(ValueError, match="device tensor"):
        ra.cache_plan(p, i(2), i(2), torch.zeros(2, 4, dtype=torch.int32), i(10), i(1), i(3), i(5), i(5), i(4))
    with pytest.raises(ValueError, match="int32"):
        ra.cache_plan(p, i(2).long(), i(2), torch.zeros(2, 4, dtype=torch.int32), i(10), i(1), i(3), i(5), i(5), i(4))
    for bad, word in ((x.float(), "bfloat16"), (x[:2], "shape"), (x.transpose(0, 1), "shape"), ("k", "tensor"),
                      (torch.zeros(3, 2, 256, dtype=torch.bfloat16)[..., ::2], "adjacent"),
                      (torch.zeros(3, 2, 132, dtype=torch.bfloat16)[..., :128], "adjacent")):
        with pytest.raises(ValueError, match=word):
            ra._cache_tensor(bad, "k", torch.bfloat16, (3, 2, 128), None, strided=True)
    with pytest.raises(ValueError, match="contiguous"):
        ra._cache_tensor(torch.arange(8.0).view(2, 4).t(), "x", torch.float32, (4, 2), None)
    # an axis of one element may have any stride
    one = torch.zeros(1, 4, 2, 128, dtype=torch.bfloat16)[:, 0].as_strided((1, 2, 128), (3, 128, 1))
    with pytest.raises(ValueError, match="device tensor"):
        ra._cache_tensor(one, "k", torch.bfloat16, (1, 2, 128), None, strided=True)
    assert ra._cache_rows(one) == (0, 128)
    with pytest.raises(ValueError, match="positions"):
        ra._cache_rope(p, torch.zeros(2, 2), None)
