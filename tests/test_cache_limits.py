"""Sizes of the paged KV cache's attention that would not fit a launch are refused before any HIP call (CPU only)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def ra():
    import os
    from paper_2607_02584_amd import rotate_attn as m
    if not os.path.exists(m.LIB_PATH):
        pytest.skip("library not built")
    return m


# 2^32 work-items along the grid: 2^24 workgroups, of which 4096 are kept for split requests
@pytest.mark.parametrize("Hq,Hkv,R,T,ok", [
    (1024, 1024, 16380, 1, False), (1024, 1024, 16379, 1, True), (256, 256, 65536, 65536, False),
    (256, 128, 65536, 65536, True), (1024, 1, 1, 1 << 21, False), (1024, 1, 1, (1 << 21) - 1024, True),
    (8, 2, 65536, 1 << 24, True), (128, 128, 1, 1 << 24, False),
])
def test_more_pieces_than_a_launch_holds_are_refused(ra, Hq, Hkv, R, T, ok):
    p = ra.make_cache_params(Hq, Hkv, 64, page_size=16, num_pages=8, max_blocks=8)
    n = ctypes.c_size_t()
    L, ptr = ra.lib(), ctypes.c_void_p(0x1000)
    assert L.rotate_attn_cache_workspace_size(ctypes.byref(p), R, T, T, ctypes.byref(n)) == (0 if ok else -2)
    # a workspace of one byte: what fits is refused for that, and nothing is launched
    rc = L.rotate_attn_cache_attn(ctypes.byref(p), R, T, T, ptr, 64, 64, ptr, ptr, ptr, ptr, None, 0, ptr, None, ptr, 1, None)
    assert rc == (-3 if ok else -2), L.rotate_attn_last_error()
    if not ok:
        assert b"R * Hkv" in L.rotate_attn_last_error()
