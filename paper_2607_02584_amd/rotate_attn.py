"""Thin ctypes binding of librotate_attn.so (argument marshalling only).

Every step of the path runs in the HIP kernels of the library; this module
only turns torch tensors into device pointers, fills ``ra_params`` and raises
on a non-zero status.  If the library is not built the import of the first
call fails loudly: there is no fallback.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "librotate_attn.so")

ROT_NONE, ROT_INTERLEAVED, ROT_HALF, ROT_HADAMARD = 0, 1, 2, 3
PQ_RANGE15, PQ_SYM7 = 0, 1
VROT_NONE, VROT_HADAMARD = 0, 1
SMOOTH_K, SMOOTH_V, SMOOTH_Q = 1, 2, 4
BF16, FP16, FP32 = 0, 1, 2
CODES_INT4, CODES_E2M3 = 0, 1
PATH_INT4, PATH_FP16 = 0, 1


class RAError(RuntimeError):
    def __init__(self, status: int, where: str, message: str):
        super().__init__(f"{where} failed with status {status}: {message}")
        self.status = status


class Params(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("N", ctypes.c_int32), ("D", ctypes.c_int32),
        ("grid", ctypes.c_int32 * 3), ("rope_split", ctypes.c_int32 * 3), ("rope_theta", ctypes.c_float),
        ("rotation", ctypes.c_int32), ("rot_blocks", ctypes.POINTER(ctypes.c_double)),
        ("p_quant", ctypes.c_int32), ("smooth", ctypes.c_int32),
        ("q_group", ctypes.c_int32), ("k_group", ctypes.c_int32), ("v_group", ctypes.c_int32),
        ("kv_block", ctypes.c_int32), ("sm_scale", ctypes.c_float),
        ("in_dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32), ("code_format", ctypes.c_int32),
        ("v_rotation", ctypes.c_int32), ("l_quant", ctypes.c_int32),
    ]


class Layout(ctypes.Structure):
    _fields_ = [("n_pad", ctypes.c_int64), ("qk_code_bytes", ctypes.c_int64), ("q_scale_count", ctypes.c_int64),
                ("k_scale_count", ctypes.c_int64), ("v_code_bytes", ctypes.c_int64),
                ("v_scale_count", ctypes.c_int64), ("mu_count", ctypes.c_int64), ("k_bias_count", ctypes.c_int64)]


class CacheParams(ctypes.Structure):
    _fields_ = [("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("num_pages", ctypes.c_int32), ("max_blocks", ctypes.c_int32),
                ("rotation", ctypes.c_int32), ("v_rotation", ctypes.c_int32), ("causal", ctypes.c_int32),
                ("window", ctypes.c_int32), ("sm_scale", ctypes.c_float), ("in_dtype", ctypes.c_int32),
                ("out_dtype", ctypes.c_int32)]


class CacheSizes(ctypes.Structure):
    _fields_ = [("head_bytes", ctypes.c_int64), ("page_bytes", ctypes.c_int64), ("cache_bytes", ctypes.c_int64),
                ("v_codes", ctypes.c_int64), ("k_scales", ctypes.c_int64), ("v_scales", ctypes.c_int64)]


class CacheTables(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("seq_lens", "block_table", "page_refs", "free_pages", "free_count")]


_lib = None


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                               "(python -c 'import __graft_entry__ as g; g.build()')")
        # torch (which provides the device memory and streams) brings its own HIP
        # runtime under the same soname; loading it first makes the library bind
        # to that one instead of starting a second runtime in the process
        import torch  # noqa: F401
        L = ctypes.CDLL(LIB_PATH)
        P = ctypes.c_void_p
        PP = ctypes.POINTER(Params)
        CP, I, S = ctypes.POINTER(CacheParams), ctypes.c_int32, ctypes.c_int64
        TP = ctypes.POINTER(CacheTables)
        sig = {
            "rotate_attn_layout": [PP, ctypes.POINTER(Layout)],
            "rotate_attn_workspace_size": [PP, ctypes.c_int, ctypes.POINTER(ctypes.c_size_t)],
            "rotate_attn_quantize_qk": [PP, P, P, P, P, P, P, P, P, P, P, ctypes.c_size_t, P],
            "rotate_attn_quantize_v": [PP, P, P, P, P, P, ctypes.c_size_t, P],
            "rotate_attn_quantize_qkv": [PP, P, P, P, P, P, P, P, P, P, P, P, P, P, P, ctypes.c_size_t, P],
            "rotate_attn_attn_int4": [PP, P, P, P, P, P, P, P, P, P, P],
            "rotate_attn_attn_int4_debug": [PP, P, P, P, P, P, P, P, P, P, ctypes.c_int32, ctypes.c_int32,
                                            ctypes.c_int32, P, P, P, P],
            "rotate_attn_fwd_int4": [PP, P, P, P, P, P, ctypes.c_size_t, P],
            "rotate_attn_prepare_fp16": [PP, P, P, P, P, ctypes.c_size_t, P],
            "rotate_attn_attn_fp16": [PP, P, ctypes.c_size_t, P, P],
            "rotate_attn_fwd_fp16": [PP, P, P, P, P, P, ctypes.c_size_t, P],
            "rotate_attn_fwd": [PP, ctypes.c_int, P, P, P, P, P, ctypes.c_size_t, P],
            "rotate_attn_fwd_int4_noalloc": [PP, P, P, P, P, P],
            "rotate_attn_cache_layout": [CP, ctypes.POINTER(CacheSizes)],
            "rotate_attn_cache_workspace_size": [CP, I, I, I, ctypes.POINTER(ctypes.c_size_t)],
            "rotate_attn_cache_plan": [CP, I, I] + [P] * 13,
            "rotate_attn_cache_append": [CP, I, P, S, S, P, S, S, P, P, P, I, P, P],
            "rotate_attn_cache_read": [CP, I, P, P, P, P, P],
            "rotate_attn_cache_attn_sinks": [CP, I, I, I, I, P, S, S, P, P, P, P, P, I, P, P, P, ctypes.c_size_t, P],
            "rotate_attn_cache_shared_workspace_size": [CP, I, I, I, ctypes.POINTER(ctypes.c_size_t)],
            "rotate_attn_cache_attn_shared": [CP, I, I, I, P, S, S, P, P, P, P, P, P, P, P, I, P, P, P, ctypes.c_size_t, P],
            "rotate_attn_cache_pages_workspace_size": [CP, I, ctypes.POINTER(ctypes.c_size_t)],
            "rotate_attn_cache_fork": [CP, I, I, P, P, P, TP, TP, P, P, ctypes.c_size_t, P, P],
            "rotate_attn_cache_trim": [CP, I, P, I, TP, TP, P, P, ctypes.c_size_t, P, P],
            "rotate_attn_cache_compact": [CP, I, TP, TP, P, P, ctypes.c_size_t, P, P],
            "rotate_attn_cache_attn": [CP, I, I, I, P, S, S, P, P, P, P, P, I, P, P, P, ctypes.c_size_t, P],
        }
        for name, args in sig.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = ctypes.c_int
        L.rotate_attn_error_string.argtypes = [ctypes.c_int]
        L.rotate_attn_error_string.restype = ctypes.c_char_p
        L.rotate_attn_last_error.argtypes = []
        L.rotate_attn_last_error.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _check(status: int, where: str):
    if status != 0:
        raise RAError(status, where, lib().rotate_attn_last_error().decode())


def make_params(B, H, grid, split=(44, 42, 42), theta=10000.0, *, rotation=ROT_INTERLEAVED, rot_blocks=None,
                p_quant=PQ_RANGE15, smooth=SMOOTH_K | SMOOTH_V, q_group=128, k_group=128, v_group=128,
                kv_block=128, sm_scale=0.0, in_dtype=BF16, out_dtype=BF16, code_format=CODES_E2M3, D=128,
                v_rotation=VROT_NONE, l_quant=0) -> Params:
    p = Params()
    p.B, p.H, p.D = B, H, D
    p.N = int(grid[0] * grid[1] * grid[2])
    p.grid[:] = [int(g) for g in grid]
    p.rope_split[:] = [int(s) for s in split]
    p.rope_theta = float(theta)
    p.rotation = rotation
    if rot_blocks is not None:
        arr = np.ascontiguousarray(rot_blocks, dtype=np.float64).reshape(D // 2, 2, 2)
        p._rot_keep = arr  # keep alive with the struct
        p.rot_blocks = arr.ctypes.data_as(ctypes.POINTER(ctypes.c_double))
    p.p_quant, p.smooth = p_quant, smooth
    p.q_group, p.k_group, p.v_group, p.kv_block = q_group, k_group, v_group, kv_block
    p.sm_scale = float(sm_scale)
    p.in_dtype, p.out_dtype = in_dtype, out_dtype
    p.code_format = code_format
    p.v_rotation = v_rotation
    p.l_quant = int(l_quant)
    return p


def layout(p: Params) -> dict:
    out = Layout()
    _check(lib().rotate_attn_layout(ctypes.byref(p), ctypes.byref(out)), "rotate_attn_layout")
    return {f: getattr(out, f) for f, _ in Layout._fields_}


def workspace_size(p: Params, path: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().rotate_attn_workspace_size(ctypes.byref(p), path, ctypes.byref(n)), "rotate_attn_workspace_size")
    return n.value


def _ptr(t):
    if t is None:
        return None
    return ctypes.c_void_p(t.data_ptr())


def _need(t, nbytes, name, optional=False):
    """The library takes raw pointers: check here that a tensor is a contiguous
    device tensor holding at least the bytes the call will touch."""
    if t is None:
        if optional:
            return
        raise ValueError(f"{name} is required")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.numel() * t.element_size() < nbytes:
        raise ValueError(f"{name} holds {t.numel() * t.element_size()} bytes, the call needs {nbytes}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")


def _io_bytes(p):
    n = int(p.B) * int(p.H) * int(p.N) * int(p.D)
    return 2 * n, n * (4 if p.out_dtype == FP32 else 2)


def _check_codes(p, L, q_codes=None, q_scale=None, k_codes=None, k_scale=None, v_codes=None, v_scale=None,
                 mu=(), k_bias=None, need_bias=False):
    for t, nb, name in ((q_codes, L["qk_code_bytes"], "q_codes"), (k_codes, L["qk_code_bytes"], "k_codes"),
                        (q_scale, 4 * L["q_scale_count"], "q_scale"), (k_scale, 4 * L["k_scale_count"], "k_scale"),
                        (v_codes, L["v_code_bytes"], "v_codes"), (v_scale, 4 * L["v_scale_count"], "v_scale")):
        if nb and t is not False:
            _need(t, nb, name)
    for t, name in mu:
        _need(t, 4 * L["mu_count"], name, optional=True)
    if need_bias or k_bias is not None:
        _need(k_bias, 4 * L["k_bias_count"], "k_bias", optional=not need_bias)


def _stream(stream):
    if stream is not None:
        return ctypes.c_void_p(stream)
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _nbytes(t) -> int:
    return t.numel() * t.element_size()


def quantize_qk(p, q, k, q_codes, q_scale, k_codes, k_scale, mu_k, ws, stream=None, mu_q=None, k_bias=None):
    L = layout(p)
    nin, _ = _io_bytes(p)
    _need(q, nin, "q")
    _need(k, nin, "k")
    _check_codes(p, L, q_codes=q_codes, q_scale=q_scale, k_codes=k_codes, k_scale=k_scale, v_codes=False,
                 v_scale=False, mu=((mu_k, "mu_k"), (mu_q, "mu_q")), k_bias=k_bias,
                 need_bias=bool(p.smooth & SMOOTH_Q))
    _need(ws, workspace_size(p, PATH_INT4), "workspace")
    _check(lib().rotate_attn_quantize_qk(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(q_codes), _ptr(q_scale),
                                         _ptr(k_codes), _ptr(k_scale), _ptr(mu_k), _ptr(mu_q), _ptr(k_bias),
                                         _ptr(ws), _nbytes(ws), _stream(stream)), "rotate_attn_quantize_qk")


def quantize_v(p, v, v_codes, v_scale, mu_v, ws, stream=None):
    L = layout(p)
    _need(v, _io_bytes(p)[0], "v")
    _check_codes(p, L, q_codes=False, q_scale=False, k_codes=False, k_scale=False, v_codes=v_codes, v_scale=v_scale,
                 mu=((mu_v, "mu_v"),))
    _need(ws, workspace_size(p, PATH_INT4), "workspace")
    _check(lib().rotate_attn_quantize_v(ctypes.byref(p), _ptr(v), _ptr(v_codes), _ptr(v_scale), _ptr(mu_v),
                                        _ptr(ws), _nbytes(ws), _stream(stream)), "rotate_attn_quantize_v")


def quantize_qkv(p, q, k, v, q_codes, q_scale, k_codes, k_scale, v_codes, v_scale, ws, stream=None, mu_k=None,
                 mu_q=None, mu_v=None, k_bias=None):
    """quantize_qk and quantize_v in one call."""
    L = layout(p)
    nin, _ = _io_bytes(p)
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        _need(t, nin, name)
    _check_codes(p, L, q_codes, q_scale, k_codes, k_scale, v_codes, v_scale,
                 mu=((mu_k, "mu_k"), (mu_q, "mu_q"), (mu_v, "mu_v")), k_bias=k_bias,
                 need_bias=bool(p.smooth & SMOOTH_Q))
    _need(ws, workspace_size(p, PATH_INT4), "workspace")
    _check(lib().rotate_attn_quantize_qkv(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(q_codes), _ptr(q_scale),
                                          _ptr(k_codes), _ptr(k_scale), _ptr(v_codes), _ptr(v_scale), _ptr(mu_k),
                                          _ptr(mu_q), _ptr(mu_v), _ptr(k_bias), _ptr(ws), _nbytes(ws),
                                          _stream(stream)), "rotate_attn_quantize_qkv")


def attn_int4(p, q_codes, q_scale, k_codes, k_scale, v_codes, v_scale, mu_v, o, stream=None, k_bias=None):
    L = layout(p)
    _check_codes(p, L, q_codes, q_scale, k_codes, k_scale, v_codes, v_scale, mu=((mu_v, "mu_v"),), k_bias=k_bias,
                 need_bias=bool(p.smooth & SMOOTH_Q))
    _need(o, _io_bytes(p)[1], "o")
    _check(lib().rotate_attn_attn_int4(ctypes.byref(p), _ptr(q_codes), _ptr(q_scale), _ptr(k_codes), _ptr(k_scale),
                                       _ptr(v_codes), _ptr(v_scale), _ptr(mu_v), _ptr(k_bias), _ptr(o),
                                       _stream(stream)), "rotate_attn_attn_int4")


def attn_int4_debug(p, q_codes, q_scale, k_codes, k_scale, v_codes, v_scale, mu_v, o, bh, row0, rows,
                    s_out=None, u_out=None, m_out=None, stream=None, k_bias=None):
    L = layout(p)
    _check_codes(p, L, q_codes, q_scale, k_codes, k_scale, v_codes, v_scale, mu=((mu_v, "mu_v"),), k_bias=k_bias,
                 need_bias=bool(p.smooth & SMOOTH_Q))
    _need(o, _io_bytes(p)[1], "o")
    nb = -(-int(p.N) // int(p.kv_block))
    _need(s_out, 4 * rows * int(p.N), "s_out", optional=True)
    _need(u_out, rows * int(p.N), "u_out", optional=True)
    _need(m_out, 4 * rows * nb, "m_out", optional=True)
    _check(lib().rotate_attn_attn_int4_debug(ctypes.byref(p), _ptr(q_codes), _ptr(q_scale), _ptr(k_codes),
                                             _ptr(k_scale), _ptr(v_codes), _ptr(v_scale), _ptr(mu_v),
                                             _ptr(k_bias), _ptr(o),
                                             bh, row0, rows, _ptr(s_out), _ptr(u_out), _ptr(m_out),
                                             _stream(stream)), "rotate_attn_attn_int4_debug")


def _check_fwd(p, q, k, v, o, ws, path):
    nin, nout = _io_bytes(p)
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        _need(t, nin, name)
    _need(o, nout, "o")
    _need(ws, workspace_size(p, path), "workspace")


def fwd_int4(p, q, k, v, o, ws, stream=None):
    _check_fwd(p, q, k, v, o, ws, PATH_INT4)
    _check(lib().rotate_attn_fwd_int4(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(ws), _nbytes(ws),
                                      _stream(stream)), "rotate_attn_fwd_int4")


NOALLOC_SCRATCH_BYTES = 128 << 20


def fwd_int4_noalloc(p, q, k, v, o, stream=None):
    """The INT4 forward on the library's static per-GPU scratch (no workspace,
    nothing allocated); calls that overlap on one GPU race."""
    nin, nout = _io_bytes(p)
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        _need(t, nin, name)
    _need(o, nout, "o")
    _check(lib().rotate_attn_fwd_int4_noalloc(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _stream(stream)),
           "rotate_attn_fwd_int4_noalloc")


def prepare_fp16(p, q, k, v, ws, stream=None):
    nin, _ = _io_bytes(p)
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        _need(t, nin, name)
    _need(ws, workspace_size(p, PATH_FP16), "workspace")
    _check(lib().rotate_attn_prepare_fp16(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(ws), _nbytes(ws),
                                          _stream(stream)), "rotate_attn_prepare_fp16")


def attn_fp16(p, ws, o, stream=None):
    _need(ws, workspace_size(p, PATH_FP16), "workspace")
    _need(o, _io_bytes(p)[1], "o")
    _check(lib().rotate_attn_attn_fp16(ctypes.byref(p), _ptr(ws), _nbytes(ws), _ptr(o), _stream(stream)),
           "rotate_attn_attn_fp16")


def fwd_fp16(p, q, k, v, o, ws, stream=None):
    _check_fwd(p, q, k, v, o, ws, PATH_FP16)
    _check(lib().rotate_attn_fwd_fp16(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(ws), _nbytes(ws),
                                      _stream(stream)), "rotate_attn_fwd_fp16")


def fwd(p, fallback, q, k, v, o, ws, stream=None):
    _check_fwd(p, q, k, v, o, ws, PATH_FP16 if fallback else PATH_INT4)
    _check(lib().rotate_attn_fwd(ctypes.byref(p), int(bool(fallback)), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(ws),
                                 _nbytes(ws), _stream(stream)), "rotate_attn_fwd")


# ------------------------------------------------------ 4-bit paged KV cache --

def make_cache_params(Hq, Hkv, D=128, *, page_size=64, num_pages, max_blocks, rotation=ROT_HADAMARD,
                      v_rotation=VROT_NONE, causal=True, window=0, sm_scale=0.0, in_dtype=BF16,
                      out_dtype=BF16) -> CacheParams:
    p = CacheParams()
    p.Hq, p.Hkv, p.D = Hq, Hkv, D
    p.page_size, p.num_pages, p.max_blocks = page_size, num_pages, max_blocks
    p.rotation, p.v_rotation = rotation, v_rotation
    p.causal, p.window = int(causal), window
    p.sm_scale = float(sm_scale)
    p.in_dtype, p.out_dtype = in_dtype, out_dtype
    return p


def cache_layout(p: CacheParams) -> dict:
    out = CacheSizes()
    _check(lib().rotate_attn_cache_layout(ctypes.byref(p), ctypes.byref(out)), "rotate_attn_cache_layout")
    return {f: getattr(out, f) for f, _ in CacheSizes._fields_}


def cache_workspace_size(p: CacheParams, R: int, T: int, max_q: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().rotate_attn_cache_workspace_size(ctypes.byref(p), R, T, max_q, ctypes.byref(n)),
           "rotate_attn_cache_workspace_size")
    return n.value


# The cache calls are made once per layer and token: what is checked stays one
# comparison per tensor while all is well (a call with its launches takes 9 to 16
# us of host time), the reasons are worked out on the way to the error.

_dtypes = None


def _cache_dtypes():
    global _dtypes
    if _dtypes is None:
        import torch
        _dtypes = {BF16: torch.bfloat16, FP16: torch.float16, FP32: torch.float32, "i32": torch.int32,
                   "u8": torch.uint8}
    return _dtypes


def _cache_tensor(t, name, dtype, shape, device=None, strided=False):
    """A device tensor of this type and shape, contiguous; `strided`: channels
    adjacent, the other strides multiples of 8 elements."""
    if device is not None:   # all is well, as a rule
        try:
            if t.dtype is dtype and t.shape == shape and t.get_device() == device.index and t.is_contiguous():
                return t.data_ptr()
        except AttributeError:
            pass
    import torch
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a tensor")
    if t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if not t.is_contiguous():
        if not strided:
            raise ValueError(f"{name} must be contiguous")
        # the stride of an axis of one element is never used, whatever it says
        if t.stride(-1) != 1 or any(t.stride(i) % 8 or t.stride(i) < 0 for i in (0, 1) if shape[i] > 1):
            raise ValueError(f"{name} needs adjacent channels and other strides that are multiples of 8 elements")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, the cache call runs on {device}")
    return t.data_ptr()


def _cache_rows(t):
    """Token and head stride of [T, heads, D] (0 on an axis of one element)."""
    n, h, _ = t.shape
    a, b, _ = t.stride()
    return a if n > 1 else 0, b if h > 1 else 0


def _cache_rope(p, rope, device):
    """rope [rows, D/2, 2]: every position the block table can hold has a row."""
    import torch
    if rope is None:
        return None, 0
    if not isinstance(rope, torch.Tensor) or rope.dim() != 3:
        raise ValueError("rope must be a tensor of shape [positions, D/2, 2]")
    rows = rope.shape[0]
    ptr = _cache_tensor(rope, "rope", _cache_dtypes()[FP32], (rows, p.D // 2, 2), device)
    if rows < p.max_blocks * p.page_size:
        raise ValueError(f"rope has {rows} positions, max_blocks * page_size is {p.max_blocks * p.page_size}")
    if rows > 0x7fffffff:
        raise ValueError("rope has more than 2^31 - 1 positions")
    return ptr, rows


def _cache_ints(device, *what):
    """Addresses of int32 tensors, given as (tensor, name, shape)."""
    i32, index = _cache_dtypes()["i32"], device.index
    try:   # all is well, as a rule
        at = [t.data_ptr() for t, _, shape in what
              if t.dtype is i32 and t.shape == shape and t.get_device() == index and t.is_contiguous()]
        if len(at) == len(what):
            return at
    except AttributeError:
        pass
    return [_cache_tensor(t, name, i32, shape, device) for t, name, shape in what]


def _current_stream(device):
    """The device's current stream: its handle alone where torch hands that out
    (0.1 us of host time instead of 1.9)."""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(device.index) if raw else torch.cuda.current_stream(device).cuda_stream


def _cache_call(fn, where, device, stream, *args):
    """fn(*args, stream) with the tensors' device current, on `stream` or that
    device's current stream."""
    import torch
    if stream is None:
        stream = _current_stream(device)
    if torch.cuda.current_device() == device.index:
        status = fn(*args, stream)
    else:
        with torch.cuda.device(device):
            status = fn(*args, stream)
    if status != 0:
        _check(status, where)


def _cache_pages(p, cache, u8):
    return _cache_tensor(cache, "cache", u8, (p.num_pages, p.Hkv * p.page_size * (p.D + 8)))


def cache_plan(p, seq_lens, new_lens, block_table, free_pages, free_count, q_start, positions, slots, status,
               release=None, seq_out=None, count_out=None, stream=None):
    """Block tables, offsets, positions and slots of a step from its lengths
    (all int32; rotate_attn.h has the rules).  seq_lens and free_count are
    updated in place unless seq_out and count_out are given.  The call only
    enqueues: status is read by whoever wants to know."""
    i32 = _cache_dtypes()["i32"]
    R, T = seq_lens.numel(), slots.numel()
    dev, per_request, per_token = seq_lens.device, (R,), (T,)
    lens = _cache_tensor(seq_lens, "seq_lens", i32, per_request)
    table = _cache_tensor(block_table, "block_table", i32, (R, p.max_blocks), dev)
    count = _cache_tensor(free_count, "free_count", i32, (1,), dev)
    _cache_call(
        lib().rotate_attn_cache_plan, "rotate_attn_cache_plan", dev, stream, ctypes.byref(p), R, T, lens,
        _cache_tensor(new_lens, "new_lens", i32, per_request, dev),
        None if release is None else _cache_tensor(release, "release", i32, per_request, dev), table,
        _cache_tensor(free_pages, "free_pages", i32, (p.num_pages,), dev), count,
        lens if seq_out is None else _cache_tensor(seq_out, "seq_out", i32, per_request, dev),
        count if count_out is None else _cache_tensor(count_out, "count_out", i32, (1,), dev),
        _cache_tensor(q_start, "q_start", i32, (R + 1,), dev), _cache_tensor(positions, "positions", i32, per_token, dev),
        _cache_tensor(slots, "slots", i32, per_token, dev), _cache_tensor(status, "status", i32, (4,), dev))


def cache_append(p, k, v, slots, cache, positions=None, rope=None, stream=None):
    """Tokens k, v [T, Hkv, D] into their slots of the cache: RoPE by position
    where rope is given, rotation, 4-bit codes."""
    dt = _cache_dtypes()
    pages, dev, T = _cache_pages(p, cache, dt["u8"]), cache.device, slots.numel()
    shape, kind = (T, p.Hkv, p.D), dt[p.in_dtype]
    if rope is not None and positions is None:
        raise ValueError("rope needs positions")
    table, rows = _cache_rope(p, rope, dev)
    _cache_call(
        lib().rotate_attn_cache_append, "rotate_attn_cache_append", dev, stream, ctypes.byref(p), T,
        _cache_tensor(k, "k", kind, shape, dev, True), *_cache_rows(k),
        _cache_tensor(v, "v", kind, shape, dev, True), *_cache_rows(v),
        _cache_tensor(slots, "slots", dt["i32"], (T,), dev),
        None if positions is None else _cache_tensor(positions, "positions", dt["i32"], (T,), dev), table, rows, pages)


def cache_read(p, cache, slots, k, v, stream=None):
    """The values that cached tokens stand for, into k, v [T, Hkv, D] of out_dtype."""
    dt = _cache_dtypes()
    pages, dev, T = _cache_pages(p, cache, dt["u8"]), cache.device, slots.numel()
    shape, kind = (T, p.Hkv, p.D), dt[p.out_dtype]
    _cache_call(
        lib().rotate_attn_cache_read, "rotate_attn_cache_read", dev, stream, ctypes.byref(p), T, pages,
        _cache_tensor(slots, "slots", dt["i32"], (T,), dev), _cache_tensor(k, "k", kind, shape, dev),
        _cache_tensor(v, "v", kind, shape, dev))


def cache_attn(p, q, cache, block_table, q_start, seq_lens, max_q, o, ws, lse=None, rope=None, stream=None):
    """Attention of packed queries q [T, Hq, D] to their requests' cached
    tokens into o [T, Hq, D] (and lse [T, Hq])."""
    dt = _cache_dtypes()
    pages, dev, R, T = _cache_pages(p, cache, dt["u8"]), cache.device, seq_lens.numel(), q.shape[0]
    shape, i32 = (T, p.Hq, p.D), dt["i32"]
    table, rows = _cache_rope(p, rope, dev)
    nws = _nbytes(ws)
    _cache_call(
        lib().rotate_attn_cache_attn, "rotate_attn_cache_attn", dev, stream, ctypes.byref(p), R, T, max_q,
        _cache_tensor(q, "q", dt[p.in_dtype], shape, dev, True), *_cache_rows(q), pages,
        _cache_tensor(block_table, "block_table", i32, (R, p.max_blocks), dev),
        _cache_tensor(q_start, "q_start", i32, (R + 1,), dev), _cache_tensor(seq_lens, "seq_lens", i32, (R,), dev),
        table, rows, _cache_tensor(o, "o", dt[p.out_dtype], shape, dev),
        None if lse is None else _cache_tensor(lse, "lse", dt[FP32], shape[:2], dev),
        _cache_tensor(ws, "workspace", dt["u8"], (nws,), dev), nws)


def cache_attn_sinks(p, sinks, q, cache, block_table, q_start, seq_lens, max_q, o, ws, lse=None, rope=None, stream=None):
    """cache_attn under the params' window, beside which each request's first
    `sinks` tokens stay visible (workspace as cache_attn's)."""
    dt = _cache_dtypes()
    pages, dev, R, T = _cache_pages(p, cache, dt["u8"]), cache.device, seq_lens.numel(), q.shape[0]
    shape = T, p.Hq, p.D
    table, rows = _cache_rope(p, rope, dev)
    nws = _nbytes(ws)
    _cache_call(
        lib().rotate_attn_cache_attn_sinks, "rotate_attn_cache_attn_sinks", dev, stream, ctypes.byref(p), sinks, R, T, max_q,
        _cache_tensor(q, "q", dt[p.in_dtype], shape, dev, True), *_cache_rows(q), pages,
        *_cache_ints(dev, (block_table, "block_table", (R, p.max_blocks)), (q_start, "q_start", (R + 1,)),
                     (seq_lens, "seq_lens", (R,))), table, rows, _cache_tensor(o, "o", dt[p.out_dtype], shape, dev),
        None if lse is None else _cache_tensor(lse, "lse", dt[FP32], shape[:2], dev),
        _cache_tensor(ws, "workspace", dt["u8"], (nws,), dev), nws)


def cache_attn_shared(p, q, cache, block_table, q_start, seq_lens, positions, group_start, prefix_lens, o, ws, lse=None,
                      rope=None, stream=None):
    """cache_attn of requests in groups that hold the same first tokens: requests
    group_start[g] .. group_start[g + 1] - 1 share prefix_lens[g] of them, which are
    read once for all (positions as cache_plan leaves them)."""
    dt = _cache_dtypes()
    pages, dev, R, T = _cache_pages(p, cache, dt["u8"]), cache.device, seq_lens.numel(), q.shape[0]
    shape, groups = (T, p.Hq, p.D), prefix_lens.numel()
    table, rows = _cache_rope(p, rope, dev)
    nws = _nbytes(ws)
    _cache_call(
        lib().rotate_attn_cache_attn_shared, "rotate_attn_cache_attn_shared", dev, stream, ctypes.byref(p), R, T, groups,
        _cache_tensor(q, "q", dt[p.in_dtype], shape, dev, True), *_cache_rows(q), pages,
        *_cache_ints(dev, (block_table, "block_table", (R, p.max_blocks)), (q_start, "q_start", (R + 1,)),
                     (seq_lens, "seq_lens", (R,)), (positions, "positions", (T,)),
                     (group_start, "group_start", (groups + 1,)), (prefix_lens, "prefix_lens", (groups,))), table, rows,
        _cache_tensor(o, "o", dt[p.out_dtype], shape, dev),
        None if lse is None else _cache_tensor(lse, "lse", dt[FP32], shape[:2], dev),
        _cache_tensor(ws, "workspace", dt["u8"], (nws,), dev), nws)


def cache_shared_workspace(p: CacheParams, R: int, groups: int, T: int, device="cuda"):
    """Workspace of cache_attn_shared."""
    import torch
    n = ctypes.c_size_t()
    _check(lib().rotate_attn_cache_shared_workspace_size(ctypes.byref(p), R, groups, T, ctypes.byref(n)),
           "rotate_attn_cache_shared_workspace_size")
    return torch.empty(max(n.value, 256), dtype=torch.uint8, device=device)


def _page_tables(p, seq_lens, block_table, page_refs, free_pages, free_count, cache, ws, status, seq_out, table_out,
                 refs_out, free_out, count_out):
    """R, the device, and (tables, out, cache, workspace, its bytes, status) as the library takes them."""
    R, u8 = seq_lens.numel(), _cache_dtypes()["u8"]
    pages, dev = _cache_pages(p, cache, u8), cache.device
    per_request, per_page, rows, one = (R,), (p.num_pages,), (R, p.max_blocks), (1,)
    at = _cache_ints(dev, (seq_lens, "seq_lens", per_request), (block_table, "block_table", rows),
                     (page_refs, "page_refs", per_page), (free_pages, "free_pages", per_page),
                     (free_count, "free_count", one),
                     (seq_lens if seq_out is None else seq_out, "seq_out", per_request),
                     (block_table if table_out is None else table_out, "table_out", rows),
                     (page_refs if refs_out is None else refs_out, "refs_out", per_page),
                     (free_pages if free_out is None else free_out, "free_out", per_page),
                     (free_count if count_out is None else count_out, "count_out", one), (status, "status", (4,)))
    nws = _nbytes(ws)
    return R, dev, (CacheTables(*at[:5]), CacheTables(*at[5:10]), pages, _cache_tensor(ws, "workspace", u8, (nws,), dev), nws,
                    at[10])


def cache_fork(p, parents, children, seq_lens, block_table, page_refs, free_pages, free_count, cache, ws, status,
               lens=None, seq_out=None, table_out=None, refs_out=None, free_out=None, count_out=None, stream=None):
    """Requests children[i], which hold nothing, begin with the first lens[i] (all,
    where None) tokens of parents[i]: full pages are shared, the page that the
    tokens end in is copied (all int32; rotate_attn.h has the rules).  Tables are
    updated in place unless arrays for their new state are given."""
    R, dev, rest = _page_tables(p, seq_lens, block_table, page_refs, free_pages, free_count, cache, ws, status, seq_out,
                                table_out, refs_out, free_out, count_out)
    n = (parents.numel(),)
    what = (parents, "parents", n), (children, "children", n), (lens, "lens", n)
    _cache_call(lib().rotate_attn_cache_fork, "rotate_attn_cache_fork", dev, stream, ctypes.byref(p), R, n[0],
                *((*_cache_ints(dev, *what[:2]), None) if lens is None else _cache_ints(dev, *what)), *rest)


def cache_trim(p, seq_lens, block_table, page_refs, free_pages, free_count, cache, ws, status, keep=None, sinks=-1,
               seq_out=None, table_out=None, refs_out=None, free_out=None, count_out=None, stream=None):
    """Requests keep their first keep[r] tokens (all where negative, 0 ends them);
    with sinks >= 0 they also lose the pages between the first `sinks` tokens and
    the params' window.  Pages that nobody holds any more go back on the stack."""
    R, dev, rest = _page_tables(p, seq_lens, block_table, page_refs, free_pages, free_count, cache, ws, status, seq_out,
                                table_out, refs_out, free_out, count_out)
    _cache_call(lib().rotate_attn_cache_trim, "rotate_attn_cache_trim", dev, stream, ctypes.byref(p), R,
                None if keep is None else _cache_ints(dev, (keep, "keep", (R,)))[0], sinks, *rest)


def cache_compact(p, seq_lens, block_table, page_refs, free_pages, free_count, cache, ws, status, seq_out=None,
                  table_out=None, refs_out=None, free_out=None, count_out=None, stream=None):
    """Moves the pages in use to the front of the cache; tables, holders and the
    stack of free pages follow."""
    R, dev, rest = _page_tables(p, seq_lens, block_table, page_refs, free_pages, free_count, cache, ws, status, seq_out,
                                table_out, refs_out, free_out, count_out)
    _cache_call(lib().rotate_attn_cache_compact, "rotate_attn_cache_compact", dev, stream, ctypes.byref(p), R, *rest)


def cache_pages_workspace(p: CacheParams, R: int, device="cuda"):
    """Workspace of cache_fork, cache_trim and cache_compact."""
    import torch
    n = ctypes.c_size_t()
    _check(lib().rotate_attn_cache_pages_workspace_size(ctypes.byref(p), R, ctypes.byref(n)),
           "rotate_attn_cache_pages_workspace_size")
    return torch.empty(n.value, dtype=torch.uint8, device=device)


def alloc_cache(p: CacheParams, R: int, device="cuda"):
    """The state of R requests: pages, block table, lengths, the stack of free
    pages, all free, and the pages' further holders, none."""
    import torch
    i32 = dict(dtype=torch.int32, device=device)
    return dict(
        cache=torch.empty((int(p.num_pages), cache_layout(p)["page_bytes"]), dtype=torch.uint8, device=device),
        block_table=torch.full((R, int(p.max_blocks)), -1, **i32),
        seq_lens=torch.zeros(R, **i32),
        free_pages=torch.arange(int(p.num_pages) - 1, -1, -1, **i32),
        free_count=torch.full((1,), int(p.num_pages), **i32),
        page_refs=torch.zeros(int(p.num_pages), **i32),
    )


def cache_workspace(p: CacheParams, R: int, T: int, max_q: int, device="cuda"):
    import torch
    return torch.empty(max(cache_workspace_size(p, R, T, max_q), 256), dtype=torch.uint8, device=device)


# ---------------------------------------------------------------- helpers --

def alloc_int4(p: Params, device="cuda"):
    """Caller-side buffers for the quantize / attention entry points."""
    import torch
    L = layout(p)
    return dict(
        q_codes=torch.zeros(L["qk_code_bytes"], dtype=torch.uint8, device=device),
        k_codes=torch.zeros(L["qk_code_bytes"], dtype=torch.uint8, device=device),
        v_codes=torch.zeros(L["v_code_bytes"], dtype=torch.uint8, device=device),
        q_scale=torch.zeros(L["q_scale_count"], dtype=torch.float32, device=device),
        k_scale=torch.zeros(L["k_scale_count"], dtype=torch.float32, device=device),
        v_scale=torch.zeros(L["v_scale_count"], dtype=torch.float32, device=device),
        mu_k=torch.zeros(L["mu_count"], dtype=torch.float32, device=device),
        mu_v=torch.zeros(L["mu_count"], dtype=torch.float32, device=device),
        mu_q=torch.zeros(L["mu_count"], dtype=torch.float32, device=device),
        k_bias=torch.zeros(L["k_bias_count"], dtype=torch.float32, device=device),
    )


def workspace(p: Params, path: int, device="cuda"):
    import torch
    return torch.empty(max(workspace_size(p, path), 256), dtype=torch.uint8, device=device)


def to_device_bits(x_bits: np.ndarray, device="cuda"):
    """uint16 bit patterns -> int16 device tensor holding the same bits."""
    import torch
    return torch.from_numpy(np.ascontiguousarray(x_bits).view(np.int16)).to(device)
