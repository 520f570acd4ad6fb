"""Wait states between the paged KV cache's matrix products and the uses of their results (CPU only), with the
distances that the compiler itself keeps in code without branches: 8 wait states behind a 4-pass product, 12 behind an
8-pass one, before a vector instruction or another product's first or second operand reads it.  (test_cache_isa asks for 6 and
10 and does not look at a product's operands.)
"""
import os
import re
import shutil
import subprocess

import pytest

from test_cache_isa import CSRC, HIPCC, ROOT, _blocks, _regs

needs_hipcc = pytest.mark.skipif(not shutil.which(HIPCC) and not os.path.exists(HIPCC), reason="hipcc not available")
PRODUCTS = {"v_mfma_f32_16x16x32": 8, "v_mfma_f32_32x32x16": 12}

PROBE = """
#include <hip/hip_runtime.h>
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
#define A16(a, b, c) __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0)
#define A32(a, b, c) __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0)
extern "C" __global__ void vector_16(const v8bf* a, v4f* o) { o[threadIdx.x] = A16(a[0], a[1], o[0]) * 3.0f; }
extern "C" __global__ void vector_32(const v8bf* a, v16f* o) { o[threadIdx.x] = A32(a[0], a[1], o[0]) * 3.0f; }
extern "C" __global__ void operand_16(const v8bf* a, v4f* o) {
  const v4f r = A16(a[0], a[1], o[0]);
  o[threadIdx.x] = A16(__builtin_bit_cast(v8bf, r), a[2], o[0]);
}
extern "C" __global__ void operand_32(const v8bf* a, v16f* o) {
  const v16f r = A32(a[0], a[1], o[0]);
  const v4f q = {r[0], r[1], r[2], r[3]};
  o[threadIdx.x] = A32(a[2], __builtin_bit_cast(v8bf, q), o[0]);
}
"""


def _kernels(src, out):
    cmd = [HIPCC, "-O3", "-std=c++17", "--offload-arch=gfx950", "-ffp-contract=off", "-Xclang", "-target-feature",
           "-Xclang", "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"), "--cuda-device-only", "-S", "-x", "hip",
           str(src), "-o", str(out)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    kernels, body = {}, None
    for ln in out.read_text().splitlines():
        m = re.match(r"([A-Za-z_]\S*):\s", ln + " ")
        if m:
            body = kernels.setdefault(m.group(1), [])
        elif ln.startswith(".Lfunc_end"):
            body = None
        elif body is not None:
            body.append(ln)
    return {k: v for k, v in kernels.items() if any("mfma" in x for x in v)}


def _uses(t, regs):
    """Whether instruction t needs the finished result in regs: any register of another instruction, the first two
    operands of a product, an accumulator that overlaps it without being it."""
    if t.startswith("s_"):
        return False
    if "mfma" not in t:
        return bool(_regs(t) & regs)
    dst, a, b, c = [_regs(x) for x in t.split(None, 1)[1].split(",")[:4]]
    return bool((a | b) & regs) or (c != regs and (bool(c & regs) or (bool(dst & regs) and dst != regs)))


def _takes_over(t, regs):
    """The next product of a chain (its sum may go to other registers, which is in order), or a new result."""
    if "mfma" not in t:
        return False
    dst, _, _, c = [_regs(x) for x in t.split(None, 1)[1].split(",")[:4]]
    return c == regs or dst == regs


def _nearest(blocks, succ, name, at, regs, need):
    """Wait states to the nearest use on any path from behind instruction `at`, None from `need` on."""
    best, seen, todo = None, {}, [(name, at + 1, 0)]
    while todo:
        n, i, d = todo.pop()
        if d >= need or seen.get((n, i), need) <= d:
            continue
        seen[(n, i)] = d
        while d < need:
            if i >= len(blocks[n]):
                if succ[n][1]:
                    todo.append((succ[n][1], 0, d))
                break
            t = blocks[n][i]
            if t.startswith("s_endpgm"):
                break
            if _uses(t, regs):
                best = d if best is None else min(best, d)
                break
            if _takes_over(t, regs):
                break
            d += int(t.split()[1], 0) + 1 if t.startswith("s_nop") else 1
            if t.startswith(("s_branch", "s_cbranch")):
                todo.append((t.split()[-1], 0, d))
                if t.startswith("s_branch"):
                    break
            i += 1
    return best


def _too_near(body, products=PRODUCTS):
    blocks, succ = _blocks(body)
    found = []
    for n, ins in blocks.items():
        for i, t in enumerate(ins):
            for k, need in products.items():
                if t.startswith(k):
                    d = _nearest(blocks, succ, n, i, _regs(t.split(",")[0]), need)
                    if d is not None:
                        found.append((n, t, d))
    return found


@needs_hipcc
def test_the_distances_are_those_of_code_without_branches(tmp_path):
    src = tmp_path / "probe.hip"
    src.write_text(PROBE)
    far = {k: 64 for k in PRODUCTS}
    kernels = _kernels(src, tmp_path / "probe.s")
    assert len(kernels) == 4
    for name, body in kernels.items():
        # the first product (of an operand probe the one that the second reads)
        d = _too_near(body, far)[0][2]
        need = PRODUCTS["v_mfma_f32_16x16x32" if name.endswith("16") else "v_mfma_f32_32x32x16"]
        assert d == need if name.startswith("vector") else d >= need, (name, d)


P16 = "\tv_mfma_f32_16x16x32_bf16 v[2:5], v[6:9], v[10:13], 0"
P32 = "\tv_mfma_f32_32x32x16_bf16 v[16:31], v[6:9], v[10:13], 0"
USE = {"vector": "\tv_mul_f32_e32 v0, v1, v{0}", "store": "\tglobal_store_dword v0, v{0}, s[0:1]",
       "first operand": "\tv_mfma_f32_16x16x32_bf16 v[40:43], v[{0}:{1}], v[10:13], 0",
       "second operand": "\tv_mfma_f32_16x16x32_bf16 v[40:43], v[10:13], v[{0}:{1}], 0",
       "part of an accumulator": "\tv_mfma_f32_16x16x32_bf16 v[{1}:{2}], v[10:13], v[6:9], v[{1}:{2}]"}


@pytest.mark.parametrize("product,first,need", [(P16, 2, 8), (P32, 16, 12)])
@pytest.mark.parametrize("use", USE)
def test_the_walk_finds_uses_one_wait_state_too_near(product, first, need, use):
    use = USE[use].format(first, first + 3, first + 6)
    for behind, near in ((need, False), (need - 1, True)):
        straight = [product, f"\ts_nop {behind - 1}", use]
        skip = [product, f"\ts_nop {behind - 2}", "\ts_cbranch_vccnz .LBB0_2", *["\tv_mov_b32_e32 v50, v51"] * 12,
                ".LBB0_2:", use]
        loop = [".LBB0_1:", use, *["\tv_mov_b32_e32 v50, v51"] * 12, product, f"\ts_nop {behind - 2}",
                "\ts_cbranch_scc1 .LBB0_1", "\ts_endpgm"]
        for body in (straight, skip, loop):
            assert bool(_too_near(body)) == near, (behind, body)


def test_the_walk_takes_a_chain_as_one():
    chain = [P16, "\tv_mfma_f32_16x16x32_bf16 v[2:5], v[6:9], v[10:13], v[2:5]", "\ts_nop 7", "\tv_mul_f32_e32 v0, v1, v3"]
    assert not _too_near(chain)
    assert _too_near(chain[:2] + ["\ts_nop 6"] + chain[3:])
    moved = [P16, "\tv_mfma_f32_16x16x32_bf16 v[4:7], v[6:9], v[10:13], v[2:5]", "\ts_nop 7", "\tv_mul_f32_e32 v0, v1, v5"]
    assert not _too_near(moved)
    assert _too_near(moved[:2] + ["\ts_nop 6"] + moved[3:])


@needs_hipcc
def test_no_product_of_the_cache_kernels_is_used_too_early(tmp_path):
    bad = {k: _too_near(v)[:3] for k, v in _kernels(os.path.join(CSRC, "ra_cache_attn.hip"), tmp_path / "k.s").items()}
    assert sum("k_few" in k for k in bad) and sum("k_rows" in k for k in bad)
    bad = {k: v for k, v in bad.items() if v}
    assert not bad, f"products used too early: {bad}"
