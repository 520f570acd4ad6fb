"""Static checks of the machine code of the paged KV cache's kernels (CPU only).

A matrix product's result may be used by other instructions only some wait
states after it was issued.  The compiler counts them, but where a branch
skips a block between a product and a use, it has been seen to count along the
longer path alone: the use then read the first result register too early, and
the scores of every fourth key were wrong.  This test walks all paths from
every product to the first other instruction that names one of its result
registers and demands a distance of at least the product's passes.
"""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_02584_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# wait states that a use needs: 4-pass and 8-pass products
NEED = {"v_mfma_f32_16x16x32": 6, "v_mfma_f32_32x32x16": 10}


def _regs(text):
    out = set()
    for a, b in re.findall(r"\bv\[(\d+):(\d+)\]", text):
        out.update(range(int(a), int(b) + 1))
    out.update(int(a) for a in re.findall(r"\bv(\d+)\b", text))
    return out


def _blocks(body):
    """Instructions by block and the blocks' successors."""
    blocks, order, name = {"entry": []}, ["entry"], "entry"
    for ln in body:
        m = re.match(r"(\.L\w+):", ln)
        if m:
            name = m.group(1)
            blocks[name] = []
            order.append(name)
            continue
        t = ln.split(";")[0].strip()
        if ln[:1].isspace() and re.match(r"[a-z]", t):
            blocks[name].append(t)
    succ = {}
    for i, n in enumerate(order):
        nxt = order[i + 1] if i + 1 < len(order) else None
        parts, cur, ends = [], [], False
        for t in blocks[n]:
            cur.append(t)
            if t.startswith(("s_branch", "s_cbranch")):
                parts.append((cur, t.split()[-1]))
                cur = []
                ends = t.startswith("s_branch")
            elif t.startswith("s_endpgm"):
                ends = True
        # leave at any branch, or fall through at the end
        succ[n] = (parts, None if ends and not cur else nxt)
    return blocks, succ


def _paths_end(blocks, succ, name, at, regs, need):
    """Shortest distance from behind instruction `at` to a use of regs, cut at need; None if none so near."""
    best, seen, todo = None, {}, [(name, at + 1, 0)]
    while todo:
        n, i, d = todo.pop()
        if d >= need or seen.get((n, i), need) <= d:
            continue
        seen[(n, i)] = d
        ins = blocks[n]
        while i < len(ins) and d < need:
            t = ins[i]
            if t.startswith("s_nop"):
                d += int(t.split()[1]) + 1
            elif t.startswith(("s_branch", "s_cbranch")):
                d += 1
                todo.append((t.split()[-1], 0, d))
                if t.startswith("s_branch"):
                    break
            elif t.startswith("s_endpgm"):
                break
            elif "mfma" not in t and not t.startswith("s_") and _regs(t) & regs:
                best = d if best is None else min(best, d)
                break
            elif "mfma" in t and _regs(t.split(",")[0]) & regs:
                break            # the next product of a chain takes over
            else:
                d += 1
            i += 1
        else:
            nxt = succ[n][1]
            if d < need and nxt and i >= len(ins):
                todo.append((nxt, 0, d))
    return best


def _violations(body):
    blocks, succ = _blocks(body)
    bad = []
    for n, ins in blocks.items():
        for i, t in enumerate(ins):
            for k, need in NEED.items():
                if t.startswith(k):
                    d = _paths_end(blocks, succ, n, i, _regs(t.split(",")[0]), need)
                    if d is not None:
                        bad.append((n, t, d))
    return bad


def test_the_walk_finds_a_use_behind_a_skipped_block():
    product = "\tv_mfma_f32_16x16x32_bf16 v[2:5], v[6:9], v[10:13], 0"
    skip = [product, "\ts_cbranch_vccnz .LBB0_2", *["\tv_mov_b32_e32 v20, v21"] * 12, ".LBB0_2:",
            "\tv_mul_f32_e32 v30, v31, v2"]
    assert _violations(skip)
    waits = [product, "\ts_nop 7", "\ts_cbranch_vccnz .LBB0_2", "\ts_nop 0", ".LBB0_2:", "\tv_mul_f32_e32 v30, v31, v2"]
    assert not _violations(waits)
    chain = [product, "\tv_mfma_f32_16x16x32_bf16 v[2:5], v[6:9], v[10:13], v[2:5]", "\ts_nop 7", "\tv_mul_f32_e32 v0, v1, v3"]
    assert not _violations(chain)


@pytest.mark.skipif(not shutil.which(HIPCC) and not os.path.exists(HIPCC), reason="hipcc not available")
def test_no_product_is_used_too_early(tmp_path):
    out = tmp_path / "k.s"
    cmd = [HIPCC, "-O3", "-std=c++17", "--offload-arch=gfx950", "-ffp-contract=off", "-Xclang", "-target-feature",
           "-Xclang", "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"), "--cuda-device-only", "-S", "-x", "hip",
           os.path.join(CSRC, "ra_cache_attn.hip"), "-o", str(out)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    kernels, body = {}, None
    for ln in out.read_text().splitlines():
        m = re.match(r"(_Z\S+):", ln)
        if m:
            body = kernels.setdefault(m.group(1), [])
        elif ln.startswith(".Lfunc_end"):
            body = None
        elif body is not None:
            body.append(ln)
    kernels = {k: v for k, v in kernels.items() if any("mfma" in x for x in v)}
    assert sum("k_few" in k for k in kernels) == 4 and sum("k_rows" in k for k in kernels) == 8
    bad = {k: _violations(v)[:3] for k, v in kernels.items()}
    bad = {k: v for k, v in bad.items() if v}
    assert not bad, f"products used too early: {bad}"
