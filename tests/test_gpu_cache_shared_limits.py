"""Prefix lengths that no request has: what is defined of such a call's outputs, and its tensors' neighbours."""
import numpy as np
import pytest

from cache_case import Case, i32

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ra():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_02584_amd import rotate_attn as m
    m.lib()
    return m


@pytest.mark.parametrize("out", ["bf16", "fp32"])
@pytest.mark.parametrize("queries", [1, 20])
@pytest.mark.parametrize("long,low", [(2 ** 31 - 1, -2 ** 31), (1 << 30, -1), (1000, 0), (151, -64)])
def test_impossible_prefixes(ra, long, low, queries, out):
    """A negative prefix shares nothing.  One longer than the group's first request is cut to what this holds, so that the
    first request has its own outputs; the others hold other tokens there, and something finite.  A third group is as it
    should be."""
    groups = [(0, 6, 150), (6, 11, 90), (11, 14, 70)]
    lens = [150 + queries - 1 + 3 * i for i in range(6)] + [90 + queries + 5 * i for i in range(5)] + [70 + queries + i for i in range(3)]
    c = Case(ra, 4, 2, 128, 16, lens, [queries] * 14, groups=groups, rope=True, had=True, out=out, seed=queries, pad=3)
    G, T = 3, c.T
    size = ra.cache_shared_workspace(c.p, 14, G, T).numel()
    ws = torch.full((size + 4096,), 0x33, dtype=torch.uint8, device="cuda")
    o = torch.full((T + 64, 4, 128), 7.0, dtype=c.o.dtype, device="cuda")
    lse = torch.full((T + 64, 4), 7.0, device="cuda")
    # places behind the ends of the cache's requests are NaN: something finite needs finite ones
    c.scales()[:] = np.where(np.isnan(c.scales()), np.float32(0.5), c.scales())
    ra.cache_attn_shared(c.p, c.q, torch.from_numpy(c.cache).cuda(), i32(c.table), i32(c.start), i32(c.lens), c.positions,
                         i32([0, 6, 11, 14]), i32([long, low, 70]), o[32:32 + T], ws[2048:2048 + size], lse=lse[32:32 + T],
                         rope=c.rope())
    torch.cuda.synchronize()
    want = c.want()
    for a, b in ((0, queries), (6 * queries, 14 * queries)):
        c.check(False, got=(o[32 + a:32 + b], lse[32 + a:32 + b]), want=[x[a:b] for x in want])
    live = 14 * queries
    assert torch.isfinite(o[32:32 + live]).all() and torch.isfinite(lse[32:32 + live]).all()
    for t in (o, lse):
        assert (t[:32] == 7.0).all() and (t[32 + live:] == 7.0).all()
    assert (ws[:2048] == 0x33).all() and (ws[2048 + size:] == 0x33).all()


@pytest.mark.parametrize("Hq,Hkv,had", [(8, 2, True), (6, 6, False)])
def test_prompts_behind_a_prefix(ra, Hq, Hkv, had):
    """Hundreds to thousands of new tokens a request behind a cached prefix, beside requests that decode: what cache_attn
    gives, both within 2^-18 of 64-bit results with binary32 outputs."""
    qs = [2000, 1, 700, 3300, 1, 0, 513]
    lens = [3000 + 1 + 7 * i + q for i, q in enumerate(qs)]
    c = Case(ra, Hq, Hkv, 128, 64, lens, qs, out="fp32", rope=True, had=had, groups=[(0, 5, 3000), (5, 7, 3000)], seed=9, pad=30)
    x, lse = (t.clone() for t in c.run())
    c.groups = []
    y, lse2 = c.run()
    assert (x - y).abs().max() <= 2.0 ** -17 * y.abs().max() and (lse - lse2).abs().max() <= 2.0 ** -17
