"""Queries with channels far larger than the rest where the keys are 0: scores come from the small channels alone, and
lse has to be as exact as binary32 arithmetic there (cache_attn_sinks, cache_attn_shared)."""
import numpy as np
import pytest

import cache_ref as ref
from cache_case import Case

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ra():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_02584_amd import rotate_attn as m
    m.lib()
    return m


def _blank(c, channels):
    """K's codes of these channels are 0 in every page and head."""
    p = c.p
    heads = c.cache.reshape(p.num_pages, p.Hkv, -1)
    for d in channels:
        at = ref.k_byte(p.D, np.arange(p.page_size), d)
        heads[:, :, at] &= 0x0F if d % 2 else 0xF0


@pytest.mark.parametrize("dt,out", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "fp32")])
@pytest.mark.parametrize("D,Hq,Hkv", [(128, 8, 2), (64, 6, 1)])
@pytest.mark.parametrize("times", [10, 100, 1000, 10000])
@pytest.mark.parametrize("kind", ["few", "many", "large"])
def test_large_channels_that_no_key_has(ra, dt, out, D, Hq, Hkv, times, kind):
    """Rows of few-row and of many-row requests, of few and of many queries."""
    qs = {"few": [1, 3], "many": [1, 40], "large": [150, 2]}[kind]
    times = min(times, 1000) if dt == "fp16" else times
    for rope in (False, True):
        for kw in (dict(window=90, sinks=20), dict(groups=[(0, 2, 120)])):
            c = Case(ra, Hq, Hkv, D, 32, [300, 160], qs, dt, out, rope=rope, seed=times + D, gain=2.0, **kw)
            large = (6, 7) if rope else (7,)      # a pair that RoPE turns
            _blank(c, large)
            c.q[:, :, list(large)] *= times
            c.run()
            c.check_lse()


@pytest.mark.parametrize("D", [128, 64])
def test_half_of_the_channels_large(ra, D):
    for kw in (dict(window=90, sinks=20), dict(groups=[(0, 2, 120)])):
        c = Case(ra, 4, 1, D, 16, [300, 160], [30, 20], seed=D, gain=2.0, **kw)
        _blank(c, range(0, D, 2))
        c.q[:, :, 0::2] *= 3000
        c.run()
        c.check_lse()


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("times", [1, 30, 1000])
def test_large_channels_in_a_rotated_cache(ra, D, times):
    """The rotation spreads them over the row; binary32's own rotation then rounds at their size."""
    for kw in (dict(window=90, sinks=20), dict(groups=[(0, 2, 120)])):
        c = Case(ra, 4, 1, D, 16, [300, 160], [30, 1], rope=True, had=True, seed=D, gain=2.0, **kw)
        c.q[:, :, 8:10] *= times
        c.run()
        c.check_lse()
