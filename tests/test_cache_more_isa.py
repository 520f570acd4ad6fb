"""The wait states of test_cache_isa and test_cache_isa_waits in the kernels of cache_attn_sinks and cache_attn_shared
(CPU only)."""
import os

import pytest

from test_cache_isa import CSRC, _violations
from test_cache_isa_waits import _kernels, _too_near, needs_hipcc
from test_isa_hazards import CONV, _violations as _conversions

# products of 4-bit keys and 6-bit queries: 8 passes, as 32x32x16 (the scaled form is two instruction words)
SMALL = {"v_mfma_f32_32x32x64_f8f6f4": 12, "v_mfma_scale_f32_32x32x64_f8f6f4": 12}


def _packed_too_near(body):
    """Conversions to 6 bits whose next instruction but one is a product that reads the result."""
    text = [t for t in (ln.split(";")[0].strip() for ln in body) if t and not t.endswith(":") and not t.startswith(".")]
    bad = []
    for i, t in enumerate(text):
        if t.startswith(CONV):
            first = t.split(None, 1)[1].split(",")[0]
            bad += [(t, u) for u in text[i + 1:i + 2] if "mfma" in u and first in u]
    return bad


@needs_hipcc
@pytest.mark.parametrize("name,kinds", [("ra_cache_sinks.hip", {"k_few": 4, "k_fine_few": 4, "k_rows": 8, "k_fine_rows": 4, "k_both": 12}),
                                        ("ra_cache_shared.hip", {"k_few": 2, "k_fine_few": 2, "k_both": 12})])
def test_no_product_is_used_too_early(tmp_path, name, kinds):
    kernels = _kernels(os.path.join(CSRC, name), tmp_path / "k.s")
    for kind, n in kinds.items():
        assert sum(f"{len(kind)}{kind}I" in k for k in kernels) == n, kind
    small = {k: sum(x.strip().startswith(tuple(SMALL)) for x in v) for k, v in kernels.items()}
    assert all(n == 0 if "k_few" in k or "k_fine_few" in k else n >= 20 for k, n in small.items()), small
    bad = {k: (_violations(v) + _too_near(v) + _too_near(v, SMALL) + _packed_too_near(v) + _conversions([x.strip() for x in v]))[:3]
           for k, v in kernels.items()}
    bad = {k: v for k, v in bad.items() if v}
    assert not bad, f"products used too early: {bad}"
