"""The wait states of test_cache_isa and test_cache_isa_waits in the kernels of cache_attn_sinks and cache_attn_shared
(CPU only)."""
import os

import pytest

from test_cache_isa import CSRC, _violations
from test_cache_isa_waits import _kernels, _too_near, needs_hipcc


@needs_hipcc
@pytest.mark.parametrize("name,kinds", [("ra_cache_sinks.hip", {"k_few": 4, "k_fine_few": 4, "k_rows": 8, "k_fine_rows": 4}),
                                        ("ra_cache_shared.hip", {"k_few": 2, "k_fine_few": 2, "k_both": 12})])
def test_no_product_is_used_too_early(tmp_path, name, kinds):
    kernels = _kernels(os.path.join(CSRC, name), tmp_path / "k.s")
    for kind, n in kinds.items():
        assert sum(f"{len(kind)}{kind}I" in k for k in kernels) == n, kind
    bad = {k: (_violations(v) + _too_near(v))[:3] for k, v in kernels.items()}
    bad = {k: v for k, v in bad.items() if v}
    assert not bad, f"products used too early: {bad}"
