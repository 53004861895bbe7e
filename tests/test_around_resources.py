"""Register budgets of the kernels of embedding, norm and vocabulary loss, as the other kernels'."""
import re

import pytest

from test_kernel_resources import kernels  # noqa: F401  (a fixture)

BUDGETS = [
    # (kernel, vector registers): waves per SIMD of the products by their tiles' edge: one, two, four
    (r"loss_(part|grad|out)_kernelI.*Li256E", 512),
    (r"loss_(part|grad|out)_kernelI.*Li128E", 256),
    (r"loss_(part|grad|out)_kernelI.*Li64E", 128),
    (r"embed_order_kernel", 128),
    (r"embed_(bin|join)_kernel", 80),
    (r"embed_sum_kernel", 96),
    (r"11norm_kernelI.*Li64ELi[124]E", 128),
    (r"15norm_bwd_kernelI.*Li64ELi[124]E", 256),
]


@pytest.mark.parametrize("pattern,most", BUDGETS)
def test_register_budget(kernels, pattern, most):  # noqa: F811
    found = {k: v["vgpr_count"] for k, v in kernels.items() if re.search(pattern, k)}
    assert found, f"no kernel matches {pattern}"
    over = {k: v for k, v in found.items() if v > most}
    assert not over, over
