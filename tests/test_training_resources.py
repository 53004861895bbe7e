"""Register budgets of the attention and optimizer kernels, as the other kernels'."""
import re

import pytest

from test_kernel_resources import kernels  # noqa: F401  (a fixture)

BUDGETS = [
    # (kernel, vector registers): four, three and two waves per SIMD
    (r"16attention_kernelIDF16bLi(32|64)E", 128),
    (r"16attention_kernelIDF16bLi(96|128)E", 256),
    (r"attention_dq_kernelIDF16bLi64E", 168),
    (r"attention_d(q|kv)_kernelIDF16bLi", 256),
    (r"attention_split_kernelIDF16bLi", 256),
    (r"adamw_kernel", 80),
]


@pytest.mark.parametrize("pattern,most", BUDGETS)
def test_register_budget(kernels, pattern, most):  # noqa: F811
    found = {k: v["vgpr_count"] for k, v in kernels.items() if re.search(pattern, k)}
    assert found, f"no kernel matches {pattern}"
    over = {k: v for k, v in found.items() if v > most}
    assert not over, over
