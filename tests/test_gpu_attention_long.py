"""As many keys as 32 bits count, all of them one row in memory: every query's place among
them passes 2^31 on the way."""
import math

import pytest
import torch

from paper_2607_20652_amd import binding as dpb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def test_the_last_queries_of_the_longest_sequence_see_their_keys():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    n, rows, D = 2 ** 31 - 256, 300, 8
    q = torch.zeros(1, rows, 1, D, dtype=torch.bfloat16, device=DEV)
    q[0, :, 0, 0] = 0.5
    k = torch.ones(1, 1, 1, D, dtype=torch.bfloat16, device=DEV).expand(1, n, 1, D)
    out, lse = dpb.attention(q, k, k, True, 1.0)
    seen = torch.arange(n - rows + 1, n + 1, dtype=torch.float64)
    # every weight is the same and every value 1: the sums are whole numbers of 2^31 / 408 at most in each wave's
    # part, exact in fp32, and joined with a rounding each
    assert bool(((out.double().cpu() - 1).abs() <= 2.0 ** -8).all())
    assert bool(((lse[0, :, 0].double().cpu() - (0.5 + seen.log())).abs() < 1e-5 + 22 * 2.0 ** -22).all())
    assert math.isfinite(float(lse.sum()))
