"""What is rounded to bf16 on its way out of the norm and its gradient: every upper half of an fp32 number with the
lower halves next to a tie, NaNs of all payloads among them, against the rounding that torch has."""
import pytest
import torch

from paper_2607_20652_amd import binding as dpb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dpb.load()


def numbers():
    upper = torch.arange(1 << 16, dtype=torch.int64)[:, None] << 16
    lower = torch.tensor([0, 1, 0x7FFF, 0x8000, 0x8001, 0xC000, 0xFFFE, 0xFFFF])
    return (upper | lower).flatten().to(torch.int32).view(torch.float32)     # (the last ones are NaNs of all bits)


def same(got, x):
    """The nearest bf16 numbers, NaN for NaN.  What is under 2^-126 may have become 0."""
    got, want = got.detach().cpu().float().flatten(), x.cpu().bfloat16().float().flatten()
    assert torch.equal(got.isnan(), x.cpu().isnan().flatten())
    bad = ~(got.isnan() | (got == want) | ((got - want).abs() <= 2.0 ** -126))
    assert not bad.any(), (x.cpu().flatten()[bad][:4], got[bad][:4])


@pytest.mark.parametrize("dim", [512, 4096, 1 << 19])
def test_an_fp32_call_s_gradient_of_a_bf16_weight(dim):
    """A single row of ones: the weight's gradient is the row's."""
    w, ones, rstd = torch.ones(dim, device=DEV, dtype=torch.bfloat16), torch.ones(1, dim, device=DEV), torch.ones(1, device=DEV)
    for g in numbers().to(DEV).split(dim)[::max(1, 8192 // dim)]:
        same(dpb.rms_norm_bwd(g[None], ones, w, rstd)[1], g)
    g = numbers().to(DEV)[-dim:]
    same(dpb.rms_norm_bwd(g[None], ones, w, rstd)[1], g)


@pytest.mark.parametrize("offset", [0, 1], ids=["", "by elements"])
@pytest.mark.parametrize("dim", [512, 4096, 16384, 32768])
def test_a_bf16_norm_with_an_fp32_weight(dim, offset):
    """A single row of ones, whose mean square is 1 for widths of a power of two: the norm is the weight."""
    x = torch.ones(1, dim + offset, device=DEV, dtype=torch.bfloat16)[:, offset:]
    for w in (numbers().to(DEV)[:dim], numbers().to(DEV)[-dim:], numbers().to(DEV)[3 << 16:][:dim]):
        same(dpb.rms_norm(x, w.clone(), eps=0.0)[0], w)


@pytest.mark.parametrize("dim", [4096, 8192])
def test_a_gradient_of_rows_whose_rstd_is_nan(dim):
    """An rstd of all bits set, as memory that was never written may have: the row's gradient is NaN, by chunks and by elements."""
    rstd = torch.full((2,), -1, dtype=torch.int32, device=DEV).view(torch.float32)
    rstd[1] = 1.0
    for offset in (0, 1):
        g = torch.ones(2, dim + offset, device=DEV, dtype=torch.bfloat16)[:, offset:]
        dx, _ = dpb.rms_norm_bwd(g, g, None, rstd)
        assert dx[0].isnan().all() and torch.isfinite(dx[1]).all()
