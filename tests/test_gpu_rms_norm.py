"""RMS norm with the residual's addition, and its gradients, against fp64."""
import pytest
import torch

import around_util as R
from paper_2607_20652_amd import binding as dpb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dpb.load()


def draw(rows, dim, dtype, seed=0):
    g = torch.Generator().manual_seed(seed + rows * 31 + dim)
    x, r, go, gt = (torch.randn(rows, dim, generator=g).to(DEV, dtype) for _ in range(4))
    return x, r, go, gt, (torch.randn(dim, generator=g) * 0.2 + 1).to(DEV)


# every form of the kernels: a wave and a workgroup a row, one and several elements a lane, rows read twice
SIZES = [(1, 1), (3, 7), (1, 64), (5, 511), (130, 512), (17, 500), (1000, 768), (33, 501), (9, 1024), (2, 1032), (40, 2048), (6, 2056),
         (5, 4096), (3, 4100), (7, 8192), (2, 8200), (4, 16384), (3, 16392), (2, 20001), (9000, 72)]


@TYPES
@pytest.mark.parametrize("rows,dim", SIZES)
@pytest.mark.parametrize("residual", [False, True], ids=["", "residual"])
def test_norm_and_gradients(rows, dim, residual, dtype):
    x, r, go, gt, w = draw(rows, dim, dtype)
    w = w.to(dtype)
    out, total, rstd = dpb.rms_norm(x, w, r if residual else None, eps=1e-5)
    if residual:
        want = x.double() + r.double()
        R.check("total", total, want, R.U[dtype] * want.abs())
    else:
        assert total is x
    want_out, want_rstd = R.rms_norm(total, w, 1e-5)
    R.check("out", out, *want_out)
    R.check("rstd", rstd, *want_rstd)
    for grad_total in (None, gt):
        dx, dw = dpb.rms_norm_bwd(go, total, w, rstd, grad_total)
        want_dx, want_dw = R.rms_norm_bwd(go, total, w, rstd, grad_total)
        R.check("dx", dx, *want_dx)
        R.check("dweight", dw, *want_dw)
        again = dpb.rms_norm_bwd(go, total, w, rstd, grad_total)
        assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])


@TYPES
def test_weights_of_another_type_and_none(dtype):
    x, r, go, gt, w = draw(50, 96, dtype)
    for weight in (w.float(), w.bfloat16(), None):
        out, total, rstd = dpb.rms_norm(x, weight, r)
        R.check("out", out, *R.rms_norm(total, weight, 1e-6)[0])
        dx, dw = dpb.rms_norm_bwd(go, total, weight, rstd, gt)
        want_dx, want_dw = R.rms_norm_bwd(go, total, weight, rstd, gt)
        R.check("dx", dx, *want_dx)
        if weight is None:
            assert dw is None
        else:
            assert dw.dtype == weight.dtype
            R.check("dweight", dw, *want_dw)


@TYPES
@pytest.mark.parametrize("dim,step,offset", [(64, 8, 0), (64, 0, 8), (64, 3, 1), (512, 1, 0), (5000, 7, 0), (2048, 8, 8)])
def test_rows_that_start_anywhere(dim, step, offset, dtype):
    torch.manual_seed(1)
    cut = lambda: torch.randn(6, 5, dim + step + offset, device=DEV).to(dtype)[..., offset:offset + dim]  # noqa: E731
    x, r, go, gt = cut(), cut(), cut(), cut()
    w = torch.rand(dim + 1, device=DEV).to(dtype)[1:]      # a weight that starts off 16 bytes
    whole = [t.contiguous() for t in (x, r, go, gt)]
    got, want = dpb.rms_norm(x, w, r), dpb.rms_norm(whole[0], w.clone(), whole[1])
    # (another number of lanes may share a row: the sums' order differs)
    for a, b in zip(got, want):
        assert torch.allclose(a.float(), b.float(), rtol=2.0 ** -7 if dtype == torch.bfloat16 else 1e-5, atol=0)
    assert torch.equal(got[1], want[1])
    dx, dw = dpb.rms_norm_bwd(go, got[1], w, got[2], gt)
    want_dx, want_dw = R.rms_norm_bwd(whole[2], got[1], w, got[2], whole[3])
    R.check("dx", dx, *want_dx)
    R.check("dweight", dw, *want_dw)


@TYPES
@pytest.mark.parametrize("dim", [64, 501, 2048, 8192, 20000])
def test_in_place(dim, dtype):
    x, r, go, gt, w = draw(20, dim, dtype)
    want = dpb.rms_norm(x, w, r)
    z, y = r.clone(), x.clone()
    got = dpb.rms_norm(y, w, z, out=y, total=z)            # the decode loop's form: nothing new but rstd
    assert got[0] is y and got[1] is z and all(torch.equal(a, b) for a, b in zip(got, want))
    z, y = r.clone(), x.clone()
    got = dpb.rms_norm(y, w, z, out=z, total=y)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    wanted = dpb.rms_norm_bwd(go, want[1], w, want[2], gt)
    for place in (0, 1):
        grads = [go.clone(), gt.clone()]
        got = dpb.rms_norm_bwd(grads[0], want[1], w, want[2], grads[1], dx=grads[place])
        assert got[0] is grads[place] and all(torch.equal(a, b) for a, b in zip(got, wanted))


def test_rows_of_zeros_and_what_is_not_finite():
    x = torch.randn(5, 256, device=DEV)
    x[1] = 0
    x[2, 7] = float("nan")
    x[3, 9] = float("inf")
    w = torch.ones(256, device=DEV)
    out, _, rstd = dpb.rms_norm(x, w, eps=1e-6)
    assert not out[1].any() and abs(float(rstd[1]) - 1e3) < 1e-3 * 4
    assert out[2].isnan().all() and out[3, 9].isnan() and not out[3, :9].any()
    assert torch.isfinite(out[[0, 4]]).all()
    assert dpb.rms_norm(torch.zeros(1, 8, device=DEV), None, eps=0.0)[0].isnan().all()
    assert dpb.rms_norm(torch.zeros(0, 8, device=DEV), None)[0].shape == (0, 8)
    dx, dw = dpb.rms_norm_bwd(torch.zeros(0, 8, device=DEV), torch.zeros(0, 8, device=DEV), w[:8].clone(),
                              torch.zeros(0, device=DEV))
    assert dx.shape == (0, 8) and not dw.any()
    one = torch.randn(64, device=DEV)                       # a single row without a dimension for rows
    out, _, rstd = dpb.rms_norm(one, w[:64].clone())
    assert out.shape == (64,) and rstd.shape == ()
    R.check("out", out, *R.rms_norm(one, w[:64], 1e-6)[0])


def test_gradients_against_differences():
    """Central differences of step h in fp64 on the CPU from the kernel's own formula's values: the kernel's gradient
    against how its outputs change. Outputs are fp32: their rounding (2^-24 of values up to 4, 64 terms) over h."""
    torch.manual_seed(3)
    x, w, g = torch.randn(2, 32, device=DEV), torch.rand(32, device=DEV) + 0.5, torch.randn(2, 32, device=DEV)
    out, total, rstd = dpb.rms_norm(x, w)
    dx, dw = dpb.rms_norm_bwd(g, total, w, rstd)
    h = 2.0 ** -7
    f = lambda x, w: float((dpb.rms_norm(x, w)[0].double() * g.double()).sum())  # noqa: E731
    noise = 64 * 4 * 4 * 2.0 ** -24 / h + 20 * h * h
    for i in (0, 13, 31):
        d = torch.zeros_like(x)
        d[1, i] = h
        assert abs((f(x + d, w) - f(x - d, w)) / (2 * h) - float(dx[1, i])) < noise
        assert abs((f(x, w + d[1]) - f(x, w - d[1])) / (2 * h) - float(dw[i])) < noise
