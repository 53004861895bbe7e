"""Softmax cross entropy over a vocabulary, and its gradients, against fp64."""
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


def draw(rows, dim, vocab, dtype, learnt=3.0):
    g = torch.Generator().manual_seed(rows * 7 + dim * 3 + vocab)
    w = (torch.randn(vocab, dim, generator=g) * 1.5 / dim ** 0.5).to(DEV, dtype)
    t = torch.randint(-1, vocab + 1, (rows,), generator=g).to(DEV)
    at = t.clamp(0, vocab - 1)
    h = torch.randn(rows, dim, generator=g).to(DEV) + torch.rand(rows, 1, generator=g).to(DEV) * learnt * w[at].float()
    ga, ge = ((torch.rand(rows, generator=g) - 0.2).to(DEV) for _ in range(2))
    return h.to(dtype), w, t, ga, ge * 0.1


SIZES = [  # rows, dim, vocab
    (1, 8, 1), (1, 64, 24), (2, 1, 5), (65, 64, 1000), (24, 100, 333), (33, 1024, 4099), (300, 200, 1003), (257, 72, 2000),
    (130, 1, 3000), (64, 129, 64), (63, 200, 65), (128, 64, 256), (255, 320, 257), (512, 256, 512), (1023, 96, 517), (700, 768, 3001),
    (2050, 520, 1500), (4100, 64, 200), (40, 64, 40000), (1500, 1000, 5000),
]


@TYPES
@pytest.mark.parametrize("rows,dim,vocab", SIZES)
def test_loss_and_gradients(rows, dim, vocab, dtype):
    h, w, t, ga, ge = draw(rows, dim, vocab, dtype)
    scale = 0.7
    loss, lse = dpb.cross_entropy(h, w, t, scale)
    want_loss, want_lse, _ = R.cross_entropy(h, w, t, scale)
    R.check("loss", loss, *want_loss)
    R.check("lse", lse, *want_lse)
    for a, e in ((ga, None), (ga, ge), (None, ge)):
        dh, dw = dpb.cross_entropy_bwd(a, h, w, t, lse, scale, grad_lse=e)
        want_dh, want_dw = R.cross_entropy_bwd(a, h, w, t, lse, scale, e)
        R.check("dhidden", dh, *want_dh)
        R.check("dweight", dw, *want_dw)
    again = dpb.cross_entropy_bwd(None, h, w, t.int(), lse, scale, grad_lse=ge)
    assert torch.equal(dh, again[0]) and torch.equal(dw, again[1])
    assert all(torch.equal(x, y) for x, y in zip((loss, lse), dpb.cross_entropy(h, w, t.int(), scale)))
    only = dpb.cross_entropy_bwd(None, h, w, t, lse, scale, grad_lse=ge, weight_grad=False)
    assert only[1] is None and torch.equal(only[0], dh)
    only = dpb.cross_entropy_bwd(None, h, w, t, lse, scale, grad_lse=ge, hidden_grad=False)
    assert only[0] is None and torch.equal(only[1], dw)


@TYPES
def test_pieces_of_the_vocabulary(dtype):
    """So many rows that the gradient's scores go through in pieces (more than 1 GiB of them): rows of a
    small width, checked at some of the rows and at all of the vocabulary."""
    rows, dim, vocab = (66000, 32, 9001) if dtype == torch.bfloat16 else (66000, 16, 5003)
    h, w, t, ga, _ = draw(rows, dim, vocab, dtype)
    loss, lse = dpb.cross_entropy(h, w, t)
    dh, dw = dpb.cross_entropy_bwd(ga, h, w, t, lse)
    want_h, want_w, bound_w = [], torch.zeros(vocab, dim, dtype=torch.float64, device=DEV), 0
    for at in range(0, rows, 6000):
        s = slice(at, at + 6000)
        (h64, h_off), (w64, w_off) = R.cross_entropy_bwd(ga[s], h[s], w, t[s], lse[s], 1.0)
        want_w += w64
        bound_w = bound_w + w_off
        if at in (0, 60000):
            R.check("dhidden", dh[s], h64, h_off)
    R.check("dweight", dw, want_w, bound_w + 11 * R.E * bound_w + 2 * R.U[dtype] * want_w.abs() + rows * R.E * want_w.abs())
    R.check("loss", loss[:6000], *R.cross_entropy(h[:6000], w, t[:6000], 1.0)[0])


@TYPES
@pytest.mark.parametrize("step,offset", [(8, 0), (0, 8), (24, 8), (1, 0), (5, 0)])
def test_rows_evenly_apart(step, offset, dtype):
    h, w, t, ga, _ = draw(70, 96, 300, dtype)
    cut = lambda x: torch.cat([torch.full((len(x), offset), 7.0, device=DEV).to(dtype), x, torch.full((len(x), step), float("nan"), device=DEV).to(dtype)], 1)[:, offset:offset + 96]  # noqa: E731,E501
    h2, w2 = cut(h), cut(w)
    want = dpb.cross_entropy(h, w, t)
    got = dpb.cross_entropy(h2, w2, t)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(torch.equal(a, b) for a, b in zip(dpb.cross_entropy_bwd(ga, h2, w2, t, got[1]), dpb.cross_entropy_bwd(ga, h, w, t, want[1])))


@TYPES
def test_leading_dimensions_and_one_row_for_all(dtype):
    h, w, t, ga, _ = draw(24, 64, 100, dtype)
    loss, lse = dpb.cross_entropy(h.view(2, 12, 64), w, t.view(2, 12))
    assert loss.shape == (2, 12) and torch.equal(loss.flatten(), dpb.cross_entropy(h, w, t)[0])
    dh, dw = dpb.cross_entropy_bwd(ga.view(2, 12), h.view(2, 12, 64), w, t.view(2, 12), lse)
    assert dh.shape == (2, 12, 64)
    same = h[:1].expand(24, 64)
    for a, b in zip(dpb.cross_entropy(same, w, t), dpb.cross_entropy(same.contiguous(), w, t)):
        assert torch.equal(a, b)
    one = dpb.cross_entropy(h[3], w, t[3])
    assert one[0].shape == () and torch.equal(one[1], lse.flatten()[3]) is True


@TYPES
def test_large_and_sure_scores(dtype):
    """Scores far from 0 and probabilities that are 0 and 1: no overflow, and the loss of a sure target is next to 0,
    not below it.  Its sum of exponentials is 2^(s log2(e) - b) with b the rounded exponent, 1 + x with x up to some
    1e-5 here, rounded at 2^-24; its logarithm cancels x, which the kernel forms exactly, up to that rounding and its own
    (of some 2^-24 x): 2^-23 covers both."""
    dim, vocab = 64, 700
    w = torch.zeros(vocab, dim, device=DEV)
    w[:, 0] = torch.linspace(-1, 1, vocab, device=DEV)
    w[5] = 0
    w[5, 1] = 1.0
    h = torch.zeros(4, dim, device=DEV)
    h[0, 0], h[1, 0], h[2, 1], h[3, 0] = 3e4, -3e4, 200.0, 60.0
    h, w = h.to(dtype), w.to(dtype)
    t = torch.tensor([vocab - 1, vocab - 1, 5, 0], device=DEV)
    loss, lse = dpb.cross_entropy(h, w, t)
    (want, off), (want_lse, lse_off), _ = R.cross_entropy(h, w, t, 1.0)
    R.check("loss", loss, want, off)
    R.check("lse", lse, want_lse, lse_off)
    assert 0.0 <= float(loss[2]) <= 2.0 ** -23 and float(loss[0]) >= 0.0
    ga = torch.ones(4, device=DEV)
    for got, ref in zip(dpb.cross_entropy_bwd(ga, h, w, t, lse), R.cross_entropy_bwd(ga, h, w, t, lse, 1.0)):
        R.check("grad", got, *ref)


@TYPES
def test_what_is_not_finite_stays_in_its_row(dtype):
    h, w, t, ga, _ = draw(300, 72, 1000, dtype)
    t = t.clamp(0, 999)
    want = dpb.cross_entropy(h, w, t)
    h = h.clone()
    h[7, 3], h[130, 5] = float("nan"), float("inf")
    loss, lse = dpb.cross_entropy(h, w, t)
    fine = torch.ones(300, dtype=torch.bool, device=DEV)
    fine[[7, 130]] = False
    assert torch.equal(loss[fine], want[0][fine]) and torch.equal(lse[fine], want[1][fine])
    assert not torch.isfinite(loss[~fine]).any()
    dh, _ = dpb.cross_entropy_bwd(ga, h, w, t, lse)
    assert torch.equal(dh[fine], dpb.cross_entropy_bwd(ga, *(x for x in (torch.where(fine[:, None], h, torch.zeros_like(h)), w, t, torch.where(fine, lse, want[1]))))[0][fine])


def test_rows_without_a_gradient_leave_nothing():
    """Targets outside the vocabulary and gradients of 0: exact zeros, whatever the row's lse says."""
    h, w, t, ga, _ = draw(90, 64, 500, torch.bfloat16)
    t[::3] = -100
    t[1::3] = 500
    lse = dpb.cross_entropy(h, w, t)[1]
    lse[0] = float("-inf")
    loss = dpb.cross_entropy(h, w, t)[0]
    out = (t < 0) | (t >= 500)
    assert not loss[out].any() and loss[~out].all()
    dh, dw = dpb.cross_entropy_bwd(ga, h, w, t, lse)
    assert not dh[out].any()
    keep = torch.nonzero(~out)[:, 0]
    want = R.cross_entropy_bwd(ga[keep], h[keep], w, t[keep], lse[keep], 1.0)
    R.check("dweight", dw, *want[1])
    assert not dpb.cross_entropy_bwd(ga, h, w, torch.full_like(t, -100), lse)[1].any()


def test_gradients_against_differences():
    """Central differences of the fp32 loss: its rounding, 90 times 2^-21, over the step h, and the third derivative's part."""
    h, w, t, ga, ge = draw(90, 40, 300, torch.float32)
    loss, lse = dpb.cross_entropy(h, w, t)
    dh, dw = dpb.cross_entropy_bwd(ga, h, w, t, lse, grad_lse=ge)

    def f(h, w):
        loss, lse = dpb.cross_entropy(h, w, t)
        return float((loss.double() * ga.double() + lse.double() * ge.double()).sum())

    step = 2.0 ** -6
    for i, j in ((0, 0), (41, 17), (89, 39)):
        d = torch.zeros_like(h)
        d[i, j] = step
        assert abs((f(h + d, w) - f(h - d, w)) / (2 * step) - float(dh[i, j])) < 90 * 2.0 ** -21 / step + 2 * step ** 2
        d = torch.zeros_like(w)
        d[i, j] = step
        assert abs((f(h, w + d) - f(h, w - d)) / (2 * step) - float(dw[i, j])) < 90 * 2.0 ** -21 / step + 90 * step ** 2


def test_nothing_to_do_and_given_outputs():
    w = torch.randn(50, 16, device=DEV)
    none = torch.zeros(0, dtype=torch.int64, device=DEV)
    loss, lse = dpb.cross_entropy(torch.zeros(0, 16, device=DEV), w, none)
    assert loss.shape == lse.shape == (0,)
    dh, dw = dpb.cross_entropy_bwd(loss, torch.zeros(0, 16, device=DEV), w, none, lse)
    assert dh.shape == (0, 16) and dw.shape == (50, 16) and not dw.any()
    h, t = torch.randn(9, 16, device=DEV), torch.arange(9, device=DEV)
    with pytest.raises(dpb.DPBError):
        dpb.cross_entropy(h, w[:0], t)
    want = dpb.cross_entropy(h, w, t)
    outs = [torch.empty(9, device=DEV) for _ in range(2)]
    versions = [x._version for x in outs]
    assert all(torch.equal(a, b) for a, b in zip(dpb.cross_entropy(h, w, t, loss=outs[0], lse=outs[1]), want))
    assert all(x._version > v for x, v in zip(outs, versions))
    grads = [torch.empty_like(h), torch.empty_like(w)]
    got = dpb.cross_entropy_bwd(want[0], h, w, t, want[1], dhidden=grads[0], dweight=grads[1])
    assert got[0] is grads[0] and all(torch.equal(a, b) for a, b in zip(got, dpb.cross_entropy_bwd(want[0], h, w, t, want[1])))


@TYPES
def test_a_logit_of_minus_infinity_is_no_entry(dtype):
    """Loss and log-sum-exp are those of the vocabulary without it, and what is one token's stays with it."""
    h, w, t, _, _ = draw(200, 72, 700, dtype)
    h, t = h.abs() + 0.5, t.clamp(0, 699)
    t[t == 400] = 0
    w = w.clone()
    w[400] = 1.0
    w[400, 7] = float("-inf")
    rest = torch.cat([w[:400], w[401:]])
    (want, off), (want_lse, lse_off), _ = R.cross_entropy(h, rest, t - (t > 400).long(), 0.3)
    loss, lse = dpb.cross_entropy(h, w, t, 0.3)
    R.check("loss", loss, want, off)
    R.check("lse", lse, want_lse, lse_off)
    t[3], h[5, 7], h[6, 0] = 400, -1.0, float("nan")      # the target's logit is -inf; +inf; NaN
    loss, lse = dpb.cross_entropy(h, w, t, 0.3)
    assert loss[3] == float("inf") and torch.isfinite(lse[3])
    assert not torch.isfinite(loss[5:7]).any() and not torch.isfinite(lse[5:7]).any()
    fine = torch.ones(200, dtype=torch.bool, device=DEV)
    fine[[3, 5, 6]] = False
    R.check("loss", loss[fine], want[fine], off[fine])
    R.check("lse", lse[fine], want_lse[fine], lse_off[fine])
