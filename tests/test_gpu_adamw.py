"""The AdamW step against the same formulas in fp64: types, masters, odd sizes,
unaligned tensors, many tensors, 8-bit states and their rounding, non-finite
gradients, refusals."""
import math

import pytest
import torch

from paper_2607_20652_amd import binding as dpb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
SIZES = [1, 255, 256, 257, 3, 4096, 8191, 8192, 8193, 0, 70001, 12]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dpb.load()


def make(sizes, ptype, gtype, seed=0, offset=0):
    """Tensors on the GPU, `offset` elements into buffers of their own."""
    gen = torch.Generator().manual_seed(seed)
    put = lambda x, t: torch.cat([torch.zeros(offset), x]).to(t).to(DEV)[offset:]  # noqa: E731
    params = [put(torch.randn(n, generator=gen) * 0.1, ptype) for n in sizes]
    grads = [put(torch.randn(n, generator=gen) * 10 ** (-(i % 4)), gtype) for i, n in enumerate(sizes)]
    return params, grads


def flat(tensors):
    """Tensors as the states lie, in fp64: each at a multiple of 256 elements, zeros between."""
    n = [-(-t.numel() // 256) * 256 for t in tensors]
    out, at = torch.zeros(sum(n), dtype=torch.float64), 0
    for t, k in zip(tensors, n):
        out[at:at + t.numel()] = t.detach().double().cpu().reshape(-1)
        at += k
    return out


def formulas(w, g, m, v, step, lr, betas, eps, decay):
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    w = (1 - lr * decay) * w - lr * (m / (1 - betas[0] ** step)) / ((v / (1 - betas[1] ** step)).sqrt() + eps)
    return w, m, v


def near(got, want, tol):
    """Within tol of each value, or of the update's scale where a value is smaller."""
    got = got.double().cpu()
    off = (got - want).abs()
    assert bool((off <= tol * want.abs().clamp_min(1e-3)).all()), float((off / want.abs().clamp_min(1e-3)).max())


@pytest.mark.parametrize("offset", [0, 1], ids=["aligned", "unaligned"])
@pytest.mark.parametrize("master", [False, True], ids=["", "master"])
@pytest.mark.parametrize("gtype", [F32, BF16], ids=["g32", "g16"])
@pytest.mark.parametrize("ptype", [F32, BF16], ids=["p32", "p16"])
def test_states_in_32_bits(ptype, gtype, master, offset):
    params, grads = make(SIZES, ptype, gtype, 1, offset)
    m, v, scales, weights = dpb.adamw_state(params, 32, master)
    decay = [0.1 * (i % 3) for i in range(len(SIZES))]
    each = torch.cat([torch.full((-(-n // 256) * 256,), d, dtype=torch.float64) for n, d in zip(SIZES, decay)])
    w64, m64, v64 = flat(params), flat([]).new_zeros(m.numel()), flat([]).new_zeros(m.numel())
    gs = torch.tensor([0.5], device=DEV)
    for step in (1, 2, 3):
        g64 = flat(grads) * 0.5
        dpb.adamw_step(params, grads, m, v, master=weights, step=step, lr=1e-2, betas=(0.9, 0.99), eps=1e-6,
                       weight_decay=decay, grad_scale=gs)
        w64, m64, v64 = formulas(w64, g64, m64, v64, step, 1e-2, (0.9, 0.99), 1e-6, each)
        # a handful of fp32 roundings a step
        near(m, m64, 3e-6)
        near(v, v64, 3e-6)
        if weights is not None:
            near(weights, w64, 3e-5)     # an update of 1e-2 against 1e-3 of the scale: 1e-2 * 1e-6 / 1e-3 each
        if ptype == F32:
            near(flat(params), w64, 3e-5)
        else:
            # rounded once from the master, or once a step; then go on from what is stored
            off = (flat(params) - w64).abs()
            assert bool((off <= 2.0 ** -8 * w64.abs() + 1e-6).all())
            if weights is None:
                w64 = flat(params)


def test_more_tensors_than_one_launch_holds():
    sizes = [(37 * i) % 700 for i in range(230)]
    params, grads = make(sizes, F32, F32, 2)
    m, v, _, _ = dpb.adamw_state(params)
    w64 = flat(params)
    want, m64, v64 = formulas(w64, flat(grads), 0 * w64, 0 * w64, 1, 1e-2, (0.9, 0.999), 1e-8, 0.01)
    dpb.adamw_step(params, grads, m, v, step=1, lr=1e-2, weight_decay=0.01)
    near(m, m64, 3e-6)
    near(v, v64, 3e-6)
    near(flat(params), want, 3e-5)


def neighbours(x, scale):
    """The two 8-bit values around x / scale (fp64), times the scale."""
    a = (x / scale).abs().clamp(max=448.0)
    step = torch.exp2(torch.floor(torch.log2(a.clamp_min(2.0 ** -6))) - 3)
    down = torch.floor(a / step) * step
    return down * scale, (down + step) * scale


@pytest.mark.parametrize("ptype,gtype,master", [(F32, F32, False), (BF16, BF16, True), (BF16, F32, False)])
def test_states_in_8_bits(ptype, gtype, master):
    params, grads = make(SIZES, ptype, gtype, 3)
    m, v, scales, weights = dpb.adamw_state(params, 8, master)
    for step in (1, 2, 3):
        each = scales.double().cpu().repeat_interleave(256, 0)
        w64 = flat(params) if weights is None else weights.double().cpu()
        m0, v0 = m.double().cpu() * each[:, 0], (v.double().cpu() * each[:, 1]) ** 2
        dpb.adamw_step(params, grads, m, v, scales, weights, step=step, lr=1e-2, betas=(0.9, 0.99), eps=1e-6,
                       weight_decay=0.1, seed=step)
        w1, m1, v1 = formulas(w64, flat(grads), m0, v0, step, 1e-2, (0.9, 0.99), 1e-6, 0.1)
        u1 = v1.sqrt()
        top = torch.stack([m1.abs().view(-1, 256).amax(1), u1.view(-1, 256).amax(1)], 1) / 448
        assert bool(((scales.double().cpu() - top).abs() <= 1e-6 * top).all())
        each = scales.double().cpu().repeat_interleave(256, 0)
        for code, want, sc in ((m, m1, each[:, 0]), (v, u1, each[:, 1])):
            got, safe = code.double().cpu() * sc, sc.clamp_min(1e-300)
            lo, hi = neighbours(want, safe)
            # either neighbour; an fp32 value next to one may be taken for it
            slack = 1e-5 * want.abs()
            assert bool(((got.abs() >= lo - slack) & (got.abs() <= hi + slack)).all())
            assert bool((got * want >= 0).all())
        assert bool(((v.float() > 0).cpu() == (u1 > 0)).all())     # never to zero
        if weights is not None:
            near(weights, w1, 3e-5)
        if ptype == F32:
            near(flat(params), w1, 3e-5)
        else:
            assert bool(((flat(params) - w1).abs() <= 2.0 ** -8 * w1.abs() + 1e-6).all())


def test_rounding_keeps_the_mean():
    """Over many seeds the 8-bit states average to the values they stand for."""
    n, rounds = 4096, 400
    gen = torch.Generator().manual_seed(4)
    g = torch.randn(n, generator=gen).to(DEV)
    total = torch.zeros(2, n, dtype=torch.float64, device=DEV)
    for seed in range(rounds):
        p = [torch.zeros(n, device=DEV)]
        m, v, scales, _ = dpb.adamw_state(p, 8)
        dpb.adamw_step(p, [g], m, v, scales, step=1, lr=1e-3, seed=seed)
        each = scales.double().repeat_interleave(256, 0)
        total[0] += m.double() * each[:, 0]
        total[1] += v.double() * each[:, 1]
    mean = (total / rounds).cpu()
    for got, want in ((mean[0], 0.1 * g.double().cpu()), (mean[1], math.sqrt(1e-3) * g.double().cpu().abs())):
        lo, hi = neighbours(want, (want.abs().view(-1, 256).amax(1) / 448).repeat_interleave(256))
        # a coin with sides hi and lo thrown `rounds` times: its mean strays by at most (hi - lo) / 2 / sqrt(rounds)
        # in one standard deviation; over 4096 places five and a half are not passed (and the 2^-16 grid of the coin)
        off = (got - want).abs() - 2.0 ** -16 * (hi - lo)
        live = lo > 0
        assert bool((off[live] <= 5.5 * (hi - lo)[live] / 2 / math.sqrt(rounds)).all())


def test_same_seed_same_bits():
    params, grads = make(SIZES, F32, F32, 5)
    got = []
    for _ in range(2):
        p = [x.clone() for x in params]
        m, v, scales, _ = dpb.adamw_state(p, 8)
        for step in (1, 2):
            dpb.adamw_step(p, grads, m, v, scales, step=step, lr=1e-3, seed=77 + step)
        got.append([*p, m.view(torch.uint8), v.view(torch.uint8), scales])
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_gradients_that_are_not_finite():
    for bad in (math.nan, math.inf):
        p, g = [torch.ones(1000, device=DEV)], [torch.full((1000,), 0.1, device=DEV)]
        g[0][300] = bad
        m, v, scales, _ = dpb.adamw_state(p, 8)
        dpb.adamw_step(p, g, m, v, scales, step=1, lr=1e-3)
        hit = p[0].isnan().cpu()
        assert hit[300] and hit.sum() == 1                       # this step: that element alone
        assert not torch.isfinite(scales[1]).any() and torch.isfinite(scales[[0, 2, 3]]).all()
        m, v, _, _ = dpb.adamw_state(p)
        q = [torch.ones(1000, device=DEV)]
        dpb.adamw_step(q, g, m, v, step=1, lr=1e-3)
        assert (~torch.isfinite(m)).sum() == 1 and (~torch.isfinite(v)).sum() == 1


@pytest.mark.parametrize("bits", [8, 32])
def test_a_tensor_of_more_than_2_to_the_31_elements(bits):
    n, tail = 2**31 + 2**20 + 77, 5000
    p = [torch.zeros(n, dtype=BF16, device=DEV)]
    g = [torch.zeros(n, dtype=BF16, device=DEV)]
    gen = torch.Generator().manual_seed(7)
    p[0][-tail:] = torch.randn(tail, generator=gen).to(BF16).to(DEV)
    g[0][-tail:] = torch.randn(tail, generator=gen).to(BF16).to(DEV)
    w64, g64 = p[0][-tail:].double().cpu(), g[0][-tail:].double().cpu()
    m, v, scales, _ = dpb.adamw_state(p, bits)
    dpb.adamw_step(p, g, m, v, scales, step=1, lr=1e-2, weight_decay=0.1, seed=3)
    want, m1, v1 = formulas(w64, g64, 0 * w64, 0 * w64, 1, 1e-2, (0.9, 0.999), 1e-8, 0.1)
    assert bool(((p[0][-tail:].double().cpu() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-6).all())
    assert not p[0][:-tail].any() and not g[0][:-tail].any()
    got = m[n - tail:n].double().cpu()
    if bits == 8:
        got *= scales[torch.arange(n - tail, n, device=DEV) // 256, 0].double().cpu()
        assert bool(((got - m1).abs() <= 0.13 * m1.abs() + 0.1 * 2.0 ** -9 / 448 * 5).all())   # a neighbour: at most 1/8 off
    else:
        near(got, m1, 3e-6)


def test_zero_gradients_and_tiny_ones():
    p, g = [torch.ones(512, device=DEV)], [torch.zeros(512, device=DEV)]
    g[0][256:] = 1e-41
    m, v, scales, _ = dpb.adamw_state(p, 8)
    dpb.adamw_step(p, g, m, v, scales, step=1, lr=1e-3, weight_decay=0.5)
    assert torch.isfinite(p[0]).all() and (p[0] - (1 - 5e-4)).abs().max() < 1e-6
    assert torch.isfinite(scales).all() and not m.float()[:256].any() and not v.float()[:256].any()


def test_refusals():
    p, g = make([300], F32, F32, 6)
    m, v, _, _ = dpb.adamw_state(p)
    good = dict(step=1, lr=1e-3)
    for bad in (dict(step=0), dict(lr=math.nan), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=0.0),
                dict(weight_decay=math.inf)):
        with pytest.raises(dpb.DPBError) as e:
            dpb.adamw_step(p, g, m, v, **(good | bad))
        assert e.value.status == -1
    with pytest.raises(dpb.DPBError):
        dpb.adamw_step(p, g, torch.zeros(516, device=DEV)[1:513], v, **good)     # states not aligned
    with pytest.raises(AssertionError):
        dpb.adamw_step(p, g, m[:256], v, **good)
    with pytest.raises(AssertionError):
        dpb.adamw_step(p, [g[0][:299]], m, v, **good)
    with pytest.raises(AssertionError):
        dpb.adamw_step(p, g, m.to(F8), v, **good)
    with pytest.raises(ValueError):
        dpb.adamw_step([x.cpu() for x in p], g, m, v, **good)
    with pytest.raises(ValueError):
        dpb.adamw_step([torch.zeros(600, device=DEV)[::2]], g, m, v, **good)
    dpb.adamw_step([], [], m, v, **good)
