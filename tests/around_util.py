"""Embedding, norm and vocabulary loss in fp64 with the error bounds of the kernels' arithmetic."""
import torch

# a result's last rounding, and one of a bf16 operand: half a step of its type
U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
E = 2.0 ** -24     # of one fp32 operation
# fp32 numbers under 2^-126 may become 0: each term of a sum of up to 2^16 of them, times operands up to 2^10
TINY = 2.0 ** -100


def check(name, got, value, bound):
    got, value, bound = got.detach().double().cpu(), value.double().cpu(), bound.double().cpu()
    assert got.shape == value.shape, name
    off = (got - value).abs()
    bad = ~(off <= bound + TINY)
    assert not bad.any(), (f"{name}: {int(bad.sum())} of {bad.numel()} out of bounds, worst "
                           f"{float((off / bound.clamp_min(1e-300)).nan_to_num(1e30).max()):.3g} times the bound, at {bad.nonzero()[:4].tolist()}")


def embedding_bwd(grad, tokens, vocab, scale):
    """(value, bound) of the table's gradient: as many additions as the row has tokens, a product, a rounding."""
    g, t = grad.double().flatten(0, -2), tokens.flatten().long()
    live = (t >= 0) & (t < vocab)
    of = lambda x: torch.zeros(vocab, x.shape[1], dtype=torch.float64, device=x.device).index_add_(0, t[live], x[live])  # noqa: E731
    n = of(torch.ones(len(t), 1, dtype=torch.float64, device=g.device))
    value, size = of(g) * scale, of(g.abs()) * abs(scale)
    return value, n * E * size + 2 * U[grad.dtype] * value.abs()


def rms_norm(total, weight, eps):
    """(value, bound) of out and rstd from the sum as it was kept.  A row's squares are added up by 64 or
    more lanes, then across them."""
    z = total.double()
    w = torch.ones(z.shape[-1], dtype=torch.float64, device=z.device) if weight is None else weight.double()
    f = (z.shape[-1] / 64 + 20) * E
    rstd = (z.square().mean(-1) + eps).rsqrt()
    out = z * rstd[..., None] * w
    return (out, (f + U[total.dtype]) * out.abs()), (rstd, f * rstd)


def rms_norm_bwd(grad, total, weight, rstd, grad_total=None):
    """(value, bound) of dx and dweight from the forward's total and rstd."""
    g, z, rho = grad.double(), total.double(), rstd.double()[..., None]
    w = torch.ones(z.shape[-1], dtype=torch.float64, device=z.device) if weight is None else weight.double()
    n, u = z * rho, g * w
    dx = rho * (u - n * (u * n).mean(-1, keepdim=True))
    size = rho * (u.abs() + n.abs() * (u * n).abs().mean(-1, keepdim=True))
    if grad_total is not None:
        dx = dx + grad_total.double()
        size = size + grad_total.double().abs()
    dims = tuple(range(z.dim() - 1))
    rows = z.numel() // z.shape[-1]
    dw, dws = (g * n).sum(dims), (g * n).abs().sum(dims)
    f = (z.shape[-1] / 64 + 20) * E
    # a weight's sum: by workgroups that take rows in turn, then over those
    uw = U[total.dtype if weight is None else weight.dtype]
    return (dx, f * size + U[total.dtype] * dx.abs()), (dw, (rows / 64 + 80) * E * dws + uw * dw.abs())


def cross_entropy(hidden, weight, targets, scale):
    """(value, bound) of loss and lse, and what the gradients need: (p, the bound of each score).

    A score is a sum of dim products; the sums of exponentials add up relative errors of their terms (scores'
    errors and some 8 steps of the exponential and its argument, which is under some 2^5) and of at most 64 + 64 +
    16 additions one behind the other."""
    h, w = hidden.double().flatten(0, -2), weight.double()
    t = targets.flatten().long()
    logits = h @ w.T * scale
    off = (h.shape[1] + 4) * E * scale * (h.abs() @ w.abs().T)
    lse = torch.logsumexp(logits, 1)
    p = torch.exp(logits - lse[:, None])
    lse_off = (p * off).sum(1) + 400 * E + 4 * E * lse.abs()
    live = (t >= 0) & (t < w.shape[0])
    at = torch.where(live, t, 0)[:, None]
    loss = torch.where(live, lse - logits.gather(1, at)[:, 0], 0.0)
    loss_off = torch.where(live, lse_off + off.gather(1, at)[:, 0] + 4 * E * loss.abs() + 4 * E * logits.gather(1, at)[:, 0].abs(), 0.0)
    return (loss, loss_off), (lse, lse_off), (p, off, lse, live, at)


def cross_entropy_bwd(grad_loss, hidden, weight, targets, lse, scale, grad_lse=None):
    """(value, bound) of dhidden and dweight from the forward's lse."""
    h, w = hidden.double().flatten(0, -2), weight.double()
    zeros = torch.zeros(h.shape[0], dtype=torch.float64, device=h.device)
    _, _, (p, off, exact, live, at) = cross_entropy(hidden, weight, targets, scale)
    given = lse.double().flatten()
    p = p * torch.exp(exact - given)[:, None]          # for the lse that the call has
    a = torch.where(live, zeros if grad_loss is None else grad_loss.double().flatten(), 0.0)
    e = zeros if grad_lse is None else grad_lse.double().flatten()
    d = p * (a + e)[:, None]
    # the exponential of a score: its error, and a rounding each of lse log2(e), of the argument and in the power
    p_off = (p * (off + (8 + 4 * given.abs()[:, None] + 64) * E)) * (a + e).abs()[:, None]
    d.scatter_add_(1, at, -(a * live)[:, None])
    u = U[hidden.dtype] if hidden.dtype == torch.bfloat16 else E
    d_off = p_off + u * d.abs() + 2 * E * a.abs()[:, None] * torch.zeros_like(d).scatter_(1, at, 1.0)
    sums = lambda n, size: (n + 80) * E * size  # noqa: E731
    dh, dw = d @ w * scale, d.T @ h * scale
    dh_off = scale * (d_off @ w.abs() + sums(w.shape[0], d.abs() @ w.abs())) + 2 * U[hidden.dtype] * dh.abs()
    dw_off = scale * (d_off.T @ h.abs() + sums(h.shape[0], d.abs().T @ h.abs())) + 2 * U[hidden.dtype] * dw.abs()
    return (dh, dh_off), (dw, dw_off)
