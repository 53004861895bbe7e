"""Plain attention in fp64 with the error bounds of the kernels' arithmetic."""
import math

import torch

# Half a step of bf16 (8 significant bits) is 2^-9 of the value: twice that for each rounding.
U = {torch.bfloat16: 2.0 ** -8, torch.float32: 0.0}
# fp32 products and sums over up to a few thousand terms, exp of arguments up to about 30 in magnitude:
# 30 * 2^-24 * log2(e) is 2.6e-6 of a weight, the sums' and products' errors are of that order.
F32 = 2e-5


def visible(qn, kn, causal, device="cpu"):
    """[qn, kn]: key j is seen by query i."""
    i = torch.arange(qn, device=device)[:, None]
    j = torch.arange(kn, device=device)[None, :]
    return j <= i + kn - qn if causal else torch.ones(qn, kn, dtype=torch.bool, device=device)


def one_head(q, k, v, causal, scale, g=None):
    """fp64 results of one sequence and head, with bounds: {name: (value, bound for bf16 steps, bound for fp32)}.

    out:  weights rounded to bf16 as operands, and the result rounded.
    grads: P and dS rounded as operands; delta is taken from the rounded out."""
    q, k, v = q.double(), k.double(), v.double()
    see = visible(q.shape[0], k.shape[0], causal, q.device)
    s = (q @ k.T * scale).masked_fill(~see, -math.inf)
    lse = torch.logsumexp(s, 1) if k.shape[0] else torch.full((q.shape[0],), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.where(see, torch.exp(s - lse[:, None].nan_to_num(neginf=0.0)), 0.0)
    out = p @ v
    av = p @ v.abs()
    res = {"out": (out, av + out.abs(), av), "lse": (lse, torch.zeros_like(lse), 1 + lse.abs().nan_to_num(posinf=0.0))}
    if g is None:
        return res
    g = g.double()
    dp, delta = g @ v.T, (g * out).sum(1, keepdim=True)
    ds = p * (dp - delta) * scale
    # what may be off in dS: its own rounding, delta by rounded outputs; in fp32 every term of dP and delta
    size = (g.abs() * out.abs()).sum(1, keepdim=True)
    ds16 = ds.abs() + p * size * scale
    ds32 = p * (g.abs() @ v.abs().T + (g.abs() * av).sum(1, keepdim=True)) * scale
    dv, dq, dk = p.T @ g, ds @ k, ds.T @ q
    pv = p.T @ g.abs()
    res["dv"] = (dv, pv + dv.abs(), pv)
    res["dq"] = (dq, ds16 @ k.abs() + dq.abs(), ds32 @ k.abs())
    res["dk"] = (dk, ds16.T @ q.abs() + dk.abs(), ds32.T @ q.abs())
    return res


def reference(q, k, v, causal, scale, g=None, q_lens=None, k_lens=None):
    """The same for [B, S, H, D] tensors (CPU): rows that take no part are 0 (lse -inf)."""
    B, Q, H, D = q.shape
    K, G = k.shape[1], k.shape[2]
    zeros = lambda x: [torch.zeros(x.shape, dtype=torch.float64) for _ in range(3)]  # noqa: E731
    res = {"out": zeros(q), "lse": zeros(q[..., 0])}
    res["lse"][0].fill_(-math.inf)
    if g is not None:
        res |= {"dq": zeros(q), "dk": zeros(k), "dv": zeros(k)}
    for b in range(B):
        qn = Q if q_lens is None else min(max(int(q_lens[b]), 0), Q)
        kn = K if k_lens is None else min(max(int(k_lens[b]), 0), K)
        for h in range(H):
            e = h // (H // G)
            got = one_head(q[b, :qn, h], k[b, :kn, e], v[b, :kn, e], causal, scale, None if g is None else g[b, :qn, h])
            for name, parts in got.items():
                for to, x in zip(res[name], parts):
                    if name in ("dk", "dv"):
                        to[b, :kn, e] += x
                    else:
                        to[b, :qn, h] = x
    return res


def check(name, got, ref, dtype):
    """got against (value, bf16 bound, fp32 bound), infinities and NaN in the same places."""
    value, b16, b32 = ref
    got = got.double().cpu()
    assert got.shape == value.shape
    fine = torch.isfinite(value)
    assert torch.equal(got[~fine].isnan(), value[~fine].isnan()), name
    assert torch.equal(got[~fine].nan_to_num(0.0), value[~fine].nan_to_num(0.0)), name
    u = 0.0 if name == "lse" else U[dtype]
    bound = u * b16 + F32 * b32
    off = (got - value).abs()
    bad = fine & ~(off <= bound)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} out of bounds, worst {float((off / bound.clamp_min(1e-300))[fine].max()):.3g} times the bound at {bad.nonzero()[:4].tolist()}"
