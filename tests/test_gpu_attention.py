"""Attention and its gradients against plain fp64 attention: head widths, shared
heads, lengths from none to several tiles, causal masks that leave rows empty,
packed sequences, strides, streams, non-finite values behind the lengths."""
import math

import pytest
import torch

from attention_util import check, reference
from paper_2607_20652_amd import binding as dpb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dpb.load()


def make(seed, B, Q, K, H, G, D, dtype):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return (2 * r(B, Q, H, D)).to(dtype), r(B, K, G, D).to(dtype), r(B, K, G, D).to(dtype), r(B, Q, H, D).to(dtype)


def run(q, k, v, g, causal, scale=None, **kw):
    """The calls on the GPU: out, lse, dq, dk, dv."""
    q, k, v, g = (x if x.is_cuda else x.to(DEV) for x in (q, k, v, g))
    out, lse = dpb.attention(q, k, v, causal, scale, **kw)
    dq, dk, dv = dpb.attention_bwd(g, q, k, v, out, lse, causal, scale, **kw)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def agree(got, ref, dtype):
    torch.cuda.synchronize()
    for name in ref:
        check(name, got[name], ref[name], dtype)


SHAPES = [
    # B, Q, K, H, G, D
    (1, 1, 1, 1, 1, 8),
    (2, 1, 2, 2, 1, 64),
    (1, 7, 5, 3, 3, 16),
    (2, 31, 33, 4, 2, 64),
    (1, 32, 64, 1, 1, 128),
    (2, 64, 32, 2, 2, 40),
    (1, 65, 129, 6, 2, 72),
    (1, 127, 128, 5, 1, 128),
    (3, 130, 70, 2, 2, 96),
    (1, 257, 300, 4, 4, 64),
    (1, 300, 257, 7, 1, 24),
    (1, 5, 700, 8, 2, 128),
    (1, 1, 1031, 7, 7, 64),
    (2, 1, 515, 16, 2, 112),
    (1, 520, 1, 2, 1, 32),
]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True], ids=["all", "causal"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_padded_full(shape, causal, dtype):
    B, Q, K, H, G, D = shape
    q, k, v, g = make(1, B, Q, K, H, G, D, dtype)
    ref = reference(q, k, v, causal, D ** -0.5, g)
    agree(run(q, k, v, g, causal), ref, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True], ids=["all", "causal"])
@pytest.mark.parametrize("Q,K,H,G,D", [(70, 150, 4, 2, 64), (1, 200, 6, 3, 128), (3, 90, 2, 2, 64), (200, 40, 3, 1, 80)])
def test_lengths_with_anything_behind_them(Q, K, H, G, D, causal, dtype):
    B = 6
    q, k, v, g = make(2, B, Q, K, H, G, D, dtype)
    ql = torch.tensor([Q, Q, 0, max(Q - 3, 0), 1, Q + 9], dtype=torch.int32)
    kl = torch.tensor([K, 0, K, 33, -5, 1], dtype=torch.int32)
    ref = reference(q, k, v, causal, 0.3, g, ql, kl)
    for b in range(B):
        # rows that take no part hold what memory may hold
        n, m = min(max(int(ql[b]), 0), Q), min(max(int(kl[b]), 0), K)
        for x, at in ((q, n), (g, n), (k, m), (v, m)):
            x[b, at:] = math.nan
            x[b, at:, :, ::2] = math.inf
    agree(run(q, k, v, g, causal, 0.3, q_lens=ql.to(DEV), k_lens=kl.to(DEV)), ref, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True], ids=["all", "causal"])
@pytest.mark.parametrize("same", [True, False], ids=["self", "cross"])
def test_packed(same, causal, dtype):
    ql = [1, 130, 0, 64, 17, 200]
    kl = ql if same else [140, 3, 9, 0, 64, 1]
    H, G, D = 4, 2, 64
    B, Q, K = len(ql), max(ql), max(kl)
    q, k, v, g = make(3, B, Q, K, H, G, D, dtype)
    ref = reference(q, k, v, causal, D ** -0.5, g, ql, kl)
    pack = lambda x, n: torch.cat([x[b, :n[b]] for b in range(B)])  # noqa: E731
    starts = lambda n: torch.tensor([sum(n[:i]) for i in range(B + 1)], dtype=torch.int32, device=DEV)  # noqa: E731
    # some room behind the sequences, and a longest sequence told too long
    got = run(pack(q, ql), pack(k, kl), pack(v, kl), pack(g, ql), causal, q_starts=starts(ql), k_starts=starts(kl),
              max_q=Q + 5, max_k=K + 70)
    packed = {n: tuple(pack(x, kl if n in ("dk", "dv") else ql) for x in r) for n, r in ref.items()}
    agree(got, packed, dtype)


def test_packed_starts_out_of_range_stay_inside():
    q, k, v, g = (x[0].to(DEV) for x in make(4, 1, 40, 40, 2, 2, 64, BF16))
    bad = torch.tensor([-7, 20, 12, 90], dtype=torch.int32, device=DEV)
    got = run(q, k, v, g, True, q_starts=bad, k_starts=bad, max_q=40, max_k=40)
    ref = reference(q[None, :20].cpu(), k[None, :20].cpu(), v[None, :20].cpu(), True, 0.125)
    check("out", got["out"][None, :12], tuple(x[:, :12] for x in ref["out"]), BF16)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_strides(dtype):
    B, Q, K, H, G, D = 2, 70, 90, 4, 2, 64
    q, k, v, g = make(5, B, Q, K, H, G, D, dtype)
    ref = reference(q, k, v, True, D ** -0.5, g)
    heads_first = lambda x: x.to(DEV).transpose(1, 2).contiguous().transpose(1, 2)  # noqa: E731

    def beside(x):      # rows of a wider tensor, at an offset
        wide = torch.full((x.shape[0], x.shape[1] + 3, x.shape[2] + 1, D + 16), math.nan, dtype=dtype, device=DEV)
        wide[:, 3:, 1:, 8:8 + D] = x.to(DEV)
        return wide[:, 3:, 1:, 8:8 + D]

    tokens_first = lambda x: x.to(DEV).permute(1, 0, 2, 3).contiguous().permute(1, 0, 2, 3)  # noqa: E731
    for a, b, c in ((heads_first, beside, tokens_first), (beside, tokens_first, heads_first)):
        qd, kd, vd, gd = a(q), b(k), c(v), b(g)
        out = a(torch.zeros_like(q))
        out, lse = dpb.attention(qd, kd, vd, True, out=out)
        dq, dk, dv = (f(torch.zeros_like(x)) for f, x in ((c, q), (a, k), (b, v)))
        dpb.attention_bwd(gd, qd, kd, vd, out, lse, True, dq=dq, dk=dk, dv=dv)
        agree({"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}, ref, dtype)


def test_broadcast_inputs():
    """One key sequence and one query row for all, through strides of 0."""
    q, k, v, g = make(6, 3, 5, 100, 4, 1, 64, F32)
    q = q[:, :1].expand(-1, 5, -1, -1)
    k, v = k[:1].expand(3, -1, -1, -1), v[:1].expand(3, -1, -1, -1)
    ref = reference(q, k, v, False, 0.125, g)
    qd = q[:, :1].to(DEV).expand(-1, 5, -1, -1)
    kd, vd = (x[:1].to(DEV).expand(3, -1, -1, -1) for x in (k, v))
    agree(run(qd, kd, vd, g, False), ref, F32)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_rows_far_apart(dtype):
    """Rows 4 MiB apart: the last ones lie 5 GB behind the first."""
    pitch, n, D = (4 << 20) // (2 if dtype == BF16 else 4), 1250, 64
    q, k, v, g = make(14, 1, 3, n, 2, 1, D, dtype)
    ref = reference(q, k, v, True, D ** -0.5, g)
    far = []
    for x in (k, v):
        room = torch.empty(pitch * (n - 1) + D, dtype=dtype, device=DEV)
        far.append(room.as_strided((1, n, 1, D), (0, pitch, D, 1)))
        far[-1].copy_(x)
    out, lse = dpb.attention(q.to(DEV), *far, True)
    dk, dv = (torch.empty(1, n, 1, D, dtype=dtype, device=DEV) for _ in range(2))
    dq, dk, dv = dpb.attention_bwd(g.to(DEV), q.to(DEV), *far, out, lse, True, dk=dk, dv=dv)
    agree({"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}, ref, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_large_scores(dtype):
    """Scores far apart: the softmax picks one key; no overflow, no NaN."""
    q, k, v, g = make(7, 1, 80, 200, 2, 2, 64, dtype)
    q, k = q * 16, k * 16
    out, lse = dpb.attention(q.to(DEV), k.to(DEV), v.to(DEV), True, 1.0)
    ref = reference(q, k, v, True, 1.0)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    # fp32 scores of magnitude 1e4 are off by 1e-3 or so: what counts is the winner
    top = ref["lse"][0].abs().max()
    assert (lse.cpu().double() - ref["lse"][0]).abs().max() < 64 * 2.0 ** -24 * top
    sure = (out.cpu().double() - ref["out"][0]).abs().amax(-1) < 0.05
    assert sure.double().mean() > 0.95


def test_a_nan_reaches_its_own_rows_only():
    q, k, v, g = make(8, 2, 150, 150, 2, 2, 64, BF16)
    q[0, 100, 1, 3] = math.nan
    out, lse = dpb.attention(q.to(DEV), k.to(DEV), v.to(DEV), True)
    bad = torch.zeros(2, 150, 2, dtype=torch.bool)
    bad[0, 100, 1] = True
    assert torch.equal(out.isnan().any(-1).cpu(), bad) and torch.equal(lse.isnan().cpu(), bad)


def test_same_bits_every_run_and_on_another_stream():
    q, k, v, g = (x.to(DEV) for x in make(9, 2, 200, 900, 8, 2, 128, BF16))
    first = run(q, k, v, g, True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = run(q, k, v, g, True)
    side.synchronize()
    for n in first:
        assert torch.equal(first[n], again[n]), n


@pytest.mark.parametrize("causal", [False, True], ids=["all", "causal"])
def test_gradients_against_differences(causal):
    """fp32 gradients along random directions against central differences of fp64 attention."""
    B, Q, K, H, G, D = 1, 37, 45, 4, 2, 24
    q, k, v, g = make(10, B, Q, K, H, G, D, F32)
    got = run(q, k, v, g, causal)
    gen = torch.Generator().manual_seed(11)
    loss = lambda q, k, v: float((reference(q, k, v, causal, D ** -0.5)["out"][0] * g.double()).sum())  # noqa: E731
    for at, name in enumerate(("dq", "dk", "dv")):
        x = [q.double(), k.double(), v.double()]
        d = torch.randn(x[at].shape, generator=gen, dtype=torch.float64)
        h = 1e-4
        up, down = list(x), list(x)
        up[at], down[at] = x[at] + h * d, x[at] - h * d
        slope = (loss(*up) - loss(*down)) / (2 * h)
        grad = got[name].double().cpu()
        mine = float((grad * d).sum())
        # differences: third-order terms of about h^2; the gradient: fp32 sums
        assert abs(mine - slope) < 1e-5 * float((grad * d).abs().sum()) + 1e-6


def test_forward_values_survive_a_graph():
    q, k, v, g = (x.to(DEV) for x in make(12, 2, 1, 2000, 8, 2, 64, BF16))
    out, lse = dpb.attention(q, k, v)
    lib_ws = torch.empty(1 << 22, dtype=torch.float32, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o2, l2 = torch.empty_like(out), torch.empty_like(lse)
    with torch.cuda.stream(side):
        dpb.attention(q, k, v, out=o2, lse=l2, workspace=lib_ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dpb.attention(q, k, v, out=o2, lse=l2, workspace=lib_ws)
    for i in range(3):
        q.mul_(0.5)
        want, _ = dpb.attention(q, k, v)
        o2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o2, want), i


def test_refusals():
    q, k, v, g = (x.to(DEV) for x in make(13, 1, 8, 8, 4, 2, 64, BF16))

    def status(*a, **kw):
        with pytest.raises(dpb.DPBError) as e:
            dpb.attention(*a, **kw)
        return e.value.status

    wide = torch.zeros(1, 8, 4, 136, dtype=BF16, device=DEV)
    assert status(wide, wide, wide) == -2                              # head_dim over 128
    odd = torch.zeros(1, 8, 4, 60, dtype=BF16, device=DEV)
    assert status(odd, odd, odd) == -2                                 # head_dim not a multiple of 8
    assert status(q[:, :, :3], k, v) == -1                             # 3 heads over 2 key heads
    for scale in (0.0, -1.0, math.inf, math.nan):
        assert status(q, k, v, scale=scale) == -1
    off = torch.zeros(1 * 8 * 4 * 64 + 8, dtype=BF16, device=DEV)
    assert status(off[1:2049].view(1, 8, 4, 64), k, v) == -1           # not 16-byte aligned
    pitch = torch.zeros(1, 8, 4, 68, dtype=BF16, device=DEV)[..., :64]
    assert status(pitch, k, v) == -1                                   # strides not a multiple of 16 bytes
    with pytest.raises(ValueError):
        dpb.attention(q.cpu(), k, v)
    with pytest.raises(ValueError):
        dpb.attention(q.transpose(1, 3).contiguous().transpose(1, 3), k, v)
    with pytest.raises(AssertionError):
        dpb.attention(q, k.float(), v)
    with pytest.raises(AssertionError):
        dpb.attention(q, k, v[:, :4])
    with pytest.raises(TypeError):
        dpb.attention(q.half(), k.half(), v.half())
    out, lse = dpb.attention(q, k, v)
    with pytest.raises(dpb.DPBError):
        dpb.attention_bwd(g, q, k, v, out, lse, workspace=torch.empty(4, device=DEV))
    with pytest.raises(dpb.DPBError):
        dpb.attention_bwd(g, q, k, v, out, lse, dk=k)
    empty = q[:, :0]
    out, lse = dpb.attention(empty, k, v)
    assert out.shape == empty.shape and lse.shape == (1, 0, 4)
    dq, dk, dv = dpb.attention_bwd(empty, empty, k, v, out, lse)
    assert not dk.any() and not dv.any()
    out, lse = dpb.attention(q, k[:, :0], v[:, :0])
    assert not out.any() and torch.isinf(lse).all()
