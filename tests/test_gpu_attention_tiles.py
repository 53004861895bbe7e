"""Attention by tiles of 128 query rows (training batches and prompts) against plain fp64
attention.  A call takes that kernel only where its rows fill the chip, so every test
here checks that its sizes do: head widths of all instances in both types, shared
heads, ragged and packed sequences, empty rows, strides, streams, graphs,
non-finite values, and rows far apart."""
import ctypes
import math

import pytest
import torch

from attention_util import check, reference
from paper_2607_20652_amd import binding as dpb

gpu = pytest.mark.gpu

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
CAUSAL = pytest.mark.parametrize("causal", [False, True], ids=["all", "causal"])

SHAPES = [
    # B, Q, K, H, G, D
    (43, 50, 1, 3, 3, 16),
    (8, 130, 150, 16, 16, 32),
    (7, 129, 61, 12, 12, 40),
    (16, 257, 257, 4, 4, 64),
    (32, 64, 65, 4, 4, 64),
    (6, 150, 90, 21, 3, 72),
    (32, 33, 40, 4, 4, 96),
    (2, 300, 700, 22, 22, 112),
    (8, 66, 300, 16, 8, 128),
    (5, 256, 128, 13, 13, 128),
]
PACKED = [1, 130, 0, 64, 17, 200, 128, 129, 33]
RAGGED = [(33, 70, 150, 4, 4, 64), (33, 200, 40, 6, 2, 128), (33, 90, 129, 4, 4, 32), (65, 40, 33, 2, 2, 80)]
FAR = (1, 130, 1250, 128, 1, 64)


def splits(B, Q, K, H, G):
    """Parts of the keys in a call of these sizes; 0 is the kernel tested here.  (A function of the library's
    own, not of its C ABI: without a GPU it goes by the 256 compute units of an MI355X.)"""
    fn = dpb.load()._ZN3dpb16attention_splitsEiiiii
    fn.restype, fn.argtypes = ctypes.c_int, [ctypes.c_int] * 5
    return fn(B, Q, K, H, G)


def test_the_sizes_take_the_tiled_kernel_in_all_its_instances():
    for B, Q, K, H, G, _ in SHAPES + RAGGED + [FAR]:
        assert splits(B, Q, K, H, G) == 0, (B, Q, K, H, G)
    assert splits(len(PACKED), max(PACKED), max(PACKED), 16, 8) == 0
    assert {-(-D // 32) for *_, D in SHAPES} == {1, 2, 3, 4}
    # the smallest such call, and one row and one pair less
    assert splits(32, 33, 100, 4, 4) == 0 and splits(32, 32, 100, 4, 4) == 1 and splits(127, 33, 100, 1, 1) == 1


@pytest.fixture(scope="module")
def device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dpb.load()


def make(seed, B, Q, K, H, G, D, dtype):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return (2 * r(B, Q, H, D)).to(dtype), r(B, K, G, D).to(dtype), r(B, K, G, D).to(dtype), r(B, Q, H, D).to(dtype)


def run(q, k, v, g, causal, scale=None, **kw):
    q, k, v, g = (x if x.is_cuda else x.to(DEV) for x in (q, k, v, g))
    B = len(kw["q_starts"]) - 1 if "q_starts" in kw else q.shape[0]
    assert splits(B, kw.get("max_q", q.shape[-3]), kw.get("max_k", k.shape[-3]), q.shape[-2], k.shape[-2]) == 0
    out, lse = dpb.attention(q, k, v, causal, scale, **kw)
    dq, dk, dv = dpb.attention_bwd(g, q, k, v, out, lse, causal, scale, **kw)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def agree(got, ref, dtype):
    torch.cuda.synchronize()
    for name in ref:
        check(name, got[name], ref[name], dtype)


@gpu
@TYPES
@CAUSAL
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_padded_full(device, shape, causal, dtype):
    q, k, v, g = make(21, *shape, dtype)
    ref = reference(q, k, v, causal, shape[-1] ** -0.5, g)
    agree(run(q, k, v, g, causal), ref, dtype)


@gpu
@TYPES
@CAUSAL
@pytest.mark.parametrize("shape", RAGGED, ids=lambda s: "x".join(map(str, s)))
def test_lengths_with_anything_behind_them(device, shape, causal, dtype):
    B, Q, K, H, G, D = shape
    q, k, v, g = make(22, *shape, dtype)
    gen = torch.Generator().manual_seed(23)
    ql = torch.randint(0, Q + 1, (B,), generator=gen, dtype=torch.int32)
    kl = torch.randint(0, K + 1, (B,), generator=gen, dtype=torch.int32)
    ql[:6] = torch.tensor([Q, Q, 0, max(Q - 3, 0), 1, Q + 9])
    kl[:6] = torch.tensor([K, 0, K, 33, -5, 1])
    ref = reference(q, k, v, causal, 0.3, g, ql, kl)
    for b in range(B):
        n, m = min(max(int(ql[b]), 0), Q), min(max(int(kl[b]), 0), K)
        for x, at in ((q, n), (g, n), (k, m), (v, m)):
            x[b, at:] = math.nan
            x[b, at:, :, ::2] = math.inf
    agree(run(q, k, v, g, causal, 0.3, q_lens=ql.to(DEV), k_lens=kl.to(DEV)), ref, dtype)


@gpu
@TYPES
@CAUSAL
@pytest.mark.parametrize("same", [True, False], ids=["self", "cross"])
def test_packed(device, same, causal, dtype):
    ql = PACKED
    kl = ql if same else [140, 3, 9, 0, 64, 1, 129, 30, 200]
    H, G, D = 16, 8, 64
    B, Q, K = len(ql), max(ql), max(kl)
    q, k, v, g = make(24, B, Q, K, H, G, D, dtype)
    ref = reference(q, k, v, causal, D ** -0.5, g, ql, kl)
    pack = lambda x, n: torch.cat([x[b, :n[b]] for b in range(B)])  # noqa: E731
    starts = lambda n: torch.tensor([sum(n[:i]) for i in range(B + 1)], dtype=torch.int32, device=DEV)  # noqa: E731
    got = run(pack(q, ql), pack(k, kl), pack(v, kl), pack(g, ql), causal, q_starts=starts(ql), k_starts=starts(kl),
              max_q=Q + 5, max_k=K + 70)
    packed = {n: tuple(pack(x, kl if n in ("dk", "dv") else ql) for x in r) for n, r in ref.items()}
    agree(got, packed, dtype)


@gpu
def test_packed_starts_out_of_range_stay_inside(device):
    q, k, v, g = (x[0].to(DEV) for x in make(25, 1, 140, 140, 32, 32, 64, BF16))
    bad = torch.tensor([-7, 70, 50, 300], dtype=torch.int32, device=DEV)
    got = run(q, k, v, g, True, q_starts=bad, k_starts=bad, max_q=140, max_k=140)
    ref = reference(q[None, :70].cpu(), k[None, :70].cpu(), v[None, :70].cpu(), True, 0.125)
    # (rows 50 to 69 lie in two sequences)
    check("out", got["out"][None, :50], tuple(x[:, :50] for x in ref["out"]), BF16)
    check("lse", got["lse"][None, :50], tuple(x[:, :50] for x in ref["lse"]), BF16)


@gpu
@TYPES
def test_strides(device, dtype):
    B, Q, K, H, G, D = 9, 133, 90, 16, 8, 64
    q, k, v, g = make(26, B, Q, K, H, G, D, dtype)
    ref = reference(q, k, v, True, D ** -0.5, g)
    assert splits(B, Q, K, H, G) == 0
    heads_first = lambda x: x.to(DEV).transpose(1, 2).contiguous().transpose(1, 2)  # noqa: E731
    tokens_first = lambda x: x.to(DEV).permute(1, 0, 2, 3).contiguous().permute(1, 0, 2, 3)  # noqa: E731

    def beside(x):
        wide = torch.full((x.shape[0], x.shape[1] + 3, x.shape[2] + 1, D + 16), math.nan, dtype=dtype, device=DEV)
        wide[:, 3:, 1:, 8:8 + D] = x.to(DEV)
        return wide[:, 3:, 1:, 8:8 + D]

    for a, b, c in ((heads_first, beside, tokens_first), (beside, tokens_first, heads_first)):
        qd, kd, vd, gd = a(q), b(k), c(v), b(g)
        out = b(torch.zeros_like(q))
        out, lse = dpb.attention(qd, kd, vd, True, out=out)
        dq, dk, dv = (f(torch.zeros_like(x)) for f, x in ((c, q), (a, k), (b, v)))
        dpb.attention_bwd(gd, qd, kd, vd, out, lse, True, dq=dq, dk=dk, dv=dv)
        agree({"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}, ref, dtype)


@gpu
def test_broadcast_inputs(device):
    """One key sequence for all, and one query row for all tokens, through strides of 0."""
    q, k, v, g = make(27, 17, 65, 100, 8, 8, 64, F32)
    q = q[:, :1].expand(-1, 65, -1, -1)
    k, v = k[:1].expand(17, -1, -1, -1), v[:1].expand(17, -1, -1, -1)
    ref = reference(q, k, v, True, 0.125, g)
    qd = q[:, :1].to(DEV).expand(-1, 65, -1, -1)
    kd, vd = (x[:1].to(DEV).expand(17, -1, -1, -1) for x in (k, v))
    agree(run(qd, kd, vd, g, True), ref, F32)


@gpu
@TYPES
def test_large_scores(device, dtype):
    """Scores far apart: the softmax picks one key; no overflow, no NaN, and the base follows."""
    q, k, v, g = make(28, 8, 140, 200, 8, 8, 64, dtype)
    q, k = q * 16, k * 16
    assert splits(8, 140, 200, 8, 8) == 0
    out, lse = dpb.attention(q.to(DEV), k.to(DEV), v.to(DEV), True, 1.0)
    ref = reference(q, k, v, True, 1.0)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    # fp32 scores of magnitude 1e4 are off by 1e-3 or so: what counts is the winner
    top = ref["lse"][0].abs().max()
    assert (lse.cpu().double() - ref["lse"][0]).abs().max() < 64 * 2.0 ** -24 * top
    sure = (out.cpu().double() - ref["out"][0]).abs().amax(-1) < 0.05
    assert sure.double().mean() > 0.95


@gpu
def test_a_nan_reaches_its_own_rows_only(device):
    q, k, v, g = make(29, 4, 270, 270, 12, 12, 64, BF16)
    q[0, 100, 1, 3] = math.nan
    q[3, 269, 11, 63] = math.nan
    assert splits(4, 270, 270, 12, 12) == 0
    out, lse = dpb.attention(q.to(DEV), k.to(DEV), v.to(DEV), True)
    bad = torch.zeros(4, 270, 12, dtype=torch.bool)
    bad[0, 100, 1] = bad[3, 269, 11] = True
    assert torch.equal(out.isnan().any(-1).cpu(), bad) and torch.equal(lse.isnan().cpu(), bad)


@gpu
@TYPES
def test_same_bits_every_run_and_on_another_stream(device, dtype):
    q, k, v, g = (x.to(DEV) for x in make(30, 4, 300, 300, 12, 12, 128, dtype))
    first = run(q, k, v, g, True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = run(q, k, v, g, True)
    side.synchronize()
    for n in first:
        assert torch.equal(first[n], again[n]), n


@gpu
def test_values_survive_a_graph(device):
    q, k, v, g = (x.to(DEV) for x in make(31, 8, 200, 200, 8, 8, 64, BF16))
    got = run(q, k, v, g, True)
    room = torch.empty(dpb.load().dpb_attention_bwd_workspace_bytes(
        dpb._attn(q, k, v, True, None, None, None, None, None, None, None)) // 4 + 4, device=DEV)

    def calls():
        dpb.attention(q, k, v, True, out=got["out"], lse=got["lse"])
        dpb.attention_bwd(g, q, k, v, got["out"], got["lse"], True, dq=got["dq"], dk=got["dk"], dv=got["dv"],
                          workspace=room)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(3):
        q.mul_(0.5)
        want = run(q, k, v, g, True)
        for x in got.values():
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for n in want:
            assert torch.equal(got[n], want[n]), (i, n)


@gpu
@TYPES
def test_rows_far_apart(device, dtype):
    """Keys 4 MiB apart: the last ones lie 5 GB behind the first."""
    B, Q, n, H, G, D = FAR
    pitch = (4 << 20) // (2 if dtype == BF16 else 4)
    q, k, v, g = make(32, *FAR, dtype)
    ref = reference(q, k, v, True, D ** -0.5, g)
    far = []
    for x in (k, v):
        room = torch.empty(pitch * (n - 1) + D, dtype=dtype, device=DEV)
        far.append(room.as_strided((1, n, 1, D), (0, pitch, D, 1)))
        far[-1].copy_(x)
    got = run(q, *far, g, True)
    # (dK and dV add up 16,640 rows: some 129, the square root, roundings of 2^-24 of the terms' magnitudes, 8e-6)
    agree(got, ref, dtype)
