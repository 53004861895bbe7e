"""How far a NaN in a place that a causal mask hides can reach: as far as the header says, in
the kernel of few rows, in the one of tiles, and in both kernels of the backward."""
import math

import pytest
import torch

from paper_2607_20652_amd import binding as dpb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BEFORE, BEHIND = 95, 62
# B, Q, K, H, G, D: few rows, tiles; K - Q moves the keys' tiles against the rows'
SHAPES = [(1, 300, 333, 2, 2, 64), (1, 31, 400, 2, 1, 128), (1, 290, 290, 2, 2, 96), (13, 300, 333, 4, 4, 64),
          (9, 290, 355, 16, 8, 128), (13, 300, 299, 4, 4, 32)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dpb.load()


def make(shape, dtype):
    B, Q, K, H, G, D = shape
    gen = torch.Generator().manual_seed(50)
    return [torch.randn(B, n, h, D, generator=gen).to(dtype).to(DEV) for n, h in ((Q, H), (K, G), (K, G), (Q, H))]


def bad_rows(x):
    """[tokens, heads] of the first sequence: something there is not finite."""
    return (~torch.isfinite(x[0].float())).any(-1).cpu()


@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_in_the_forward(shape, dtype, value):
    B, Q, K, H, G, D = shape
    first = K - Q                                  # query i sees keys up to i + first
    for key in sorted({K - 1, K - 64, K - 65, (K + first) // 2, max(first + 1, K - 130)} & set(range(max(first + 1, 0), K))):
        sees = torch.arange(Q) >= key - first
        for name in ("k", "v"):
            q, k, v, _ = make(shape, dtype)
            {"k": k, "v": v}[name][0, key, 0, 5] = value
            out, lse = dpb.attention(q, k, v, True)
            bad = bad_rows(out)
            mine = torch.arange(H) // (H // G) == 0
            assert not bad[:, ~mine].any() and torch.isfinite(out[1:]).all()
            if name == "v" or math.isnan(value):
                assert bad[sees][:, mine].all()
            reach = BEFORE if name == "v" else 0
            assert not bad[torch.arange(Q) < key - first - reach].any(), (name, key)
            if name == "v":
                assert not lse.isnan().any() and not (lse == math.inf).any()      # (-inf: a row that sees no key)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_in_the_backward(shape, dtype):
    B, Q, K, H, G, D = shape
    first = K - Q
    mine_k, mine_q = torch.arange(G) == 0, torch.arange(H) // (H // G) == 0
    q, k, v, g = make(shape, dtype)
    out, lse = dpb.attention(q, k, v, True)
    rows, keys = torch.arange(Q), torch.arange(K)
    for at in (K - 1, K - 70, max(first + 1, K - 140)):
        for name in ("k", "v"):
            x = {"k": k.clone(), "v": v.clone()}
            x[name][0, at, 0, 7] = math.nan
            dq, dk, dv = dpb.attention_bwd(g, q, x["k"], x["v"], out, lse, True)
            bad = bad_rows(dq)
            assert bad[rows >= at - first][:, mine_q].all() and not bad[rows < at - first - BEFORE].any() and not bad[:, ~mine_q].any()
            assert torch.isfinite(dq[1:]).all() and torch.isfinite(dk[1:]).all() and torch.isfinite(dv[1:]).all()
    for at in (0, Q // 2, Q - 1):
        for name in ("q", "g", "out", "lse"):
            x = {"q": q.clone(), "g": g.clone(), "out": out.clone(), "lse": lse.clone()}
            if name == "lse":
                x["lse"][0, at, 0] = math.nan
            else:
                x[name][0, at, 0, 7] = math.nan
            dq, dk, dv = dpb.attention_bwd(x["g"], x["q"], k, v, x["out"], x["lse"], True)
            sees = at + first                       # its last key
            bad = bad_rows(dq)
            if sees >= 0:
                assert bad[at, 0]
            bad[at, 0] = False
            assert not bad.any(), (name, at)
            for d in (dk, dv):
                bad = bad_rows(d)
                assert not bad[keys > sees + BEHIND].any() and not bad[:, ~mine_k].any(), (name, at)
            if sees >= 0:
                assert bad_rows(dk)[:sees + 1, 0].all(), (name, at)
