"""Embedding and the gradient of its table against fp64: tokens that repeat, that no row is for, tables and
gradients of all alignments, more rows than are ordered at once, the same bits every time."""
import pytest
import torch

import around_util as R
from paper_2607_20652_amd import binding as dpb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dpb.load()


def tokens_of(kind, n, vocab, g):
    if kind == "all":          # some outside the table
        return torch.randint(-2, vocab + 2, (n,), generator=g)
    if kind == "one":
        return torch.full((n,), vocab // 2)
    if kind == "none":
        return torch.where(torch.arange(n) % 2 == 0, -100, vocab)
    if kind == "cycle":
        return torch.arange(n) % vocab
    if kind == "edges":        # the long rows' ends fall on, before and behind 64 places
        sizes = [64, 65, 63, 1, 128, 127, 66, 2, 300]
        return torch.cat([torch.full((k,), i % vocab) for i, k in enumerate(sizes)])[:n][torch.randperm(min(n, sum(sizes)), generator=g)]
    u = torch.rand(n, generator=g, dtype=torch.float64)
    return (torch.exp(u * torch.log(torch.tensor(vocab + 1.0))) - 1).long().clamp(0, vocab - 1)


CASES = [  # tokens, vocab, dim, kind
    (1, 1, 1, "one"), (5, 3, 7, "all"), (64, 10, 64, "one"), (65, 10, 64, "one"), (816, 9, 40, "edges"), (1023, 50, 72, "all"),
    (1025, 1024, 100, "cycle"), (3000, 50304, 128, "text"), (5000, 777, 1000, "text"), (4097, 2000, 33, "one"),
    (300, 1025, 8, "none"), (2049, 70000, 16, "text"), (20000, 24, 520, "all"), (1000, 3_000_000, 4, "all"),
    # more than are ordered out of the tokens themselves: binned
    (16385, 50304, 64, "text"), (17000, 9, 16, "one"), (40000, 2000, 24, "cycle"), (33000, 3_000_000, 4, "text"), (70001, 1025, 8, "all"),
    (16384, 700, 40, "text"), (20000, 1025, 8, "none"),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,dim,kind", CASES)
def test_lookup_and_gradient(n, vocab, dim, kind, dtype):
    g = torch.Generator().manual_seed(n + vocab)
    t = tokens_of(kind, n, vocab, g).to(DEV)
    table = torch.randn(vocab, dim, generator=g).to(DEV, dtype)
    out = dpb.embedding(t, table, scale=1.7)
    live = (t >= 0) & (t < vocab)
    want = torch.where(live[:, None], (table[torch.where(live, t, 0)].float() * 1.7), 0.0).to(dtype)
    assert torch.equal(out, want)
    assert torch.equal(dpb.embedding(t.int(), table), torch.where(live[:, None], table[torch.where(live, t, 0)], torch.zeros((), dtype=dtype, device=DEV)))
    grad = torch.randn(len(t), dim, generator=g).to(DEV, dtype)
    dw = dpb.embedding_bwd(grad, t, vocab, scale=0.3)
    R.check("dweight", dw, *R.embedding_bwd(grad, t, vocab, 0.3))
    assert torch.equal(dw, dpb.embedding_bwd(grad, t.int(), vocab, scale=0.3))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("step,offset", [(8, 0), (0, 8), (3, 1), (1, 0)])
def test_rows_that_start_anywhere(step, offset, dtype):
    torch.manual_seed(0)
    wide = torch.randn(60, 64 + step + offset, device=DEV).to(dtype)
    table = wide[:, offset:offset + 64]
    t = torch.randint(0, 60, (4, 33), device=DEV)
    assert torch.equal(dpb.embedding(t, table), table[t])
    big = torch.randn(4 * 33, 64 + step + offset, device=DEV).to(dtype)
    grad = big.view(4, 33, -1)[..., offset:offset + 64]
    assert torch.equal(dpb.embedding_bwd(grad, t, 60), dpb.embedding_bwd(grad.contiguous(), t, 60))


def test_expanded_gradient_and_what_is_not_finite():
    t = torch.tensor([3, 1, 3, 0, 3], device=DEV)
    ones = torch.ones(1, 1, device=DEV).expand(5, 16)
    with pytest.raises(ValueError):
        dpb.embedding_bwd(ones, t, 4)                       # contiguous along its last dimension
    row = torch.arange(16.0, device=DEV).expand(5, 16)      # one row for all
    assert torch.equal(dpb.embedding_bwd(row, t, 4), torch.tensor([1.0, 1, 0, 3], device=DEV)[:, None] * row[0])
    g = torch.randn(5, 16, device=DEV)
    g[1, 2] = float("nan")
    g[0, 3] = float("inf")
    dw = dpb.embedding_bwd(g, t, 4)
    assert dw[1].isnan().sum() == 1 and dw[3].isinf().sum() == 1 and torch.isfinite(dw[0]).all() and not dw[2].any()


def test_sums_keep_their_order_and_bits():
    g = torch.Generator().manual_seed(9)
    t = tokens_of("text", 30000, 500, g).to(DEV)
    grad = torch.randn(30000, 256, generator=g).to(DEV)
    first = dpb.embedding_bwd(grad, t, 500)
    for _ in range(3):
        assert torch.equal(first, dpb.embedding_bwd(grad, t, 500))


def test_given_outputs_and_nothing_to_do():
    t = torch.zeros(0, dtype=torch.int64, device=DEV)
    table = torch.randn(7, 24, device=DEV)
    assert dpb.embedding(t, table).shape == (0, 24)
    dw = torch.full((7, 24), 3.0, device=DEV)
    assert dpb.embedding_bwd(torch.zeros(0, 24, device=DEV), t, 7, dweight=dw) is dw and not dw.any()
    assert dpb.embedding_bwd(torch.zeros(3, 24, device=DEV), torch.zeros(3, dtype=torch.int64, device=DEV), 0).shape == (0, 24)
    out = torch.empty(2, 24, device=DEV)
    version = out._version
    assert dpb.embedding(torch.tensor([5, 9], device=DEV), table, out=out) is out and out._version > version
    assert torch.equal(out[0], table[5]) and not out[1].any()
    assert dpb.embedding(torch.tensor(4, device=DEV), table).shape == (24,)


def test_an_empty_table_gives_zeros():
    assert not dpb.embedding(torch.tensor([0, 1], device=DEV), torch.empty(0, 8, device=DEV)).any()
