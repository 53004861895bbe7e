"""Inputs whose rows share memory, as windows over one stretch do: what their copies give, bit by bit."""
import pytest
import torch

from paper_2607_20652_amd import binding as dpb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dpb.load()


def windows(n, dim, step, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((n - 1) * step + dim, generator=g).to(DEV, dtype).as_strided((n, dim), (step, 1))


@TYPES
@pytest.mark.parametrize("step", [8, 24, 0])
@pytest.mark.parametrize("rows,dim,vocab", [(70, 64, 300), (300, 200, 1003), (4100, 328, 9000)])
def test_loss(rows, dim, vocab, step, dtype):
    h, w = windows(rows, dim, step, dtype, 1), windows(vocab, dim, 8, dtype, 2)
    t = torch.randint(-1, vocab, (rows,), device=DEV)
    ga = torch.rand(rows, device=DEV)
    got, want = (dpb.cross_entropy(x, y, t, 0.2) for x, y in ((h, w), (h.contiguous(), w.contiguous())))
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.isfinite(got[1]).all()
    got, want = (dpb.cross_entropy_bwd(ga, x, y, t, want[1], 0.2) for x, y in ((h, w), (h.contiguous(), w.contiguous())))
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.isfinite(a).all() for a in got)


@TYPES
@pytest.mark.parametrize("step", [8, 3, 0])
def test_embedding_and_norm(step, dtype):
    table, x, r, go = (windows(90, 64, step, dtype, i) for i in range(4))
    t = torch.randint(-1, 90, (90,), device=DEV)
    assert torch.equal(dpb.embedding(t, table), dpb.embedding(t, table.contiguous()))
    assert torch.equal(dpb.embedding_bwd(go, t, 90), dpb.embedding_bwd(go.contiguous(), t, 90))
    w = torch.rand(64, device=DEV)
    out, total, rstd = dpb.rms_norm(x, w, r)
    want = dpb.rms_norm(x.contiguous(), w, r.contiguous())
    assert torch.equal(total, want[1])
    if step % 8 == 0:    # (else the rows are read by elements, their squares added up in another order)
        assert torch.equal(out, want[0]) and torch.equal(rstd, want[2])
    got, want = (dpb.rms_norm_bwd(g, total, w, rstd, g) for g in (go, go.contiguous()))
    assert step % 8 or all(torch.equal(a, b) for a, b in zip(got, want))
