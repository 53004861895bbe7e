"""Embedding, norm and vocabulary loss as differentiable functions, without a GPU: the library's calls are the
same formulas in torch, so that what is tested is how the results meet autograd."""
import pytest
import torch

from paper_2607_20652_amd import autograd as A
from paper_2607_20652_amd import binding as B


def embedding(tokens, table, scale=1.0):
    live = (tokens >= 0) & (tokens < table.shape[0])
    return torch.where(live[..., None], table[torch.where(live, tokens, 0)] * scale, 0.0)


def rms_norm(x, weight, residual=None, eps=1e-6):
    total = x if residual is None else x + residual
    rstd = (total.square().mean(-1) + eps).rsqrt()
    out = total * rstd[..., None]
    return out if weight is None else out * weight, total, rstd


def cross_entropy(hidden, weight, targets, scale=1.0):
    logits = hidden @ weight.T * scale
    lse = logits.logsumexp(-1)
    live = (targets >= 0) & (targets < weight.shape[0])
    return torch.where(live, lse - logits.gather(-1, torch.where(live, targets, 0)[..., None])[..., 0], 0.0), lse


def grads(f, inputs, given):
    """Gradients of f's outputs for those of `given` that are not None."""
    with torch.enable_grad():
        x = [t.detach().requires_grad_() for t in inputs]
        outs = [(o, g) for o, g in zip(f(*x), given) if g is not None]
        return torch.autograd.grad([o for o, _ in outs], x, [g for _, g in outs], allow_unused=True)


@pytest.fixture
def plain(monkeypatch):
    off = torch.no_grad()
    monkeypatch.setattr(B, "embedding", off(embedding))
    monkeypatch.setattr(B, "embedding_bwd", lambda grad, tokens, vocab, scale=1.0: grads(
        lambda w: [embedding(tokens, w, scale)], [grad.new_zeros(vocab, grad.shape[-1])], [grad])[0])
    monkeypatch.setattr(B, "rms_norm", off(rms_norm))

    def rms_norm_bwd(grad, total, weight, rstd, grad_total=None):
        eps = (rstd.double() ** -2 - total.double().square().mean(-1)).flatten()[0].item()
        if weight is None:
            return grads(lambda z: rms_norm(z, None, None, eps)[:2], [total], [grad, grad_total])[0], None
        return grads(lambda z, w: rms_norm(z, w, None, eps)[:2], [total, weight], [grad, grad_total])

    monkeypatch.setattr(B, "rms_norm_bwd", rms_norm_bwd)
    monkeypatch.setattr(B, "cross_entropy", off(cross_entropy))

    def cross_entropy_bwd(ga, hidden, weight, targets, lse, scale=1.0, grad_lse=None, hidden_grad=True, weight_grad=True):
        dh, dw = grads(lambda h, w: cross_entropy(h, w, targets, scale), [hidden, weight], [ga, grad_lse])
        return dh if hidden_grad else None, dw if weight_grad else None

    monkeypatch.setattr(B, "cross_entropy_bwd", cross_entropy_bwd)


def randn(*shape):
    return torch.randn(*shape, dtype=torch.float64, generator=torch.Generator().manual_seed(len(shape))).requires_grad_()


def test_gradients_are_the_formulas(plain):
    t = torch.tensor([[0, 3, -1], [3, 6, 2]])
    assert torch.autograd.gradcheck(lambda w: A.embedding_layer(t, w, 1.5), (randn(6, 4),))
    x, r, w = randn(2, 3, 5), randn(2, 3, 5).detach().mul(0.5).requires_grad_(), randn(5)
    assert torch.autograd.gradcheck(lambda x, w: A.rms_norm_layer(x, w)[0], (x, w))
    assert torch.autograd.gradcheck(lambda x, w, r: A.rms_norm_layer(x, w, r), (x, w, r))
    assert torch.autograd.gradcheck(lambda x, r: A.rms_norm_layer(x, None, r), (x, r))
    h, w = randn(2, 3, 4), randn(7, 4)
    assert torch.autograd.gradcheck(lambda h, w: A.cross_entropy_layer(h, w, t, 0.7), (h, w))


def test_only_what_is_wanted(plain):
    """The sum's gradient alone passes by the norm; a frozen head costs no product; nothing comes from nothing."""
    x, r, w = randn(3, 5), randn(3, 5).detach().add(1.0).requires_grad_(), randn(5)
    _, total = A.rms_norm_layer(x, w, r)
    total.sum().backward()
    assert torch.equal(x.grad, torch.ones_like(x)) and torch.equal(r.grad, x.grad) and w.grad is None
    out, none = A.rms_norm_layer(x, w)
    assert none is None
    h, v, t = randn(3, 4), randn(7, 4).detach(), torch.tensor([1, 2, 0])
    loss, lse = A.cross_entropy_layer(h, v, t)
    (loss.mean() + 1e-2 * lse.square().mean()).backward()
    want = grads(lambda h: [(lambda a: a[0].mean() + 1e-2 * a[1].square().mean())(cross_entropy(h, v, t))], [h], [torch.ones((), dtype=torch.float64)])
    assert torch.allclose(h.grad, want[0])
    table = randn(4, 2)
    assert not A.embedding_layer(t, table.detach()).requires_grad


def test_a_second_derivative_is_an_error(plain):
    t = torch.tensor([1, 2, 0])
    for f, x in ((lambda w: A.embedding_layer(t, w).square(), randn(4, 2)), (lambda x: A.rms_norm_layer(x, None)[0].square(), randn(3, 5)),
                 (lambda h: A.cross_entropy_layer(h, randn(7, 4), t)[0].square(), randn(3, 4))):
        (first,) = torch.autograd.grad(f(x).sum() + (x ** 3).sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            first.sum().backward()


def test_rows_reach_the_library_even_and_aligned(plain, monkeypatch):
    """A slice of every sequence, a gradient joined to a number, expanded ones: copied where they have to be."""
    seen = []
    for name in ("embedding_bwd", "rms_norm", "rms_norm_bwd", "cross_entropy"):
        def note(*args, _f=getattr(B, name), **kw):
            for a in args[:2]:
                if isinstance(a, torch.Tensor) and a.is_floating_point() and a.dim() > 1:
                    B._rows(a, "rows")
                    seen.append(a.data_ptr() % 16)
            return _f(*args, **kw)
        monkeypatch.setattr(B, name, note)
    x, w, head = randn(2, 6, 4), randn(4), randn(7, 4)
    t = torch.randint(0, 7, (2, 5))
    y = A.rms_norm_layer(x[:, 1:], w, x[:, :-1])[0]
    loss = A.cross_entropy_layer(y, head, t)[0].sum()
    (joined,) = [torch.cat([w.sum()[None], A.rms_norm_layer(x, w)[0].flatten(), A.embedding_layer(t, head).flatten()])]
    (loss + (joined * torch.arange(len(joined))).sum() + A.embedding_layer(t, head).sum()).backward()
    assert len(seen) >= 8 and not any(seen)


def test_model_refuses_places_that_it_has_not(plain):
    class Plan:
        d = 8

    model = A.ParityTransformer(Plan(), 11, 6, 0, 2, 16)
    z, _ = model.hidden(torch.zeros(2, 6, dtype=torch.int64))
    assert z.shape == (2, 6, 8) and model(torch.zeros(2, 4, dtype=torch.int64), start=2).shape == (2, 4, 11)
    for tokens, start in ((7, 0), (3, 4), (1, -1)):
        with pytest.raises(ValueError):
            model(torch.zeros(2, tokens, dtype=torch.int64), start=start)
    t = torch.tensor([[1, 2, 3], [4, 5, -100]])
    loss, _ = model.loss(t.clamp(0), t)
    want = torch.nn.functional.cross_entropy(model(t.clamp(0)).flatten(0, 1), t.flatten())
    assert torch.allclose(loss, want)
    loss.backward()
    assert all(p.grad is not None for p in model.parameters())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("far", ["hidden", "weight", "both"])
def test_rows_far_apart_reach_the_loss_within_its_strides(plain, monkeypatch, dtype, far):
    """The last token of each sequence of a long batch: rows of 8 MiB and more apart, which the library does not read
    where they are, are copied; what it then gets has a workspace (a description that it refuses has none)."""
    lib, seen = B.load(), []
    for name in ("cross_entropy", "cross_entropy_bwd"):
        def note(*args, _name=name, _f=getattr(B, name), **kw):
            hidden, weight, targets = args[1:4] if _name.endswith("bwd") else args[:3]
            a, _ = B._logits(hidden, weight, targets, 0.5)
            seen.append(getattr(lib, f"dpb_{_name}_workspace_bytes")(a, B._dtype_code(hidden)))
            return _f(*args, **kw)
        monkeypatch.setattr(B, name, note)
    step = (1 << 23) // torch.empty((), dtype=dtype).element_size()
    wide = lambda n: torch.zeros(n * step, dtype=dtype).as_strided((n, 8), (step, 1))  # noqa: E731
    near = lambda n: torch.zeros(n, 8, dtype=dtype)  # noqa: E731
    h, w = (wide if far != "weight" else near)(4), (wide if far != "hidden" else near)(3)
    h.copy_(torch.randn(4, 8, generator=torch.Generator().manual_seed(0)))
    w.copy_(torch.randn(3, 8, generator=torch.Generator().manual_seed(1)))
    h, w, t = h.requires_grad_(), w.requires_grad_(), torch.tensor([0, 2, 1, 0])
    loss, lse = A.cross_entropy_layer(h, w, t, 0.5)
    (loss.sum() + lse.sum()).backward()
    assert len(seen) == 2 and all(seen)
    assert torch.equal(loss, cross_entropy(h, w, t, 0.5)[0]) and h.grad.shape == h.shape and w.grad.shape == w.shape
