"""The differentiable functions without a GPU: the library's calls are replaced by the same
formulas in torch, so that what is tested is how the results meet autograd."""
import math

import pytest
import torch

from paper_2607_20652_amd import autograd as A
from paper_2607_20652_amd import binding as B


def plain_attention(q, k, v, causal=False, scale=None, q_lens=None, k_lens=None):
    k, v = (x.repeat_interleave(q.shape[2] // x.shape[2], 2) for x in (k, v))
    s = torch.einsum("bihd,bjhd->bhij", q, k) * (q.shape[-1] ** -0.5 if scale is None else scale)
    if causal:
        n, m = s.shape[-2:]
        s = s.masked_fill(torch.arange(m) > torch.arange(n)[:, None] + m - n, -math.inf)
    return torch.einsum("bhij,bjhd->bihd", s.softmax(-1), v), s.logsumexp(-1).transpose(1, 2)


def plain_attention_bwd(grad, q, k, v, out, lse, causal=False, scale=None, q_lens=None, k_lens=None):
    with torch.enable_grad():
        x = [t.detach().requires_grad_() for t in (q, k, v)]
        return torch.autograd.grad(plain_attention(*x, causal, scale)[0], x, grad)


@pytest.fixture
def plain(monkeypatch):
    """The calls of attention as they are without a graph (the library records none)."""
    monkeypatch.setattr(B, "attention", torch.no_grad()(plain_attention))
    monkeypatch.setattr(B, "attention_bwd", lambda *a, **kw: tuple(t.detach() for t in plain_attention_bwd(*a, **kw)))


def qkv(dtype=torch.float64):
    g = torch.Generator().manual_seed(0)
    return [torch.randn(2, 5, h, 8, generator=g, dtype=dtype).requires_grad_() for h in (4, 2, 2)]


def test_gradients_are_the_formulas(plain):
    q, k, v = qkv()
    assert torch.autograd.gradcheck(lambda *x: A.attention_layer(*x, True), (q, k, v))


def test_a_second_derivative_through_attention_is_an_error(plain):
    """A gradient penalty whose loss has another path to q: without the error it lacked attention's part."""
    q, k, v = qkv()
    (first,) = torch.autograd.grad((A.attention_layer(q, k, v, True) ** 2).sum() + (q ** 3).sum(), q, create_graph=True)
    want = plain_attention_bwd(2 * plain_attention(q, k, v, True)[0].detach(), q, k, v, None, None, True)[0] + 3 * q ** 2
    assert torch.allclose(first, want)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        first.square().sum().backward()


def test_a_second_derivative_through_the_bottleneck_is_an_error(monkeypatch):
    """A bottleneck that doubles its input, whose gradient is not differentiable either."""
    class Plan:
        pass

    monkeypatch.setattr(B, "encode", lambda plan, x: (torch.zeros(1, dtype=torch.int32), x.detach().clone()))
    monkeypatch.setattr(B, "decode", lambda plan, idx, coef, dtype: 2 * coef)
    monkeypatch.setattr(B, "decode_bwd_ex", lambda plan, idx, gu, **kw: (None, 2 * gu.detach()))
    x = torch.randn(3, 4, requires_grad=True)
    y, _ = A.dpb_layer(x, Plan(), normalized=False)
    (first,) = torch.autograd.grad((y ** 2).sum() + (x ** 3).sum(), x, create_graph=True)
    assert torch.allclose(first, 8 * x + 3 * x ** 2)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        first.sum().backward()


def test_gradients_that_start_anywhere_reach_the_library_aligned(plain, monkeypatch):
    """The result joined to a single number: its gradient is contiguous, four bytes into the whole's."""
    seen, bwd = [], B.attention_bwd

    def note(grad, *args):
        seen.append((grad.data_ptr() % 16, grad.is_contiguous()))
        return bwd(grad, *args)

    monkeypatch.setattr(B, "attention_bwd", note)
    w = torch.randn(1 + 2 * 5 * 4 * 8)
    q, k, v = qkv(torch.float32)
    (torch.cat([q.sum()[None], A.attention_layer(q, k, v, True).flatten()]) * w).sum().backward()
    x = [t.detach().clone().requires_grad_() for t in (q, k, v)]
    ((A.attention_layer(*x, True).flatten() * w[1:].clone()).sum() + x[0].sum() * w[0]).backward()
    assert seen == [(0, True)] * 2
    for a, b in zip((q, k, v), x):
        assert torch.allclose(a.grad, b.grad)


@pytest.mark.parametrize("cached", [False, True], ids=["", "cache"])
def test_sublayer_under_autocast(monkeypatch, cached):
    """The projection is bf16 there and the cache fp32, as the weights are."""
    def calls(q, k, v, *args):
        assert q.dtype == k.dtype == v.dtype
        out, lse = plain_attention(q, k, v, *args)
        return out, lse.float()

    monkeypatch.setattr(B, "attention", calls)
    torch.manual_seed(0)
    layer = A.CausalAttention(32, 4, 2)
    h = torch.randn(2, 6, 32)
    with torch.no_grad():
        want = layer(h)
        with torch.autocast("cpu", torch.bfloat16):
            if cached:
                cache = layer.cache(2, 6)
                got = torch.cat([layer(h[:, :4], cache), layer(h[:, 4:5], cache), layer(h[:, 5:], cache)], 1)
            else:
                got = layer(h)
    # three roundings to bf16 of values of about 1
    assert (got.float() - want).abs().max() < 3 * 2.0 ** -8 * want.abs().max()
