"""ParityTransformer's modules are called as modules: hooks run, wrappers and replaced modules have their effect.
Without a GPU: the library's calls are formulas in torch, the bottleneck doubles its input."""
import pytest
import torch

from paper_2607_20652_amd import autograd as A
from paper_2607_20652_amd import binding as B
from test_around_autograd_host import plain  # noqa: F401  (a fixture)
from test_autograd_host import plain_attention, plain_attention_bwd


class Plan:
    d = 8


@pytest.fixture
def model(plain, monkeypatch):  # noqa: F811
    monkeypatch.setattr(B, "attention", torch.no_grad()(plain_attention))
    monkeypatch.setattr(B, "attention_bwd", lambda *a, **kw: tuple(t.detach() for t in plain_attention_bwd(*a, **kw)))
    monkeypatch.setattr(B, "encode", lambda plan, x: (torch.zeros(1, dtype=torch.int32), x.detach().clone()))
    monkeypatch.setattr(B, "decode", lambda plan, idx, coef, dtype: 2 * coef)
    monkeypatch.setattr(B, "decode_bwd_ex", lambda plan, idx, gu, **kw: (None, 2 * gu))
    torch.manual_seed(0)
    return A.ParityTransformer(Plan(), 11, 6, 2, 2, 16, std=0.5, normalized=False)


def tokens():
    return torch.randint(11, (3, 6), generator=torch.Generator().manual_seed(1))


def stream(model, t):
    """The model's hidden rows, addition by addition."""
    h = model.embed(t) + model.position(torch.arange(t.shape[1]).expand_as(t))
    for block in model.blocks:
        h = h + block.attention.mix(block.attention.norm(h))
        h = h + block.mlp.feed(block.mlp.norm(h).flatten(0, 1))[0].view(h.shape)
    return model.norm(h)


def near(a, b):
    return (a - b).abs().max() < 1e-5 * b.abs().max()     # (fp32 sums of 8 and 16 terms, through two blocks)


def test_hooks_run(model):
    modules = {n: m for n, m in model.named_modules() if n and not isinstance(m, torch.nn.ModuleList)}
    assert {"embed", "position", "norm", "blocks.1", "blocks.0.attention", "blocks.0.attention.norm", "blocks.1.mlp", "blocks.1.mlp.norm",
            "blocks.0.mlp.fc1"} <= set(modules)
    for call in (lambda: model.hidden(tokens()), lambda: model.loss(tokens(), tokens())[0].backward(), lambda: model(tokens()),
                 lambda: model(tokens()[:, :2], model.caches(3, 6))):
        before, after = [], []
        hooks = [m.register_forward_pre_hook(lambda *_, n=n: before.append(n)) for n, m in modules.items()]
        hooks += [m.register_forward_hook(lambda *_, n=n: after.append(n)) for n, m in modules.items()]
        call()
        assert sorted(before) == sorted(after) == sorted(modules)
        for hook in hooks:
            hook.remove()


def test_what_a_hook_gives_back_is_used(model):
    t = tokens()
    with torch.no_grad():
        hook = model.position.register_forward_hook(lambda m, a, y: torch.zeros_like(y))
        got = model.hidden(t)[0]
        hook.remove()
        model.position.weight.zero_()
        assert torch.equal(got, model.hidden(t)[0])
        # a block that leaves the stream as it was: its two terms
        hook = model.blocks[0].register_forward_hook(lambda m, a, y: ((torch.zeros_like(y[0][0]), a[0] + a[2]), y[1]))
        got = model.hidden(t)[0]
        hook.remove()
        del model.blocks[0]
        assert near(got, model.hidden(t)[0])


def test_blocks_are_the_stream_s_additions(model):
    t = tokens()
    with torch.no_grad():
        assert near(model.hidden(t)[0], stream(model, t))
        h = torch.randn(2, 5, 8)
        whole, _ = model.blocks[0](h)
        (x, rest), _ = model.blocks[0](0.25 * h, None, 0.75 * h)
        assert near(x + rest, whole)


def test_a_wrapper_around_a_block(model):
    class Wrapper(torch.nn.Module):
        def __init__(self, block):
            super().__init__()
            self.block, self.calls = block, 0

        def forward(self, *args, **kwargs):
            self.calls += 1
            return torch.utils.checkpoint.checkpoint(self.block, *args, use_reentrant=False, **kwargs)

    t = tokens()
    model.loss(t, t)[0].backward()
    want = [p.grad.clone() for p in model.parameters()]
    model.zero_grad()
    model.blocks[1] = Wrapper(model.blocks[1])
    model.loss(t, t)[0].backward()
    assert model.blocks[1].calls == 1
    assert all(torch.equal(p.grad, g) for p, g in zip(model.parameters(), want))


@pytest.mark.parametrize("where", ["attention", "mlp", "last"])
def test_another_norm_in_a_norm_s_place(model, where):
    other = torch.nn.LayerNorm(8)
    if where == "last":
        model.norm = other
    else:
        getattr(model.blocks[0], where).norm = other
    t = tokens()
    with torch.no_grad():
        assert near(model.hidden(t)[0], stream(model, t))
    model.loss(t, t)[0].backward()
    assert other.bias.grad is not None
