"""The training operators as a model uses them: the attention sublayer against plain
torch in fp64, the cache against the whole sequence, the optimizer against
torch's AdamW, and a small Parity Transformer that learns."""
import importlib.util
import os

import pytest
import torch

from paper_2607_20652_amd import binding as dpb
from paper_2607_20652_amd.autograd import CausalAttention, ParityBlock, attention_layer
from paper_2607_20652_amd.optim import AdamW

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dpb.load()


def plain_sublayer(m, h):
    """CausalAttention in fp64 on the CPU, from its parameters."""
    x = torch.nn.functional.rms_norm(h, (h.shape[-1],), m["norm.weight"], torch.finfo(torch.float32).eps)
    return x @ m["qkv.weight"].T, x


def reference(m, h, heads, kv_heads):
    d = h.shape[-1] // heads
    y, _ = plain_sublayer(m, h)
    q, k, v = y.unflatten(-1, (-1, d)).split((heads, kv_heads, kv_heads), 2)
    k, v = (t.repeat_interleave(heads // kv_heads, 2) for t in (k, v))
    s = torch.matmul(q.transpose(1, 2), k.permute(0, 2, 3, 1)) * d ** -0.5
    n = h.shape[1]
    s = s.masked_fill(torch.ones(n, n).triu(1).bool(), float("-inf")).softmax(-1)
    return h + torch.matmul(s, v.transpose(1, 2)).transpose(1, 2).flatten(-2) @ m["out.weight"].T


@pytest.mark.parametrize("heads,kv_heads,d", [(4, 4, 64), (4, 2, 96), (6, 1, 240)])
def test_sublayer_and_its_gradients(heads, kv_heads, d):
    torch.manual_seed(0)
    layer = CausalAttention(d, heads, kv_heads, device=DEV)
    h = torch.randn(3, 70, d, device=DEV, requires_grad=True)
    g = torch.randn(3, 70, d, device=DEV)
    out = layer(h)
    out.backward(g)
    m = {n: p.detach().double().cpu().requires_grad_() for n, p in layer.named_parameters()}
    h64 = h.detach().double().cpu().requires_grad_()
    want = reference(m, h64, heads, kv_heads)
    want.backward(g.double().cpu())
    # fp32 matrix products of up to 240 terms and sums over 210 rows around the attention
    for got, ref in [(out, want), (h.grad, h64.grad)] + [(p.grad, m[n].grad) for n, p in layer.named_parameters()]:
        off, top = (got.detach().double().cpu() - ref.detach()).abs().max(), ref.detach().abs().max()
        assert float(off) < 2e-5 * float(top) + 1e-6


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_cache_gives_what_the_whole_sequence_gives(dtype):
    torch.manual_seed(1)
    layer = CausalAttention(256, 4, 2, dtype=dtype, device=DEV)
    h = torch.randn(2, 40, 256, device=DEV, dtype=dtype)
    with torch.no_grad():
        whole = layer(h)
        cache = layer.cache(2, 40)
        parts = [layer(h[:, :17], cache), layer(h[:, 17:24], cache)] + [layer(h[:, i:i + 1], cache) for i in range(24, 40)]
        with pytest.raises(ValueError):
            layer(h[:, :1], cache)
    off = (torch.cat(parts, 1) - whole).abs().max()
    # the same arithmetic in another order; in bf16 each of three roundings may fall to the other side
    assert float(off) < (1e-5 if dtype == torch.float32 else 3 * 2.0 ** -8) * float(whole.abs().max())


def test_expanded_gradients_and_lengths():
    torch.manual_seed(2)
    q, k, v = (torch.randn(2, 30, 2, 32, device=DEV, requires_grad=True) for _ in range(3))
    lens = torch.tensor([30, 11], dtype=torch.int32, device=DEV)
    attention_layer(q, k, v, True, None, lens, lens).sum().backward()     # a gradient of stride 0
    first = [t.grad.clone() for t in (q, k, v)]
    for t in (q, k, v):
        t.grad = None
    attention_layer(q, k, v, True, None, lens, lens).backward(torch.ones(2, 30, 2, 32, device=DEV))
    for a, t in zip(first, (q, k, v)):
        assert torch.equal(a, t.grad)
        assert not t.grad[1, 11:].any()


@pytest.mark.parametrize("decay", [0.0, 0.1])
def test_optimizer_against_torch(decay):
    torch.manual_seed(3)
    mine = [torch.nn.Parameter(torch.randn(s, device=DEV)) for s in ((7, 9), (300,), (64, 65), (1,))]
    theirs = [torch.nn.Parameter(p.detach().double().cpu()) for p in mine]
    a = AdamW([(p, decay) for p in mine], lr=1e-2, betas=(0.8, 0.95), eps=1e-6)
    b = torch.optim.AdamW(theirs, lr=1e-2, betas=(0.8, 0.95), eps=1e-6, weight_decay=decay)
    for step in range(5):
        for p, q in zip(mine, theirs):
            p.grad = torch.randn_like(p) * (step + 1)
            q.grad = p.grad.double().cpu()
        a.step()
        b.step()
    for p, q in zip(mine, theirs):
        # five updates of about 1e-2, each off by a few fp32 roundings of itself and of the weight
        assert (p.detach().double().cpu() - q.detach()).abs().max() < 5 * (1e-2 * 3e-6 + 4 * 2.0 ** -24)


@pytest.mark.parametrize("bits", [8, 32])
def test_optimizer_state_goes_on_where_it_was_saved(bits):
    torch.manual_seed(4)
    start = [torch.randn(50, 60, device=DEV).to(t) for t in (torch.float32, torch.bfloat16, torch.bfloat16)]
    grads = [[torch.randn_like(p) for p in start] for _ in range(4)]

    def run(params, opt, which):
        for g in which:
            for p, x in zip(params, g):
                p.grad = x
            opt.step()

    one = [torch.nn.Parameter(p.clone()) for p in start]
    opt = AdamW(one, bits=bits, weight_decay=0.01)
    run(one, opt, grads[:2])
    two = [torch.nn.Parameter(p.detach().clone()) for p in one]
    again = AdamW(two, bits=bits, weight_decay=0.01)
    again.load_state_dict(opt.state_dict())
    run(one, opt, grads[2:])
    run(two, again, grads[2:])
    assert all(torch.equal(p, q) for p, q in zip(one, two))
    other = AdamW(two[:2], bits=bits)
    with pytest.raises(ValueError):
        other.load_state_dict(opt.state_dict())
    two[0].grad = None
    with pytest.raises(ValueError):
        again.step()
    with pytest.raises(TypeError):
        AdamW([torch.nn.Parameter(torch.zeros(3, device=DEV, dtype=torch.float16))])


def test_block_is_its_two_sublayers():
    torch.manual_seed(5)
    plan = dpb.Plan(64, 12, 3, 16, 4, 8, 0)
    block = ParityBlock(plan, heads=4, d_ff=96, kv_heads=2, device=DEV, n_min=4)
    h = torch.randn(2, 33, 64, device=DEV, requires_grad=True)
    out, loss = block(h)
    (out.square().mean() + 0.05 * loss).backward()
    got = [h.grad.clone()] + [p.grad.clone() for p in block.parameters()]
    h.grad = None
    block.zero_grad()
    out2, loss2 = block.mlp(block.attention(h))
    (out2.square().mean() + 0.05 * loss2).backward()
    assert torch.equal(out, out2)
    for a, b in zip(got, [h.grad] + [p.grad for p in block.parameters()]):
        # (the variance loss adds up in an order that may change)
        assert torch.allclose(a, b, rtol=1e-4, atol=1e-6)
    assert all(x.abs().sum() > 0 for x in got)


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "parity_transformer.py")
    spec = importlib.util.spec_from_file_location("parity_transformer_example", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_a_small_parity_transformer_learns_and_goes_on():
    ex = example()
    model, losses = ex.train(120, say=lambda *_: None)
    assert losses[-1] < 0.1 * losses[0]
    x = ex.batch(4, torch.Generator().manual_seed(2))
    n = 4 * ex.LAG
    made = model.generate(x[:, :n], 12)
    assert torch.equal(made[:, :n], x[:, :n])
    with torch.no_grad():
        whole = model(made[:, :-1])[:, n - 1:].argmax(-1)
    assert (whole == made[:, n:]).double().mean() > 0.95      # a tie within rounding may fall either way
    assert (made[:, n:] == x[:, n:n + 12]).double().mean() > 0.9
