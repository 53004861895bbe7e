"""Masters follow parameters that somebody else changed between two steps, and keep what
bf16 cannot hold of those that nobody did."""
import pytest
import torch

from paper_2607_20652_amd import binding as dpb
from paper_2607_20652_amd.optim import AdamW

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dpb.load()


def model(seed):
    torch.manual_seed(seed)
    return torch.nn.Sequential(torch.nn.Linear(20, 30), torch.nn.Linear(30, 7)).to(DEV, BF16)


def step(opt, m, size=1.0):
    for p in m.parameters():
        p.grad = torch.full_like(p, size)
    opt.step()


@pytest.mark.parametrize("bits", [8, 32])
def test_a_model_that_is_loaded_stays_loaded(bits):
    m, other = model(0), model(1)
    opt = AdamW(m.parameters(), lr=1e-3, bits=bits)
    m.load_state_dict(other.state_dict())                  # before the first step
    step(opt, m)
    for p, q in zip(m.parameters(), other.parameters()):
        assert (p - q).abs().max() < 2e-3 + 2.0 ** -8
    step(opt, m)
    m.load_state_dict(other.state_dict())                  # and between two
    opt.lr = 0.0
    step(opt, m)
    for p, q in zip(m.parameters(), other.parameters()):
        assert torch.equal(p, q)


def test_what_nobody_changed_keeps_its_low_bits():
    p = torch.nn.Parameter(torch.ones(600, device=DEV, dtype=BF16))
    q = torch.nn.Parameter(torch.ones(5, device=DEV, dtype=BF16))
    opt = AdamW([q, p], lr=1e-4)
    for _ in range(3):
        p.grad, q.grad = torch.ones_like(p), torch.ones_like(q)
        opt.step()
    g = opt.groups[0]
    was = g["master"].clone()
    assert bool((p == 1).all()) and bool((was[256:856] < 1).all())     # too little for bf16
    with torch.no_grad():
        p[100:110] = 3.0
    p.grad, q.grad = torch.zeros_like(p), torch.zeros_like(q)
    opt.lr = 0.0
    opt.step()
    same = torch.ones(856, dtype=torch.bool, device=DEV)
    same[356:366] = False
    assert torch.equal(g["master"][:856][same], was[:856][same]) and bool((g["master"][356:366] == 3).all())
    assert bool((p[100:110] == 3).all()) and bool((p[110:] == 1).all())
    # a write of what was there already loses nothing either
    with torch.no_grad():
        p.copy_(p.clone())
    opt.step()
    assert torch.equal(g["master"][:856][same], was[:856][same])


def test_writes_through_data_are_taken_over_when_told():
    p = torch.nn.Parameter(torch.ones(8, device=DEV, dtype=BF16))
    opt = AdamW([p], lr=0.0)
    p.grad = torch.ones_like(p)
    opt.step()
    p.data.fill_(5.0)
    opt.take_parameters()
    opt.step()
    assert bool((p == 5).all())


def test_a_checkpoint_of_model_and_optimizer_goes_on_to_the_bit():
    one, two = model(2), model(3)
    a, b = (AdamW(m.parameters(), lr=1e-3, bits=8) for m in (one, two))
    for _ in range(3):
        step(a, one, 0.3)
    two.load_state_dict(one.state_dict())
    b.load_state_dict(a.state_dict())
    for _ in range(2):
        step(a, one, -0.2)
        step(b, two, -0.2)
    assert all(torch.equal(x, y) for x, y in zip(one.parameters(), two.parameters()))
    assert torch.equal(a.groups[0]["master"], b.groups[0]["master"])
