"""A step that is refused changes nothing: not the parameters and states of the types
before the one at fault, and not the count of steps."""
import copy
import math

import pytest
import torch

from paper_2607_20652_amd import binding as dpb
from paper_2607_20652_amd.optim import AdamW

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dpb.load()


def params():
    gen = torch.Generator().manual_seed(1)
    return [torch.nn.Parameter(torch.randn(n, generator=gen).to(t).to(DEV)) for n, t in
            ((300, torch.float32), (40, torch.float32), (500, torch.bfloat16), (7, torch.bfloat16))]


def give_gradients(ps):
    gen = torch.Generator().manual_seed(2)
    for p in ps:
        p.grad = torch.randn(p.shape, generator=gen).to(p.dtype).to(DEV)


def lacking(ps):
    ps[3].grad = None


def of_another_device(ps):
    ps[2].grad = None
    ps[2].data = ps[2].data.cpu()
    ps[2].grad = torch.zeros(500, dtype=torch.bfloat16)


def not_contiguous(ps):
    ps[2].data = torch.stack([ps[2].data, ps[2].data], 1)[:, 0]


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("fault", [lacking, not_contiguous, of_another_device])
def test_nothing_changes_before_an_error(fault, bits):
    ps = params()
    opt = AdamW(ps, lr=0.1, bits=bits)
    give_gradients(ps)
    opt.step()
    fault(ps)
    before = [p.detach().clone() for p in ps]
    state = copy.deepcopy(opt.state_dict())
    with pytest.raises(ValueError):
        opt.step()
    assert opt.steps == 1
    assert all(torch.equal(a, b) for a, b in zip(ps, before))
    for now, was in zip(opt.state_dict()["groups"], state["groups"]):
        for k in now:
            assert now[k] is None and was[k] is None or torch.equal(now[k].view(torch.uint8), was[k].view(torch.uint8)), k


def test_the_step_after_a_refused_one_is_the_next():
    one, two = params(), params()
    a, b = AdamW(one, lr=0.1, bits=8), AdamW(two, lr=0.1, bits=8)
    give_gradients(one)
    give_gradients(two)
    one[3].grad = None
    with pytest.raises(ValueError):
        a.step()
    give_gradients(one)
    a.lr = math.nan
    with pytest.raises(dpb.DPBError):
        a.step()
    a.lr = 0.1
    for _ in range(2):
        a.step()
        b.step()
    assert a.steps == b.steps == 2
    assert all(torch.equal(p, q) for p, q in zip(one, two))
