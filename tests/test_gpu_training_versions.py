"""What the training operators write in place is known to autograd: a graph that saved a
tensor before it was written cannot be gone through afterwards."""
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


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [8, 32])
def test_a_step_between_forward_and_backward_is_an_error(bits, dtype):
    torch.manual_seed(0)
    w = torch.nn.Parameter(torch.randn(32, 32, device=DEV, dtype=dtype))
    x = torch.randn(4, 32, device=DEV, dtype=dtype)
    opt = AdamW([w], bits=bits)
    for _ in range(2):                           # forward, backward, step: as it should be
        opt.zero_grad()
        torch.tanh(x @ w @ w).sum().backward()
        opt.step()
    late = torch.tanh(x @ w @ w).sum()
    opt.step()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        late.backward()


def test_states_and_masters_have_new_versions():
    p = [torch.zeros(300, device=DEV, dtype=torch.bfloat16)]
    g = [torch.ones(300, device=DEV, dtype=torch.bfloat16)]
    m, v, scales, master = dpb.adamw_state(p, 8, True)
    written, read = [*p, m, v, scales, master], g
    before = [t._version for t in written + read]
    dpb.adamw_step(p, g, m, v, scales, master, step=1, lr=1e-3)
    assert [t._version - b for t, b in zip(written + read, before)] == [1] * len(written) + [0]
    with pytest.raises(dpb.DPBError):
        dpb.adamw_step(p, g, m, v, scales, master, step=0, lr=1e-3)
    assert p[0]._version == before[0] + 1        # nothing was written


def test_outputs_that_are_given():
    q, k, v = (torch.randn(1, 40, 2, 32, device=DEV) for _ in range(3))
    out, lse, w = torch.empty_like(q), torch.empty(1, 40, 2, device=DEV), torch.ones_like(q, requires_grad=True)
    late = (out * w).sum()
    dpb.attention(q, k, v, out=out, lse=lse)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        late.backward()
    grads = [torch.empty_like(q) for _ in range(3)]
    before = [t._version for t in grads]
    dpb.attention_bwd(v, q, k, v, out, lse, dq=grads[0], dv=grads[2])
    assert [t._version - b for t, b in zip(grads, before)] == [1, 0, 1]
    assert [t._version for t in (q, k, v)] == [0, 0, 0]


def test_inference_tensors_have_no_versions():
    with torch.inference_mode():
        p, g = [torch.ones(10, device=DEV)], [torch.ones(10, device=DEV)]
        m, v, _, _ = dpb.adamw_state(p)
        dpb.adamw_step(p, g, m, v, step=1, lr=0.5)
        q = torch.randn(1, 8, 2, 16, device=DEV)
        out = torch.full_like(q, 9.0)
        dpb.attention(q, q, q, out=out)
    assert bool(((p[0] - 0.5).abs() < 1e-5).all()) and not bool((out == 9.0).any())
