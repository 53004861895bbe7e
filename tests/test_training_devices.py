"""The training operators have no plan and run on the current device: the binding makes
that the tensors' one, and refuses tensors of several. Without a GPU, with fake tensors
and a library that notes what it is called with."""
import contextlib

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2607_20652_amd import binding as dpb

pytestmark = pytest.mark.filterwarnings("ignore:Accessing the data pointer")


class Library:
    """Notes (call, current device, stream) and has every call succeed."""

    def __init__(self):
        self.calls, self.current = [], 0

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, self.current, args[-1]))
            return 2048 if name.endswith("bytes") else 1 if name.endswith("blocks") else 0
        return call


@pytest.fixture
def lib(monkeypatch):
    lib = Library()

    @contextlib.contextmanager
    def device(index):
        lib.current, was = index, lib.current
        yield
        lib.current = was

    monkeypatch.setattr(dpb, "load", lambda: lib)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: lib.current, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 1000 + index, raising=False)
    with FakeTensorMode():
        yield lib


def qkv(q="cuda:0", k="cuda:0", v="cuda:0"):
    return [torch.empty(2, 8, 4, 64, dtype=torch.bfloat16, device=d) for d in (q, k, v)]


def states(device, n=300):
    p, g = (torch.empty(n, device=device) for _ in range(2))
    return p, g, torch.empty(512, device=device), torch.empty(512, device=device)


@pytest.mark.parametrize("at", [0, 1, 3])
def test_calls_run_where_the_tensors_are(lib, at):
    dev = f"cuda:{at}"
    q, k, v = qkv(dev, dev, dev)
    out, lse = dpb.attention(q, k, v)
    dpb.attention_bwd(out, q, k, v, out, lse)
    p, g, m, w = states(dev)
    dpb.adamw_step([p], [g], m, w, step=1, lr=1.0)
    launches = [c for c in lib.calls if not c[0].endswith("blocks")]
    assert [c[0] for c in launches] == ["dpb_attention_workspace_bytes", "dpb_attention", "dpb_attention_bwd_workspace_bytes",
                                        "dpb_attention_bwd", "dpb_adamw_step"]
    assert all(current == at for _, current, _ in launches)
    assert all(stream == 1000 + at for name, _, stream in launches if not name.endswith("bytes"))
    assert lib.current == 0


@pytest.mark.parametrize("name", ["k", "v", "out", "lse", "q_lens", "k_lens", "workspace"])
def test_attention_refuses_a_tensor_of_another_device(lib, name):
    q, k, v = qkv()
    new = {"k": lambda: qkv(k="cuda:1")[1], "v": lambda: qkv(v="cuda:1")[2], "out": lambda: qkv("cuda:1")[0],
           "lse": lambda: torch.empty(2, 8, 4, device="cuda:1"), "workspace": lambda: torch.empty(4096, device="cuda:1"),
           "q_lens": lambda: torch.empty(2, dtype=torch.int32, device="cuda:1")}
    x = new.get(name, new["q_lens"])()
    args = dict(q=q, k=k, v=v) | {name: x}
    with pytest.raises(ValueError, match="device"):
        dpb.attention(**args)
    assert not [c for c in lib.calls if c[0] == "dpb_attention"]


@pytest.mark.parametrize("name", ["grad_out", "k", "v", "out", "lse", "dq", "dk", "dv", "workspace"])
def test_its_backward_refuses_a_tensor_of_another_device(lib, name):
    q, k, v = qkv()
    args = dict(grad_out=q, q=q, k=k, v=v, out=q, lse=torch.empty(2, 8, 4, device="cuda:0"))
    shape, dtype = ((4096,), torch.float32) if name == "workspace" else ((2, 8, 4), torch.float32) if name == "lse" \
        else ((2, 8, 4, 64), torch.bfloat16)
    with pytest.raises(ValueError, match="device"):
        dpb.attention_bwd(**(args | {name: torch.empty(shape, dtype=dtype, device="cuda:1")}))
    assert not [c for c in lib.calls if c[0] == "dpb_attention_bwd"]


@pytest.mark.parametrize("name", ["params", "grads", "m", "v", "master", "grad_scale"])
def test_a_step_refuses_a_tensor_of_another_device(lib, name):
    p, g, m, v = states("cuda:0")
    args = dict(params=[p, p], grads=[g, g], m=m, v=v, master=None, grad_scale=None, step=1, lr=1.0)
    x = torch.empty(1 if name == "grad_scale" else 300 if name in ("params", "grads") else 512, device="cuda:1")
    args[name] = [args[name][0], x] if name in ("params", "grads") else x
    with pytest.raises(ValueError, match="device"):
        dpb.adamw_step(**args)
    assert not [c for c in lib.calls if c[0] == "dpb_adamw_step"]
