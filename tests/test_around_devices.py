"""Embedding, norm and vocabulary loss run on their tensors' device, and refuse tensors of several. Without a GPU,
with fake tensors and a library that notes what it is called with."""
import pytest
import torch

from paper_2607_20652_amd import binding as dpb
from test_training_devices import lib  # noqa: F401  (a fixture)

pytestmark = pytest.mark.filterwarnings("ignore:Accessing the data pointer")


def parts(d):
    def make(*shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device=d)
    rows, f = make(2, 8, 64), torch.float32
    return {"tokens": make(2, 8, dtype=torch.int64), "targets": make(2, 8, dtype=torch.int64), "table": make(100, 64), "weight": make(100, 64),
            "grad_out": rows, "x": rows, "residual": make(2, 8, 64), "out": make(2, 8, 64), "total": make(2, 8, 64), "hidden": rows,
            "rstd": make(2, 8, dtype=f), "lse": make(2, 8, dtype=f), "loss": make(2, 8, dtype=f), "grad_loss": make(2, 8, dtype=f),
            "grad_lse": make(2, 8, dtype=f), "grad_total": make(2, 8, 64), "dx": make(2, 8, 64), "dhidden": make(2, 8, 64),
            "dweight": make(100, 64), "workspace": make(4096, dtype=f), "row": make(64)}


CALLS = {   # call: (its tensors, the rest)
    "embedding": (["tokens", "table", "out"], {}),
    "embedding_bwd": (["grad_out", "tokens", "dweight", "workspace"], {"vocab": 100}),
    "rms_norm": (["x", "weight", "residual", "out", "total", "rstd"], {}),
    "rms_norm_bwd": (["grad_out", "total", "weight", "rstd", "grad_total", "dx", "dweight", "workspace"], {}),
    "cross_entropy": (["hidden", "weight", "targets", "loss", "lse", "workspace"], {}),
    "cross_entropy_bwd": (["grad_loss", "hidden", "weight", "targets", "lse", "grad_lse", "dhidden", "dweight", "workspace"], {}),
}


def arguments(call, d):
    names, rest = CALLS[call]
    p = parts(d)
    norm = call.startswith("rms_norm")
    return {n: p["row" if norm and n in ("weight", "dweight") else n] for n in names} | rest


@pytest.mark.parametrize("at", [0, 1, 3])
@pytest.mark.parametrize("call", CALLS)
def test_calls_run_where_the_tensors_are(lib, call, at):  # noqa: F811
    getattr(dpb, call)(**arguments(call, f"cuda:{at}"))
    assert [c[0] for c in lib.calls if not c[0].endswith("bytes")] == [f"dpb_{call}"]
    assert all(current == at for _, current, _ in lib.calls)     # the workspace's size too: it goes by the device's units
    assert all(stream == 1000 + at for name, _, stream in lib.calls if not name.endswith("bytes"))
    assert lib.current == 0


@pytest.mark.parametrize("call,name", [(c, n) for c, (names, _) in CALLS.items() for n in names])
def test_a_tensor_of_another_device_is_refused(lib, call, name):  # noqa: F811
    args = arguments(call, "cuda:0") | {name: arguments(call, "cuda:1")[name]}
    with pytest.raises(ValueError, match="device"):
        getattr(dpb, call)(**args)
    assert not [c for c in lib.calls if c[0] == f"dpb_{call}"]
