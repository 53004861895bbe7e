"""An optimizer step over memory that overlaps is refused before anything is enqueued: two
workgroups of one launch would read and write the same weights."""
import ctypes

import pytest
import torch

from paper_2607_20652_amd import binding as dpb
from paper_2607_20652_amd.optim import AdamW

EINVAL = -1
MB = 1 << 20


def step(params, grads, sizes, m=300 * MB, v=400 * MB, scales=None, master=None, gs=None, bits=32, pt=0, gt=0):
    n = len(sizes)
    o = dpb._AdamW(1e-3, 0.9, 0.99, 1e-8, 1, 0)
    return dpb.load().dpb_adamw_step(ctypes.byref(o), n, (ctypes.c_void_p * n)(*params), (ctypes.c_void_p * n)(*grads),
                                     (ctypes.c_int64 * n)(*sizes), None, pt, gt, bits, m, v, scales, master, gs, None)


P, G = (1 * MB, 2 * MB), (10 * MB, 11 * MB)


@pytest.mark.parametrize("bad", [
    dict(params=(MB, MB)),                                     # the same tensor twice
    dict(params=(MB, MB + 1196)),                              # a view's last element is another's first
    dict(params=(MB + 1196, MB)),
    dict(params=(2 * MB, MB), sizes=(1, MB // 4 + 1)),         # one inside another
    dict(params=(MB, MB + 598), pt=1),                         # bf16: 600 bytes each
    dict(grads=(MB, 11 * MB)),                                 # a gradient that is the weight
    dict(grads=(10 * MB, 2 * MB + 1196)),
    dict(grads=(10 * MB, 2 * MB - 598), gt=1),
    dict(v=300 * MB),                                          # both states at one place
    dict(m=400 * MB + 4 * 1008), dict(m=MB), dict(v=10 * MB),
    dict(master=300 * MB), dict(master=2 * MB), dict(gs=2 * MB + 1196), dict(gs=400 * MB + 4 * 1020),
    dict(bits=8, scales=300 * MB + 1008), dict(bits=8, scales=MB + 1184), dict(bits=8, scales=500 * MB, gs=500 * MB + 28),
])
def test_what_is_written_may_not_overlap(bad):
    assert step(**({"params": P, "grads": G, "sizes": (300, 300)} | bad)) == EINVAL


def test_many_tensors():
    n = 300
    params = [MB + 4 * i * 7 for i in range(n)]
    assert step([*params[:-1], params[5]], [64 * MB] * n, [7] * n) == EINVAL


def test_a_parameter_given_twice():
    p, q = (torch.nn.Parameter(torch.zeros(4)) for _ in range(2))
    with pytest.raises(ValueError, match="twice"):
        AdamW([p, q, p])
    with pytest.raises(ValueError, match="twice"):
        AdamW([(p, 0.1), (q, 0.0), (p, 0.0)])


@pytest.mark.gpu
def test_neighbours_and_shared_gradients_are_fine():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    room = torch.ones(1 + 300 + 7 + 256, device="cuda")
    one, two, three = room[1:301], room[301:308], room[308:]
    g = torch.full((300,), 0.5, device="cuda")
    params, grads = [two, three, one], [g[:7], g[:256], g]     # end to end, and gradients that share memory
    m, v, scales, _ = dpb.adamw_state(params, 8)
    dpb.adamw_step(params, grads, m, v, scales, step=1, lr=0.25)
    assert float(room[0]) == 1.0 and bool(((room[1:] - 0.75).abs() < 1e-5).all())
    for bad in ([one, one], [room[1:301], room[300:600]], [one, room[250:260]]):
        grads = [torch.zeros_like(x) for x in bad]
        m, v, _, _ = dpb.adamw_state(bad)
        with pytest.raises(dpb.DPBError) as e:
            dpb.adamw_step(bad, grads, m, v, step=1, lr=1.0)
        assert e.value.status == EINVAL
    with pytest.raises(dpb.DPBError):
        dpb.adamw_step([one], [one], *dpb.adamw_state([one])[:2], step=1, lr=1.0)
    assert float(room[0]) == 1.0 and bool(((room[1:] - 0.75).abs() < 1e-5).all())
