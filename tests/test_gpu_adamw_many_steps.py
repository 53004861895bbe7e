"""8-bit optimizer states over thousands of steps, against 32-bit ones of the same gradients.

u = sqrt(v) is rounded up or down with its mean kept, and v is its square, so every
rounding adds its variance to v.  Where that settles, for independent normal gradients of
one size: in a step u moves by d = r (g^2 - u^2) / (2 u), r = 1 - beta2, far less than the
distance h of its neighbours, so it goes to one of them with probability |d| / h. The
drift is -r (u - sqrt(v)) near sqrt(v) and the mean square of a move E|d| h, so that u
scatters with the relative variance
    s^2 = (h / u) E|g^2 / v - 1| / 4,    E|g^2 / v - 1| = 4 phi(1) = 0.968 (phi: the normal density),
whatever beta2 is: with h / u from 1/16 to 1/8, s is 12.3 to 17.4%.  No mean move,
E[(v - u^2) / u] = 0, then gives E[u^2] = v (1 + s^2)^2: 3.0 to 6.1% above v.
The 32-bit v scatters by itself by r (relative variance of v; a quarter of it in u)."""
import pytest
import torch

from paper_2607_20652_amd import binding as dpb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
N = 1 << 16


@pytest.mark.parametrize("beta2,steps", [(0.99, 1500), (0.999, 8000)])
def test_where_the_states_settle(beta2, steps):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gen = torch.Generator(device=DEV).manual_seed(11)
    # blocks of different sizes; within a block one
    size = torch.exp(torch.randn(N // 256, 1, device=DEV, generator=gen)).expand(-1, 256).reshape(-1)
    p8, p32 = [torch.zeros(N, device=DEV)], [torch.zeros(N, device=DEV)]
    s8, s32 = dpb.adamw_state(p8, 8), dpb.adamw_state(p32, 32)
    for step in range(1, steps + 1):
        g = [torch.randn(N, device=DEV, generator=gen) * size]
        kw = dict(step=step, lr=0.0, betas=(0.9, beta2))
        dpb.adamw_step(p8, g, *s8[:3], seed=step, **kw)
        dpb.adamw_step(p32, g, *s32[:2], **kw)
    each = s8[2].double().repeat_interleave(256, 0)
    m8, u8 = s8[0].double() * each[:, 0], s8[1].double() * each[:, 1]
    m32, v32, size = s32[0].double(), s32[1].double(), size.double()
    u8, m8, m32, v32 = u8 / size, m8 / size, m32 / size, v32 / size ** 2
    print(f"v {float((u8 ** 2).mean() / v32.mean()):.4f}  u {float(u8.mean()):.4f}  scatter {float(u8.std() / u8.mean()):.4f}")
    # (a percent and a tenth on either side for what the drift's curvature adds; 65,536 elements stray by 0.1%)
    assert 1.02 < float((u8 ** 2).mean() / v32.mean()) < 1.08
    assert 0.11 < float(u8.std() / u8.mean()) < 0.2
    # m is linear in what is rounded: unbiased. Its roundings, each at most half of a distance of 1/8, of which
    # the last ten or so count, stray by a third of m or less: 65,536 of them by 0.2%
    assert abs(float((m8 * m32).mean() / (m32 * m32).mean()) - 1) < 0.01
