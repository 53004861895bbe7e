"""The training operators' C ABI without a GPU: sizes, refusals before anything is
enqueued, calls with nothing to do, and the random rounding's hash."""
import ctypes
import math

import pytest
import torch

from paper_2607_20652_amd import binding as dpb

EINVAL, EUNSUPPORTED, OK = -1, -2, 0


def attn(batch=2, q_len=5, k_len=7, q_rows=0, k_rows=0, heads=4, kv_heads=2, dim=64, causal=0, scale=0.125,
         q_lens=0, k_lens=0, q_starts=0, k_starts=0):
    return dpb._ATTN.pack(batch, q_len, k_len, q_rows, k_rows, heads, kv_heads, dim, causal, scale, q_lens, k_lens,
                          q_starts, k_starts)


def heads(data=1 << 20, batch=4096, token=256, head=64):
    return dpb._HEADS.pack(data, batch, token, head)


def forward(a, dtype=1, q=None, k=None, v=None, out=None, lse=1 << 20, ws=None, n=0):
    return dpb.load().dpb_attention(a, dtype, q or heads(), k or heads(), v or heads(), out or heads(2 << 20),
                                    lse, ws, n, None)


def backward(a, dtype=1, outs=(2 << 20, 3 << 20, 4 << 20), lse=1 << 20, ws=1 << 20, n=1 << 40):
    return dpb.load().dpb_attention_bwd(a, dtype, heads(), heads(), heads(), heads(), heads(), lse, heads(outs[0]),
                                        heads(outs[1]), heads(outs[2]), ws, n, None)


@pytest.mark.parametrize("bad", [
    dict(batch=-1), dict(q_len=-1), dict(k_len=-2), dict(heads=0), dict(kv_heads=0), dict(heads=5), dict(dim=0),
    dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(q_starts=1 << 20),
    dict(k_starts=1 << 20), dict(q_starts=1 << 20, k_starts=1 << 20, k_lens=1 << 20),
    dict(q_starts=1 << 20, k_starts=1 << 20, q_rows=-1),
])
def test_sizes_that_mean_nothing(bad):
    assert forward(attn(**bad)) == EINVAL and backward(attn(**bad)) == EINVAL
    assert dpb.load().dpb_attention_workspace_bytes(attn(**bad)) == 0
    assert dpb.load().dpb_attention_bwd_workspace_bytes(attn(**bad)) == 0


@pytest.mark.parametrize("large", [
    dict(dim=136), dict(dim=60), dict(q_len=1 << 31), dict(k_len=1 << 31), dict(batch=1 << 31),
    dict(batch=1 << 16, q_len=1 << 20, heads=64, kv_heads=64), dict(q_len=1 << 30, heads=64, kv_heads=1),
])
def test_sizes_beyond_the_kernels(large):
    assert forward(attn(**large)) == EUNSUPPORTED and backward(attn(**large)) == EUNSUPPORTED


def test_bad_tensors():
    a = attn()
    assert forward(None) == EINVAL
    assert forward(a, dtype=7) == EINVAL
    for x in (heads(data=0), heads(data=(1 << 20) + 8), heads(token=260), heads(head=-64), heads(batch=4)):
        for name in ("q", "k", "v", "out"):
            assert forward(a, **{name: x}) == EINVAL, name
    assert forward(a, k=heads(token=1 << 23)) == EUNSUPPORTED      # 16 MiB a token
    assert forward(a, lse=0) == EINVAL and forward(a, lse=(1 << 20) + 4) == EINVAL
    # the strides along which there is one entry say nothing
    one = attn(batch=1, q_len=1, heads=1, kv_heads=1, k_len=0)
    assert backward(one, outs=(0, 3 << 20, 4 << 20)) == EINVAL


def test_bad_workspaces_and_overlaps():
    a = attn(batch=1, q_len=1, k_len=4096, heads=2, kv_heads=1)
    need = dpb.load().dpb_attention_workspace_bytes(a)
    assert need > 0
    assert forward(a) == EINVAL and forward(a, ws=1 << 20, n=need - 1) == EINVAL
    assert forward(a, ws=(1 << 20) + 4, n=need) == EINVAL
    a = attn()
    for name in ("q", "k", "v"):
        assert forward(a, **{name: heads(5 << 20)}, out=heads(5 << 20)) == EINVAL, name
    need = dpb.load().dpb_attention_bwd_workspace_bytes(a)
    assert need >= 2 * 4 * 2 * 5 * 4
    assert backward(a, n=need - 1) == EINVAL and backward(a, ws=0) == EINVAL
    assert backward(a, outs=(1 << 20, 3 << 20, 4 << 20)) == EINVAL
    assert backward(a, outs=(2 << 20, 2 << 20, 4 << 20)) == EINVAL


def test_nothing_to_do():
    assert forward(attn(batch=0)) == OK and backward(attn(batch=0)) == OK
    assert forward(attn(q_len=0)) == OK
    assert dpb.load().dpb_attention_workspace_bytes(attn(q_len=0)) == 0


def test_state_blocks():
    assert dpb.adamw_blocks([]) == 0
    assert dpb.adamw_blocks([0, 1, 256, 257, 0, 512]) == 0 + 1 + 1 + 2 + 0 + 2
    assert dpb.load().dpb_adamw_blocks(None, 3) == 0


def step(count=1, params=(1 << 20,), grads=(2 << 20,), sizes=(300,), decay=None, pt=0, gt=0, bits=32, m=3 << 20,
         v=4 << 20, scales=None, master=None, gs=None, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, t=1):
    n = len(sizes)
    ptrs = lambda p: (ctypes.c_void_p * max(1, n))(*p)  # noqa: E731
    o = dpb._AdamW(lr, b1, b2, eps, t, 0)
    return dpb.load().dpb_adamw_step(ctypes.byref(o), count, ptrs(params), ptrs(grads), (ctypes.c_int64 * max(1, n))(*sizes),
                                     None if decay is None else (ctypes.c_float * n)(*decay), pt, gt, bits, m, v, scales,
                                     master, gs, None)


@pytest.mark.parametrize("bad", [
    dict(count=-1), dict(pt=2), dict(gt=-1), dict(bits=16), dict(bits=8), dict(lr=math.nan), dict(b1=1.0), dict(b1=-0.1),
    dict(b2=math.nan), dict(eps=0.0), dict(eps=1e-60), dict(eps=math.inf), dict(t=0), dict(sizes=(-3,)), dict(params=(0,)),
    dict(grads=(0,)), dict(params=((1 << 20) + 2,)), dict(grads=((1 << 20) + 1,), gt=1), dict(decay=(math.inf,)), dict(m=0),
    dict(v=(4 << 20) + 4), dict(master=8), dict(gs=2), dict(bits=8, scales=4),
])
def test_steps_that_mean_nothing(bad):
    assert step(**bad) == EINVAL


def test_steps_of_nothing():
    assert step(count=0) == OK
    assert step(sizes=(0,), params=(0,), grads=(0,)) == OK


def test_calls_ask_for_device_tensors():
    q = torch.zeros(1, 2, 4, 64)
    for call in (lambda: dpb.attention(q, q, q), lambda: dpb.attention_bwd(q, q, q, q, q, q[..., 0].contiguous())):
        with pytest.raises((ValueError, AssertionError)):
            call()
    with pytest.raises(ValueError):
        dpb.adamw_step([q], [q], q, q, step=1, lr=1.0)


def test_the_rounding_s_random_bits_are_even_and_unrelated():
    """Both halves of the hash over places and seeds: counts in 1024 bins (chi-square of 1023 degrees, six
    standard deviations of 45), and no correlation between neighbours, halves and seeds (five times 1 / sqrt(n))."""
    low, n = 0xFFFFFFFF, 1 << 20

    def bits(seed, start=0):
        x = torch.arange(start, start + n)
        x = ((x & low) * 0x9E3779B9 + (x >> 32) * 0x6A09E667 + seed) & low
        x = ((x ^ (x >> 16)) * 0x6A09E667) & low
        x = ((x ^ (x >> 15)) * 0x9E3779B9) & low
        return x ^ (x >> 16)

    def related(a, b):
        return abs(float(torch.corrcoef(torch.stack([a.double(), b.double()]))[0, 1])) > 5 / math.sqrt(n)

    one, two, far = bits(1), bits(2), bits(1, 1 << 33)
    for x in (one, two, far):
        for half in (x & 0xFFFF, x >> 16):
            count = torch.bincount(half >> 6, minlength=1024).double()
            chi = float(((count - n / 1024) ** 2).sum() / (n / 1024))
            assert abs(chi - 1023) < 6 * 45.3
        assert not related(x[:-1], x[1:]) and not related(x[:-64], x[64:]) and not related(x & 0xFFFF, x >> 16)
    assert not related(one, two) and not related(one, far)
