"""Outputs of attention whose rows share memory (an expanded tensor, say) are refused before
anything is enqueued: every row would be written by several workgroups."""
import pytest

from paper_2607_20652_amd import binding as dpb

EINVAL = -1
SIZES = dict(batch=2, q_len=5, k_len=7, q_rows=0, k_rows=0, heads=4, kv_heads=2, dim=64, causal=0, scale=0.125, q_lens=0,
             k_lens=0, q_starts=0, k_starts=0)
PACKED = SIZES | dict(q_rows=20, k_rows=20, q_starts=1 << 20, k_starts=1 << 20)


def heads(data, batch=4096, token=256, head=64):
    return dpb._HEADS.pack(data, batch, token, head)


def calls(sizes, at, **strides):
    """Statuses of the three calls with these strides at output `at` of (q's, k's) where they have one."""
    a, lib = dpb._ATTN.pack(*sizes.values()), dpb.load()
    good, bad = [heads(i << 20) for i in (2, 3, 4)], heads(5 << 20, **strides)
    outs = list(good)
    outs[at] = bad
    x, got = heads(1 << 20), []
    if at == 0:
        got.append(lib.dpb_attention(a, 1, x, x, x, bad, 1 << 20, 1 << 20, 1 << 40, None))
    got.append(lib.dpb_attention_bwd(a, 1, x, x, x, x, x, 1 << 20, *outs, 1 << 20, 1 << 40, None))
    got.append(lib.dpb_attention_clear(a, 1, outs[0], None, outs[1], outs[2], None))
    return got


@pytest.mark.parametrize("at", [0, 1, 2])
@pytest.mark.parametrize("strides", [dict(batch=0), dict(token=0), dict(head=0), dict(batch=8), dict(token=32), dict(head=56)])
def test_rows_that_share_memory(strides, at):
    assert set(calls(SIZES, at, **strides)) == {EINVAL}
    if "batch" not in strides:
        assert set(calls(PACKED, at, **strides)) == {EINVAL}


def test_strides_along_one_entry_say_nothing():
    """Refused for another reason, after the strides were taken: no log-sum-exp."""
    one = SIZES | dict(batch=1, q_len=1, k_len=1, heads=1, kv_heads=1)
    lib, a, x = dpb.load(), dpb._ATTN.pack(*one.values()), heads(1 << 20)
    flat = [heads(i << 20, 0, 0, 0) for i in (2, 3, 4)]
    assert lib.dpb_attention_clear(a, 1, *flat[:1], None, *flat[1:], None) == 0
    assert lib.dpb_attention_bwd(a, 1, x, x, x, x, x, 0, *flat, 1 << 20, 1 << 40, None) == EINVAL
    assert lib.dpb_attention_bwd(dpb._ATTN.pack(*(one | dict(batch=0)).values()), 1, x, x, x, x, x, 0, *flat, None, 0, None) == 0
