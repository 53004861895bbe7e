"""The largest calls: refused where a launch would have 2^32 threads, on both sides of that
line, and nothing below it. A size that is accepted is told by the refusal that comes
after it, of a missing log-sum-exp, so nothing is launched."""
import pytest

from paper_2607_20652_amd import binding as dpb

EINVAL, EUNSUPPORTED = -1, -2
T = 1 << 20     # an address


def attn(batch, q_len, k_len, heads, kv_heads, dim=64, causal=0, packed=False):
    rows = dict(q=1000, k=1000) if packed else dict(q=0, k=0)
    starts = T if packed else 0
    return dpb._ATTN.pack(batch, q_len, k_len, rows["q"], rows["k"], heads, kv_heads, dim, causal, 0.125, 0, 0, starts, starts)


def forward(a):
    x, y = dpb._HEADS.pack(T, 1 << 30, 1 << 20, 64), dpb._HEADS.pack(2 * T, 1 << 30, 1 << 20, 64)
    return dpb.load().dpb_attention(a, 1, x, x, x, y, None, T, 1 << 60, None)


def backward(a):
    x, y = dpb._HEADS.pack(T, 1 << 30, 1 << 20, 64), [dpb._HEADS.pack(i * T, 1 << 30, 1 << 20, 64) for i in (2, 3, 4)]
    return dpb.load().dpb_attention_bwd(a, 1, x, x, x, x, x, None, *y, T, 1 << 60, None)


N = 1 << 24     # workgroups of 256 threads that are one too many

FORWARD = [
    # accepted, and refused
    ((1, 1, 100, N - 1, N - 1), (1, 1, 100, N, N)),                     # few rows: one workgroup each
    ((N - 1, 32, 100, 1, 1), (N, 32, 100, 1, 1)),
    ((N // 2 - 1, 129, 100, 1, 1), (N // 2, 129, 100, 1, 1)),           # tiles of 128 rows
    ((1 << 10, 65536, 65536, 16, 16), (1 << 10, 65536, 65536, 32, 32)),
    ((1, 2 ** 31 - 256, 1, 1, 1), (1, 2 ** 31 - 255, 1, 1, 1)),         # rows in 32 bits
    ((1, 1, 2 ** 31 - 256, 8, 1), (1, 1, 2 ** 31 - 255, 8, 1)),
    ((1 << 20, 1, 1 << 20, 8, 8), (1 << 21, 1, 1 << 20, 8, 8)),         # keys are no workgroups of the forward
]


@pytest.mark.parametrize("packed", [False, True], ids=["padded", "packed"])
@pytest.mark.parametrize("fits,too_large", FORWARD)
def test_the_largest_forward(fits, too_large, packed):
    assert forward(attn(*fits, packed=packed)) == EINVAL
    assert forward(attn(*too_large, packed=packed)) == EUNSUPPORTED
    assert dpb.load().dpb_attention_workspace_bytes(attn(*too_large, packed=packed)) == 0


BACKWARD = [
    ((N - 1, 2, 2, 1, 1), (N, 2, 2, 1, 1)),
    ((N // 2 - 1, 129, 128, 1, 1), (N // 2, 129, 128, 1, 1)),
    ((N // 2 - 1, 100, 129, 1, 1), (N // 2, 100, 129, 1, 1)),
    ((N // 4 - 1, 100, 512, 1, 1), (N // 4, 100, 512, 1, 1)),           # keys are
    ((1 << 10, 65536, 65536, 16, 16), (1 << 10, 65536, 65536, 32, 32)),
]


@pytest.mark.parametrize("causal", [0, 1], ids=["all", "causal"])
@pytest.mark.parametrize("packed", [False, True], ids=["padded", "packed"])
@pytest.mark.parametrize("fits,too_large", BACKWARD)
def test_the_largest_backward(fits, too_large, packed, causal):
    size = dpb.load().dpb_attention_bwd_workspace_bytes
    assert backward(attn(*fits, packed=packed, causal=causal)) == EINVAL
    assert size(attn(*fits, packed=packed, causal=causal)) > 0
    assert backward(attn(*too_large, packed=packed, causal=causal)) == EUNSUPPORTED
    assert size(attn(*too_large, packed=packed, causal=causal)) == 0


def test_a_workspace_of_sizes_near_the_line_is_counted_in_64_bits():
    rows = (N // 2 - 1) * 129
    assert dpb.load().dpb_attention_bwd_workspace_bytes(attn(N // 2 - 1, 129, 128, 1, 1)) >= 2 * 4 * rows
    # one sequence of 2^30 rows of one head, 2^24 keys: the keys' parts of 16,777,216 rows
    assert dpb.load().dpb_attention_bwd_workspace_bytes(attn(1, 1 << 30, 1 << 24, 1, 1, 128)) >= 2 * 4 * (1 << 30)
