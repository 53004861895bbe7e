"""Packed rows that belong to no sequence: room before the first, behind the last, and
behind a longest sequence told too short.  Outputs made by the call hold zeros
there (log-sum-exp -inf), outputs that are given keep what they held."""
import math

import pytest
import torch

from attention_util import check, reference
from paper_2607_20652_amd import binding as dpb

gpu = pytest.mark.gpu

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
CASES = [
    # query starts, rows; key starts, rows; longest; heads, key heads, width
    ([3, 10, 10, 40], 60, [0, 20, 25, 25], 30, (64, 64), (4, 2, 64)),
    ([0, 50, 90], 90, [7, 40, 100], 131, (20, 33), (3, 3, 40)),
    ([5, 205, 405], 1500, [5, 205, 405], 1500, (170, 200), (32, 32, 128)),
    ([0, 0], 33, [0, 0], 5, (1, 1), (2, 1, 8)),
    ([11], 17, [2], 9, (4, 4), (2, 2, 16)),
    (list(range(1, 1302)), 1310, list(range(0, 2602, 2)), 2700, (1, 1), (2, 1, 32)),
]


def attn(q_starts=0, k_starts=0, dim=64):
    return dpb._ATTN.pack(2, 5, 7, 20, 20, 4, 2, dim, 0, 0.125, 0, 0, q_starts, k_starts)


def test_refusals_and_calls_with_nothing_to_do():
    clear, x = dpb.load().dpb_attention_clear, dpb._HEADS.pack(1 << 20, 4096, 256, 64)
    packed = attn(1 << 20, 1 << 20)
    assert clear(None, 1, x, None, None, None, None) == -1
    assert clear(packed, 7, x, None, None, None, None) == -1
    assert clear(attn(1 << 20, 1 << 20, dim=136), 1, x, None, None, None, None) == -2
    for bad in (dpb._HEADS.pack(0, 0, 256, 64), dpb._HEADS.pack((1 << 20) + 8, 0, 256, 64), dpb._HEADS.pack(1 << 20, 0, 260, 64)):
        for at in (2, 4, 5):
            args = [packed, 1, None, None, None, None, None]
            args[at] = bad
            assert clear(*args) == -1
    assert clear(packed, 1, x, (1 << 20) + 4, None, None, None) == -1
    assert clear(packed, 1, None, None, None, None, None) == 0
    assert clear(attn(), 1, x, 1 << 20, x, x, None) == 0            # padded: no such rows


def poison(*shapes_and_types):
    """What the allocator hands out next held NaN."""
    held = [torch.full(s, math.nan, dtype=t, device=DEV) for s, t in shapes_and_types]
    torch.cuda.synchronize()
    del held


def spans(starts, rows, longest):
    return [(min(s, rows), min(e - s, longest)) for s, e in zip(starts, starts[1:])]


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_rows_of_no_sequence(case, dtype):
    qs, qn, ks, kn, (mq, mk), (H, G, D) = CASES[case]
    gen = torch.Generator().manual_seed(40 + case)
    r = lambda n, h: torch.randn(n, h, D, generator=gen).to(dtype)  # noqa: E731
    q, k, v, g = r(qn, H), r(kn, G), r(kn, G), r(qn, H)
    want = {n: [torch.zeros(x.shape, dtype=torch.float64) for _ in range(3)]
            for n, x in (("out", q), ("lse", q[..., 0]), ("dq", q), ("dk", k), ("dv", v))}
    want["lse"][0].fill_(-math.inf)
    for (a, n), (b, m) in zip(spans(qs, qn, mq), spans(ks, kn, mk)):
        one = reference(q[None, a:a + n], k[None, b:b + m], v[None, b:b + m], True, D ** -0.5, g[None, a:a + n])
        for name, parts in one.items():
            at = slice(b, b + m) if name in ("dk", "dv") else slice(a, a + n)
            for to, x in zip(want[name], parts):
                to[at] = x[0]
    # rows of no sequence hold what memory may hold, and are not read
    for x, starts, longest in ((q, qs, mq), (g, qs, mq), (k, ks, mk), (v, ks, mk)):
        live = torch.zeros(x.shape[0], dtype=torch.bool)
        for a, n in spans(starts, x.shape[0], longest):
            live[a:a + n] = True
        x[~live] = math.nan
    q, k, v, g = (x.to(DEV) for x in (q, k, v, g))
    kw = dict(q_starts=torch.tensor(qs, dtype=torch.int32, device=DEV), k_starts=torch.tensor(ks, dtype=torch.int32, device=DEV),
              max_q=mq, max_k=mk)
    poison((q.shape, dtype), (q.shape[:-1], F32))
    out, lse = dpb.attention(q, k, v, True, **kw)
    poison((q.shape, dtype), (k.shape, dtype), (k.shape, dtype))
    dq, dk, dv = dpb.attention_bwd(g, q, k, v, out, lse, True, **kw)
    got = {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
    for name in want:
        check(name, got[name], want[name], dtype)

    # the same into tensors that are given: equal where there is a sequence, untouched elsewhere
    mark = {n: torch.full_like(x, 7.0) for n, x in got.items()}
    dpb.attention(q, k, v, True, out=mark["out"], lse=mark["lse"], **kw)
    dpb.attention_bwd(g, q, k, v, out, lse, True, dq=mark["dq"], dk=mark["dk"], dv=mark["dv"], **kw)
    for name, x in mark.items():
        starts, longest = (ks, mk) if name in ("dk", "dv") else (qs, mq)
        live = torch.zeros(x.shape[0], dtype=torch.bool)
        for a, n in spans(starts, x.shape[0], longest):
            live[a:a + n] = True
        assert torch.equal(x[live], got[name][live]) and bool((x[~live] == 7).all()), name


@gpu
def test_only_the_outputs_that_are_made_are_cleared():
    q, k, v = (torch.randn(30, 2, 32, device=DEV) for _ in range(3))
    starts = torch.tensor([4, 20], dtype=torch.int32, device=DEV)
    kw = dict(q_starts=starts, k_starts=starts, max_q=16, max_k=16)
    given = torch.full((30, 2, 32), 7.0, device=DEV)
    poison(((30, 2), F32))
    out, lse = dpb.attention(q, k, v, out=given, **kw)
    assert out is given and bool((given[:4] == 7).all()) and bool((given[20:] == 7).all())
    assert bool((lse[:4] == -math.inf).all()) and bool((lse[20:] == -math.inf).all()) and torch.isfinite(lse[4:20]).all()
    dk = torch.full((30, 2, 32), 7.0, device=DEV)
    poison(((30, 2, 32), F32), ((30, 2, 32), F32))
    dq, _, dv = dpb.attention_bwd(v, q, k, v, out, lse, dk=dk, **kw)
    for x, held in ((dq, 0.0), (dk, 7.0), (dv, 0.0)):
        assert bool((x[:4] == held).all()) and bool((x[20:] == held).all()) and torch.isfinite(x).all()


@gpu
def test_heads_in_another_order_and_a_graph():
    """Gaps in outputs whose heads lie apart; the call in a graph, replayed over dirty outputs."""
    q, k, v = (torch.randn(2, 50, 48, device=DEV).to(BF16).transpose(0, 1) for _ in range(3))
    starts = torch.tensor([6, 20, 41], dtype=torch.int32, device=DEV)
    a = dpb._attn(q, k, v, True, None, None, None, starts, starts, 16, 21)
    out = torch.full((2, 50, 48), 7.0, dtype=BF16, device=DEV).transpose(0, 1)
    lse = torch.full((50, 2), 7.0, device=DEV)

    def clear():
        dpb._check("clear", dpb.load().dpb_attention_clear(a, dpb.DPB_BF16, dpb._heads(out, "out"), dpb._dev(lse, "lse"),
                                                           None, None, dpb._stream(q)))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        clear()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        clear()
    loose = torch.ones(50, dtype=torch.bool, device=DEV)
    loose[6:20] = False
    loose[20:36] = False                    # 16 of its 21 rows
    for _ in range(3):
        out.fill_(7.0)
        lse.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert bool((out[loose] == 0).all()) and bool((out[~loose] == 7).all())
        assert bool((lse[loose] == -math.inf).all()) and bool((lse[~loose] == 7).all())
