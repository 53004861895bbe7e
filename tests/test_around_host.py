"""The C ABI of embedding, norm and vocabulary loss without a GPU: refusals before anything is enqueued, workspace
sizes, calls with nothing to do; and the binding's checks."""
import math

import pytest
import torch

from paper_2607_20652_amd import binding as dpb

EINVAL, EUNSUPPORTED, OK = -1, -2, 0
MB = 1 << 20
GB = 1 << 30


def embed(dtype=1, table=GB, stride=64, vocab=100, dim=64, tokens=2 * GB, bits=64, count=10, scale=1.0, out=3 * GB):
    return dpb.load().dpb_embedding(dtype, table, stride, vocab, dim, tokens, bits, count, scale, out, None)


def embed_bwd(dtype=1, grad=GB, stride=64, tokens=2 * GB, bits=64, count=10, vocab=100, dim=64, scale=1.0, out=3 * GB, ws=4 * GB, n=GB):
    return dpb.load().dpb_embedding_bwd(dtype, grad, stride, tokens, bits, count, vocab, dim, scale, out, ws, n, None)


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(dtype=-1), dict(stride=-1), dict(vocab=-1), dict(dim=0), dict(count=-1), dict(bits=16), dict(bits=0),
    dict(scale=math.inf), dict(scale=math.nan), dict(tokens=0), dict(tokens=2 * GB + 4), dict(tokens=2 * GB + 2, bits=32),
    dict(out=0), dict(out=3 * GB + 8), dict(out=2 * GB), dict(out=2 * GB - 16), dict(stride=1 << 60),
])
def test_lookups_that_mean_nothing(bad):
    assert embed(**bad) == EINVAL
    assert embed_bwd(**bad) == EINVAL


def test_lookups_over_their_own_memory():
    assert embed(table=0) == EINVAL and embed(table=GB + 1) == EINVAL
    assert embed(out=GB) == EINVAL and embed(out=GB + 99 * 128 + 112) == EINVAL and embed(out=GB - 16) == EINVAL
    assert embed_bwd(grad=0) == EINVAL and embed_bwd(grad=GB + 1) == EINVAL
    for x in (dict(out=GB), dict(out=4 * GB), dict(ws=3 * GB), dict(ws=GB - 16), dict(ws=2 * GB), dict(ws=0), dict(ws=4 * GB + 4), dict(n=100)):
        assert embed_bwd(**x) == EINVAL, x


def test_lookups_of_nothing_and_of_too_much():
    assert embed(count=0, tokens=0, out=0) == OK and embed_bwd(vocab=0, out=0, ws=0) == OK
    lib = dpb.load()
    assert lib.dpb_embedding_bwd_workspace_bytes(0, 64, 10) == 0
    assert lib.dpb_embedding_bwd_workspace_bytes(-1, 64, 10) == 0 and lib.dpb_embedding_bwd_workspace_bytes(5, 0, 10) == 0
    for big in (dict(vocab=(1 << 31) - 65536, dim=1, stride=1), dict(count=(1 << 31) - 65536, dim=1, stride=1), dict(count=1 << 30, dim=1 << 20, stride=0),
                dict(vocab=1 << 30, dim=1 << 20)):
        assert embed_bwd(**big) == EUNSUPPORTED, big
        assert lib.dpb_embedding_bwd_workspace_bytes(big.get("vocab", 100), big.get("dim", 64), big.get("count", 10)) == 0


@pytest.mark.parametrize("vocab,dim,count", [(1, 1, 0), (1, 1, 1), (50304, 1024, 16384), (50304, 1024, 16385), (1025, 33, 65), (3_000_000, 4, 1000)])
def test_sorting_space(vocab, dim, count):
    """Two words a token of whole bins (above 16,384 of them), two more, starts of buckets and rows, and two parts of
    each 32 tokens."""
    shift, bins = 0, -(-count // 1024) if count > 16384 else 0
    while (vocab - 1) >> shift >= (1024 if bins else 512):
        shift += 1
    buckets, chunks = ((vocab - 1) >> shift) + 1, -(-count // 32)
    up = lambda n: -(-n // 16) * 16  # noqa: E731
    want = up(bins * 8192) + up(bins * (buckets + 1) * 4) + 2 * up(count * 4) + up((vocab + 1) * 4) + up(chunks * 8 * (-(-dim // 4) * 4))
    assert dpb.load().dpb_embedding_bwd_workspace_bytes(vocab, dim, count) == want


def norm(dtype=1, x=GB, xs=64, r=2 * GB, rs=64, w=3 * GB, wt=1, rows=10, dim=64, eps=1e-6, out=4 * GB, total=5 * GB, rstd=6 * GB):
    return dpb.load().dpb_rms_norm(dtype, x, xs, r, rs, w, wt, rows, dim, eps, out, total, rstd, None)


def norm_bwd(dtype=1, g=GB, gs=64, h=2 * GB, hs=64, z=3 * GB, zs=64, w=4 * GB, wt=1, rstd=5 * GB, rows=10, dim=64, dx=6 * GB, dw=7 * GB,
             ws=8 * GB, n=GB):
    return dpb.load().dpb_rms_norm_bwd(dtype, g, gs, h, hs, z, zs, w, wt, rstd, rows, dim, dx, dw, ws, n, None)


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(wt=2), dict(rows=-1), dict(dim=0), dict(eps=-1e-6), dict(eps=math.nan), dict(eps=math.inf), dict(xs=-1),
    dict(rs=-1), dict(x=0), dict(out=0), dict(total=0), dict(x=GB + 1), dict(r=2 * GB + 1), dict(out=4 * GB + 1), dict(total=5 * GB + 1),
    dict(w=3 * GB + 1), dict(rstd=6 * GB + 2),
    dict(out=GB + 16), dict(out=GB, xs=128), dict(total=2 * GB - 2), dict(total=2 * GB, rs=72), dict(out=3 * GB), dict(out=5 * GB + 64),
    dict(rstd=GB), dict(rstd=2 * GB + 1272), dict(rstd=3 * GB), dict(rstd=4 * GB + 4), dict(total=6 * GB),
])
def test_norms_that_mean_nothing(bad):
    assert norm(**bad) == EINVAL


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(wt=-1), dict(rows=-1), dict(dim=0), dict(gs=-1), dict(hs=-2), dict(zs=-1), dict(g=0), dict(z=0), dict(rstd=0),
    dict(g=GB + 1), dict(h=2 * GB + 1), dict(z=3 * GB + 1), dict(rstd=5 * GB + 2), dict(dx=6 * GB + 1), dict(dw=7 * GB + 1), dict(ws=0),
    dict(ws=8 * GB + 4), dict(n=100), dict(dx=GB + 16), dict(dx=GB, gs=65), dict(dx=2 * GB, hs=128), dict(dx=3 * GB), dict(dx=4 * GB),
    dict(dx=5 * GB), dict(dx=7 * GB), dict(dx=8 * GB), dict(dw=GB), dict(dw=2 * GB), dict(dw=3 * GB + 2), dict(dw=4 * GB), dict(dw=8 * GB),
    dict(ws=GB), dict(ws=3 * GB), dict(ws=5 * GB),
])
def test_norm_gradients_that_mean_nothing(bad):
    assert norm_bwd(**bad) == EINVAL


def test_norms_of_nothing():
    assert norm(rows=0, x=0, out=0, r=0) == OK
    assert norm_bwd(dx=0, dw=0) == OK
    lib = dpb.load()
    assert lib.dpb_rms_norm_bwd_workspace_bytes(0, 64) == 0 and lib.dpb_rms_norm_bwd_workspace_bytes(3, 0) == 0
    assert lib.dpb_rms_norm_bwd_workspace_bytes(3, 100) >= 400


def test_rows_past_what_is_counted():
    top, most = (1 << 31) - 1, (1 << 31) - 65536
    lib = dpb.load()
    assert embed(dim=top, count=0) == embed(dim=most + 1, stride=0) == EUNSUPPORTED and embed(dim=most, count=0) == OK
    assert embed(count=1 << 60) == EUNSUPPORTED and embed_bwd(dim=top, vocab=1) == EUNSUPPORTED
    assert lib.dpb_embedding_bwd_workspace_bytes(1, top, 1) == 0
    for big in (dict(dim=(1 << 22) + 1), dict(dim=top), dict(rows=1 << 60, dim=1)):
        if "rows" in big:
            assert norm(**big, xs=0, rs=0) == EUNSUPPORTED and norm_bwd(**big, gs=0, hs=0, zs=0) == EUNSUPPORTED
        else:
            assert norm(**big) == EUNSUPPORTED and norm_bwd(**big) == EUNSUPPORTED
            assert lib.dpb_rms_norm_bwd_workspace_bytes(10, big["dim"]) == 0
    assert norm(rows=0, dim=1 << 22) == OK and lib.dpb_rms_norm_bwd_workspace_bytes(10, 1 << 22) >= 1 << 24


def logits(hidden=GB, weight=2 * GB, hs=64, ws=64, rows=10, vocab=100, dim=64, scale=1.0):
    return dpb._LOGITS.pack(hidden, weight, hs, ws, rows, vocab, dim, scale)


def loss(dtype=1, targets=3 * GB, bits=64, loss=4 * GB, lse=5 * GB, space=6 * GB, n=GB, **a):
    return dpb.load().dpb_cross_entropy(logits(**a), dtype, targets, bits, loss, lse, space, n, None)


def loss_bwd(dtype=1, targets=3 * GB, bits=64, ga=4 * GB, ge=5 * GB, lse=6 * GB, dh=7 * GB, dw=8 * GB, space=9 * GB, n=GB, **a):
    return dpb.load().dpb_cross_entropy_bwd(logits(**a), dtype, targets, bits, ga, ge, lse, dh, dw, space, n, None)


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(rows=-1), dict(vocab=-1), dict(dim=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan),
    dict(hs=-1), dict(vocab=0), dict(bits=8), dict(targets=0), dict(targets=3 * GB + 4), dict(hidden=0), dict(weight=0),
    dict(hidden=GB + 8), dict(weight=2 * GB + 2), dict(lse=0), dict(lse=5 * GB + 2), dict(space=0), dict(space=9 * GB + 8), dict(n=64),
    dict(space=GB), dict(space=2 * GB), dict(space=3 * GB), dict(ws=-1),
])
def test_losses_that_mean_nothing(bad):
    assert loss(**bad) == EINVAL
    assert loss_bwd(**bad) == EINVAL


def test_losses_over_their_own_memory():
    for x in (dict(loss=0), dict(loss=5 * GB + 8), dict(loss=GB), dict(lse=2 * GB + 16), dict(loss=3 * GB + 4), dict(lse=6 * GB + 8), dict(loss=4 * GB + 2)):
        assert loss(**x) == EINVAL, x
    for x in (dict(dh=GB), dict(dh=2 * GB + 16), dict(dw=GB), dict(dw=2 * GB), dict(dh=8 * GB + 16), dict(dh=9 * GB), dict(dw=9 * GB + 32), dict(dh=3 * GB),
              dict(dw=4 * GB), dict(dw=5 * GB), dict(dh=6 * GB), dict(dh=7 * GB + 8), dict(dw=8 * GB + 4), dict(ga=4 * GB + 1), dict(ge=5 * GB + 2)):
        assert loss_bwd(**x) == EINVAL, x


def test_losses_of_nothing_and_of_too_much():
    lib = dpb.load()
    assert dpb.load().dpb_cross_entropy(None, 1, 0, 64, 0, 0, 0, 0, None) == EINVAL
    assert loss(rows=0, hidden=0, targets=0, space=0, n=0) == OK
    assert loss_bwd(dh=0, dw=0) == OK and loss_bwd(rows=0, vocab=0) == OK and loss_bwd(rows=0) == EINVAL
    for big in (dict(rows=1 << 31), dict(vocab=1 << 31), dict(hs=1 << 22), dict(ws=1 << 22), dict(dim=1 << 22, hs=1 << 22), dict(rows=1 << 24, vocab=1 << 24)):
        assert loss(**big) == EUNSUPPORTED and loss_bwd(**big) == EUNSUPPORTED, big
        assert lib.dpb_cross_entropy_workspace_bytes(logits(**big), 1) == 0 and lib.dpb_cross_entropy_bwd_workspace_bytes(logits(**big), 1) == 0
    assert lib.dpb_cross_entropy_workspace_bytes(logits(rows=0), 1) == 0 and lib.dpb_cross_entropy_workspace_bytes(None, 1) == 0


@pytest.mark.parametrize("rows,dim,vocab", [(16384, 1024, 50304), (66000, 64, 50304), (262144, 512, 100_000), (10, 64, 100)])
def test_the_gradient_s_space_is_bounded(rows, dim, vocab):
    """A piece of 1 GiB (or 1,024 entries), an fp32 sum of each gradient and what a split product takes: never the logits."""
    n = dpb.load().dpb_cross_entropy_bwd_workspace_bytes(logits(rows=rows, dim=dim, vocab=vocab, hs=dim, ws=dim), 1)
    piece = min(max(GB, rows * 2048), rows * 2 * vocab)
    assert piece // 2 <= n <= 1.01 * piece + 1024 + 65 * 4 * max(rows, min(vocab, 65536)) * dim if rows < 1000 else n <= 1.02 * piece + 8 * (rows + vocab) * dim * 4


def test_rows_that_need_no_copy_take_none():
    lib = dpb.load()
    size = lambda **a: lib.dpb_cross_entropy_workspace_bytes(logits(**a), 1)  # noqa: E731
    plain = size()
    assert size(hs=72) == plain and size(hs=65) == plain + 10 * 128 and size(ws=65) == plain + 100 * 128
    assert size(hs=0) == plain and size(rows=1, hs=65) == size(rows=1)


def test_binding_checks():
    t, f = torch.zeros(3, dtype=torch.int64), torch.zeros(3, 8)
    calls = [
        lambda: dpb.embedding(t, f), lambda: dpb.embedding_bwd(f, t, 4), lambda: dpb.rms_norm(f, None),
        lambda: dpb.rms_norm_bwd(f, f, None, f[:, 0]), lambda: dpb.cross_entropy(f, f, t),
        lambda: dpb.cross_entropy_bwd(f[:, 0], f, f, t, f[:, 0]),
    ]
    for call in calls:       # host tensors
        with pytest.raises((ValueError, AssertionError)):
            call()
    wrong = [
        lambda: dpb.embedding(t, f[0]), lambda: dpb.embedding(t, f, out=torch.zeros(3, 9)), lambda: dpb.embedding(t, torch.zeros(3, 0)),
        lambda: dpb.embedding_bwd(f, t[:2], 4), lambda: dpb.embedding_bwd(f, t, -1), lambda: dpb.embedding_bwd(f, t, 4, dweight=f),
        lambda: dpb.rms_norm(f, f[0, :7]), lambda: dpb.rms_norm(f, None, f[:2]), lambda: dpb.rms_norm(f, None, f.bfloat16()),
        lambda: dpb.rms_norm(f, None, total=f), lambda: dpb.rms_norm(f, None, out=f[:, :4]), lambda: dpb.rms_norm(f, None, rstd=f),
        lambda: dpb.rms_norm_bwd(f, f, None, f), lambda: dpb.rms_norm_bwd(f, f, None, f[:, 0], dweight=f[0]),
        lambda: dpb.rms_norm_bwd(f.bfloat16(), f, None, f[:, 0]), lambda: dpb.rms_norm_bwd(f, f, f[0], f[:, 0], grad_total=f[0]),
        lambda: dpb.cross_entropy(f, f[:, :4], t), lambda: dpb.cross_entropy(f, f.bfloat16(), t), lambda: dpb.cross_entropy(f, f, t[:2]),
        lambda: dpb.cross_entropy(f, f, t, loss=f), lambda: dpb.cross_entropy_bwd(f, f, f, t, f[:, 0]),
        lambda: dpb.cross_entropy_bwd(f[:, 0], f, f, t, f[:, 0], dhidden=f, hidden_grad=False),
        lambda: dpb.cross_entropy_bwd(f[:, 0].double(), f, f, t, f[:, 0]),
    ]
    for call in wrong:
        with pytest.raises(AssertionError):
            call()


def test_rows_in_memory():
    x = torch.zeros(4, 5, 24)
    assert dpb._rows(x, "x") == (20, 24) and dpb._rows(x[..., :8], "x") == (20, 24) and dpb._rows(x[:, 2], "x") == (4, 120)
    assert dpb._rows(x[:, :1, :8], "x") == (4, 120) and dpb._rows(x[0, 0], "x") == (1, 24) and dpb._rows(x[:0], "x")[0] == 0
    assert dpb._rows(torch.zeros(24).expand(7, 24), "x") == (7, 0) and dpb._rows(x.transpose(0, 1)[:, :1], "x") == (5, 24)
    assert dpb._rows(torch.zeros(3, 1)[:, :1], "x") == (3, 1) and dpb._rows(torch.zeros(1, 1).expand(6, 1), "x")[0] == 6
    for bad in (x[:, :3], x.transpose(0, 1), x[..., ::2], x.transpose(1, 2)):
        with pytest.raises(ValueError):
            dpb._rows(bad, "x")


def test_a_scale_whose_exponents_overflow_is_refused():
    """exp(l) is 2^(l log2(e)): scale log2(e) has to be an fp32 number as well."""
    lib, most = dpb.load(), 3.4028234e38 / 1.4426952
    for scale in (2.4e38, 3e38, 3.4028234e38):
        assert loss(scale=scale) == EUNSUPPORTED and loss_bwd(scale=scale) == EUNSUPPORTED
        assert lib.dpb_cross_entropy_workspace_bytes(logits(scale=scale), 1) == 0
        assert lib.dpb_cross_entropy_bwd_workspace_bytes(logits(scale=scale), 1) == 0
    for scale in (0.9999 * most, 1e-30):
        assert lib.dpb_cross_entropy_workspace_bytes(logits(scale=scale), 1) == lib.dpb_cross_entropy_workspace_bytes(logits(), 1) > 0
