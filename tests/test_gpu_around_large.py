"""Embedding, norm and vocabulary loss at sizes where tiles are largest, products are split, the vocabulary goes in
pieces or offsets pass 32 bits; and the layers' backward in a captured graph."""
import threading

import pytest
import torch

import around_util as R
from paper_2607_20652_amd import autograd as A
from paper_2607_20652_amd import binding as dpb
from test_gpu_cross_entropy import DEV, TYPES, draw

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dpb.load()


@TYPES
@pytest.mark.parametrize("rows,dim,vocab", [
    (5000, 1001, 12000),     # tiles of 256 in bf16, dH in parts, rows that do not start on 16 bytes
    (5000, 1000, 20011),     # whole tiles, and the rest of dW in parts
    (3000, 1024, 30001),     # a last entry in a tile of its own
    (9000, 264, 9001),       # tiles of 128, both results in parts
    (3, 8, 5_000_000),       # pieces for the length of a token's row
    (4500, 4096, 2000),      # rows much longer than the vocabulary's tiles
])
def test_large_tiles_and_parts(rows, dim, vocab, dtype):
    h, w, t, ga, ge = draw(rows, dim, vocab, dtype)
    loss, lse = dpb.cross_entropy(h, w, t, 0.7)
    want_loss, want_lse, _ = R.cross_entropy(h, w, t, 0.7)
    R.check("loss", loss, *want_loss)
    R.check("lse", lse, *want_lse)
    dh, dw = dpb.cross_entropy_bwd(ga, h, w, t, lse, 0.7, grad_lse=ge)
    want_dh, want_dw = R.cross_entropy_bwd(ga, h, w, t, lse, 0.7, ge)
    R.check("dhidden", dh, *want_dh)
    R.check("dweight", dw, *want_dw)
    again = dpb.cross_entropy_bwd(ga, h, w, t, lse, 0.7, grad_lse=ge)
    assert torch.equal(dh, again[0]) and torch.equal(dw, again[1])


@TYPES
@pytest.mark.parametrize("dim", [1032, 1035])
def test_pieces_with_a_result_in_parts(dim, dtype):
    """Two pieces in bf16, three in fp32: each adds its product to the sum so far, of whole tiles and of parts.
    The sum of the pieces is at most three additions more."""
    rows, vocab = 20000, 30000
    h, w, t, ga, _ = draw(rows, dim, vocab, dtype)
    loss, lse = dpb.cross_entropy(h, w, t)
    dh, dw = dpb.cross_entropy_bwd(ga, h, w, t, lse)
    want_w, bound_w = torch.zeros(vocab, dim, dtype=torch.float64, device=DEV), 0
    for at in range(0, rows, 5000):
        s = slice(at, at + 5000)
        R.check("loss", loss[s], *R.cross_entropy(h[s], w, t[s], 1.0)[0])
        (h64, h_off), (w64, w_off) = R.cross_entropy_bwd(ga[s], h[s], w, t[s], lse[s], 1.0)
        R.check("dhidden", dh[s], h64, h_off + 4 * R.E * h_off)
        want_w += w64
        bound_w = bound_w + w_off
    # the bounds of the parts hold (5,000 + 80) steps of each sum: 20,000 in all, four times those
    R.check("dweight", dw, want_w, 4 * bound_w)


def test_rows_past_32_bits():
    """Tables, rows and gradients of more than 2^31 elements (and 2^32 bytes)."""
    rows, dim = 70000, 32768
    big = torch.zeros(rows, dim, device=DEV, dtype=torch.bfloat16)
    ends = torch.tensor([0, 1, 65535, 65536, 65537, rows - 2, rows - 1], device=DEV)
    torch.manual_seed(3)
    big[ends] = torch.randn(len(ends), dim, device=DEV).bfloat16()
    assert torch.equal(dpb.embedding(ends, big), big[ends])
    tokens = torch.arange(rows, device=DEV)
    out = dpb.embedding(tokens, big)
    assert torch.equal(out[ends], big[ends]) and torch.equal(out[1000:1010], big[1000:1010])
    dw = dpb.embedding_bwd(big, tokens, rows)                        # every row has the one token
    assert torch.equal(dw[ends], big[ends]) and not dw[60000:60010].any()
    few = dpb.embedding_bwd(big, tokens % 3, 3)
    for i in range(3):
        some = big[ends[ends % 3 == i]].double()
        R.check("sum", few[i], some.sum(0), rows * R.E * some.abs().sum(0) + 2 * R.U[big.dtype] * some.sum(0).abs())
    w = torch.randn(dim, device=DEV).bfloat16()
    y, total, rstd = dpb.rms_norm(big, w, out, out=dw)
    assert torch.equal(total[ends], big[ends] + out[ends])
    want, want_rstd = R.rms_norm(total[ends], w, 1e-6)
    R.check("out", y[ends], *want)
    R.check("rstd", rstd[ends], *want_rstd)
    dx, _ = dpb.rms_norm_bwd(big, total, w, rstd, dx=out)
    R.check("dx", dx[ends], *R.rms_norm_bwd(big[ends], total[ends], w, rstd[ends])[0])


def test_hidden_rows_far_apart():
    """600 rows of a hidden state, and of a vocabulary, that 8 MiB lie between."""
    step = (1 << 22) - 8
    wide = torch.empty(600 * step, dtype=torch.bfloat16, device=DEV)
    far_h, far_w = wide.as_strided((600, 64), (step, 1)), wide.as_strided((600, 64), (step, 1), 64)
    h, w, t, ga, _ = draw(600, 64, 600, torch.bfloat16)
    far_h.copy_(h)
    far_w.copy_(w)
    got, want = dpb.cross_entropy(far_h, far_w, t), dpb.cross_entropy(h, w, t)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    got, want = (dpb.cross_entropy_bwd(ga, x, y, t, want[1]) for x, y in ((far_h, far_w), (h, w)))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_one_workspace_for_calls_of_all_sizes():
    """Whatever an earlier call has left in it; and one that is too small is refused."""
    space = torch.full((1 << 24,), float("nan"), device=DEV)
    for rows, dim, vocab in ((700, 129, 2000), (40, 64, 40000), (3000, 256, 300)):
        h, w, t, ga, _ = draw(rows, dim, vocab, torch.bfloat16)
        loss, lse = dpb.cross_entropy(h, w, t)
        got = dpb.cross_entropy(h, w, t, workspace=space)
        assert torch.equal(got[0], loss) and torch.equal(got[1], lse)
        for a, b in zip(dpb.cross_entropy_bwd(ga, h, w, t, lse, workspace=space), dpb.cross_entropy_bwd(ga, h, w, t, lse)):
            assert torch.equal(a, b)
        assert torch.equal(dpb.embedding_bwd(h, t, vocab, workspace=space), dpb.embedding_bwd(h, t, vocab))
        weight = w[0].contiguous()
        _, total, rstd = dpb.rms_norm(h, weight)
        for a, b in zip(dpb.rms_norm_bwd(h, total, weight, rstd, workspace=space), dpb.rms_norm_bwd(h, total, weight, rstd)):
            assert torch.equal(a, b)
        for call in (lambda: dpb.cross_entropy(h, w, t, workspace=space[:4]), lambda: dpb.cross_entropy_bwd(ga, h, w, t, lse, workspace=space[:4]),
                     lambda: dpb.embedding_bwd(h, t, vocab, workspace=space[:4]), lambda: dpb.rms_norm_bwd(h, total, weight, rstd, workspace=space[:4])):
            with pytest.raises(RuntimeError):
                call()


def test_calls_of_two_threads():
    """Each on a stream of its own, at once."""
    def work(seed, out):
        torch.cuda.set_device(0)
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(10):
                h, w, t, ga, lse = inputs[seed]
                out.append((*dpb.cross_entropy(h, w, t), *dpb.cross_entropy_bwd(ga, h, w, t, lse), dpb.embedding_bwd(h, t, len(w))))
            torch.cuda.current_stream().synchronize()

    inputs, want = [], []
    for size in ((600, 96, 1500), (50, 128, 9000)):
        h, w, t, ga, _ = draw(*size, torch.bfloat16)
        loss, lse = dpb.cross_entropy(h, w, t)
        inputs.append((h, w, t, ga, lse))
        want.append((loss, lse, *dpb.cross_entropy_bwd(ga, h, w, t, lse), dpb.embedding_bwd(h, t, len(w))))
    torch.cuda.synchronize()
    got = [[], []]
    threads = [threading.Thread(target=work, args=(i, got[i])) for i in range(2)]
    for thread in threads:
        thread.start()
    for thread in threads:
        thread.join()
    for outs, one in zip(got, want):
        assert len(outs) == 10 and all(torch.equal(a, b) for out in outs for a, b in zip(out, one))


def test_a_captured_backward_of_the_layers():
    """From tokens to the gradients of all leaves in one graph, replayed between eager passes."""
    g = torch.Generator(device=DEV).manual_seed(2)
    tokens = torch.randint(0, 500, (4, 75), device=DEV, generator=g)
    targets = torch.randint(-1, 500, (4, 75), device=DEV, generator=g)
    ga = torch.rand(4, 75, device=DEV, generator=g)
    leaves = [torch.randn(s, device=DEV, generator=g).requires_grad_() for s in ((500, 64), (64,), (4, 75, 64))]

    def step(leaves):
        table, w, residual = leaves
        out, _ = A.rms_norm_layer(A.embedding_layer(tokens, table), w, residual)
        loss, _ = A.cross_entropy_layer(out, table, targets)
        return torch.autograd.grad(loss, leaves, ga)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(leaves)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        grads = step(leaves)
    for seed in range(4):
        g.manual_seed(seed)
        tokens.copy_(torch.randint(-1, 501, (4, 75), device=DEV, generator=g))
        targets.copy_(torch.randint(-1, 501, (4, 75), device=DEV, generator=g))
        with torch.no_grad():
            leaves[0].copy_(torch.randn(500, 64, device=DEV, generator=g))
        graph.replay()
        got = [x.clone() for x in grads]
        torch.cuda.synchronize()
        others = [x.detach().clone().requires_grad_() for x in leaves]   # (leaves of their own)
        assert all(torch.equal(a, b) for a, b in zip(got, step(others)))


@pytest.mark.parametrize("dtype,length", [(torch.bfloat16, 4096), (torch.bfloat16, 5000), (torch.float32, 2048)])
def test_the_last_token_of_each_long_sequence(dtype, length):
    """Hidden rows 8 MiB and more apart, through the layer: what their copy gives."""
    h, w, t, ga, _ = draw(4, 1024, 600, dtype)
    stream = torch.zeros(4, length, 1024, dtype=dtype, device=DEV)
    stream[:, -1] = h
    stream.requires_grad_()
    far, near, table = stream[:, -1], h.clone().requires_grad_(), w.clone().requires_grad_()
    for x in (far, near):
        loss, lse = A.cross_entropy_layer(x, table, t)
        if x is far:
            first = loss, lse, *torch.autograd.grad((loss * ga).sum() + lse.sum(), (stream, table))
        else:
            second = loss, lse, *torch.autograd.grad((loss * ga).sum() + lse.sum(), (near, table))
    assert all(torch.equal(first[i], second[i]) for i in (0, 1, 3))
    assert torch.equal(first[2][:, -1], second[2]) and not first[2][:, :-1].any()


@TYPES
@pytest.mark.parametrize("rows,dim,vocab", [
    (8192, 200, 20000),     # scores in tiles of 256 with seven steps: four and three
    (4096, 320, 16384),     # ten: twice four and two
    (4096, 570, 16384),     # eighteen, the last of which is not full
])
def test_steps_that_are_no_multiple_of_the_stages(rows, dim, vocab, dtype):
    h, w, t, ga, ge = draw(rows, dim, vocab, dtype)
    loss, lse = dpb.cross_entropy(h, w, t, 0.7)
    want_loss, want_lse, _ = R.cross_entropy(h, w, t, 0.7)
    R.check("loss", loss, *want_loss)
    R.check("lse", lse, *want_lse)
    got = dpb.cross_entropy_bwd(ga, h, w, t, lse, 0.7, grad_lse=ge)
    for name, x, want in zip(("dhidden", "dweight"), got, R.cross_entropy_bwd(ga, h, w, t, lse, 0.7, ge)):
        R.check(name, x, *want)
    assert all(torch.equal(a, b) for a, b in zip(got, dpb.cross_entropy_bwd(ga, h, w, t, lse, 0.7, grad_lse=ge)))
