"""The calls around the transformer blocks whose speed is measured, and their plain forms.

A case names an operator and its sizes:

  embedding          dpb.embedding: rows of a table for tokens, times a scale
  embedding_bwd      dpb.embedding_bwd: the table's gradient
  rms_norm           dpb.rms_norm: the residual's addition and the root-mean-square norm of the sum
  rms_norm_bwd       dpb.rms_norm_bwd: gradients of the sum and of the norm's weight
  cross_entropy      dpb.cross_entropy: softmax cross entropy of hidden rows over a vocabulary's matrix
  cross_entropy_bwd  dpb.cross_entropy_bwd: gradients of the rows and of the matrix, from the log-sum-exp

The plain forms are elementary torch operations in 32 bits; `exact` has the
results in 64 bits from the operators' definitions.

  embedding      y = scale table[token]; a token outside [0, vocab) gives a row of zeros and no gradient
  rms_norm       z = x + r, rounded to their type;  y = z (mean z^2 + eps)^-1/2 w
  cross_entropy  l = scale H W^T, lse = log sum exp l, loss = lse - l[target]; a target outside
                 [0, vocab) gives a loss of 0 (lse is the row's all the same)
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def _embed(name, op, tokens, dim, vocab, dtype, order):
    return dict(name=name, op=op, tokens=tokens, dim=dim, vocab=vocab, dtype=dtype, order=order)


def _norm(name, op, rows, dim, dtype, residual):
    return dict(name=name, op=op, rows=rows, dim=dim, dtype=dtype, residual=residual)


def _loss(name, op, rows, dim, vocab, dtype, ignored):
    return dict(name=name, op=op, rows=rows, dim=dim, vocab=vocab, dtype=dtype, ignored=ignored)


def listed():
    return [
        # the new tokens of 16 sequences in a generation step: latency
        _embed("embed_step_16", "embedding", 16, 1024, 50304, "bf16", "text"),
        # the tokens of a training batch, 16 sequences of 1024
        _embed("embed_train_16k", "embedding", 16384, 1024, 50304, "bf16", "text"),
        # the table's gradient for that batch: some tokens come often, most rows of the table not at all
        _embed("embed_bwd_train_16k", "embedding_bwd", 16384, 1024, 50304, "bf16", "text"),
        # the gradient of learned positions of an fp32 model: few rows, each once per sequence
        _embed("embed_bwd_positions", "embedding_bwd", 16384, 768, 1024, "f32", "positions"),
        # the norm before a sublayer in a generation step of 16 sequences: latency
        _norm("norm_step_16", "rms_norm", 16, 1024, "bf16", True),
        # the addition of a sublayer's output and the next sublayer's norm, training batch
        _norm("norm_train_16k", "rms_norm", 16384, 1024, "bf16", True),
        # its backward, the later layers' gradient of the sum added
        _norm("norm_bwd_train_16k", "rms_norm_bwd", 16384, 1024, "bf16", True),
        # a first norm without residual, fp32, a width that fills no lines
        _norm("norm_bwd_odd_f32", "rms_norm_bwd", 10007, 500, "f32", False),
        # scoring a few given tokens: the vocabulary's matrix read once
        _loss("loss_score_24", "cross_entropy", 24, 1024, 50304, "bf16", 0.0),
        # the loss of a training batch
        _loss("loss_train_16k", "cross_entropy", 16384, 1024, 50304, "bf16", 0.02),
        # its gradients
        _loss("loss_bwd_train_16k", "cross_entropy_bwd", 16384, 1024, 50304, "bf16", 0.02),
        # the gradients of a padded batch of a small fp32 model, sizes that fit no tile
        _loss("loss_bwd_small_f32", "cross_entropy_bwd", 1023, 200, 10007, "f32", 0.3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embedding", "embedding_bwd", "rms_norm", "rms_norm_bwd", "cross_entropy", "cross_entropy",
                     "cross_entropy_bwd", "cross_entropy_bwd"])
    dtype = "f32" if rng.random() < 0.35 else "bf16"
    dim = rng.choice([64, 72, 100, 128, 200, 256, 384, 500, 512, 640, 768, 1000, 1024, 1024, 1536, 2048])
    rows = _log(rng, 1, 16384 if dim <= 1024 else 8192)
    if op in ("embedding", "embedding_bwd"):
        vocab = _log(rng, 24, 50304 if dim <= 1024 else 25152)
        case = _embed("", op, rows, dim, vocab, dtype, rng.choice(["text", "text", "uniform", "positions", "one"]))
    elif op in ("rms_norm", "rms_norm_bwd"):
        case = _norm("", op, rows, dim + rng.choice([0, 0, 0, 1, 3]), dtype, rng.random() < 0.7)
    else:
        vocab = _log(rng, 24, 50304)
        # at most the largest listed call's products; in fp32 a tenth of them
        most = 16384 * 1024 * 50304 * (0.1 if dtype == "f32" else 1.0)
        while rows * dim * vocab > most:
            rows = max(1, rows * 5 // 8)
        case = _loss("", op, rows, dim, vocab, dtype, rng.choice([0.0, 0.02, 0.3]))
    del case["name"]
    return case


def work(case):
    b, d = (2 if case["dtype"] == "bf16" else 4), case["dim"]
    if case["op"] == "embedding":
        met = min(case["tokens"], case["vocab"])
        return {"bytes": b * d * (met + case["tokens"]) + 8 * case["tokens"], "flops": d * case["tokens"]}
    if case["op"] == "embedding_bwd":
        return {"bytes": b * d * (case["vocab"] + case["tokens"]) + 8 * case["tokens"], "flops": d * case["tokens"]}
    n = case["rows"] * d
    if case["op"] == "rms_norm":
        return {"bytes": b * n * (4 if case["residual"] else 2) + b * d + 4 * case["rows"], "flops": 5 * n}
    if case["op"] == "rms_norm_bwd":
        return {"bytes": b * n * (4 if case["residual"] else 3) + 2 * b * d + 4 * case["rows"], "flops": 10 * n}
    both = b * (n + case["vocab"] * d) + 8 * case["rows"]
    if case["op"] == "cross_entropy":
        return {"bytes": both + 8 * case["rows"], "flops": 2 * n * case["vocab"]}
    return {"bytes": 2 * both, "flops": 6 * n * case["vocab"]}


# ---------------------------------------------------------------- inputs

def _rng(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(1_000_003 * seed + stream)
    return g


def _text(n, vocab, g):
    """Tokens as frequent as words are: the n-th of the vocabulary 1/n times the first."""
    u = torch.rand(n, device=DEV, dtype=torch.float64, generator=g)
    return torch.exp(u * math.log(vocab + 1)).sub_(1).long().clamp_(0, vocab - 1)


def _tokens(case, g):
    n, vocab = case["tokens"], case["vocab"]
    if case["order"] == "positions":
        return torch.arange(n, device=DEV) % vocab
    if case["order"] == "one":         # padding throughout
        return torch.randint(vocab, (1,), device=DEV, generator=g).repeat(n)
    if case["order"] == "uniform":
        return torch.randint(vocab, (n,), device=DEV, generator=g)
    return _text(n, vocab, g)


def prepare(case, seed):
    g, dt, d = _rng(seed, 1), DTYPES[case["dtype"]], case["dim"]
    randn = lambda *shape: torch.randn(*shape, device=DEV, dtype=dt, generator=g)  # noqa: E731
    if case["op"] in ("embedding", "embedding_bwd"):
        s = {"case": case, "tokens": _tokens(case, g), "scale": math.sqrt(d)}
        if case["op"] == "embedding":
            s["table"] = randn(case["vocab"], d).mul_(0.02)
        else:
            s["grad"] = randn(case["tokens"], d).mul_(1e-3)
        return s
    n = case["rows"]
    if case["op"] in ("rms_norm", "rms_norm_bwd"):
        # a stream that grows from layer to layer, its rows of different sizes
        size = torch.exp(torch.randn(n, 1, device=DEV, generator=g) * 0.5).to(dt)
        s = {"case": case, "x": randn(n, d).mul_(size), "weight": randn(d).mul_(0.1).add_(1.0)}
        s["residual"] = randn(n, d).mul_(size * 3) if case["residual"] else None
        if case["op"] == "rms_norm_bwd":
            _, s["total"], s["rstd"] = _plain_rms_norm(s)
            s["grad"] = randn(n, d).mul_(1e-3)
            s["grad_total"] = randn(n, d).mul_(1e-3) if case["residual"] else None
        return s
    vocab = case["vocab"]
    s = {"case": case, "scale": 1.0, "weight": randn(vocab, d).mul_(1.5 / math.sqrt(d)), "targets": _text(n, vocab, g)}
    # hidden rows that have learnt something: their target's score lies up to some 9 above the others'
    learnt = torch.rand(n, 1, device=DEV, generator=g).mul_(4.0)
    s["hidden"] = torch.randn(n, d, device=DEV, generator=g).add_(learnt * s["weight"][s["targets"]].float()).to(dt)
    if case["ignored"]:
        out = torch.rand(n, device=DEV, generator=g) < case["ignored"]
        s["targets"] = torch.where(out, -100, s["targets"])
    if case["op"] == "cross_entropy_bwd":
        _, s["lse"] = _plain_cross_entropy(s)
        # the mean's gradient, tokens weighted
        s["grad"] = torch.rand(n, device=DEV, generator=g).add_(0.5).div_(n)
    return s


# ---------------------------------------------------------------- plain forms

def _plain_embedding(s):
    table, tokens = s["table"], s["tokens"]
    valid = (tokens >= 0) & (tokens < table.shape[0])
    y = table[torch.where(valid, tokens, 0)].float() * s["scale"]
    return torch.where(valid[:, None], y, 0.0).to(table.dtype)


def _plain_embedding_bwd(s):
    tokens, vocab = s["tokens"], s["case"]["vocab"]
    valid = (tokens >= 0) & (tokens < vocab)
    dw = torch.zeros(vocab + 1, s["grad"].shape[1], device=DEV)
    dw.index_add_(0, torch.where(valid, tokens, vocab), s["grad"].float() * s["scale"])
    return dw[:vocab].to(s["grad"].dtype)


def _plain_rms_norm(s):
    x = s["x"]
    z = x if s["residual"] is None else (x.float() + s["residual"].float()).to(x.dtype)
    f = z.float()
    rstd = 1 / ((f * f).sum(1) / f.shape[1] + EPS).sqrt()
    return (f * rstd[:, None] * s["weight"].float()).to(x.dtype), z, rstd


def _plain_rms_norm_bwd(s):
    g, rstd = s["grad"].float(), s["rstd"][:, None]
    n = s["total"].float() * rstd
    u = g * s["weight"].float()
    dx = rstd * (u - n * ((u * n).sum(1, keepdim=True) / n.shape[1]))
    if s["grad_total"] is not None:
        dx = dx + s["grad_total"].float()
    return dx.to(s["total"].dtype), (g * n).sum(0).to(s["weight"].dtype)


def _plain_logits(s):
    return (s["hidden"].float() @ s["weight"].float().t()).mul_(s["scale"])


def _plain_targets(s):
    valid = (s["targets"] >= 0) & (s["targets"] < s["weight"].shape[0])
    return valid, torch.where(valid, s["targets"], 0)[:, None]


def _plain_cross_entropy(s):
    logits = _plain_logits(s)
    valid, at = _plain_targets(s)
    top = logits.amax(1, keepdim=True)
    own_logit = logits.gather(1, at)
    lse = top + logits.sub_(top).exp_().sum(1, keepdim=True).log()
    return torch.where(valid, (lse - own_logit)[:, 0], 0.0), lse[:, 0]


def _plain_cross_entropy_bwd(s):
    p = _plain_logits(s).sub_(s["lse"][:, None]).exp_()
    valid, at = _plain_targets(s)
    g = torch.where(valid, s["grad"], 0.0)[:, None]
    p.scatter_add_(1, at, -valid[:, None].float()).mul_(g)
    dh = (p @ s["weight"].float()).mul_(s["scale"])
    dw = (p.t() @ s["hidden"].float()).mul_(s["scale"])
    return dh.to(s["hidden"].dtype), dw.to(s["weight"].dtype)


# ---------------------------------------------------------------- one pass

def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2607_20652_amd import binding as dpb
    if op == "embedding":
        return {"out": dpb.embedding(s["tokens"], s["table"], scale=s["scale"]) if own else _plain_embedding(s)}
    if op == "embedding_bwd":
        return {"dweight": dpb.embedding_bwd(s["grad"], s["tokens"], s["case"]["vocab"], scale=s["scale"]) if own
                else _plain_embedding_bwd(s)}
    if op == "rms_norm":
        out, total, rstd = dpb.rms_norm(s["x"], s["weight"], s["residual"], eps=EPS) if own else _plain_rms_norm(s)
        return {"out": out, "total": total, "rstd": rstd}
    if op == "rms_norm_bwd":
        dx, dw = dpb.rms_norm_bwd(s["grad"], s["total"], s["weight"], s["rstd"], grad_total=s["grad_total"]) if own \
            else _plain_rms_norm_bwd(s)
        return {"dx": dx, "dweight": dw}
    if op == "cross_entropy":
        loss, lse = dpb.cross_entropy(s["hidden"], s["weight"], s["targets"], scale=s["scale"]) if own \
            else _plain_cross_entropy(s)
        return {"loss": loss, "lse": lse}
    dh, dw = dpb.cross_entropy_bwd(s["grad"], s["hidden"], s["weight"], s["targets"], s["lse"], scale=s["scale"]) if own \
        else _plain_cross_entropy_bwd(s)
    return {"dhidden": dh, "dweight": dw}


# ---------------------------------------------------------------- 64 bits

def _exact_embedding(case, s):
    live = (s["tokens"] >= 0) & (s["tokens"] < case["vocab"])
    if case["op"] == "embedding":
        out = torch.zeros(case["tokens"], case["dim"], dtype=torch.float64, device=DEV)
        out[live] = s["table"].double()[s["tokens"][live]] * s["scale"]
        return {"out": out}
    # sums of the sorted tokens' rows, as differences of running sums within blocks of columns
    order = torch.argsort(s["tokens"][live], stable=True)
    toks, counts = torch.unique_consecutive(s["tokens"][live][order], return_counts=True)
    ends = counts.cumsum(0)
    dw = torch.zeros(case["vocab"], case["dim"], dtype=torch.float64, device=DEV)
    if len(toks):
        run_sum = s["grad"][live][order].double().cumsum(0)[ends - 1]
        dw[toks] = torch.diff(run_sum, dim=0, prepend=torch.zeros_like(run_sum[:1])) * s["scale"]
    return {"dweight": dw}


def _exact_norm(case, s):
    z = s["x"].double()
    if case["residual"]:
        z = z + s["residual"].double()
        total = z
        z = z.to(s["x"].dtype).double()      # the norm is of the sum as it is kept
    else:
        total = z
    if case["op"] == "rms_norm":
        rstd = (z.square().mean(1) + EPS).rsqrt()
        return {"out": z * rstd[:, None] * s["weight"].double(), "total": total, "rstd": rstd}
    z, rstd, g, w = s["total"].double(), s["rstd"].double()[:, None], s["grad"].double(), s["weight"].double()
    dx = rstd * g * w - z * rstd ** 3 * (g * w * z).mean(1, keepdim=True)
    if case["residual"]:
        dx = dx + s["grad_total"].double()
    return {"dx": dx, "dweight": torch.mv((g * z).t(), rstd[:, 0])}


def _exact_loss(case, s):
    back, n = case["op"] == "cross_entropy_bwd", case["rows"]
    h, w, t = s["hidden"].double(), s["weight"].double(), s["targets"]
    part = max(1, 2 ** 27 // case["vocab"])
    losses, lses, dhs, dw = [], [], [], torch.zeros_like(w) if back else None
    for at in range(0, n, part):
        x, c = h[at:at + part], t[at:at + part]
        logits = torch.mm(x, w.t()) * s["scale"]
        rows = torch.nonzero((c >= 0) & (c < case["vocab"]))[:, 0]
        if back:
            p = torch.exp(logits - s["lse"][at:at + part].double()[:, None])
            p[rows, c[rows]] -= 1
            keep = torch.zeros(len(c), dtype=torch.float64, device=DEV)
            keep[rows] = s["grad"][at:at + part][rows].double() * s["scale"]
            p *= keep[:, None]
            dhs.append(torch.mm(p, w))
            dw += torch.mm(p.t(), x)
        else:
            lse = torch.logsumexp(logits, 1)
            loss = torch.zeros_like(lse)
            loss[rows] = lse[rows] - logits[rows, c[rows]]
            losses.append(loss)
            lses.append(lse)
    return {"dhidden": torch.cat(dhs), "dweight": dw} if back else {"loss": torch.cat(losses), "lse": torch.cat(lses)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("embedding", "embedding_bwd"):
        return _exact_embedding(case, s)
    if case["op"] in ("rms_norm", "rms_norm_bwd"):
        return _exact_norm(case, s)
    return _exact_loss(case, s)
