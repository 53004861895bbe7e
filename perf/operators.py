"""The calls of the training operators whose speed is measured, and their plain forms.

A case names an operator and its sizes:

  attention      dpb.attention: softmax attention, for a batch or for one new token over a cache
  attention_bwd  dpb.attention_bwd: its gradients, from the forward's output and log-sum-exp
  adamw          dpb.adamw_step: one AdamW step over all tensors of a model

The plain forms are elementary torch operations in 32 bits; `exact` has the
results in 64 bits from the operators' definitions.  Inputs are drawn from
the seed; the lengths of ragged batches belong to the case.

Attention: sequences are padded ([B, S, heads, D], with lengths in mode
"lens") or packed one behind the other ([tokens, heads, D] with their starts,
mode "packed").  Key j is visible to query i of the same sequence when
j < k_len and, if causal, j <= i + k_len - q_len; a query that sees no key
gets zeros and a log-sum-exp of -inf.

AdamW: the tensors lie in one buffer, each at a multiple of 256 elements (as
their states do); states are fp32 (m, v) or 8-bit floats (m and sqrt(v), one
scale per 256 elements, rounded up or down at random by a hash of the seed and
the element's place).
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 256          # elements that share the scales of 8-bit states
LR, BETAS, EPS, DECAY, STEP = 1e-4, (0.9, 0.999), 1e-8, 0.1, 1000


def _attn(name, op, batch, q_len, k_len, heads, kv_heads, dim, dtype, causal=True, mode="full", layout="bshd"):
    return dict(name=name, op=op, batch=batch, q_len=q_len, k_len=k_len, heads=heads, kv_heads=kv_heads, dim=dim,
                dtype=dtype, causal=causal, mode=mode, layout=layout)


def _adamw(name, width, layers, vocab, dtype, bits, master):
    return dict(name=name, op="adamw", width=width, layers=layers, vocab=vocab, dtype=dtype, bits=bits, master=master)


def listed():
    return [
        # one new token of each of 16 sequences over their caches, as many key heads as query heads: a generation step
        _attn("attn_token_16", "attention", 16, 1, 1024, 16, 16, 64, "bf16", mode="lens"),
        # one new token over long caches with shared key heads: few rows, a long axis
        _attn("attn_token_long", "attention", 3, 1, 131072, 32, 8, 128, "bf16", mode="lens"),
        # the forward of a training batch: 16 sequences of 1024 tokens
        _attn("attn_train_16k", "attention", 16, 1024, 1024, 16, 16, 64, "bf16"),
        # a long prompt with shared key heads
        _attn("attn_prompt_16k", "attention", 1, 16384, 16384, 16, 4, 128, "bf16"),
        # documents of all lengths packed one behind the other, 16 heads
        _attn("attn_packed_docs", "attention", 37, 2048, 2048, 16, 16, 64, "bf16", mode="packed"),
        # the gradients of two short sequences of a small fp32 model: latency
        _attn("bwd_small_f32", "attention_bwd", 2, 65, 65, 4, 4, 32, "f32"),
        # the backward of the training batch
        _attn("bwd_train_16k", "attention_bwd", 16, 1024, 1024, 16, 16, 64, "bf16"),
        # the backward of long sequences with shared key heads
        _attn("bwd_long_8k", "attention_bwd", 2, 8192, 8192, 16, 4, 128, "bf16"),
        # fp32 analysis of a padded batch that attends over another sequence, head width that fits no tile
        _attn("bwd_cross_f32", "attention_bwd", 3, 511, 1203, 6, 2, 72, "f32", causal=False, mode="lens", layout="bhsd"),
        # one step of a small fp32 model: many little tensors, latency
        _adamw("adamw_small_32", 64, 4, 1000, "f32", 32, False),
        # a 12-layer model of width 1024, fp32 parameters and states
        _adamw("adamw_1024_32", 1024, 12, 50304, "f32", 32, False),
        # the same model with bf16 parameters and gradients, fp32 masters and 8-bit states
        _adamw("adamw_1024_8", 1024, 12, 50304, "bf16", 8, True),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v + 1 if v == 3072 else v


def draw(rng):
    op = rng.choice(["token", "attention", "attention", "attention_bwd", "attention_bwd", "adamw"])
    if op == "adamw":
        bits = rng.choice([8, 32])
        dtype = rng.choice(["bf16", "f32"])
        width = rng.choice([64, 100, 200, 256, 384, 500, 512, 640, 800, 1000, 1024])
        case = _adamw("", width, rng.randint(1, 12), _log(rng, 100, 50304), dtype, bits,
                      dtype == "bf16" and rng.random() < 0.7)
    elif op == "token":
        case = _draw_token(rng)
    else:
        case = _draw_attention(rng, op)
    del case["name"]
    return case


def _draw_heads(rng):
    kv = rng.choice([1, 2, 3, 4, 5, 8, 12, 16])
    heads = kv * rng.choice([g for g in (1, 1, 2, 4, 7, 8) if kv * g <= 32])
    dim = rng.choice([64, 64, 64, 128, 128, 128, 16, 32, 40, 72, 80, 96, 112])
    if 3072 in (heads * dim, kv * dim, 2 * heads * dim, 2 * kv * dim):
        dim = 40
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    return heads, kv, dim, dtype, rng.choice(["bshd", "bshd", "bhsd", "pair"]), rng.random() < 0.75


def _draw_token(rng):
    heads, kv, dim, dtype, layout, causal = _draw_heads(rng)
    k_len = _log(rng, 1, 131072)
    # at most 4e8 elements of keys
    batch = _log(rng, 1, min(256, max(1, int(4e8 / (k_len * kv * dim)))))
    return _attn("", "attention", batch, rng.choice([1, 1, 1, 2, 5]), k_len, heads, kv, dim, dtype, causal,
                 rng.choice(["full", "lens", "lens"]), layout)


def _draw_attention(rng, op):
    heads, kv, dim, dtype, layout, causal = _draw_heads(rng)
    mode = rng.choice(["full", "full", "lens", "packed"])
    # (behind a single key the gradients of q and k are what is left of a difference of equal numbers)
    least = 2 if op == "attention_bwd" else 1
    q_len = _log(rng, least, 8192)
    k_len = q_len if mode == "packed" or rng.random() < 0.6 else _log(rng, least, 8192)
    # at most a third of the largest listed call's products, and 8 GB of scores in the plain form
    most = min(16384.0 ** 2 * 16 * 128 / 6 * (0.1 if dtype == "f32" else 1) / dim, 2e9) / heads
    while q_len * k_len > most:
        q_len = max(least, q_len * 5 // 8)
        k_len = q_len if mode == "packed" else max(least, k_len * 5 // 8)
    batch = max(1, min(64, _log(rng, 1, max(1, int(most / (q_len * k_len))))))
    return _attn("", op, batch, q_len, k_len, heads, kv, dim, dtype, causal, mode, layout)


# ---------------------------------------------------------------- sizes of a case

def _lens(case):
    """Lengths of the sequences (queries, keys): the first has the full length, others are spread below it."""
    B, Q, K = case["batch"], case["q_len"], case["k_len"]
    if case["mode"] == "full":
        return [Q] * B, [K] * B
    r = random.Random(f"{B} {Q} {K} {case['heads']} {case['dim']}")
    k = [K] + [r.randint(0, K) for _ in range(B - 1)]
    if case["mode"] == "packed":
        return k, k
    q = [Q] * B if Q <= 8 else [Q] + [r.randint(0, Q) for _ in range(B - 1)]
    return q, k


def _shapes(case):
    d, ff = case["width"], 4 * case["width"]
    layer = [(d,), (d, d), (d, d), (d, d), (d, d), (d,), (ff, d), (ff,), (d, ff), (d,)]
    return [(case["vocab"], d)] + layer * case["layers"] + [(d,)]


def work(case):
    if case["op"] == "adamw":
        n = sum(math.prod(s) for s in _shapes(case))
        p = 2 if case["dtype"] == "bf16" else 4
        # gradient read, parameter written (and read where there is no master), master and both states read and written
        size = p + p + (8 if case["master"] else p) + 2 * 2 * (4 if case["bits"] == 32 else 1 + 4 / BLOCK)
        return {"bytes": n * size, "flops": n * 16}
    ql, kl = _lens(case)
    pairs = 0
    for q, k in zip(ql, kl):
        if case["causal"]:
            # query i sees max(0, min(k, i + 1 + k - q)) keys
            seen = min(q, k)
            pairs += seen * (seen + 1) // 2 + seen * (k - seen)
        else:
            pairs += q * k
    b, H, G, D = (2 if case["dtype"] == "bf16" else 4), case["heads"], case["kv_heads"], case["dim"]
    rows, cols = sum(ql) * H, sum(kl) * G
    if case["op"] == "attention":
        return {"bytes": b * D * (2 * rows + 2 * cols) + 4 * rows, "flops": 4 * D * pairs * H}
    return {"bytes": b * D * (4 * rows + 4 * cols) + 4 * rows, "flops": 10 * D * pairs * H}


# ---------------------------------------------------------------- inputs

def _rng(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(1_000_003 * seed + stream)
    return g


def _rows(case, tokens, heads, g, scale=1.0):
    """[B, tokens, heads, D] (packed: [total, heads, D]) in the case's memory order."""
    dt, D = DTYPES[case["dtype"]], case["dim"]
    if case["mode"] == "packed":
        n = sum(_lens(case)[0])
        if case["layout"] == "pair":      # beside another tensor, as in the output of one projection
            return torch.randn(n, 2, heads, D, device=DEV, dtype=dt, generator=g).mul_(scale)[:, 0]
        return torch.randn(n, heads, D, device=DEV, dtype=dt, generator=g).mul_(scale)
    B = case["batch"]
    if case["layout"] == "bhsd":
        return torch.randn(B, heads, tokens, D, device=DEV, dtype=dt, generator=g).mul_(scale).transpose(1, 2)
    if case["layout"] == "pair":
        return torch.randn(B, tokens, 2, heads, D, device=DEV, dtype=dt, generator=g).mul_(scale)[:, :, 0]
    return torch.randn(B, tokens, heads, D, device=DEV, dtype=dt, generator=g).mul_(scale)


def _sequences(case):
    """What a program says of its sequences, as keyword arguments of the calls."""
    ql, kl = _lens(case)
    of = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    if case["mode"] == "packed":
        starts = [0]
        for n in ql:
            starts.append(starts[-1] + n)
        return dict(q_starts=of(starts), k_starts=of(starts), max_q=max(ql), max_k=max(kl))
    return dict(q_lens=of(ql), k_lens=of(kl)) if case["mode"] == "lens" else {}


def prepare(case, seed):
    g = _rng(seed, 1)
    if case["op"] != "adamw":
        s = {"case": case, "seqs": _sequences(case),
             "q": _rows(case, case["q_len"], case["heads"], g, 2.0),
             "k": _rows(case, case["k_len"], case["kv_heads"], g),
             "v": _rows(case, case["k_len"], case["kv_heads"], g)}
        if case["op"] == "attention_bwd":
            s["out"], s["lse"] = _plain_attention(s)
            s["grad"] = _rows(case, case["q_len"], case["heads"], g)
        return s
    shapes = _shapes(case)
    blocks = [-(-math.prod(x) // BLOCK) for x in shapes]
    n = sum(blocks)
    dt = DTYPES[case["dtype"]]
    live = torch.zeros(n * BLOCK, dtype=torch.bool, device=DEV)
    s = {"case": case, "seed": (12345 + 1_000_003 * seed) % 2**32}
    at, spans = 0, []
    for x, b in zip(shapes, blocks):
        spans.append((at * BLOCK, math.prod(x), x))
        live[spans[-1][0]:spans[-1][0] + spans[-1][1]] = True
        at += b
    w = torch.randn(n * BLOCK, device=DEV, generator=g).mul_(0.02).mul_(live)
    # gradients whose size changes from one output row to the next, and moments of such gradients
    size = torch.exp(torch.randn(n, 1, device=DEV, generator=g)).mul_(1e-3)
    noise = lambda: torch.randn(n * BLOCK, device=DEV, generator=g).mul_(live)  # noqa: E731
    s["param"] = w.to(dt)
    s["grad"] = noise().view(n, BLOCK).mul_(size).view(-1).to(dt)
    m = noise().view(n, BLOCK).mul_(size * 0.3)
    u = (noise().view(n, BLOCK) * 0.2 + 1).abs_().mul_(size).mul_(live.view(n, BLOCK))
    if case["bits"] == 32:
        s["m"], s["v"], s["scales"] = m.view(-1), u.square().view(-1), None
    else:
        sm, su = (x.abs().amax(1, keepdim=True).div_(448.0) for x in (m, u))
        of = lambda x, sc: (x / sc.clamp_min(1e-30)).to(torch.float8_e4m3fn).view(-1)  # noqa: E731
        s["m"], s["v"], s["scales"] = of(m, sm), of(u, su), torch.cat([sm, su], 1).contiguous()
    s["master"] = w if case["master"] else None
    s["decay"] = [DECAY if len(x) > 1 else 0.0 for x in shapes]
    s["block_decay"] = torch.tensor(s["decay"], device=DEV).repeat_interleave(torch.tensor(blocks, device=DEV))[:, None]
    s["params"] = [s["param"][a:a + k].view(x) for a, k, x in spans]
    s["grads"] = [s["grad"][a:a + k].view(x) for a, k, x in spans]
    return s


# ---------------------------------------------------------------- plain forms

def _padded(case, x, starts, longest):
    """Packed rows as [B, longest, heads, D]; places past a sequence's end hold some other row."""
    at = starts[:-1, None].long() + torch.arange(longest, device=DEV)
    return x[at.clamp_(max=x.shape[0] - 1)]


def _packed(x, lens):
    """The reverse for [B, longest, ...]: the rows of all sequences one behind the other."""
    return x[torch.arange(x.shape[1], device=DEV) < lens[:, None]]


def _plain_sides(s):
    """q, k, v in fp32 as [B, heads, S, D], the visible pairs [B, 1, Sq, Sk], and the lengths."""
    case, seqs = s["case"], s["seqs"]
    q, k, v = s["q"], s["k"], s["v"]
    if case["mode"] == "packed":
        ql = kl = (seqs["q_starts"][1:] - seqs["q_starts"][:-1]).long()
        q, k, v = (_padded(case, x, seqs["q_starts"], seqs["max_q"]) for x in (q, k, v))
    elif case["mode"] == "lens":
        ql, kl = seqs["q_lens"].long(), seqs["k_lens"].long()
    else:
        ql, kl = (torch.full((q.shape[0],), x.shape[1], device=DEV) for x in (q, k))
    i = torch.arange(q.shape[1], device=DEV)[None, :, None]
    j = torch.arange(k.shape[1], device=DEV)[None, None, :]
    seen = (i < ql[:, None, None]) & (j < kl[:, None, None])
    if case["causal"]:
        seen = seen & (j <= i + (kl - ql)[:, None, None])
    group = case["heads"] // case["kv_heads"]
    q, k, v = (x.float().transpose(1, 2) for x in (q, k, v))
    if group > 1:
        k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    return q, k, v, seen[:, None], ql


def _plain_attention(s):
    case = s["case"]
    q, k, v, seen, ql = _plain_sides(s)
    p = (q @ k.transpose(2, 3)).mul_(1 / math.sqrt(case["dim"])).masked_fill_(~seen, -math.inf)
    top = p.amax(3, keepdim=True)
    p.sub_(top.masked_fill(top == -math.inf, 0.0)).exp_()
    total = p.sum(3, keepdim=True)
    lse = (top + total.log()).squeeze(3).transpose(1, 2).contiguous()
    out = ((p @ v) / total.masked_fill(total == 0, 1.0)).transpose(1, 2).to(s["q"].dtype)
    if case["mode"] == "packed":
        return _packed(out, ql), _packed(lse, ql)
    return out.contiguous(), lse


def _plain_attention_bwd(s):
    case = s["case"]
    q, k, v, seen, ql = _plain_sides(s)
    out, lse, grad = s["out"], s["lse"], s["grad"]
    if case["mode"] == "packed":
        starts, most = s["seqs"]["q_starts"], s["seqs"]["max_q"]
        out, lse, grad = (_padded(case, x, starts, most) for x in (out, lse, grad))
    out, grad = out.float().transpose(1, 2), grad.float().transpose(1, 2)
    lse = lse.transpose(1, 2).unsqueeze(3)
    scale = 1 / math.sqrt(case["dim"])
    p = (q @ k.transpose(2, 3)).mul_(scale).sub_(lse.masked_fill(lse == -math.inf, 0.0)).masked_fill_(~seen, -math.inf).exp_()
    dv = p.transpose(2, 3) @ grad
    ds = (grad @ v.transpose(2, 3)).sub_((grad * out).sum(3, keepdim=True)).mul_(p)
    del p
    dq, dk = (ds @ k).mul_(scale), (ds.transpose(2, 3) @ q).mul_(scale)
    shared = (dk.shape[0], case["kv_heads"], -1, dk.shape[2], dk.shape[3])
    dk, dv = dk.view(shared).sum(2), dv.view(shared).sum(2)
    dq, dk, dv = (x.transpose(1, 2).to(s["q"].dtype) for x in (dq, dk, dv))
    if case["mode"] == "packed":
        return tuple(_packed(x, ql) for x in (dq, dk, dv))
    return dq, dk, dv


def _hash(n, seed):
    """32 random bits for each of the places 0..n-1, a function of the place and the seed."""
    low = 0xFFFFFFFF
    x = torch.arange(n, device=DEV)
    x = ((x & low) * 0x9E3779B9 + (x >> 32) * 0x6A09E667 + seed) & low
    x = ((x ^ (x >> 16)) * 0x6A09E667) & low
    x = ((x ^ (x >> 15)) * 0x9E3779B9) & low
    return x ^ (x >> 16)


def _plain_round8(x, bits):
    """x in [-448, 448] rounded up or down at random to an 8-bit float: 16 random bits against the part cut off."""
    a = x.abs()
    step = torch.exp2(a.clamp_min(2.0 ** -6).frexp().exponent.float() - 4)     # 3 bits behind the leading one
    up = a / step + bits.float() * 2.0 ** -16
    return torch.copysign((up.floor_() * step).clamp_(max=448.0), x).to(torch.float8_e4m3fn)


def _plain_adamw(s):
    case, (b1, b2) = s["case"], BETAS
    rows = lambda x: x.view(-1, BLOCK)  # noqa: E731
    w = rows(s["master"] if s["master"] is not None else s["param"]).float()
    g = rows(s["grad"]).float()
    if case["bits"] == 32:
        m, v = rows(s["m"]), rows(s["v"])
    else:
        m = rows(s["m"]).float() * s["scales"][:, :1]
        v = (rows(s["v"]).float() * s["scales"][:, 1:]).square()
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    u = v.sqrt()
    new = w * (1 - LR * s["block_decay"]) - m * (LR / (1 - b1 ** STEP)) / (u / math.sqrt(1 - b2 ** STEP) + EPS)
    if case["bits"] == 32:
        s["m"].view(-1, BLOCK).copy_(m)
        s["v"].view(-1, BLOCK).copy_(v)
    else:
        sc = torch.stack([m.abs().amax(1), u.amax(1)], 1) * (1 / 448.0)
        inv = (1 / sc).masked_fill_(sc < 2.0 ** -126, 0.0)
        r = rows(_hash(m.numel(), s["seed"]))
        c = _plain_round8((u * inv[:, 1:]).clamp_(max=448.0), r >> 16)
        tiny = torch.tensor(2.0 ** -9, device=DEV).to(torch.float8_e4m3fn)
        c = torch.where((u > 0) & (c.float() == 0), tiny.view(torch.uint8), c.view(torch.uint8))
        rows(s["m"]).copy_(_plain_round8((m * inv[:, :1]).clamp_(-448.0, 448.0), r & 0xFFFF))
        rows(s["v"].view(torch.uint8)).copy_(c)
        s["scales"].copy_(sc)
    if s["master"] is not None:
        rows(s["master"]).copy_(new)
    rows(s["param"]).copy_(new)


# ---------------------------------------------------------------- one pass

def run(s):
    case = s["case"]
    if own:
        from paper_2607_20652_amd import binding as dpb
    if case["op"] == "attention":
        if own:
            out, lse = dpb.attention(s["q"], s["k"], s["v"], causal=case["causal"], **s["seqs"])
        else:
            out, lse = _plain_attention(s)
        return {"out": out, "lse": lse}
    if case["op"] == "attention_bwd":
        if own:
            dq, dk, dv = dpb.attention_bwd(s["grad"], s["q"], s["k"], s["v"], s["out"], s["lse"],
                                           causal=case["causal"], **s["seqs"])
        else:
            dq, dk, dv = _plain_attention_bwd(s)
        return {"dq": dq, "dk": dk, "dv": dv}
    if own:
        dpb.adamw_step(s["params"], s["grads"], s["m"], s["v"], scales=s["scales"], master=s["master"], step=STEP,
                       lr=LR, betas=BETAS, eps=EPS, weight_decay=s["decay"], seed=s["seed"])
    else:
        _plain_adamw(s)
    return {k: s[k] for k in ("param", "m", "v", "scales", "master") if s[k] is not None}


# ---------------------------------------------------------------- 64 bits

def _exact_head(q, k, v, causal, grad=None):
    """One sequence and head in fp64: (out, lse), or the gradients (dq, dk, dv) for `grad`; queries a part at a time."""
    n, m, scale = q.shape[0], k.shape[0], q.shape[1] ** -0.5
    part = max(1, 2 ** 25 // max(1, m))
    outs, lses, dqs, dk, dv = [], [], [], torch.zeros_like(k), torch.zeros_like(v)
    for at in range(0, n, part):
        x = q[at:at + part]
        score = torch.mm(x, k.t()) * scale
        if causal:
            last = torch.arange(at, at + x.shape[0], device=DEV) + (m - n)
            score[torch.arange(m, device=DEV) > last[:, None]] = -math.inf
        lse = torch.logsumexp(score, 1) if m else torch.full((x.shape[0],), -math.inf, device=DEV, dtype=torch.float64)
        p = torch.where(score == -math.inf, 0.0, torch.exp(score - lse[:, None]))
        o = torch.mm(p, v)
        outs.append(o)
        lses.append(lse)
        if grad is not None:
            go = grad[at:at + part]
            dv += torch.mm(p.t(), go)
            ds = p * (torch.mm(go, v.t()) - (go * o).sum(1, keepdim=True)) * scale
            dqs.append(torch.mm(ds, k))
            dk += torch.mm(ds.t(), x)
    if grad is None:
        return torch.cat(outs), torch.cat(lses)
    return torch.cat(dqs), dk, dv


def _exact_attention(case, s):
    ql, kl = _lens(case)
    packed, group, back = case["mode"] == "packed", case["heads"] // case["kv_heads"], case["op"] == "attention_bwd"
    zeros = lambda x: torch.zeros(x.shape, dtype=torch.float64, device=DEV)  # noqa: E731
    out, dq, dk, dv = zeros(s["q"]), zeros(s["q"]), zeros(s["k"]), zeros(s["v"])
    lse = torch.full(s["q"].shape[:-1], -math.inf, dtype=torch.float64, device=DEV)
    at = 0
    for b in range(case["batch"]):
        qs = (slice(at, at + ql[b]),) if packed else (b, slice(0, ql[b]))
        ks = qs if packed else (b, slice(0, kl[b]))
        at += ql[b]
        if not ql[b]:
            continue
        for h in range(case["heads"]):
            q, k, v = (s[n][x + (e,)].double() for n, x, e in (("q", qs, h), ("k", ks, h // group), ("v", ks, h // group)))
            if back:
                got = _exact_head(q, k, v, case["causal"], s["grad"][qs + (h,)].double())
                dq[qs + (h,)] = got[0]
                dk[ks + (h // group,)] += got[1]
                dv[ks + (h // group,)] += got[2]
            else:
                out[qs + (h,)], lse[qs + (h,)] = _exact_head(q, k, v, case["causal"])
    return {"dq": dq, "dk": dk, "dv": dv} if back else {"out": out, "lse": lse}


def _exact_adamw(case, s):
    (b1, b2), n = BETAS, s["m"].numel()
    start = (s["master"] if case["master"] else s["param"]).double()
    g, m, v = s["grad"].double(), s["m"].double(), s["v"].double()
    if case["bits"] == 8:
        each = s["scales"].double().repeat_interleave(BLOCK, 0)
        m, v = m * each[:, 0], (v * each[:, 1]) ** 2
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    decay = s["block_decay"].double().repeat_interleave(BLOCK, 0)[:, 0]
    w = start * (1 - LR * decay) - LR * (m / (1 - b1 ** STEP)) / ((v / (1 - b2 ** STEP)).sqrt() + EPS)
    got = {"param": w}
    if case["master"]:
        got["master"] = w
    if case["bits"] == 32:
        return got | {"m": m, "v": v}
    # where an 8-bit state falls is random; that it is one of the two neighbours has tests of its own
    scale = torch.stack([m.abs().view(-1, BLOCK).amax(1), v.view(-1, BLOCK).amax(1).sqrt()], 1) / 448
    return got | {"m": None, "v": None, "scales": scale}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_adamw(case, s) if case["op"] == "adamw" else _exact_attention(case, s)
