"""The DPB as a differentiable layer, and an MLP block that uses it.

`DPBLayer.apply(x, plan, normalized, n_min, std)` returns (y, loss_var):
  * forward: encode (§2.2 beam search; on standardized scores when a
    Standardizer is given), decode (§2.1), and, when `normalized`,
    the rescaling of the decoder output to ||x|| (§2.2 "Normalized
    Reconstruction"); loss_var is the variance auxiliary loss of the code
    (§2.2 "Auxillary losses"), or 0 when n_min is None; its per-slot
    pre-gradients stay in a workspace for the backward;
  * backward: the indices are held fixed and coef = Phi_S x (standardized:
    coef = (Phi_S x - mu) r), so
        grad_u    = backward of the normalization (dpb_normalize_bwd),
        grad_coef = Phi_S^T grad_u + g_loss * dL_var/dcoef,
        grad_x    = Phi_S (r grad_coef) + (the norm path of the normalization),
    all in the library's kernels: the normalization backward writes the
    norm-path term into the grad_x buffer and one dpb_decode_bwd_ex call adds
    the decode of grad_coef to it; a training backward then applies the EMA
    update of the standardization statistics from the batch.

`DPBMLP` places the layer in front of a GELU MLP with a residual connection
and RMSNorm, the position the paper's ParityTransformer gives it (§3.1: a
bottleneck before the input to every MLP).  The MLP's matrices are ordinary
torch layers; everything of the DPB itself runs in libdpb.so.

`AttentionLayer.apply(q, k, v, causal, scale, q_lens, k_lens)` is softmax
attention as a differentiable function (dpb_attention, dpb_attention_bwd);
`CausalAttention` the sublayer around it, with a key-value cache for generation,
and `ParityBlock` the two sublayers of one transformer block.

`EmbeddingLayer`, `RMSNormLayer` and `CrossEntropyLayer` are what stands around the
blocks as differentiable functions: the lookup of a table's rows, the residual's
addition with the norm of the sum, and the loss over a vocabulary; `Embedding` and
`RMSNorm` are torch's modules by the first two, and `ParityTransformer` is the whole model
from them (§3.1).
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding as B


class Standardizer:
    """EMA score-standardization state of one bottleneck (§2.2 "Score
    Standardization"): stats [N, 2] = (mu, r = 1/sigma) and m2 [N] (moving
    second raw moment), updated after every training backward with `momentum`."""

    def __init__(self, plan: B.Plan, momentum: float = 0.01, eps: float = 1e-6, device=None):
        self.plan, self.momentum, self.eps = plan, momentum, eps
        self.stats, self.m2 = B.std_state(plan, device)
        self.workspace = B.std_workspace(plan, self.stats.device)
        self.training = True

    def update(self, x: torch.Tensor, idx: torch.Tensor):
        B.std_update(self.plan, x, idx, self.stats, self.m2, self.momentum, self.eps, self.workspace)


class DPBLayer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x: torch.Tensor, plan: B.Plan, normalized: bool = True, n_min: int | None = None,
                std: Standardizer | None = None):
        x = x.contiguous()
        idx, coef = B.encode_std(plan, x, std.stats) if std is not None else B.encode(plan, x)
        u = B.decode(plan, idx, coef, x.dtype)
        y = B.normalize(plan, u, x) if normalized else u
        ws = None
        if n_min is not None:
            ws = B.variance_workspace(plan, x.shape[0], x.device)
            loss, _ = B.variance_loss(plan, idx, coef, n_min, with_grad=False, workspace=ws)
        else:
            loss = torch.zeros((), dtype=torch.float32, device=x.device)
        ctx.plan, ctx.normalized, ctx.n_min, ctx.std = plan, normalized, n_min, std
        ctx.save_for_backward(x, idx, coef, u, ws)
        ctx.set_materialize_grads(False)
        return y, loss

    @staticmethod
    @once_differentiable
    def backward(ctx, gy: torch.Tensor | None, gloss: torch.Tensor | None):
        plan = ctx.plan
        x, idx, coef, u, ws = ctx.saved_tensors
        if gy is None:
            gy = torch.zeros_like(x)
        gy = gy.contiguous()
        if ctx.normalized:
            gu, gx = B.normalize_bwd(plan, gy, u, x, gu_dtype=gy.dtype, gr_dtype=x.dtype)
        else:
            gu, gx = gy, None
        add_gc = None
        if gloss is not None and ctx.n_min is not None:
            # the forward left the per-slot pre-gradients in ws
            add_gc = B.variance_grad(plan, x.shape[0], ws, grad_scale=gloss.to(torch.float32).contiguous())
        std = ctx.std
        _, gx = B.decode_bwd_ex(plan, idx, gu, add_grad_coef=add_gc, add_grad_x=gx, gx_dtype=x.dtype, grad_x=gx,
                                stats=std.stats if std is not None else None)
        if std is not None and std.training:
            # the statistics this batch was encoded with are no longer needed
            std.update(x, idx)
        return gx, None, None, None, None


def dpb_layer(x: torch.Tensor, plan: B.Plan, normalized: bool = True, n_min: int | None = None,
              std: Standardizer | None = None):
    """Functional form of DPBLayer: (y, loss_var)."""
    return DPBLayer.apply(x, plan, normalized, n_min, std)


class RMSNorm(torch.nn.RMSNorm):
    """torch.nn.RMSNorm over the last dimension; with a residual, norm(x, residual) is (norm of their sum, the sum) by
    RMSNormLayer, in the residual's type."""

    def forward(self, x: torch.Tensor, residual: torch.Tensor | None = None):
        if residual is None:
            return super().forward(x)
        # (torch.nn.RMSNorm's own default, in bf16 too)
        eps = torch.finfo(torch.float32).eps if self.eps is None else self.eps
        # (under autocast a sublayer's output has not the stream's type)
        return RMSNormLayer.apply(x.to(residual.dtype), self.weight, residual, eps)


def _add_norm(norm: torch.nn.Module, x: torch.Tensor, residual: torch.Tensor):
    """(norm of the sum, the sum), in one call where the norm offers that: another may stand in its place."""
    if isinstance(norm, RMSNorm):
        return norm(x, residual)
    total = x.to(residual.dtype) + residual
    return norm(total), total


class DPBMLP(torch.nn.Module):
    """h + W2 gelu(W1 DPB(rmsnorm(h))): a transformer MLP sublayer with the
    parity bottleneck at its input.  forward returns (output, loss_var).

    With a residual, h is h + residual, and the output the two terms (W2 ..., h + residual) of
    the sum: the next norm adds them."""

    def __init__(self, plan: B.Plan, d_ff: int, normalized: bool = True, n_min: int | None = None,
                 standardize: bool = False, momentum: float = 0.01, dtype: torch.dtype = torch.float32, device=None):
        super().__init__()
        d = plan.d
        self.plan, self.normalized, self.n_min = plan, normalized, n_min
        self.std = Standardizer(plan, momentum, device=device) if standardize else None
        if self.std is not None:
            self.register_buffer("std_stats", self.std.stats)
            self.register_buffer("std_m2", self.std.m2)
        self.norm = RMSNorm(d, dtype=dtype, device=device)
        self.fc1 = torch.nn.Linear(d, d_ff, dtype=dtype, device=device)
        self.fc2 = torch.nn.Linear(d_ff, d, dtype=dtype, device=device)

    def forward(self, h: torch.Tensor, residual: torch.Tensor | None = None):
        if residual is None:
            z = self.norm(h)
        else:
            z, h = _add_norm(self.norm, h, residual)
        out, loss_var = self.feed(z.reshape(-1, z.shape[-1]))
        out = out.reshape(h.shape)
        return (h + out if residual is None else (out, h)), loss_var

    def feed(self, z: torch.Tensor):
        """The sublayer without its norm and residual, for rows z [T, d]: (W2 gelu(W1 DPB(z)), loss_var)."""
        if self.std is not None:
            self.std.training = self.training
        y, loss_var = DPBLayer.apply(z, self.plan, self.normalized, self.n_min, self.std)
        return self.fc2(torch.nn.functional.gelu(self.fc1(y))), loss_var


class AttentionLayer(torch.autograd.Function):
    """Attention of padded sequences, q [B, Sq, H, D], k and v [B, Sk, Hkv, D] -> [B, Sq, H, D];
    the backward recomputes the probabilities from the log-sum-exp.  Second derivatives are
    an error: the library's gradients have no graph."""

    @staticmethod
    def forward(ctx, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, causal: bool = False,
                scale: float | None = None, q_lens: torch.Tensor | None = None, k_lens: torch.Tensor | None = None):
        out, lse = B.attention(q, k, v, causal, scale, q_lens, k_lens)
        ctx.causal, ctx.scale = causal, scale
        ctx.save_for_backward(q, k, v, out, lse, q_lens, k_lens)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, grad: torch.Tensor):
        q, k, v, out, lse, q_lens, k_lens = ctx.saved_tensors
        # an expanded gradient, say, or one behind a single number in a tensor they were joined to
        if grad.stride() != out.stride() or grad.data_ptr() % 16:
            grad = grad.clone(memory_format=torch.contiguous_format)
        dq, dk, dv = B.attention_bwd(grad, q, k, v, out, lse, ctx.causal, ctx.scale, q_lens, k_lens)
        return dq, dk, dv, None, None, None, None


def attention_layer(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, causal: bool = False,
                    scale: float | None = None, q_lens: torch.Tensor | None = None,
                    k_lens: torch.Tensor | None = None):
    """Functional form of AttentionLayer."""
    return AttentionLayer.apply(q, k, v, causal, scale, q_lens, k_lens)


class KeyValueCache:
    """Keys and values of up to `length` tokens of `batch` sequences for one attention sublayer."""

    def __init__(self, batch: int, length: int, kv_heads: int, head_dim: int, dtype: torch.dtype, device=None):
        self.k = torch.zeros(batch, length, kv_heads, head_dim, dtype=dtype, device=device)
        self.v = torch.zeros_like(self.k)
        self.used = 0

    def append(self, k: torch.Tensor, v: torch.Tensor):
        """Adds the tokens' keys and values; all of them so far, as views."""
        end = self.used + k.shape[1]
        if end > self.k.shape[1]:
            raise ValueError(f"the cache holds {self.k.shape[1]} tokens, not {end}")
        self.k[:, self.used:end], self.v[:, self.used:end] = k, v
        self.used = end
        return self.k[:, :end], self.v[:, :end]


class CausalAttention(torch.nn.Module):
    """h + W_o attention(rmsnorm(h)), queries, keys and values from one projection; `kv_heads`
    key heads are shared by `heads` query heads.  With a cache, h holds the tokens behind
    those in it.  With a residual, h is h + residual, and (W_o ..., h + residual) comes back: the
    two terms of the output, which the next norm adds."""

    def __init__(self, d: int, heads: int, kv_heads: int | None = None, dtype: torch.dtype = torch.float32, device=None):
        super().__init__()
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads or heads, d // heads
        if self.head_dim * heads != d:
            raise ValueError(f"{heads} heads do not divide a width of {d}")
        self.norm = RMSNorm(d, dtype=dtype, device=device)
        self.qkv = torch.nn.Linear(d, (heads + 2 * self.kv_heads) * self.head_dim, bias=False, dtype=dtype, device=device)
        self.out = torch.nn.Linear(d, d, bias=False, dtype=dtype, device=device)

    def forward(self, h: torch.Tensor, cache: KeyValueCache | None = None, residual: torch.Tensor | None = None):
        if residual is None:
            return h + self.mix(self.norm(h), cache)
        z, h = _add_norm(self.norm, h, residual)
        return self.mix(z, cache), h

    def mix(self, z: torch.Tensor, cache: KeyValueCache | None = None):
        """The sublayer without its norm and residual: W_o attention(z)."""
        x = self.qkv(z).unflatten(-1, (-1, self.head_dim))
        q, k, v = x.split((self.heads, self.kv_heads, self.kv_heads), dim=2)   # views of one tensor
        if cache is not None:
            k, v = cache.append(k, v)
            q = q.to(k.dtype)   # (under autocast the projection's type is not the cache's)
        y = AttentionLayer.apply(q, k, v, True)
        return self.out(y.flatten(-2))

    def cache(self, batch: int, length: int) -> KeyValueCache:
        w = self.qkv.weight
        return KeyValueCache(batch, length, self.kv_heads, self.head_dim, w.dtype, w.device)


class ParityBlock(torch.nn.Module):
    """One block of a Parity Transformer: causal attention, then DPBMLP (§3.1).  forward
    returns (output, loss_var); with a residual, as the sublayers do, the input is
    h + residual and the output its last two terms."""

    def __init__(self, plan: B.Plan, heads: int, d_ff: int, kv_heads: int | None = None,
                 dtype: torch.dtype = torch.float32, device=None, **mlp):
        super().__init__()
        self.attention = CausalAttention(plan.d, heads, kv_heads, dtype, device)
        self.mlp = DPBMLP(plan, d_ff, dtype=dtype, device=device, **mlp)

    def forward(self, h: torch.Tensor, cache: KeyValueCache | None = None, residual: torch.Tensor | None = None):
        if residual is None:
            return self.mlp(self.attention(h, cache))
        return self.mlp(*self.attention(h, cache, residual))


def _even(t: torch.Tensor) -> torch.Tensor:
    """t, or a copy whose rows are evenly apart and start on 16 bytes."""
    try:
        B._rows(t, "rows")
    except ValueError:
        return t.contiguous()
    return t.clone(memory_format=torch.contiguous_format) if t.data_ptr() % 16 else t


def _near(t: torch.Tensor) -> torch.Tensor:
    """t, or a copy whose rows are as the loss takes them: even, and closer than it reads them from (the last token of
    each long sequence, say)."""
    t = _even(t)
    far = not t.is_contiguous() and B._rows(t, "rows")[1] * t.element_size() >= B.LOGITS_STRIDE
    return t.contiguous() if far else t


class EmbeddingLayer(torch.autograd.Function):
    """scale * table[tokens]; tokens outside the table give zeros and no gradient."""

    @staticmethod
    def forward(ctx, tokens: torch.Tensor, table: torch.Tensor, scale: float = 1.0):
        tokens = tokens.contiguous()
        ctx.save_for_backward(tokens)
        ctx.vocab, ctx.scale = table.shape[0], scale
        return B.embedding(tokens, table, scale)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad: torch.Tensor):
        tokens, = ctx.saved_tensors
        return None, B.embedding_bwd(_even(grad), tokens, ctx.vocab, ctx.scale), None


def embedding_layer(tokens: torch.Tensor, table: torch.Tensor, scale: float = 1.0):
    """Functional form of EmbeddingLayer."""
    return EmbeddingLayer.apply(tokens, table, scale)


class Embedding(torch.nn.Embedding):
    """torch.nn.Embedding by EmbeddingLayer: rows of the weight for tokens, zeros for those outside it."""

    def __init__(self, vocab: int, dim: int, dtype: torch.dtype = torch.float32, device=None):
        super().__init__(vocab, dim, dtype=dtype, device=device)

    def forward(self, tokens: torch.Tensor):
        return EmbeddingLayer.apply(tokens, self.weight)


class RMSNormLayer(torch.autograd.Function):
    """(norm of the sum, the sum) for x and residual of one type; without a residual the sum
    is x, and (norm, None) comes back."""

    @staticmethod
    def forward(ctx, x: torch.Tensor, weight: torch.Tensor | None, residual: torch.Tensor | None = None, eps: float = 1e-6):
        x = _even(x)
        out, total, rstd = B.rms_norm(x, weight, None if residual is None else _even(residual), eps)
        ctx.save_for_backward(total, weight, rstd)
        ctx.set_materialize_grads(False)
        return out, None if residual is None else total

    @staticmethod
    @once_differentiable
    def backward(ctx, grad: torch.Tensor | None, grad_total: torch.Tensor | None):
        total, weight, rstd = ctx.saved_tensors
        if grad is None:         # the norm itself was not used
            return grad_total, None, grad_total if ctx.needs_input_grad[2] else None, None
        dx, dw = B.rms_norm_bwd(_even(grad), total, weight, rstd, None if grad_total is None else _even(grad_total))
        return dx, dw, dx if ctx.needs_input_grad[2] else None, None


def rms_norm_layer(x: torch.Tensor, weight: torch.Tensor | None, residual: torch.Tensor | None = None, eps: float = 1e-6):
    """Functional form of RMSNormLayer."""
    return RMSNormLayer.apply(x, weight, residual, eps)


class CrossEntropyLayer(torch.autograd.Function):
    """(loss, lse) of hidden rows over a vocabulary's matrix, fp32 of the targets' shape, both
    differentiable (a penalty on lse, say); the backward computes the logits once more."""

    @staticmethod
    def forward(ctx, hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, scale: float = 1.0):
        hidden, weight, targets = _near(hidden), _near(weight), targets.contiguous()
        loss, lse = B.cross_entropy(hidden, weight, targets, scale)
        ctx.save_for_backward(hidden, weight, targets, lse)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return loss, lse

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_loss: torch.Tensor | None, grad_lse: torch.Tensor | None):
        hidden, weight, targets, lse = ctx.saved_tensors
        if grad_loss is None and grad_lse is None:
            return None, None, None, None
        grads = [None if g is None else g.contiguous() for g in (grad_loss, grad_lse)]
        dh, dw = B.cross_entropy_bwd(grads[0], hidden, weight, targets, lse, ctx.scale, grad_lse=grads[1],
                                     hidden_grad=ctx.needs_input_grad[0], weight_grad=ctx.needs_input_grad[1])
        return dh, dw, None, None


def cross_entropy_layer(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, scale: float = 1.0):
    """Functional form of CrossEntropyLayer: (loss, lse)."""
    return CrossEntropyLayer.apply(hidden, weight, targets, scale)


class ParityTransformer(torch.nn.Module):
    """Tied token embeddings, learned positions and RMSNorm around ParityBlocks (§3.1).

    The residual stream is carried from module to module as its two last terms, so that
    each addition is part of the next norm: block(x, cache, h) gives the next ((x, h), loss_var),
    which is what hooks and wrappers meet.  Every module is called as one; a norm
    of another kind in a norm's place follows an addition of its own.  forward gives
    logits; loss the mean loss of the tokens that count, without logits in memory."""

    def __init__(self, plan: B.Plan, vocab: int, length: int, layers: int, heads: int, d_ff: int, kv_heads: int | None = None,
                 dtype: torch.dtype = torch.float32, device=None, std: float = 0.02, **mlp):
        super().__init__()
        self.embed = Embedding(vocab, plan.d, dtype=dtype, device=device)
        self.position = Embedding(length, plan.d, dtype=dtype, device=device)
        torch.nn.init.normal_(self.embed.weight, std=std)
        torch.nn.init.normal_(self.position.weight, std=std)
        self.blocks = torch.nn.ModuleList(
            ParityBlock(plan, heads, d_ff, kv_heads, dtype=dtype, device=device, **mlp) for _ in range(layers))
        self.norm = RMSNorm(plan.d, dtype=dtype, device=device)

    def hidden(self, tokens: torch.Tensor, caches=None, start: int = 0):
        """(rows behind the last norm, the blocks' summed variance loss); with caches, tokens are
        those from place `start` on."""
        if start < 0 or start + tokens.shape[1] > self.position.num_embeddings:
            raise ValueError(f"tokens {start} to {start + tokens.shape[1]}: the model has {self.position.num_embeddings} places")
        at = torch.arange(start, start + tokens.shape[1], device=tokens.device).expand_as(tokens)
        x, h = self.embed(tokens), self.position(at)
        loss_var = 0.0
        for i, block in enumerate(self.blocks):
            (x, h), loss = block(x, None if caches is None else caches[i], h)
            loss_var = loss_var + loss
        return _add_norm(self.norm, x, h)[0], loss_var

    def forward(self, tokens: torch.Tensor, caches=None, start: int = 0):
        return torch.nn.functional.linear(self.hidden(tokens, caches, start)[0], self.embed.weight)

    def loss(self, tokens: torch.Tensor, targets: torch.Tensor):
        """(mean loss over the targets that are in the vocabulary, 0 if none is; the blocks' variance loss)."""
        z, loss_var = self.hidden(tokens)
        weight = self.embed.weight
        if torch.is_autocast_enabled("cuda") and torch.get_autocast_dtype("cuda") == torch.bfloat16:
            z, weight = z.bfloat16(), weight.bfloat16()
        loss, _ = CrossEntropyLayer.apply(z, weight, targets)
        counted = ((targets >= 0) & (targets < weight.shape[0])).sum()
        return loss.sum() / counted.clamp(min=1), loss_var

    def caches(self, batch: int, length: int) -> list[KeyValueCache]:
        return [b.attention.cache(batch, length) for b in self.blocks]

    @torch.no_grad()
    def generate(self, prompt: torch.Tensor, tokens: int):
        """`tokens` more tokens, each the likeliest: one pass over the prompt, then one token at a time."""
        caches = self.caches(prompt.shape[0], prompt.shape[1] + tokens)
        z, out = self.hidden(prompt, caches)[0][:, -1], [prompt]
        for i in range(tokens):
            out.append(torch.nn.functional.linear(z, self.embed.weight).argmax(-1, keepdim=True))
            if i + 1 < tokens:
                z = self.hidden(out[-1], caches, prompt.shape[1] + i)[0][:, -1]
        return torch.cat(out, 1)
