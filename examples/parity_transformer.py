"""A small Parity Transformer, trained and then asked to go on.

Two blocks of causal attention and a bottlenecked MLP (ParityBlock) learn
sequences in which every token is the one `lag` places before it: the
attention has to look back, and its gradient has to say where.  AdamW keeps its
states in 8 bits.  Then a few prompts are continued one token at a time over
key-value caches.

    python examples/parity_transformer.py [--steps N] [--bits 8|32]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_20652_amd import binding as dpb  # noqa: E402
from paper_2607_20652_amd.autograd import ParityBlock  # noqa: E402
from paper_2607_20652_amd.optim import AdamW  # noqa: E402

D, HEADS, KV_HEADS, D_FF, VOCAB, LENGTH, LAG, BATCH = 64, 4, 2, 192, 24, 64, 5, 64


class ParityTransformer(torch.nn.Module):
    """Learned positions, tied embeddings and RMSNorm around ParityBlocks (§3.1)."""

    def __init__(self, plan, layers: int, dtype=torch.float32, device="cuda"):
        super().__init__()
        self.embed = torch.nn.Embedding(VOCAB, plan.d, dtype=dtype, device=device)
        self.position = torch.nn.Embedding(LENGTH, plan.d, dtype=dtype, device=device)
        torch.nn.init.normal_(self.embed.weight, std=0.2)
        torch.nn.init.normal_(self.position.weight, std=0.2)
        self.blocks = torch.nn.ModuleList(
            ParityBlock(plan, HEADS, D_FF, KV_HEADS, dtype=dtype, device=device) for _ in range(layers))
        self.norm = torch.nn.RMSNorm(plan.d, dtype=dtype, device=device)

    def forward(self, tokens, caches=None, start: int = 0):
        at = torch.arange(start, start + tokens.shape[1], device=tokens.device)
        h = self.embed(tokens) + self.position(at)
        for i, block in enumerate(self.blocks):
            h, _ = block(h, None if caches is None else caches[i])
        return self.norm(h) @ self.embed.weight.t()

    @torch.no_grad()
    def generate(self, prompt, tokens: int):
        """`tokens` more tokens, each the likeliest: one pass over the prompt, then one token at a time."""
        caches = [b.attention.cache(prompt.shape[0], prompt.shape[1] + tokens) for b in self.blocks]
        logits, out = self(prompt, caches)[:, -1], [prompt]
        for i in range(tokens):
            out.append(logits.argmax(-1, keepdim=True))
            if i + 1 < tokens:
                logits = self(out[-1], caches, prompt.shape[1] + i)[:, -1]
        return torch.cat(out, 1)


def batch(n: int, generator):
    head = torch.randint(VOCAB, (n, LAG), generator=generator)
    return head.repeat(1, LENGTH // LAG + 1)[:, :LENGTH].cuda()


def train(steps: int, bits: int = 8, say=print):
    """The trained model and its losses."""
    torch.manual_seed(0)
    generator = torch.Generator().manual_seed(1)
    plan = dpb.Plan(D, 12, 3, 16, 16, 32, 0)
    model = ParityTransformer(plan, layers=2)
    matrices = [(p, 0.01 if p.dim() > 1 else 0.0) for p in model.parameters()]
    opt = AdamW(matrices, lr=3e-3, betas=(0.9, 0.98), bits=bits)
    losses = []
    for step in range(steps):
        x = batch(BATCH, generator)
        logits = model(x[:, :-1])
        loss = torch.nn.functional.cross_entropy(logits[:, LAG:].flatten(0, 1), x[:, LAG + 1:].flatten())
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.detach())
        if step % 50 == 0 or step == steps - 1:
            say(f"step {step:4d}  loss {float(losses[-1]):.4f}")
    return model, [float(v) for v in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32))
    a = ap.parse_args()
    model, _ = train(a.steps, a.bits)
    truth = batch(8, torch.Generator().manual_seed(2))
    made = model.generate(truth[:, :4 * LAG], LENGTH - 4 * LAG)
    print(f"continued as the rule says: {float((made == truth)[:, 4 * LAG:].double().mean()):.3f} of the tokens")
