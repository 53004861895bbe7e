"""A small Parity Transformer, trained and then asked to go on.

Two blocks of causal attention and a bottlenecked MLP (ParityBlock) learn
sequences in which every token is the one `lag` places before it: the
attention has to look back, and its gradient has to say where.  The loss is taken
without logits in memory, and AdamW keeps its states in 8 bits.  Then a few prompts
are continued one token at a time over key-value caches.

    python examples/parity_transformer.py [--steps N] [--bits 8|32]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_20652_amd import binding as dpb  # noqa: E402
from paper_2607_20652_amd.autograd import ParityTransformer  # noqa: E402
from paper_2607_20652_amd.optim import AdamW  # noqa: E402

D, HEADS, KV_HEADS, D_FF, VOCAB, LENGTH, LAG, BATCH = 64, 4, 2, 192, 24, 64, 5, 64


def batch(n: int, generator):
    head = torch.randint(VOCAB, (n, LAG), generator=generator)
    return head.repeat(1, LENGTH // LAG + 1)[:, :LENGTH].cuda()


def train(steps: int, bits: int = 8, say=print):
    """The trained model and its losses."""
    torch.manual_seed(0)
    generator = torch.Generator().manual_seed(1)
    plan = dpb.Plan(D, 12, 3, 16, 16, 32, 0)
    model = ParityTransformer(plan, VOCAB, LENGTH, layers=2, heads=HEADS, d_ff=D_FF, kv_heads=KV_HEADS, device="cuda", std=0.2)
    matrices = [(p, 0.01 if p.dim() > 1 else 0.0) for p in model.parameters()]
    opt = AdamW(matrices, lr=3e-3, betas=(0.9, 0.98), bits=bits)
    losses = []
    for step in range(steps):
        x = batch(BATCH, generator)
        targets = x[:, 1:].clone()
        targets[:, :LAG] = -1     # nothing says what the first tokens are
        loss, _ = model.loss(x[:, :-1], targets)
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
