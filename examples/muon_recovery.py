"""Trains a small language model whose hidden matrices take orthogonalised updates, with a dense differential checkpoint every step.

The embedding is the output head as well and goes by Adam, the two hidden matrices, one tall and one wide, by Muon. A step is

    lookup -> hidden layer and head (torch) -> log probabilities and their gradient -> gradients (torch, and the lookup's)
    -> clipped into bf16 -> snapshot -> both optimizers

and the snapshots are the differential checkpoints. At the end the model, with its optimizers' state, is recovered from the
initial weights and the snapshots, replayed in windows, and compared with the trained one bit for bit:

    python examples/muon_recovery.py [--steps N] [--window W]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2509_04084_amd import lowdiff as ld  # noqa: E402

ADAM = dict(lr=3e-3, beta1=0.9, beta2=0.98, eps=1e-8)


def gradients(weights, tokens, wanted):
    """Mean log probability's negative, and its gradients by embedding, up- and down-projection."""
    table, up, down = weights
    x = ld.ld_embed_lookup(table, tokens)
    h = x @ up.t()
    a = torch.relu(h)
    y = x + a @ down.t()
    logits = y @ table.t()
    said = ld.ld_token_logprob(logits, wanted)
    weight = torch.tensor(-1.0 / wanted.numel(), device=logits.device)
    dz = ld.ld_token_logprob_grad(logits, said.stats, wanted, weight.expand_as(wanted), out=logits)
    d_table, dy = dz.t() @ y, dz @ table
    da = dy @ down
    dh = torch.where(h > 0, da, 0.0)
    ld.ld_embed_grad(dy + dh @ up, tokens, d_table, accumulate=True)
    return -float(said.logprob.mean()), [d_table, dh.t() @ x, dy.t() @ a]


def update(weights, state, grads, step0):
    """Steps step0 + 1 .. of both optimizers, grads[t] being those of one."""
    table, up, down = weights
    ld.ld_merge_dense_adam(table, state[0], state[1], [g[0] for g in grads], step0, **ADAM)
    ld.ld_merge_dense_muon([up, down], state[2:], [g[1:] for g in grads], lr=0.02, weight_decay=0.01)


def train(steps=30, window=7, vocab=211, width=64, hidden=160, tokens_a_step=256, max_norm=1.0, device="cuda:0", tell=None):
    """Returns the losses, and whether recovery gave the trained weights and the optimizers' state."""
    gen = torch.Generator(device=device)
    gen.manual_seed(0)
    shapes = [(vocab, width), (hidden, width), (width, hidden)]
    weights = [torch.randn(*s, generator=gen, device=device).mul_(0.1) for s in shapes]
    zeros = lambda: [torch.zeros_like(weights[0]), *(torch.zeros_like(w) for w in weights)]  # noqa: E731
    base, state, losses, snapshots = [w.clone() for w in weights], zeros(), [], []
    for step in range(steps):
        tokens = torch.randint(0, vocab, (tokens_a_step,), generator=gen, device=device)
        loss, grads = gradients(weights, tokens, (tokens * 7 + 3) % vocab)
        losses.append(loss)
        snapshots.append([torch.empty_like(g, dtype=torch.bfloat16) for g in grads])
        ld.ld_clip_grad_norm(grads, max_norm, snapshots[-1])
        update(weights, state, snapshots[-1:], step)
        if tell:
            tell(f"step {step:3d}  loss {loss:.4f}")
    recovered = zeros()
    for t in range(0, steps, window):
        update(base, recovered, snapshots[t:t + window], t)
    same = all(torch.equal(a.view(torch.int32), b.view(torch.int32)) for a, b in zip(base + recovered, weights + state))
    return losses, same


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--window", type=int, default=7)
    args = ap.parse_args()
    same = train(args.steps, args.window, tell=lambda line: print(line, flush=True))[1]
    print("recovered from the initial weights and the snapshots:", "bit for bit" if same else "NOT THE SAME")
    return 0 if same else 1


if __name__ == "__main__":
    sys.exit(main())
