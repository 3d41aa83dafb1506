"""Trains a small language model whose whole weight is its embedding, with a differential checkpoint every step.

Token and position table lie in one flat parameter, the token table is the output head as well. A step is

    lookup -> head and loss (torch) -> gradient of both tables -> clipping -> top-k with error feedback -> update

and what the last two make is the differential checkpoint of the step. At the end the model is recovered from the
initial weights and the differentials, and compared with the trained one bit for bit:

    python examples/tied_embedding.py [--steps N]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2509_04084_amd import lowdiff as ld  # noqa: E402
from paper_2509_04084_amd import synth  # noqa: E402


def train(steps=40, vocab=499, width=96, context=32, batch=16, lr=4.0, max_norm=0.3, rho=(1, 20), device="cuda:0", tell=None):
    """Returns the losses, the gradient norms before clipping, and whether recovery gave the trained weights."""
    gen = torch.Generator(device=device)
    gen.manual_seed(0)
    sizes = [vocab * width, context * width]
    off, k = synth.seg_offsets(sizes), synth.seg_topk(sizes, *rho)
    w = torch.randn(int(off[-1]), generator=gen, device=device).mul_(0.02)
    base, grad, residual = w.clone(), torch.zeros_like(w), torch.zeros_like(w)
    tables = lambda flat: (flat[:off[1]].view(vocab, width), flat[off[1]:].view(context, width))  # noqa: E731
    (wte, wpe), (d_wte, d_wpe) = tables(w), tables(grad)
    scale = math.sqrt(width)
    positions = torch.arange(context, device=device).repeat(batch, 1)
    norm, losses, norms, idx, val = torch.zeros(1, device=device), [], [], [], []
    for step in range(steps):
        ids = torch.empty(batch, context + 1, dtype=torch.int64, device=device)
        ids[:, 0] = torch.randint(0, vocab, (batch,), generator=gen, device=device)
        for t in range(context):  # what the model is to learn: every token names the next
            ids[:, t + 1] = (ids[:, t] * 7 + 3) % vocab
        tokens, wanted = ids[:, :-1].contiguous(), ids[:, 1:].reshape(-1)

        x = ld.ld_embed_lookup(wte, tokens, scale, wpe, positions).view(-1, width)
        p = torch.softmax(x @ wte.t(), dim=1)
        losses.append(float(-p.gather(1, wanted[:, None]).clamp_min(1e-30).log().mean()))
        p[torch.arange(p.shape[0], device=device), wanted] -= 1.0
        p /= p.shape[0]
        dx = p @ wte
        torch.mm(p.t(), x, out=d_wte)                                        # the head's share,
        ld.ld_embed_grad(dx, tokens.view(-1), d_wte, scale, accumulate=True)  # and the lookup's on top of it
        ld.ld_embed_grad(dx, positions.view(-1), d_wpe)

        ld.ld_clip_grad_norm([grad], max_norm, norm=norm)
        norms.append(float(norm))
        i, v = ld.ld_compress_topk(grad, residual, off, k)  # the step's differential checkpoint,
        ld.ld_merge_sparse(w, [i], [v], lr)                 # and its update
        idx.append(i)
        val.append(v)
        if tell:
            tell(f"step {step:3d}  loss {losses[-1]:.4f}  gradient norm {norms[-1]:.3f}  differential {i.numel()} of {w.numel()}")
    ld.ld_merge_sparse(base, idx, val, lr)
    return losses, norms, torch.equal(base.view(torch.int32), w.view(torch.int32))


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=40)
    recovered = train(ap.parse_args().steps, tell=lambda line: print(line, flush=True))[2]
    print("recovered from the initial weights and the differentials:", "bit for bit" if recovered else "NOT THE SAME")
    return 0 if recovered else 1


if __name__ == "__main__":
    sys.exit(main())
