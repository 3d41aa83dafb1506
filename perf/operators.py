"""The operators between a model's tokens and its differential checkpoint, as cases to time: embedding lookup,
the embedding's gradient by sorted tokens, and the global gradient norm with clipping.

A case is a dict of plain values. `prepare` makes what a training or serving program holds before the call,
`run` is one pass, in the operators' plain form or through the library's entry points (`own`), `exact` is the
definition in 64 bits, `work` the bytes and operations a pass cannot do without.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
CHUNK = 1 << 24  # values drawn at a time
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "i32": 4, "i64": 8}


# ------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # Eight sequences generate a token each with GPT-2 XL: the smallest call, all latency.
        dict(name="lookup_decode", kind="lookup", T=8, V=50257, d=1600, ids="i64", table="bf16", out="bf16", scale=1.0,
             positions=1024, zipf=1.05, pad=0.0),
        # A ragged packed prompt of GPT-2 small on fp32 master weights, activations in bf16.
        dict(name="lookup_gpt2s_packed", kind="lookup", T=8191, V=50257, d=768, ids="i64", table="f32", out="bf16",
             scale=1.0, positions=1024, zipf=1.05, pad=0.02),
        # Eight sequences of 4096 tokens at the width of Llama-7B, rows scaled by sqrt(d): the largest batch.
        dict(name="lookup_llama", kind="lookup", T=32768, V=32000, d=4096, ids="i32", table="bf16", out="bf16",
             scale=64.0, positions=0, zipf=1.05, pad=0.0),
        # A few hundred tokens added to the fp32 gradient that a tied head left: the smallest training call.
        dict(name="embed_grad_few", kind="embed_grad", T=255, V=50257, d=768, ids="i64", dout="f32", grad="f32",
             scale=1.0, accumulate=True, zipf=1.05, pad=0.0),
        # One iteration of GPT-2 XL, 16 x 1024 tokens: bf16 activations' gradient into segment 0 of the flat fp32 gradient.
        dict(name="embed_grad_gpt2xl", kind="embed_grad", T=16384, V=50257, d=1600, ids="i64", dout="bf16", grad="f32",
             scale=1.0, accumulate=False, zipf=1.05, pad=0.0),
        # The position table of the same iteration: every row is named 16 times, in every sequence's order.
        dict(name="embed_grad_positions", kind="embed_grad", T=16384, V=1024, d=1600, ids="i64", dout="bf16", grad="f32",
             scale=1.0, accumulate=False, zipf=-1.0, pad=0.0),
        # Sequences of different lengths padded to one, a width that no vector divides, half of the tokens one id or padding.
        dict(name="embed_grad_ragged", kind="embed_grad", T=30011, V=32003, d=1001, ids="i32", dout="f16", grad="f32",
             scale=31.625, accumulate=False, zipf=1.4, pad=0.3),
        # Sixteen sequences of 4096 tokens at the width of Llama-7B, gradient in bf16 for the dense path: the largest.
        dict(name="embed_grad_llama", kind="embed_grad", T=65536, V=32000, d=4096, ids="i32", dout="bf16", grad="bf16",
             scale=64.0, accumulate=False, zipf=1.05, pad=0.0),
        # One flat fp32 gradient of a million parameters, clipped into the buffer that compression reads.
        dict(name="clip_flat1m", kind="clip", table="flat", n=1 << 20, src="f32", out="f32", clipped=True),
        # ResNet-50's 161 tensors in place at a step whose norm is under the limit, as most are.
        dict(name="clip_resnet50_under", kind="clip", table="resnet50", src="f32", out="", clipped=False),
        # GPT-2 small's 148 fp32 gradients clipped into the bf16 buffers of the dense path.
        dict(name="clip_gpt2s_to_bf16", kind="clip", table="gpt2s", src="f32", out="bf16", clipped=True),
        # GPT-2 XL's 580 bf16 gradients clipped out of the training buffers, 1.56 G values.
        dict(name="clip_gpt2xl", kind="clip", table="gpt2xl", src="bf16", out="bf16", clipped=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["lookup", "embed_grad", "embed_grad", "clip", "clip"])
    kinds = list(TYPES)
    if kind == "lookup":
        case = dict(kind=kind, T=_log(rng, 1, 32768), V=_log(rng, 1000, 60000), d=_log(rng, 64, 4096))
        if rng.random() < 0.6:
            case["d"] = max(64, case["d"] // 64 * 64)
        case.update(ids=rng.choice(["i32", "i64"]), table=rng.choice(kinds), out=rng.choice(kinds),
                    scale=rng.choice([1.0, 0.5, 22.625]), positions=rng.choice([0, 0, 1024, 2048]),
                    zipf=rng.choice([0.0, 1.05, 1.4]), pad=rng.choice([0.0, 0.0, 0.25]))
        return case
    if kind == "embed_grad":
        case = dict(kind=kind, T=_log(rng, 1, 65536), V=_log(rng, 1000, 60000), d=_log(rng, 64, 4096))
        if rng.random() < 0.6:
            case["d"] = max(64, case["d"] // 64 * 64)
        case.update(ids=rng.choice(["i32", "i64"]), dout=rng.choice(kinds), grad=rng.choice(kinds),
                    scale=rng.choice([1.0, 0.5, 22.625]), accumulate=rng.random() < 0.5,
                    zipf=rng.choice([-1.0, 0.0, 1.05, 1.4]), pad=rng.choice([0.0, 0.0, 0.25]))
        while work(case)["bytes"] > 0.95 * work(listed()[7])["bytes"]:
            case["T"], case["V"] = case["T"] * 3 // 4, case["V"] * 3 // 4
        return case
    clipped = rng.random() < 0.7
    src = rng.choice(kinds)
    case = dict(kind=kind, table="random", table_seed=rng.randrange(1 << 30), tensors=_log(rng, 1, 600),
                n=_log(rng, 2000, 700_000_000) | 1, src=src, out=rng.choice(kinds) if clipped else "", clipped=clipped)
    return case


def _sizes(case):
    """Elements of every tensor of a clipping case."""
    table = case["table"]
    if table == "flat":
        return [case["n"]]
    if table == "resnet50":
        out, inp = [7 * 7 * 3 * 64, 64, 64], 64
        for width, blocks in ((64, 3), (128, 4), (256, 6), (512, 3)):
            for b in range(blocks):
                out += [inp * width, width, width, 9 * width * width, width, width, 4 * width * width, 4 * width, 4 * width]
                if b == 0:
                    out += [4 * inp * width, 4 * width, 4 * width]
                inp = 4 * width
        return out + [2048 * 1000, 1000]
    if table in ("gpt2s", "gpt2xl"):
        layers, d = (12, 768) if table == "gpt2s" else (48, 1600)
        block = [d, d, 3 * d * d, 3 * d, d * d, d, d, d, 4 * d * d, 4 * d, 4 * d * d, d]
        return [50257 * d, 1024 * d] + block * layers + [d, d]
    rng = random.Random(case["table_seed"])
    share = [math.exp(rng.gauss(0.0, 2.0)) for _ in range(case["tensors"])]
    total = sum(share)
    sizes = [max(1, int(case["n"] * s / total)) for s in share]
    big = max(range(len(sizes)), key=sizes.__getitem__)
    sizes[big] = max(1, sizes[big] + case["n"] - sum(sizes))
    return sizes


# ------------------------------------------------------------------------------------------ inputs

def _gen(*seeds):
    g = torch.Generator(device=DEV)
    g.manual_seed(hash(tuple(int(s) for s in seeds)) & 0x7FFFFFFFFFFF)
    return g


def _normal(shape, std, kind, gen):
    out = torch.empty(math.prod(shape), dtype=TYPES[kind], device=DEV)
    for c0 in range(0, out.numel(), CHUNK):
        part = out[c0:c0 + CHUNK]
        part.copy_(torch.randn(part.numel(), generator=gen, device=DEV).mul_(std))
    return out.view(shape)


def _law(case):
    """Probability of each rank of a vocabulary: 0 uniform, else a Zipf law of that exponent."""
    p = (np.arange(case["V"]) + 2.7) ** -max(0.0, case["zipf"])
    return p / p.sum()


def _tokens(case, seed):
    """The batch's ids: ranks of the vocabulary's law under a random numbering, or row after row in order
    (zipf < 0, positions); a share `pad` of them is -1, which names no row."""
    T, V, gen = case["T"], case["V"], _gen(seed, 1)
    if case["zipf"] < 0:
        ids = (torch.arange(T, device=DEV) + seed % 7) % V
    else:
        cdf = torch.from_numpy(np.cumsum(_law(case))).to(DEV)
        u = torch.rand(T, generator=gen, device=DEV, dtype=torch.float64)
        rank = torch.searchsorted(cdf, u).clamp_(max=V - 1)
        ids = torch.randperm(V, generator=gen, device=DEV)[rank]
    ids = torch.where(torch.rand(T, generator=gen, device=DEV) < case["pad"], -1, ids)
    return ids.to(torch.int32 if case["ids"] == "i32" else torch.int64)


def _positions(case, seed):
    at = torch.arange(case["T"], device=DEV) + seed % 257
    return (at % case["positions"]).to(torch.int32 if case["ids"] == "i32" else torch.int64)


def _base(case):
    return 0.256 if case["src"] == "f16" else 1e-3


def _gradients(case, seed):
    """All tensors' gradients in one buffer (heavy-tailed), each tensor with a scale of its own; 16-bit floats of
    the small range are those of a loss that was scaled up."""
    sizes, gen = _sizes(case), _gen(seed, 5)
    flat = torch.empty(sum(sizes), dtype=TYPES[case["src"]], device=DEV)
    for c0 in range(0, flat.numel(), CHUNK):
        part = flat[c0:c0 + CHUNK]
        z = torch.randn(2, part.numel(), generator=gen, device=DEV)
        part.copy_(z[0].mul_(z[1].square_().add_(0.1)).mul_(_base(case)))
    scales = torch.exp(torch.randn(len(sizes), generator=gen, device=DEV)).tolist()
    parts = flat.split(sizes)
    for x, s in zip(parts, scales):
        x.mul_(s)
    return flat, list(parts)


def _limit(case):
    """A limit that the norm of _gradients is well over, or stays under."""
    return math.sqrt(sum(_sizes(case))) * _base(case) * (0.02 if case["clipped"] else 1000.0)


def prepare(case, seed):
    kind = case["kind"]
    if kind == "lookup":
        state = dict(kind=kind, ids=_tokens(case, seed), scale=case["scale"], out=TYPES[case["out"]], pos_table=None, positions=None,
                     table=_normal((case["V"], case["d"]), 0.02, case["table"], _gen(seed, 2)))
        if case["positions"]:
            state.update(positions=_positions(case, seed),
                         pos_table=_normal((case["positions"], case["d"]), 0.01, case["table"], _gen(seed, 3)))
        return state
    if kind == "embed_grad":
        state = dict(kind=kind, ids=_tokens(case, seed), scale=case["scale"], accumulate=case["accumulate"],
                     dout=_normal((case["T"], case["d"]), 1e-3, case["dout"], _gen(seed, 2)))
        # what a tied head left there, or of an earlier iteration
        state["grad"] = _normal((case["V"], case["d"]), 1e-3, case["grad"], _gen(seed, 3))
        return state
    flat, parts = _gradients(case, seed)
    state = dict(kind=kind, flat=flat, parts=parts, max_norm=_limit(case), out=None, out_parts=None)
    if case["out"]:
        state["out"] = torch.zeros(flat.numel(), dtype=TYPES[case["out"]], device=DEV)
        state["out_parts"] = list(state["out"].split([x.numel() for x in parts]))
    return state


# --------------------------------------------------------------------------------------------- run

def _plain_rows(table, ids):
    inside = (ids >= 0) & (ids < table.shape[0])
    return torch.where(inside[:, None], table[ids.clamp(0, table.shape[0] - 1).long()].float(), 0.0)


def _plain_lookup(state):
    x = _plain_rows(state["table"], state["ids"]) * state["scale"]
    if state["pos_table"] is not None:
        x = x + _plain_rows(state["pos_table"], state["positions"])
    return x.to(state["out"])


def _plain_embed_grad(state):
    grad, ids = state["grad"], state["ids"]
    V = grad.shape[0]
    row = torch.where((ids >= 0) & (ids < V), ids, V).long()  # what names no row is added to one behind the table
    total = torch.zeros(V + 1, grad.shape[1], device=DEV)
    total.index_add_(0, row, state["dout"].float())
    total = total[:V] * state["scale"]
    grad.copy_(grad.float() + total if state["accumulate"] else total)
    return grad


def _plain_clip(state):
    x = state["flat"].float()
    norm = (x * x).sum().sqrt()
    factor = torch.where(norm > state["max_norm"], state["max_norm"] / norm, 1.0)
    out = state["flat"] if state["out"] is None else state["out"]
    out.copy_(x * factor)
    return norm.reshape(1), out


def run(state):
    kind = state["kind"]
    if own:
        from paper_2509_04084_amd import lowdiff as ld
        if kind == "lookup":
            return dict(out=ld.ld_embed_lookup(state["table"], state["ids"], state["scale"], state["pos_table"],
                                               state["positions"], out_dtype=state["out"]))
        if kind == "embed_grad":
            ld.ld_embed_grad(state["dout"], state["ids"], state["grad"], state["scale"], state["accumulate"])
            return dict(grad=state["grad"])
        norm = ld.ld_clip_grad_norm(state["parts"], state["max_norm"], state["out_parts"])
        return dict(norm=norm, grads=state["flat"] if state["out"] is None else state["out"])
    if kind == "lookup":
        return dict(out=_plain_lookup(state))
    if kind == "embed_grad":
        return dict(grad=_plain_embed_grad(state))
    norm, out = _plain_clip(state)
    return dict(norm=norm, grads=out)


# ------------------------------------------------------------------------------------------- exact

def exact(case, seed):
    kind = case["kind"]
    if kind == "lookup":
        T, d = case["T"], case["d"]
        out = torch.zeros(T, d, dtype=torch.float64, device=DEV)
        table, ids = _normal((case["V"], d), 0.02, case["table"], _gen(seed, 2)), _tokens(case, seed).long()
        named = (ids >= 0).nonzero().flatten()
        out[named] = table.double().index_select(0, ids[named]) * case["scale"]
        if case["positions"]:
            more = _normal((case["positions"], d), 0.01, case["table"], _gen(seed, 3)).double()
            out += more.index_select(0, _positions(case, seed).long())
        return dict(out=out)
    if kind == "embed_grad":
        V, d = case["V"], case["d"]
        dout, ids = _normal((case["T"], d), 1e-3, case["dout"], _gen(seed, 2)), _tokens(case, seed).long()
        named = (ids >= 0).nonzero().flatten()
        grad = torch.zeros(V, d, dtype=torch.float64, device=DEV)
        for c0 in range(0, d, 512):  # columns apart from one another
            grad[:, c0:c0 + 512].index_put_((ids[named],), dout[named, c0:c0 + 512].double(), accumulate=True)
        grad *= case["scale"]
        if case["accumulate"]:
            grad += _normal((V, d), 1e-3, case["grad"], _gen(seed, 3)).double()
        return dict(grad=grad)
    flat, _ = _gradients(case, seed)
    total = 0.0
    for c0 in range(0, flat.numel(), CHUNK):
        total += float(flat[c0:c0 + CHUNK].double().square().sum())
    norm, limit = math.sqrt(total), float(np.float32(_limit(case)))
    factor = limit / norm if norm > limit else 1.0
    return dict(norm=torch.tensor([norm], dtype=torch.float64, device=DEV), grads=flat.double() * factor)


# -------------------------------------------------------------------------------------------- work

def _distinct(case):
    """Rows that a batch's tokens can be expected to name."""
    T = case["T"] * (1.0 - case["pad"])
    if case["zipf"] < 0:
        return min(T, case["V"])
    return float((1.0 - np.power(1.0 - _law(case), T)).sum())


def work(case):
    kind = case["kind"]
    if kind == "clip":
        n, size = sum(_sizes(case)), BYTES[case["src"]]
        # in place and under the limit nothing has to be written
        return dict(bytes=n * (size + (BYTES[case["out"]] if case["out"] else 0)), flops=(3 if case["clipped"] else 2) * n)
    T, V, d, rows = case["T"], case["V"], case["d"], _distinct(case)
    if kind == "lookup":
        read = rows * d * BYTES[case["table"]] + T * BYTES[case["ids"]]
        if case["positions"]:
            read += min(T, case["positions"]) * d * BYTES[case["table"]] + T * BYTES[case["ids"]]
        return dict(bytes=read + T * d * BYTES[case["out"]], flops=2 * T * d)
    read = T * (1.0 - case["pad"]) * d * BYTES[case["dout"]] + T * BYTES[case["ids"]]
    moved = 2.0 * rows * d if case["accumulate"] else float(V * d)
    return dict(bytes=read + moved * BYTES[case["grad"]], flops=(1.0 - case["pad"]) * T * d + rows * d)
