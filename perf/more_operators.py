"""The two ends of a training step around the gradient that is checkpointed, as cases to time: log probabilities of given
tokens with entropy and top alternatives, their gradient by the logits, orthogonalising updates by Newton-Schulz products,
and the replay of dense gradients through the optimizer that does so.

A case is a dict of plain values. `prepare` makes what a training or serving program holds before the call,
`run` is one pass, in the operators' plain form or through the library's entry points (`own`), `exact` is the
definition in 64 bits, `work` the bytes and operations a pass cannot do without.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
CHUNK = 1 << 24  # values drawn at a time
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "i32": 4, "i64": 8}
STEPS = 5
COEFFS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7


# ------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # Eight sequences generate a token each with a GPT-2 vocabulary, twenty alternatives reported: the smallest call, all latency.
        dict(name="score_decode", kind="score", T=8, V=50257, logits="bf16", ids="i64", scale=1.0, entropy=True, top=20,
             masked=0.0, pad=0.0),
        # A ragged prompt scored by a GPT-2 model, for comparing a recovered model with the one it replaces.
        dict(name="score_gpt2_prompt", kind="score", T=4095, V=50257, logits="f16", ids="i64", scale=1.0, entropy=False, top=0,
             masked=0.0, pad=0.02),
        # Constrained generation at a temperature: fp32 logits, a width no vector divides, a third of the vocabulary masked.
        dict(name="score_masked", kind="score", T=1023, V=32003, logits="f32", ids="i32", scale=1.25, entropy=True, top=50,
             masked=0.33, pad=0.0),
        # A batch of 16 K tokens over Llama-7B's vocabulary with entropy and five alternatives: the largest.
        dict(name="score_llama", kind="score", T=16384, V=32000, logits="bf16", ids="i64", scale=1.0, entropy=True, top=5,
             masked=0.0, pad=0.0),
        # A few hundred tokens of a GPT-2 model on fp32 logits: the smallest training call.
        dict(name="logit_grad_few", kind="logit_grad", T=255, V=50257, logits="f32", out="f32", ids="i64", scale=1.0, entropy=False,
             masked=0.0, pad=0.0),
        # A policy update with an entropy bonus: ragged, padded, at a temperature, fp16 in and fp32 out.
        dict(name="logit_grad_entropy", kind="logit_grad", T=4001, V=32003, logits="f16", out="f32", ids="i32", scale=0.75, entropy=True,
             masked=0.1, pad=0.2),
        # One iteration of GPT-2 XL, 16 x 1024 tokens, bf16 logits and gradient: the largest.
        dict(name="logit_grad_gpt2xl", kind="logit_grad", T=16384, V=50257, logits="bf16", out="bf16", ids="i64", scale=1.0, entropy=False,
             masked=0.0, pad=0.0),
        # One attention projection of GPT-2 small: the smallest update, a chain of dependent products on a mostly idle chip.
        dict(name="orthogonalize_gpt2s_proj", kind="orthogonalize", shapes="768x768", src="f32", out="f32"),
        # The four matrices of a GPT-2 XL layer, updates handed on in bf16.
        dict(name="orthogonalize_gpt2xl_layer", kind="orthogonalize", shapes="1600x4800,1600x1600,1600x6400,6400x1600", src="f32", out="bf16"),
        # Matrices of many shapes in one call: odd, tall, wide, one row, one column.
        dict(name="orthogonalize_ragged", kind="orthogonalize", shapes="1001x333,333x1001,517x517,96x1600,1x768,768x1,37x41,640x129,1023x1025",
             src="f16", out="f32"),
        # Ten iterations of GPT-2 small's attention matrices replayed from their bf16 snapshots.
        dict(name="muon_gpt2s_window", kind="muon", shapes="768x2304,768x768,768x2304,768x768", W=10, grad="bf16", decay=0.0, nesterov=True),
        # One step of a Llama-7B layer's seven matrices, 202 M parameters: the largest.
        dict(name="muon_llama_layer", kind="muon", shapes="4096x4096,4096x4096,4096x4096,4096x4096,11008x4096,11008x4096,4096x11008", W=1,
             grad="bf16", decay=0.01, nesterov=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["score", "logit_grad", "orthogonalize", "muon"])
    kinds = list(TYPES)
    most = max(work(c)["bytes"] if kind in ("score", "logit_grad") else work(c)["flops"] for c in listed() if c["kind"] == kind)
    if kind in ("score", "logit_grad"):
        case = dict(kind=kind, T=_log(rng, 1, 16384), V=_log(rng, 500, 160000), logits=rng.choice(kinds), ids=rng.choice(["i32", "i64"]),
                    scale=rng.choice([1.0, 1.0, 0.75, 1.25]), entropy=rng.random() < 0.5, masked=rng.choice([0.0, 0.0, 0.2]),
                    pad=rng.choice([0.0, 0.0, 0.25]))
        if rng.random() < 0.5:
            case["V"] = max(512, case["V"] // 64 * 64)
        if kind == "score":
            case["top"] = rng.choice([0, 0, 1, 5, 20, 50, 64])
        else:
            case["out"] = rng.choice(kinds)
        while work(case)["bytes"] > 0.95 * most:
            case["T"] = max(1, case["T"] * 3 // 4)
        return case
    shapes = [[_log(rng, 16, 4096), _log(rng, 16, 11008)] for _ in range(_log(rng, 1, 8))]
    for s in shapes:
        if rng.random() < 0.5:
            s[:] = [max(16, x // 16 * 16) for x in s]
        if rng.random() < 0.5:
            s.reverse()
    case = dict(kind=kind, shapes=shapes)
    if kind == "orthogonalize":
        case.update(src=rng.choice(kinds), out=rng.choice(kinds))
    else:
        case.update(W=_log(rng, 1, 10), grad=rng.choice(kinds), decay=rng.choice([0.0, 0.01]), nesterov=rng.random() < 0.7)
    text = lambda: ",".join(f"{r}x{c}" for r, c in shapes)  # noqa: E731
    while work(dict(case, shapes=text()))["flops"] > 0.95 * most:
        for s in shapes:
            s[:] = [max(1, x * 4 // 5) for x in s]
    case["shapes"] = text()
    return case


def _shapes(case):
    return [tuple(int(x) for x in s.split("x")) for s in case["shapes"].split(",")]


# ------------------------------------------------------------------------------------------ inputs

def _gen(*seeds):
    g = torch.Generator(device=DEV)
    g.manual_seed(hash(tuple(int(s) for s in seeds)) & 0x7FFFFFFFFFFF)
    return g


def _id_type(case):
    return torch.int32 if case["ids"] == "i32" else torch.int64


def _open_columns(case, seed):
    """Which tokens of the vocabulary may be named: the others' logits are minus infinity."""
    return torch.rand(case["V"], generator=_gen(seed, 1), device=DEV) >= case["masked"]


def _targets(case, seed):
    """The tokens that the batch goes on with; a share `pad` of them is -1."""
    T, gen = case["T"], _gen(seed, 2)
    named = _open_columns(case, seed).nonzero().flatten()
    at = (torch.rand(T, generator=gen, device=DEV, dtype=torch.float64).pow_(3) * named.numel()).long()
    ids = named[at]
    return torch.where(torch.rand(T, generator=gen, device=DEV) < case["pad"], -1, ids)


def _logits(case, seed):
    """Normal logits over a vocabulary whose tokens differ in frequency; in three of four rows the model expects the token
    that comes, more or less."""
    T, V, gen = case["T"], case["V"], _gen(seed, 3)
    out = torch.empty(T, V, dtype=TYPES[case["logits"]], device=DEV)
    bias = -0.8 * torch.log(torch.arange(V, device=DEV) + 3.0)
    bias[~_open_columns(case, seed)] = -math.inf
    ids, rows = _targets(case, seed), max(1, CHUNK // V)
    sure = 12.0 * torch.rand(T, generator=gen, device=DEV) - 3.0
    for t0 in range(0, T, rows):
        part = torch.randn(min(rows, T - t0), V, generator=gen, device=DEV).mul_(2.0).add_(bias)
        at = ids[t0:t0 + rows].clamp_min(0)[:, None]
        part.scatter_add_(1, at, sure[t0:t0 + rows, None].clamp_min(0.0))
        out[t0:t0 + rows] = part
    return out


def _token_gradients(case, seed):
    """The loss's gradient by every token's log probability (a weighted mean's) and, with an entropy bonus, by its entropy. A
    gradient in 16-bit floats of the small range is that of a loss that was scaled up."""
    gen, T = _gen(seed, 4), case["T"]
    share = (4096.0 if case["out"] == "f16" else 1.0) / T
    d_logprob = torch.randn(T, generator=gen, device=DEV).sub_(1.0).mul_(share)
    d_entropy = torch.rand(T, generator=gen, device=DEV).mul_(-0.01 * share) if case["entropy"] else None
    return d_logprob, d_entropy


def _row_chunks(T, V, most=1 << 27):
    rows = max(1, most // V)
    return [(t0, min(T, t0 + rows)) for t0 in range(0, T, rows)]


def _matrix(r, c, gen, kind, std):
    """A gradient: a few strong directions over heavy-tailed noise, rows of different scales."""
    z = torch.randn(r, c, generator=gen, device=DEV)
    x = z.mul(torch.randn(r, c, generator=gen, device=DEV).square_().add_(0.1))
    for i in range(6):
        u, v = torch.randn(r, 1, generator=gen, device=DEV), torch.randn(1, c, generator=gen, device=DEV)
        x.addcmul_(u, v, value=2.0 ** (1 - i))
    x.mul_(torch.exp(0.5 * torch.randn(r, 1, generator=gen, device=DEV))).mul_(std)
    return x.to(TYPES[kind])


def _update_scale(r, c):
    return 0.2 * math.sqrt(max(r, c))


def _optimizer(case, seed):
    shapes = _shapes(case)
    ws, ms, grads = [], [], [[] for _ in range(case["W"])]
    for i, (r, c) in enumerate(shapes):
        gen = _gen(seed, 6, i)
        ws.append(torch.randn(r, c, generator=gen, device=DEV).mul_(0.02))
        ms.append(_matrix(r, c, gen, "f32", 1e-2))
        for t in range(case["W"]):
            grads[t].append(_matrix(r, c, gen, case["grad"], 1e-3))
    return ws, ms, grads


LR, MOMENTUM = 0.02, 0.95


def prepare(case, seed):
    kind = case["kind"]
    if kind == "score":
        return dict(kind=kind, logits=_logits(case, seed), ids=_targets(case, seed).to(_id_type(case)), scale=case["scale"],
                    entropy=case["entropy"], top=case["top"])
    if kind == "logit_grad":
        logits = _logits(case, seed)
        d_logprob, d_entropy = _token_gradients(case, seed)
        # what the forward pass kept
        stats = torch.empty(case["T"], 2, device=DEV)
        entropy = torch.empty(case["T"], device=DEV) if case["entropy"] else None
        for t0, t1 in _row_chunks(case["T"], case["V"]):
            x = logits[t0:t1].double()
            stats[t0:t1, 0] = x.max(dim=1).values
            x = (x - stats[t0:t1, :1]) * case["scale"]
            stats[t0:t1, 1] = x.exp().sum(dim=1).log()
            if case["entropy"]:
                x -= stats[t0:t1, 1:].double()
                entropy[t0:t1] = -(x.exp() * x.clamp_min(-1e4)).sum(dim=1)
        return dict(kind=kind, logits=logits, ids=_targets(case, seed).to(_id_type(case)), scale=case["scale"], stats=stats,
                    d_logprob=d_logprob, entropy=entropy, d_entropy=d_entropy, out=TYPES[case["out"]])
    if kind == "orthogonalize":
        mats = [_matrix(r, c, _gen(seed, 5, i), case["src"], 1e-2) for i, (r, c) in enumerate(_shapes(case))]
        return dict(kind=kind, mats=mats, out=TYPES[case["out"]])
    ws, ms, grads = _optimizer(case, seed)
    return dict(kind=kind, ws=ws, ms=ms, grads=grads, decay=case["decay"], nesterov=case["nesterov"],
                scale=[_update_scale(r, c) for r, c in _shapes(case)])


# --------------------------------------------------------------------------------------------- run

def _plain_score(state):
    logits, ids, top = state["logits"], state["ids"], state["top"]
    V = logits.shape[1]
    x = logits.float()
    high = x.max(dim=1).values
    x = (x - high[:, None]) * state["scale"]
    e = torch.exp(x)
    total = e.sum(dim=1)
    log_total = torch.log(total)
    out = dict(stats=torch.stack([high, log_total], dim=1))
    inside = (ids >= 0) & (ids < V)
    at = torch.where(inside, ids, 0).long()[:, None]
    out["logprob"] = torch.where(inside, x.gather(1, at)[:, 0] - log_total, 0.0)
    if state["entropy"]:
        out["entropy"] = log_total - torch.where(e > 0, e * x, 0.0).sum(dim=1) / total
    if top:
        # by value, then by the lower index: both in one whole number
        bits = (logits.float() + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        key = order * (1 << 32) + (V - 1 - torch.arange(V, device=logits.device))
        best = V - 1 - (torch.topk(key, top, dim=1).values & 0xFFFFFFFF)
        out["top_ids"] = best.int()
        out["top_logprob"] = x.gather(1, best) - log_total[:, None]
    return out


def _plain_logit_grad(state):
    logits, ids, stats = state["logits"], state["ids"], state["stats"]
    T, V = logits.shape
    logp = (logits.float() - stats[:, :1]) * state["scale"] - stats[:, 1:]
    p = torch.exp(logp)
    inside = (ids >= 0) & (ids < V)
    g = torch.where(inside, state["d_logprob"], 0.0)
    d = p * -g[:, None]
    if state["d_entropy"] is not None:
        d -= torch.where(p > 0, p * (logp + state["entropy"][:, None]), 0.0) * state["d_entropy"][:, None]
    d.scatter_add_(1, torch.where(inside, ids, 0).long()[:, None], g[:, None])
    return dict(d_logits=(d * state["scale"]).to(state["out"]))


def _plain_orthogonal(u):
    x = u.float()
    if u.shape[0] > u.shape[1]:
        x = x.t().contiguous()
    x = x / (torch.sqrt((x * x).sum()) + EPS)
    a, b, c = COEFFS
    for _ in range(STEPS):
        gram = x @ x.t().contiguous()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.t() if u.shape[0] > u.shape[1] else x


def _plain_muon(state):
    for grads in state["grads"]:
        for w, m, g, s in zip(state["ws"], state["ms"], grads, state["scale"]):
            g = g.float()
            m.mul_(MOMENTUM).add_(g)
            o = _plain_orthogonal(g + MOMENTUM * m if state["nesterov"] else m)
            w.copy_(w * (1.0 - LR * state["decay"]) - (LR * s) * o)
    return dict(ws=state["ws"], ms=state["ms"])


def run(state):
    kind = state["kind"]
    if own:
        from paper_2509_04084_amd import lowdiff as ld
        if kind == "score":
            got = ld.ld_token_logprob(state["logits"], state["ids"], state["scale"], entropy=state["entropy"], top=state["top"])
            out = dict(stats=got.stats, logprob=got.logprob)
            if state["entropy"]:
                out["entropy"] = got.entropy
            if state["top"]:
                out.update(top_ids=got.top_ids, top_logprob=got.top_logprob)
            return out
        if kind == "logit_grad":
            return dict(d_logits=ld.ld_token_logprob_grad(state["logits"], state["stats"], state["ids"], state["d_logprob"], state["entropy"],
                                                          state["d_entropy"], state["scale"], out_dtype=state["out"]))
        if kind == "orthogonalize":
            return dict(mats=ld.ld_orthogonalize(state["mats"], out_dtype=state["out"]))
        ld.ld_merge_dense_muon(state["ws"], state["ms"], state["grads"], LR, MOMENTUM, nesterov=state["nesterov"],
                               weight_decay=state["decay"], scale=state["scale"])
        return dict(ws=state["ws"], ms=state["ms"])
    if kind == "score":
        return _plain_score(state)
    if kind == "logit_grad":
        return _plain_logit_grad(state)
    if kind == "orthogonalize":
        return dict(mats=[_plain_orthogonal(x).to(state["out"]).contiguous() for x in state["mats"]])
    return _plain_muon(state)


# ------------------------------------------------------------------------------------------- exact

def _exact_orthogonal(u):
    """The polynomial of the formula in the order of the matrix itself, in 64 bits."""
    x = u.double()
    x = x / (float(x.square().sum().sqrt()) + EPS)
    a, b, c = COEFFS
    for _ in range(STEPS):
        if x.shape[0] <= x.shape[1]:
            s = torch.mm(x, x.t().contiguous())
            x = a * x + b * torch.mm(s, x) + c * torch.mm(s, torch.mm(s, x))
        else:
            s = torch.mm(x.t().contiguous(), x)
            x = a * x + b * torch.mm(x, s) + c * torch.mm(torch.mm(x, s), s)
    return x


def exact(case, seed):
    kind = case["kind"]
    if kind in ("score", "logit_grad"):
        logits, ids, scale, T, V = _logits(case, seed), _targets(case, seed), case["scale"], case["T"], case["V"]
        scale = float(np.float32(scale))
    if kind == "score":
        new = lambda *shape: torch.empty(*shape, dtype=torch.float64, device=DEV)  # noqa: E731
        out = dict(stats=new(T, 2), logprob=new(T))
        if case["entropy"]:
            out["entropy"] = new(T)
        if case["top"]:
            out.update(top_ids=None, top_logprob=new(T, case["top"]))
        for t0, t1 in _row_chunks(T, V):
            x, y = logits[t0:t1].double(), ids[t0:t1]
            high = x.max(dim=1).values
            x *= scale
            lse = torch.logsumexp(x, dim=1)
            out["stats"][t0:t1, 0], out["stats"][t0:t1, 1] = high, lse - high * scale
            out["logprob"][t0:t1] = torch.where(y >= 0, x.gather(1, y.clamp_min(0)[:, None])[:, 0] - lse, 0.0)
            if case["top"]:
                out["top_logprob"][t0:t1] = x.topk(case["top"], dim=1).values - lse[:, None]
            if case["entropy"]:
                x -= lse[:, None]
                out["entropy"][t0:t1] = -torch.special.xlogy(x.exp(), x.exp()).sum(dim=1)
        return out
    if kind == "logit_grad":
        d = torch.empty(T, V, dtype=torch.float64, device=DEV)
        d_logprob, d_entropy = _token_gradients(case, seed)
        for t0, t1 in _row_chunks(T, V):
            y = ids[t0:t1]
            p = torch.softmax(logits[t0:t1].double() * scale, dim=1)
            g = torch.where(y >= 0, d_logprob[t0:t1].double(), 0.0)[:, None]
            part = -p * g
            part[torch.arange(t1 - t0, device=DEV), y.clamp_min(0)] += g[:, 0]
            if case["entropy"]:
                plogp = torch.special.xlogy(p, p)
                part -= (plogp - p * plogp.sum(dim=1, keepdim=True)) * d_entropy[t0:t1, None].double()
            d[t0:t1] = part * scale
        return dict(d_logits=d)
    if kind == "orthogonalize":
        return dict(mats=[_exact_orthogonal(_matrix(r, c, _gen(seed, 5, i), case["src"], 1e-2)) for i, (r, c) in enumerate(_shapes(case))])
    ws, ms, grads = _optimizer(case, seed)
    lr, mu, decay = (float(np.float32(v)) for v in (LR, MOMENTUM, case["decay"]))
    ws, ms = [w.double() for w in ws], [m.double() for m in ms]
    for i, (r, c) in enumerate(_shapes(case)):
        s = float(np.float32(_update_scale(r, c)))
        for t in range(case["W"]):
            g = grads[t][i].double()
            ms[i] = mu * ms[i] + g
            ws[i] = (1.0 - lr * decay) * ws[i] - lr * s * _exact_orthogonal(g + mu * ms[i] if case["nesterov"] else ms[i])
    return dict(ws=ws, ms=ms)


# -------------------------------------------------------------------------------------------- work

def _products(r, c):
    """Operations of five Newton-Schulz steps, by the cheapest way known: the Gram matrix once (a symmetric product, half of it), its
    successors and the product of the polynomials in its own size, all symmetric, and what they amount to applied once."""
    m, n = float(min(r, c)), float(max(r, c))
    return 3.0 * m * m * n + (4.0 * STEPS - 3.0) * m ** 3


def work(case):
    kind = case["kind"]
    if kind in ("score", "logit_grad"):
        n, T = float(case["T"]) * case["V"], case["T"]
        bytes_ = n * BYTES[case["logits"]] + T * BYTES[case["ids"]]
        if kind == "score":
            return dict(bytes=bytes_ + T * (12 + 4 * case["entropy"] + 8 * case["top"]), flops=(6 if case["entropy"] else 4) * n)
        return dict(bytes=bytes_ + n * BYTES[case["out"]] + T * (20 if case["entropy"] else 12), flops=(8 if case["entropy"] else 4) * n)
    elems = float(sum(r * c for r, c in _shapes(case)))
    flops = sum(_products(r, c) for r, c in _shapes(case))
    if kind == "orthogonalize":
        return dict(bytes=elems * (BYTES[case["src"]] + BYTES[case["out"]]), flops=flops)
    return dict(bytes=elems * (16 + case["W"] * BYTES[case["grad"]]), flops=case["W"] * (flops + 7 * elems))
