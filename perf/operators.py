"""The losses over the vocabulary, as measured cases: softmax cross entropy of given tokens and distillation from a teacher's top logits,
on hidden rows and an LM head, without and with their gradients.

A case names an operator (`op`), the rows of hidden state, the head's sizes, the types of both, which part of the rows counts (`share`: the
rest are prompt tokens or padding), the teacher's entries per row (`entries`), the temperature, whether gradients are taken (`grad`: a training step: loss, then the
gradients to the hidden rows and to the head), and whether every counting row weighs the same (`even`).
"""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # the log-probability of one given token after a decode step of one user: the head is read once, latency is what counts
        dict(name="score_1", op="ce", rows=1, dim=896, vocab=151936, hidden="bf16", weight="bf16", share=1.0, grad=False, even=True),
        # the same for 64 sequences, on hidden rows as a decode step hands them out (fp32) over the bf16 head
        dict(name="score_64_f32_rows", op="ce", rows=64, dim=896, vocab=151936, hidden="f32", weight="bf16", share=1.0, grad=False, even=True),
        # scoring the text of a batch of prompts under the large model
        dict(name="score_prompts_7b", op="ce", rows=1151, dim=3584, vocab=152064, hidden="bf16", weight="bf16", share=1.0, grad=False, even=True),
        # a training step of the tiny fp32 model
        dict(name="ce_step_tiny", op="ce", rows=190, dim=256, vocab=4096, hidden="f32", weight="f32", share=0.7, grad=True, even=True),
        # one training step of the small model's head on the tokens of a few answers
        dict(name="ce_step_500", op="ce", rows=500, dim=896, vocab=151936, hidden="bf16", weight="bf16", share=0.6, grad=True, even=True),
        # a full batch of packed sequences, prompts masked
        dict(name="ce_step_8192", op="ce", rows=8192, dim=896, vocab=151936, hidden="bf16", weight="bf16", share=0.75, grad=True, even=True),
        # the large model's head on a batch
        dict(name="ce_step_7b", op="ce", rows=2048, dim=3584, vocab=152064, hidden="bf16", weight="bf16", share=1.0, grad=True, even=True),
        # odd sizes, rows that are aligned to nothing, rows that weigh differently
        dict(name="ce_step_odd", op="ce", rows=1021, dim=1001, vocab=5003, hidden="bf16", weight="bf16", share=0.8, grad=True, even=False),
        # an update of the small model from the few tokens that the large model has just produced
        dict(name="distill_step_9", op="distill", rows=9, dim=896, vocab=151936, hidden="bf16", weight="bf16", share=1.0, grad=True, even=True, entries=16, t=1.0),
        # how far the small model is from the teacher on a decode batch (no gradient)
        dict(name="distill_loss_64", op="distill", rows=64, dim=896, vocab=151936, hidden="bf16", weight="bf16", share=1.0, grad=False, even=True, entries=64, t=2.0),
        # a tiny fp32 student
        dict(name="distill_step_tiny", op="distill", rows=333, dim=256, vocab=4096, hidden="f32", weight="f32", share=0.8, grad=True, even=False, entries=7, t=1.5),
        # distillation over a batch of generated text
        dict(name="distill_step_4096", op="distill", rows=4096, dim=896, vocab=151936, hidden="bf16", weight="bf16", share=0.75, grad=True, even=True, entries=32, t=2.0),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["small", "small", "small", "score", "large", "tiny", "odd", "odd"])
    op = rng.choice(["ce", "distill"])
    case = dict(op=op, share=rng.choice([1.0, round(rng.uniform(0.3, 1.0), 2)]), grad=rng.random() < 0.7, even=rng.random() < 0.6)
    if kind == "small":
        case |= dict(rows=_log(rng, 1, 8192), dim=896, vocab=151936, hidden="bf16", weight="bf16")
    elif kind == "score":
        case |= dict(rows=_log(rng, 1, 256), dim=896, vocab=151936, hidden="f32", weight="bf16", grad=False)
    elif kind == "large":
        case |= dict(rows=_log(rng, 1, 2048), dim=3584, vocab=152064, hidden="bf16", weight="bf16")
    elif kind == "tiny":
        case |= dict(rows=_log(rng, 1, 1024), dim=256, vocab=4096, hidden="f32", weight="f32")
    else:
        case |= dict(rows=_log(rng, 1, 2048), dim=_log(rng, 33, 1500), vocab=_log(rng, 100, 60000), hidden=rng.choice(["bf16", "bf16", "f32"]), weight="bf16")
        if case["hidden"] == "f32":
            case["rows"] = min(case["rows"], 512)
    if op == "distill":
        case |= dict(entries=_log(rng, 1, 64), t=rng.choice([1.0, 2.0, round(rng.uniform(0.7, 4.0), 2)]))
    return case


# ------------------------------------------------------------------ inputs

SEGMENT = 128    # rows come as sequences of this length, each with its part that does not count first


def _counting(case):
    """Which rows count, as a list of truth values: the last `share` of every sequence."""
    n = case["rows"]
    out = []
    for at in range(0, n, SEGMENT):
        m = min(SEGMENT, n - at)
        skip = m - max(1, round(m * case["share"]))
        out += [False] * skip + [True] * (m - skip)
    return out


def prepare(case, seed):
    """Head N(0, 0.02^2); hidden rows N(0, 1) plus a pull towards the row's token that differs from row to row, so that the token's probability runs from
    almost nothing to almost one, as a trained model's does. The teacher's logits fall from its first entry on; some rows have fewer entries than others."""
    g = torch.Generator(DEVICE).manual_seed(int(seed))
    n, d, v = case["rows"], case["dim"], case["vocab"]
    weight = torch.empty((v, d), dtype=torch.float32, device=DEVICE).normal_(0.0, 0.02, generator=g).to(TYPES[case["weight"]])
    k = case.get("entries", 1)
    step = torch.randint(1, max(2, v // k), (n, 1), device=DEVICE, generator=g)
    ids = (torch.randint(0, v, (n, 1), device=DEVICE, generator=g) + step * torch.arange(k, device=DEVICE)) % v     # distinct in a row
    pull = torch.rand((n, 1), device=DEVICE, generator=g) * (18.0 / (0.02 * d))
    hidden = torch.empty((n, d), dtype=torch.float32, device=DEVICE).normal_(generator=g)
    hidden = (hidden + pull * weight[ids[:, 0]].float() / 0.02).to(TYPES[case["hidden"]])
    counts = torch.tensor(_counting(case), device=DEVICE)
    st = {"case": dict(case), "hidden": hidden, "weight": weight}
    if case["op"] == "ce":
        st["targets"] = torch.where(counts, ids[:, 0], -1).to(torch.int32)
    else:
        drop = torch.empty((n, k), dtype=torch.float32, device=DEVICE).exponential_(1.0, generator=g)
        st["teacher"] = 18.0 - torch.cumsum(drop, 1)
        have = torch.randint(max(1, k // 2), k + 1, (n, 1), device=DEVICE, generator=g) * counts[:, None]
        st["ids"] = torch.where(torch.arange(k, device=DEVICE) < have, ids, -1).to(torch.int32)
    weigh = torch.ones(n, dtype=torch.float32, device=DEVICE) if case["even"] else torch.rand(n, dtype=torch.float32, device=DEVICE, generator=g) + 0.5
    st["grad_loss"] = weigh / sum(_counting(case))
    return st


# ------------------------------------------------------------------ one pass

def _own(st):
    from paper_2504_07878_amd import losses
    case, h, w = st["case"], st["hidden"], st["weight"]
    loss = st.get("loss")
    if loss is None:      # the workspace that a training program keeps
        loss = st["loss"] = losses.VocabLoss(case["rows"], case["dim"], case["vocab"], h.dtype, w.dtype, max_entries=case.get("entries", 1), device=DEVICE)
    if case["op"] == "ce":
        value, lse = loss.cross_entropy(h, w, st["targets"])
        if not case["grad"]:
            return {"loss": value, "lse": lse}
        dh, dw = loss.cross_entropy_grad(h, w, st["targets"], lse, st["grad_loss"])
    else:
        value, lse = loss.distill(h, w, st["ids"], st["teacher"], case["t"])
        if not case["grad"]:
            return {"loss": value, "lse": lse}
        dh, dw = loss.distill_grad(h, w, st["ids"], st["teacher"], case["t"], lse, st["grad_loss"])
    return {"loss": value, "lse": lse, "d_hidden": dh, "d_weight": dw}


def run(st):
    if own:
        return _own(st)
    case, hidden, weight = st["case"], st["hidden"].float(), st["weight"].float()
    z = hidden @ weight.t()
    if case["op"] == "ce":
        t, ids = 1.0, st["targets"].long()[:, None]
        has = ids >= 0
        q = has.float()
        entropy = torch.zeros_like(q)
    else:
        t, ids = case["t"], st["ids"].long()
        has = ids >= 0
        at = torch.where(has, st["teacher"] / t, -math.inf)
        top = at.amax(1, keepdim=True)
        e = torch.exp(at - torch.where(has.any(1, keepdim=True), top, 0.0))
        total = e.sum(1, keepdim=True)
        q = e / torch.where(total > 0, total, 1.0)
        entropy = torch.where(q > 0, q * torch.log(torch.where(q > 0, q, 1.0)), 0.0)
        z = z / t
    some, ids = has.any(1), ids.clamp(min=0)
    top = z.amax(1, keepdim=True)
    lse = (top + torch.log(torch.exp(z - top).sum(1, keepdim=True)))
    loss = t * t * (entropy + q * (lse - z.gather(1, ids))).sum(1)
    out = {"loss": torch.where(some, loss, 0.0), "lse": torch.where(some, lse[:, 0], 0.0)}
    if case["grad"]:
        g = torch.exp(z - lse).scatter_add(1, ids, -q) * torch.where(some, t * st["grad_loss"], 0.0)[:, None]
        out["d_hidden"] = (g @ weight).to(st["hidden"].dtype)
        out["d_weight"] = (g.t() @ hidden).to(st["weight"].dtype)
    return out


def exact(case, seed):
    """The definition in 64 bits, some rows at a time: sums over the whole vocabulary of exp(z - z of the first entry), no maximum taken (|z| stays far below 700)."""
    st = prepare(case, seed)
    w, n, t = st["weight"].double(), case["rows"], float(case.get("t", 1.0))
    loss, lse = (torch.zeros(n, dtype=torch.float64, device=DEVICE) for _ in range(2))
    dh, dw = torch.zeros((n, case["dim"]), dtype=torch.float64, device=DEVICE), torch.zeros_like(w) if case["grad"] else None
    for at in range(0, n, 1024):
        rows = slice(at, at + 1024)
        h = st["hidden"][rows].double()
        ids = (st["targets"][rows, None] if case["op"] == "ce" else st["ids"][rows]).long()
        live = (ids >= 0).double()
        share = live.clone() if case["op"] == "ce" else live * torch.exp(st["teacher"][rows].double() / t)
        total = share.sum(1, keepdim=True)
        share = share / total.clamp(min=1e-300)
        counts = (total[:, 0] > 0).double()
        r = torch.arange(h.shape[0], device=DEVICE)[:, None].expand_as(ids)
        z = torch.mm(h, w.t()) / t
        mass = torch.exp(z).sum(1)
        lse[rows] = torch.log(mass) * counts
        cross = -(share * (z[r, ids.clamp(min=0)] - torch.log(mass)[:, None])).sum(1)
        loss[rows] = t * t * counts * (cross + torch.xlogy(share, share).sum(1))
        if case["grad"]:
            dz = torch.exp(z) / mass[:, None]
            dz.index_put_((r.reshape(-1), ids.clamp(min=0).reshape(-1)), -share.reshape(-1), accumulate=True)
            dz *= (counts * t * st["grad_loss"][rows].double())[:, None]
            dh[rows] = torch.mm(dz, w)
            dw += torch.mm(dz.t().contiguous(), h)
    out = {"loss": loss, "lse": lse}
    return out | {"d_hidden": dh, "d_weight": dw} if case["grad"] else out


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    """Counting rows and the head read once, logits once; with gradients the two products of the gradient, both gradients written."""
    n, d, v = case["rows"], case["dim"], case["vocab"]
    live, hs, ws = sum(_counting(case)), 2 if case["hidden"] == "bf16" else 4, 2 if case["weight"] == "bf16" else 4
    nbytes = live * d * hs + v * d * ws + n * 8 + n * (4 if case["op"] == "ce" else 8 * case["entries"])
    flops = 2 * live * v * d
    if case["grad"]:
        nbytes += n * 4 + n * d * hs + v * d * ws
        flops *= 3
    return {"bytes": nbytes, "flops": flops}
