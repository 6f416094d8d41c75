"""Performance cases of the vocabulary operators: what a client that trains a language model (or a classifier) does at the
two ends where the vocabulary is, through the public entry points.

A case is a dict of plain values:

    op         top       the answers a client or a teacher sends: the top logits of every row (cvlc_top_logits)
               loss      distillation from such answers, the loss alone (cvlc_distill_loss)
               backward  the loss, then its gradient in a call of its own (cvlc_distill_loss, cvlc_distill_grad)
               step      loss and gradient in one call (cvlc_distill_step)
               lookup    embedding rows of the tokens, scaled (cvlc_embed)
               scatter   the embedding's gradient, added into the client's update or written out (cvlc_embed_grad)
    dtype      of logits, table and their gradients: "bf16", "fp16" or "fp32"
    rows, vocab, pad, k      logits are rows x vocab with `pad` unused elements behind each row, k records a row
    rest       what becomes of the words that are not listed: "none", "scaled" or "bucket"
    tau        temperature
    doubled    every row's list holds two clients' records, the same words among them
    masked     rows without weight, rows with an empty list and masked words among the logits
    n, dim, vocab, wide      tokens, columns; tokens in 64 instead of 32 bits
    add        scatter: added to the update that is there (U = w_0 - w_E over local steps) instead of written out
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}


def _rows(name, op, dtype, rows, vocab, k, rest="none", tau=1.0, pad=0, doubled=False, masked=False):
    return {"name": name, "op": op, "dtype": dtype, "rows": rows, "vocab": vocab, "k": k, "rest": rest, "tau": tau, "pad": pad,
            "doubled": doubled, "masked": masked}


def _tokens(name, op, dtype, n, dim, vocab, scale=1.0, wide=False, add=False):
    return {"name": name, "op": op, "dtype": dtype, "n": n, "dim": dim, "vocab": vocab, "scale": scale, "wide": wide, "add": add}


def listed():
    return [
        # one answer: the smallest call, where the launch and the way through one row are all there is
        _rows("answers_one", "top", "bf16", 1, 32000, 32),
        # a batch of answers of an odd vocabulary in padded rows, at a temperature
        _rows("answers_ragged", "top", "fp32", 333, 50021, 100, tau=2.0, pad=11),
        # a client answers for a whole batch of long prompts
        _rows("answers_large", "top", "bf16", 2048, 131072, 64),
        # evaluation on the public data: the loss alone
        _rows("loss_large", "loss", "bf16", 4096, 131072, 64, rest="bucket"),
        # the gradient when the loss's own weight is known only later
        _rows("backward_mid", "backward", "fp16", 1000, 32000, 50, tau=2.0),
        # a local step on one short prompt
        _rows("step_small", "step", "bf16", 16, 32000, 32, rest="bucket"),
        # two clients' answers joined, odd sizes, rows that count for nothing and words that are masked
        _rows("step_ragged", "step", "fp32", 500, 50021, 100, rest="scaled", tau=2.0, pad=11, doubled=True, masked=True),
        # a local step on a whole batch
        _rows("step_large", "step", "bf16", 4096, 131072, 64, rest="bucket"),
        # one token for each of eight sequences
        _tokens("lookup_small", "lookup", "bf16", 8, 1024, 32000, scale=32.0),
        # a whole batch's tokens
        _tokens("lookup_large", "lookup", "bf16", 32768, 4096, 131072, scale=64.0, wide=True),
        # a local step's gradient into the update's block of the table
        _tokens("scatter_mid", "scatter", "fp32", 8192, 1024, 32000, scale=0.1, add=True),
        # a whole batch's gradient as a table of its own, a size that is a multiple of nothing
        _tokens("scatter_large", "scatter", "bf16", 65537, 2048, 65536, scale=45.25, wide=True),
    ]


def draw(rng):
    def log_uniform(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))) if hi > lo else lo

    op = rng.choice(["top", "top", "loss", "backward", "step", "step", "lookup", "scatter", "scatter"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op in ("lookup", "scatter"):
        dim = log_uniform(16, 8192)
        if rng.random() < 0.7:
            dim = max(16, dim // 16 * 16)
        n = log_uniform(1, min(131072, (1 << 27) // dim))
        vocab = log_uniform(256, min(200000, (1 << 27) // dim))
        c = _tokens("", op, dtype, n, dim, vocab, scale=rng.choice([1.0, 0.1, round(math.sqrt(dim), 4)]), wide=rng.random() < 0.5,
                    add=op == "scatter" and rng.random() < 0.6)
    else:
        vocab = log_uniform(10, 200000)
        most = (1 << 28) if op == "top" or dtype == "fp32" else (1 << 29)
        rows = log_uniform(1, min(8192, most // vocab))
        k = min(log_uniform(1, 256), vocab)
        distill = op != "top"
        doubled = distill and k <= 128 and rng.random() < 0.25
        c = _rows("", op, dtype, rows, vocab, k, rest=rng.choice(["none", "scaled", "bucket"]) if distill else "none",
                  tau=rng.choice([1.0, 1.0, 2.0, 0.7]), pad=rng.choice([0, 0, 8, 11]), doubled=doubled,
                  masked=distill and rng.random() < 0.3)
    del c["name"]
    return c


# ---- inputs -------------------------------------------------------------------------------

def _pad(rows, vocab, pad, dtype, device):
    """rows x vocab inside rows x (vocab + pad)"""
    return torch.zeros(rows, vocab + pad, dtype=dtype, device=device)[:, :vocab]


def _logits(c, gen, device, base=None):
    """normal, a few units wide as a trained model's are; a teacher's are near the student's"""
    z = torch.randn(c["rows"], c["vocab"], generator=gen, device=device)
    z = z.mul_(2.5) if base is None else z.add_(base, alpha=0.8)
    out = _pad(c["rows"], c["vocab"], c["pad"], DTYPES[c["dtype"]], device)
    return out.copy_(z)


def _answers(logits, k, tau):
    v, ids = torch.topk(logits.float(), k, dim=1)
    lse = torch.logsumexp(logits.float() / tau, dim=1, keepdim=True)
    return ids.to(torch.int32), v / tau - lse


def prepare(case, seed):
    c = case
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev).manual_seed(seed)
    s = dict(c)
    if c["op"] in ("lookup", "scatter"):
        n, dim, vocab = c["n"], c["dim"], c["vocab"]
        # words by their rank: the i-th about as often as 1 / i; one position of twenty is padding
        u = torch.rand(n, generator=gen, device=dev, dtype=torch.float64)
        tokens = torch.exp(u * math.log(vocab + 1)).long().sub_(1).clamp_(0, vocab - 1)
        if n > 1:
            tokens[torch.rand(n, generator=gen, device=dev) < 0.05] = -1
        s["tokens"] = tokens if c["wide"] else tokens.to(torch.int32)
        if c["op"] == "lookup":
            s["table"] = torch.randn(vocab, dim, generator=gen, device=dev, dtype=torch.float32).mul_(0.02).to(DTYPES[c["dtype"]])
            s["out"] = torch.zeros(n, dim, dtype=DTYPES[c["dtype"]], device=dev)
        else:
            s["grad"] = torch.randn(n, dim, generator=gen, device=dev, dtype=torch.float32).mul_(1e-2).to(DTYPES[c["dtype"]])
            s["update"] = torch.zeros(vocab, dim, device=dev)
            if c["add"]:
                s["update"].normal_(generator=gen).mul_(1e-3)
            if own:  # a workspace that every call uses
                from paper_2402_03770_b200 import binding as B
                s["ws"] = B.alloc_bytes(B.cvlc_embed_grad_workspace_bytes(n, dim, vocab), dev)
        return s
    rows, k = c["rows"], c["k"]
    s["logits"] = _logits(c, gen, dev)
    if c["op"] == "top":
        s["ids"] = torch.zeros(rows, k, dtype=torch.int32, device=dev)
        s["logp"] = torch.zeros(rows, k, device=dev)
        return s
    s["ids"], s["logp"] = _answers(_logits(c, gen, dev, s["logits"]), k, c["tau"])
    if c["doubled"]:
        ids, logp = _answers(_logits(c, gen, dev, s["logits"]), k, c["tau"])
        s["ids"] = torch.cat([s["ids"], ids], dim=1).contiguous()
        s["logp"] = torch.cat([s["logp"] + math.log(0.3), logp + math.log(0.7)], dim=1).contiguous()
    s["weight"] = None
    if c["masked"]:
        s["weight"] = torch.rand(rows, generator=gen, device=dev)
        s["weight"][torch.rand(rows, generator=gen, device=dev) < 0.2] = 0.0
        s["ids"][torch.rand(rows, generator=gen, device=dev) < 0.05] = -1
        # words that the student may not say, none of those that the row lists
        off = torch.rand(rows, c["vocab"], generator=gen, device=dev) < 0.02
        off.scatter_(1, s["ids"].clamp(min=0).long(), False)
        s["logits"].masked_fill_(off, -math.inf)
    s["loss"] = torch.zeros(rows, device=dev)
    if c["op"] != "loss":
        s["d_logits"] = _pad(rows, c["vocab"], c["pad"], DTYPES[c["dtype"]], dev)
    if c["op"] == "backward":
        s["stats"] = torch.zeros(rows, 8, device=dev)  # what the loss keeps for its gradient
    return s


# ---- one pass -----------------------------------------------------------------------------

def _plain_top(s):
    z = s["logits"].float()
    # the value in an order of whole numbers (zeros of either sign alike), the lower index first among equals
    bits = (z + 0.0).view(torch.int32)
    bits = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF).long()
    rank = (bits << 32) | (0xFFFFFFFF - torch.arange(z.shape[1], device=z.device))
    ids = 0xFFFFFFFF - (torch.topk(rank, s["k"], dim=1).values & 0xFFFFFFFF)
    m = z.amax(dim=1, keepdim=True)
    total = torch.exp((z - m) / s["tau"]).sum(dim=1, keepdim=True)
    logp = (z.gather(1, ids) - m) / s["tau"] - torch.log(total)
    return {"ids": ids.to(torch.int32), "logp": logp}


def _plain_distill(s):
    tau, rest = s["tau"], s["rest"]
    x = s["logits"].float() / tau
    there = (s["ids"] >= 0).float()
    at = s["ids"].clamp(min=0).long()
    said = torch.exp(s["logp"].double()) * there  # 64 bits: what a list leaves over may be the small difference of its sum from one
    p = torch.zeros_like(x).scatter_add_(1, at, said.float())
    mass = said.sum(dim=1, keepdim=True)
    if rest == "scaled":
        p = p / torch.where(mass > 0, mass, 1.0).float()
        mass = (mass > 0).double()
    m = x.amax(dim=1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(dim=1, keepdim=True)
    log_q = x - m - torch.log(total)
    loss = torch.where(p > 0, p * (torch.log(p) - log_q), 0.0).sum(dim=1, keepdim=True)
    q = e / total
    if rest == "bucket":
        unlisted = torch.zeros_like(x).scatter_add_(1, at, there) == 0
        y = torch.where(unlisted, x, -math.inf)
        top = y.amax(dim=1, keepdim=True)
        some = top > -math.inf  # else the list holds every word that the student may say, and there is no bucket
        top = torch.where(some, top, 0.0)
        f = torch.exp(y - top)
        part = torch.where(some, f.sum(dim=1, keepdim=True), 1.0)
        left = torch.where(some, (1.0 - mass).clamp(min=0.0), 0.0)
        mass, left = (mass + left).float(), left.float()
        loss = loss + torch.where(left > 0, left * (torch.log(left) - (top + torch.log(part) - m - torch.log(total))), 0.0)
        d = q * mass - p - left * (f / part)
    else:
        d = q * mass.float() - p
    loss, d = loss[:, 0], d / tau
    if s["weight"] is not None:
        w = s["weight"]
        loss = torch.where(w != 0, loss * w, 0.0)
        d = torch.where(w[:, None] != 0, d * w[:, None], 0.0)
    if s["op"] == "loss":
        return {"loss": loss}
    return {"loss": loss, "d_logits": d.to(s["logits"].dtype)}


def _plain_lookup(s):
    t = s["tokens"].long()
    rows = s["table"][t.clamp(min=0)].float() * s["scale"]
    return {"out": torch.where(t[:, None] >= 0, rows, 0.0).to(s["table"].dtype)}


def _plain_scatter(s):
    t = s["tokens"].long()
    g = torch.where(t[:, None] >= 0, s["grad"].float(), 0.0)
    d = torch.zeros_like(s["update"]).index_add_(0, t.clamp(min=0), g) * s["scale"]
    if s["add"]:
        return {"update": s["update"].add_(d)}
    return {"update": d}


def _own(s):
    from paper_2402_03770_b200 import binding as B
    op = s["op"]
    if op == "top":
        B.cvlc_top_logits(s["logits"], s["ids"], s["logp"], temperature=s["tau"])
        return {"ids": s["ids"], "logp": s["logp"]}
    if op == "lookup":
        B.cvlc_embed(s["table"], s["tokens"], s["out"], scale=s["scale"])
        return {"out": s["out"]}
    if op == "scatter":
        B.cvlc_embed_grad(s["tokens"], s["grad"], s["update"], s["ws"], scale=s["scale"], accumulate=s["add"])
        return {"update": s["update"]}
    how = {"rest": {"none": B.CVLC_REST_NONE, "scaled": B.CVLC_REST_SCALED, "bucket": B.CVLC_REST_BUCKET}[s["rest"]],
           "temperature": s["tau"], "row_weight": s["weight"]}
    if op == "loss":
        B.cvlc_distill_loss(s["logits"], s["ids"], s["logp"], s["loss"], **how)
        return {"loss": s["loss"]}
    if op == "step":
        B.cvlc_distill_step(s["logits"], s["ids"], s["logp"], s["loss"], s["d_logits"], **how)
    else:
        B.cvlc_distill_loss(s["logits"], s["ids"], s["logp"], s["loss"], stats=s["stats"], **how)
        B.cvlc_distill_grad(s["logits"], s["ids"], s["logp"], s["stats"], s["d_logits"], **how)
    return {"loss": s["loss"], "d_logits": s["d_logits"]}


def run(s):
    if own:
        return _own(s)
    op = s["op"]
    return _plain_top(s) if op == "top" else _plain_lookup(s) if op == "lookup" else _plain_scatter(s) if op == "scatter" else _plain_distill(s)


def _distinct(n, vocab):
    """expected number of different words among n tokens"""
    i = torch.arange(1, vocab + 1, dtype=torch.float64)
    p = 0.95 * torch.log1p(1.0 / i) / math.log(vocab + 1)
    return float((1.0 - torch.exp(n * torch.log1p(-p))).sum())


def work(case):
    """Inputs once, outputs once.  Logits are read; a gradient is written; records are 8 bytes.  A lookup reads the rows of the
    words that occur and writes a row per token; the gradient reads a row per token and writes the table, or reads and writes
    the rows of the words that occur.  Arithmetic: a subtraction, a product, an exponential and a sum per logit, two more
    products for its gradient."""
    c, size = case, SIZE[case["dtype"]]
    if c["op"] in ("lookup", "scatter"):
        tokens = c["n"] * (8 if c["wide"] else 4)
        row = c["dim"] * size
        distinct = _distinct(c["n"], c["vocab"])
        if c["op"] == "lookup":
            return {"bytes": tokens + c["n"] * row + distinct * row, "flops": c["n"] * c["dim"]}
        table = 2 * distinct * c["dim"] * 4 if c["add"] else c["vocab"] * c["dim"] * 4
        return {"bytes": tokens + c["n"] * row + table, "flops": c["n"] * c["dim"]}
    logits = c["rows"] * c["vocab"]
    records = c["rows"] * c["k"] * (2 if c["doubled"] else 1) * 8
    graded = c["op"] in ("backward", "step")
    per_row = 0 if c["op"] == "top" else c["rows"] * (8 if c["masked"] else 4)
    return {"bytes": logits * size * (2 if graded else 1) + records + per_row, "flops": logits * (6 if graded else 4)}


# ---- the definitions in 64 bits -----------------------------------------------------------

def _exact_distill_rows(z, ids, logp, w, tau, rest):
    """loss and gradient of some rows: the gradient by differentiating the loss"""
    z = z.double().requires_grad_(True)
    log_q = torch.log_softmax(z / tau, dim=1)
    rows, vocab = z.shape
    q_t = torch.zeros(rows, vocab + 1, dtype=torch.float64, device=z.device)  # the last column takes the absent records
    at = torch.where(ids >= 0, ids, vocab).long()
    q_t.scatter_add_(1, at, logp.double().exp())
    named = torch.zeros_like(q_t, dtype=torch.bool).scatter_(1, at, True)[:, :vocab]
    q_t = q_t[:, :vocab]
    mass = q_t.sum(1)
    if rest == "scaled":
        q_t = q_t / torch.where(mass > 0, mass, torch.ones_like(mass))[:, None]
    safe = torch.where(q_t > 0, log_q, torch.zeros_like(log_q))
    loss = (torch.special.xlogy(q_t, q_t) - q_t * safe).sum(1)
    if rest == "bucket":
        unnamed = log_q.masked_fill(named, -math.inf)
        some = unnamed.amax(1) > -math.inf
        left = torch.where(some, (1.0 - mass).clamp(min=0.0), torch.zeros_like(mass))
        others = torch.logsumexp(torch.where(some[:, None], unnamed, torch.zeros_like(unnamed)), dim=1)
        loss = loss + torch.special.xlogy(left, left) - left * others
    if w is not None:
        loss = loss * w.double()
    g, = torch.autograd.grad(loss.sum(), z)
    return loss.detach(), g


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "lookup":
        t = s["tokens"].long()
        out = torch.index_select(s["table"], 0, t.clamp(min=0)).double() * c["scale"]
        out[t < 0] = 0.0
        return {"out": out}
    if c["op"] == "scatter":
        t = s["tokens"].long()
        keep = t >= 0
        d = torch.zeros(s["update"].shape, dtype=torch.float64, device=t.device)
        d.index_put_((t[keep],), s["grad"][keep].double() * c["scale"], accumulate=True)
        return {"update": d + s["update"].double() if c["add"] else d}
    few = max(1, (1 << 25) // c["vocab"])
    cuts = [slice(i, i + few) for i in range(0, c["rows"], few)]
    if c["op"] == "top":
        ids, logp = [], []
        for cut in cuts:
            z = s["logits"][cut].double()
            v, i = torch.sort(z, dim=1, descending=True, stable=True)
            ids.append(i[:, :c["k"]].to(torch.int32))
            logp.append((v[:, :c["k"]] / c["tau"]) - torch.logsumexp(z / c["tau"], dim=1, keepdim=True))
        return {"ids": torch.cat(ids), "logp": torch.cat(logp)}
    loss, grad = [], []
    for cut in cuts:
        a, b = _exact_distill_rows(s["logits"][cut], s["ids"][cut], s["logp"][cut], None if s["weight"] is None else s["weight"][cut],
                                   c["tau"], c["rest"])
        loss.append(a)
        if c["op"] != "loss":
            grad.append(b)
    if c["op"] == "loss":
        return {"loss": torch.cat(loss)}
    return {"loss": torch.cat(loss), "d_logits": torch.cat(grad)}
