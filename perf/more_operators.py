"""Performance cases of a local step's loss and optimiser: softmax cross entropy against a head matrix (the training loss of a
client whose model speaks a vocabulary), AdamW over a model's tensors and the norm its clipping needs, through the public
entry points.

A case is a dict of plain values:

    op        loss      cross entropy of hidden states against the head, the loss alone (cvlc_head_loss)
              step      loss and the gradients of hidden states and head (cvlc_head_step)
              norm      norm of all gradients (cvlc_grad_norm)
              adamw     one step over all tensors (cvlc_adamw); "clip": behind a norm of its own, or a norm that is there already
    dtype     step, loss: of hidden states, head and their gradients: "bf16" or "fp16"; norm, adamw: of the gradients: "fp32" too
    rows, dim, vocab, pad     hidden is rows x dim, head vocab x dim, with `pad` unused elements behind each row
    wide      tokens in 64 instead of 32 bits
    masked    rows without a target and rows of weight 0 among rows of different weights
    scale     of the logits
    pieces    in how many pieces of the vocabulary the gradients are made (1: all at once)
    n, tensors, flat          values in all, in how many tensors of one vector; flat: one behind the other, else each at a multiple of 256
    bits      of the states: 32, or 8 (e4m3 and e5m2 with a scale for 256 values each, rounded stochastically)
    copy      a bf16 copy of the fp32 weights is written on the way
    clip      "none", "norm" (cvlc_grad_norm in the pass) or "given" (a norm from before)
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
BLOCK = 256  # values that share a scale
BETA1, BETA2, EPS, LR, DECAY, STEP, MOST = 0.9, 0.999, 1e-8, 1e-3, 0.1, 100, 1.0


def _head(name, op, dtype, rows, dim, vocab, pad=0, wide=False, masked=False, scale=1.0, pieces=1):
    return {"name": name, "op": op, "dtype": dtype, "rows": rows, "dim": dim, "vocab": vocab, "pad": pad, "wide": wide, "masked": masked,
            "scale": scale, "pieces": pieces}


def _tensors(name, op, dtype, n, tensors, flat=False, bits=32, copy=False, clip="none"):
    return {"name": name, "op": op, "dtype": dtype, "n": n, "tensors": tensors, "flat": flat, "bits": bits, "copy": copy, "clip": clip}


def listed():
    return [
        # scoring one token for each of eight sequences: reading the head is all there is
        _head("loss_small", "loss", "bf16", 8, 1024, 32000),
        # evaluation on a whole batch
        _head("loss_large", "loss", "bf16", 4096, 4096, 131072, wide=True),
        # a local step on one short prompt
        _head("step_small", "step", "bf16", 16, 1024, 32000),
        # an odd vocabulary, padded rows, tokens that count for nothing and weights
        _head("step_ragged", "step", "fp16", 777, 1000, 50021, pad=11, masked=True, scale=0.5),
        # a batch of a model with a large vocabulary, with room for a piece of the probabilities only
        _head("step_pieces", "step", "bf16", 4096, 2048, 131072, wide=True, masked=True, pieces=8),
        # a local step on a whole batch
        _head("step_large", "step", "bf16", 8192, 4096, 131072),
        # the gradients of a small model
        _tensors("norm_small", "norm", "fp32", 1200000, 8),
        # the gradients of a large one
        _tensors("norm_large", "norm", "bf16", 500000000, 300),
        # a client's step on a convolutional model whose weights are one vector, clipped
        _tensors("adamw_flat", "adamw", "fp32", 11200000, 62, flat=True, clip="norm"),
        # fp32 weights with a bf16 copy for the products
        _tensors("adamw_large", "adamw", "bf16", 100000000, 161, copy=True),
        # many clients' states on one GPU, 8 bits each: a small model
        _tensors("adamw8_small", "adamw", "fp32", 100000, 8, bits=8),
        # and a large one
        _tensors("adamw8_large", "adamw", "bf16", 100000000, 161, bits=8, copy=True, clip="given"),
    ]


def draw(rng):
    def log_uniform(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))) if hi > lo else lo

    op = rng.choice(["loss", "step", "step", "norm", "adamw", "adamw"])
    if op in ("loss", "step"):
        dim = log_uniform(64, 4096)
        if rng.random() < 0.8:
            dim = dim // 8 * 8
        vocab = log_uniform(10, min(200000, (1 << 29) // dim))
        rows = log_uniform(1, min(8192, (1 << 41) // (dim * vocab)))
        c = _head("", op, rng.choice(["bf16", "bf16", "fp16"]), rows, dim, vocab, pad=rng.choice([0, 0, 8, 11]), wide=rng.random() < 0.5,
                  masked=rng.random() < 0.4, scale=rng.choice([1.0, 1.0, 0.5]), pieces=rng.choice([1, 1, 3, 8]) if op == "step" else 1)
    else:
        n = log_uniform(1000, 100000000)
        bits = rng.choice([32, 8]) if op == "adamw" else 32
        dtype = rng.choice(["fp32", "bf16", "fp16"])
        c = _tensors("", op, dtype, n, log_uniform(1, min(600, n // 100)), flat=rng.random() < 0.3, bits=bits,
                     copy=op == "adamw" and rng.random() < 0.5, clip="none" if op == "norm" else rng.choice(["none", "given", "norm" if bits == 32 else "none"]))
    del c["name"]
    return c


# ---- inputs -------------------------------------------------------------------------------

def _pad(rows, cols, pad, dtype, device):
    """rows x cols inside rows x (cols + pad)"""
    return torch.zeros(rows, cols + pad, dtype=dtype, device=device)[:, :cols]


def _sizes(n, tensors):
    """a model's tensors: a few hold most of the values, many are short"""
    rng = random.Random(n * 1000003 + tensors)
    w = [10.0 ** rng.uniform(0.0, 3.5) for _ in range(tensors)]
    left = n - tensors
    sizes = [1 + int(left * x / sum(w)) for x in w]
    sizes[0] += n - sum(sizes)
    return sizes


def _blocks(sizes):
    return [(k + BLOCK - 1) // BLOCK for k in sizes]


def _places(sizes, flat):
    """where the tensors begin in the vector that holds them, and its length: one behind the other, or each at a multiple of 256"""
    room = sizes if flat else [b * BLOCK for b in _blocks(sizes)]
    starts = [0]
    for k in room:
        starts.append(starts[-1] + k)
    return starts


def _spread(x, sizes, starts):
    """values one behind the other, put where the tensors are"""
    if starts[-1] == x.numel():
        return x
    out = torch.zeros(starts[-1], dtype=x.dtype, device=x.device)
    torch._foreach_copy_(_views(out, sizes, starts), list(torch.split(x, sizes)))
    return out


def _views(x, sizes, starts):
    return [x[a:a + k] for a, k in zip(starts, sizes)]


def _fill(sizes, values, device):
    """one value for all of a tensor, and the next for the next"""
    return torch.repeat_interleave(torch.as_tensor(values, dtype=torch.float32, device=device), torch.as_tensor(sizes, device=device))


def prepare(case, seed):
    c = case
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev).manual_seed(seed)
    s = dict(c)
    if c["op"] in ("loss", "step"):
        rows, dim, vocab, dt = c["rows"], c["dim"], c["vocab"], DTYPES[c["dtype"]]
        s["head"] = _pad(vocab, dim, c["pad"], dt, dev)
        s["head"].copy_(torch.randn(vocab, dim, generator=gen, device=dev).mul_(2.5 / math.sqrt(dim)))
        # words by their rank: the i-th about as often as 1 / i; the model leans to the right word, more or less
        u = torch.rand(rows, generator=gen, device=dev, dtype=torch.float64)
        t = torch.exp(u * math.log(vocab + 1)).long().sub_(1).clamp_(0, vocab - 1)
        lean = torch.rand(rows, 1, generator=gen, device=dev) * (2.4 / c["scale"])
        s["hidden"] = _pad(rows, dim, c["pad"], dt, dev)
        s["hidden"].copy_(torch.randn(rows, dim, generator=gen, device=dev) + lean * s["head"][t].float())
        s["weight"] = None
        if c["masked"]:
            s["weight"] = torch.rand(rows, generator=gen, device=dev)
            s["weight"][torch.rand(rows, generator=gen, device=dev) < 0.1] = 0.0
            t[torch.rand(rows, generator=gen, device=dev) < 0.1] = -1
        s["targets"] = t if c["wide"] else t.to(torch.int32)
        s["loss"] = torch.zeros(rows, device=dev)
        if c["op"] == "step":
            s["d_hidden"] = _pad(rows, dim, c["pad"], dt, dev)
            s["d_head"] = _pad(vocab, dim, c["pad"], dt, dev)
        if own:  # a workspace that every call uses
            from paper_2402_03770_b200 import binding as B
            s["ws"] = B.alloc_bytes(B.cvlc_head_workspace_bytes(s["hidden"], s["head"], pieces=c["pieces"] if c["op"] == "step" else 0), dev)
        return s
    n, dt = c["n"], DTYPES[c["dtype"]]
    s["sizes"] = sizes = _sizes(n, c["tensors"])
    s["starts"] = starts = _places(sizes, c["flat"])
    # layers of different scales
    width = _fill(sizes, 10.0 ** (torch.rand(c["tensors"], generator=gen, device=dev) * 2.0 - 4.0), dev)
    s["grads"] = _spread(torch.randn(n, generator=gen, device=dev).mul_(width).to(dt), sizes, starts)
    s["norm"] = torch.zeros(1, device=dev)
    if c["op"] == "adamw":
        s["params"] = _spread(torch.randn(n, generator=gen, device=dev).mul_(0.02), sizes, starts)
        m = torch.randn(n, generator=gen, device=dev).mul_(0.3).mul_(width)
        v = torch.randn(n, generator=gen, device=dev).mul_(0.2).add_(1.0).mul_(width).square_().mul_(1.0 - BETA2 ** (STEP - 1))
        s["m"], s["v"] = _spread(m, sizes, starts), _spread(v, sizes, starts)
        s["state_starts"] = starts
        if c["bits"] == 8:  # states of their own: bytes, and for 256 of them two scales
            s["state_starts"] = apart = _places(sizes, False)
            m, v = (_spread(x, sizes, apart).view(-1, BLOCK) for x in (m, v))
            a, b = m.abs().amax(dim=1, keepdim=True) / 448.0, v.amax(dim=1, keepdim=True) / 57344.0
            s["scales"] = torch.cat([a, b], dim=1)
            s["m"] = (m / a).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8).view(-1)
            s["v"] = (v / b).clamp(0.0, 57344.0).to(torch.float8_e5m2).view(torch.uint8).view(-1)
        del m, v
        if c["copy"]:
            s["copies"] = torch.zeros(starts[-1], dtype=torch.bfloat16, device=dev)
        # weight decay for the large tensors, none for the short ones
        s["decay"] = [DECAY if k > 1000 else 0.0 for k in sizes]
        s["seed"] = seed
        if c["clip"] == "given":
            s["norm"].fill_(1.0 + 3.0 * random.Random(seed).random())
    del width
    if own:
        from paper_2402_03770_b200 import binding as B
        more = {k: _views(s[k], sizes, starts) for k in ("params", "copies") if k in s}
        more |= {k: _views(s[k], sizes, s["state_starts"]) for k in ("m", "v") if k in s}
        if "scales" in s:
            more["scales"] = list(torch.split(s["scales"], _blocks(sizes)))
        s["list"] = B.AdamwTensors(_views(s["grads"], sizes, starts), weight_decay=s.get("decay"), **more)
        s["ws"] = B.alloc_bytes(B.cvlc_grad_norm_workspace_bytes(s["list"]), dev)
    return s


# ---- one pass -----------------------------------------------------------------------------

def _plain_head(s):
    h, w, t = s["hidden"].float(), s["head"].float(), s["targets"].long()
    there = (t >= 0).float()
    if s["weight"] is not None:
        there = there * s["weight"]
    t = t.clamp(min=0)[:, None]
    z = (h @ w.T).mul_(s["scale"])
    z_t = z.gather(1, t)
    m = z.amax(dim=1, keepdim=True)
    e = torch.exp(z.sub_(m))
    others = e.scatter(1, t, 0.0).sum(dim=1, keepdim=True)
    right = torch.exp(z_t - m)
    total = others + right
    # log(1 + others / right); where the right word is out of sight, by logarithms
    near = others < right
    loss = torch.where(near, torch.log1p(others / torch.where(near, right, 1.0)), torch.log(total) + m - z_t)[:, 0] * there
    if s["op"] == "loss":
        return {"loss": loss}
    g = e.scatter_(1, t, -others)
    g *= there[:, None] * s["scale"] / total
    return {"loss": loss, "d_hidden": (g @ w).to(s["hidden"].dtype), "d_head": (g.T @ h).to(s["head"].dtype)}


def _philox(c0, c1, c2, c3, k0, k1):
    """Philox4x32-10; counters as whole numbers of 64 bits that hold 32"""
    low = 0xFFFFFFFF
    for _ in range(10):
        p, q = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # of 64 bits: the upper half comes out by shift and mask
        c0, c1, c2, c3 = ((q >> 32) & low) ^ c1 ^ k0, q & low, ((p >> 32) & low) ^ c3 ^ k1, p & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _random(s, dev):
    """32 random bits for every value of every block: counter (value / 4, tensor, step), key seed"""
    quads = torch.as_tensor(_blocks(s["sizes"]), device=dev) * (BLOCK // 4)
    tensor = torch.repeat_interleave(torch.arange(len(quads), device=dev), quads)
    quad = torch.arange(len(tensor), device=dev) - torch.repeat_interleave(torch.cumsum(quads, 0) - quads, quads)
    words = _philox(quad & 0xFFFFFFFF, quad >> 32, tensor, torch.full_like(tensor, STEP), s["seed"] & 0xFFFFFFFF, s["seed"] >> 32)
    return torch.stack(words, dim=1).view(-1, BLOCK)


def _to_float8(y, random16, mantissa, bias, lowest):
    """codes of values from 0 up, rounded up with the probability of what is cut off; `lowest`: the smallest normal value"""
    cut = 23 - mantissa
    small = y < lowest
    bits = torch.where(small, y + lowest, y).view(torch.int32).long() + (random16 << (cut - 16)) + (1 << (cut - 17))
    return (bits >> cut) - ((127 - bias) << mantissa) - torch.where(small, 1 << mantissa, 0)


def _plain_norm(grads):
    return torch.sqrt(grads.float().square().sum(dtype=torch.float64)).float().view(1)


def _plain_adamw(s):
    dev, sizes, starts, apart = s["grads"].device, s["sizes"], s["starts"], s["state_starts"]
    g, p = s["grads"].float(), s["params"]
    if s["clip"] == "norm":
        s["norm"].copy_(_plain_norm(g))
    if s["clip"] != "none":
        g = g * torch.where(s["norm"] > MOST, MOST / s["norm"], 1.0)
    eight, moved = s["bits"] == 8, apart[-1] != starts[-1]
    if moved:  # the weights lie one behind the other, the states by blocks
        g, p = (_spread(torch.cat(_views(x, sizes, starts)), sizes, apart) for x in (g, p))
    if eight:
        m = (s["m"].view(-1, BLOCK).view(torch.float8_e4m3fn).float() * s["scales"][:, :1]).view(-1)
        v = (s["v"].view(-1, BLOCK).view(torch.float8_e5m2).float() * s["scales"][:, 1:]).view(-1)
    else:
        m, v = s["m"], s["v"]
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + (1.0 - BETA2) * (g * g)
    decay = _fill([b - a for a, b in zip(apart, apart[1:])], s["decay"], dev)
    p = p - LR * (decay * p + (m / (1.0 - BETA1 ** STEP)) / (torch.sqrt(v / (1.0 - BETA2 ** STEP)) + EPS))
    if eight:
        bits = _random(s, dev)
        m, v = m.view(-1, BLOCK), v.view(-1, BLOCK)
        a, b = m.abs().amax(dim=1, keepdim=True), v.amax(dim=1, keepdim=True)
        floor = 2.0 ** -100
        ia, ib = torch.where(a >= floor, 448.0 / a, 0.0), torch.where(b >= floor, 57344.0 / b, 0.0)
        a, b = torch.where(a >= floor, a / 448.0, 0.0), torch.where(b >= floor, b / 57344.0, 0.0)
        c = _to_float8((m.abs() * ia).clamp(max=448.0), bits & 0xFFFF, 3, 7, 2.0 ** -6)
        c = torch.where((m < 0) & (c > 0), c | 128, c)
        y = (v * ib).clamp(max=57344.0)
        d = _to_float8(y, bits >> 16, 2, 15, 2.0 ** -14)
        d = torch.where(y > 0, d.clamp(min=1), 0)
        s["m"].copy_(c.view(-1))
        s["v"].copy_(d.view(-1))
        s["scales"].copy_(torch.cat([a, b], dim=1))
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    if moved:
        p = torch.cat(_views(p, sizes, apart))
    s["params"].copy_(p)
    if s["copy"]:
        s["copies"].copy_(p)


def _updated(s):
    out = {k: s[k] for k in ("params", "copies", "scales") if k in s}
    eight = s["bits"] == 8
    out |= {"m": s["m"].view(torch.float8_e4m3fn) if eight else s["m"], "v": s["v"].view(torch.float8_e5m2) if eight else s["v"]}
    if s["clip"] == "norm":
        out["norm"] = s["norm"]
    return out


def _own(s):
    from paper_2402_03770_b200 import binding as B
    op = s["op"]
    if op == "loss":
        B.cvlc_head_loss(s["hidden"], s["head"], s["targets"], s["loss"], s["ws"], scale=s["scale"], row_weight=s["weight"])
        return {"loss": s["loss"]}
    if op == "step":
        B.cvlc_head_step(s["hidden"], s["head"], s["targets"], s["loss"], s["d_hidden"], s["d_head"], s["ws"], scale=s["scale"],
                         row_weight=s["weight"], pieces=s["pieces"])
        return {"loss": s["loss"], "d_hidden": s["d_hidden"], "d_head": s["d_head"]}
    if op == "norm" or s["clip"] == "norm":
        B.cvlc_grad_norm(s["list"], s["norm"], s["ws"])
    if op == "norm":
        return {"norm": s["norm"]}
    B.cvlc_adamw(s["list"], lr=LR, step=STEP, beta1=BETA1, beta2=BETA2, eps=EPS, norm=None if s["clip"] == "none" else s["norm"], max_norm=MOST,
                 seed=s["seed"])
    return _updated(s)


def run(s):
    if own:
        return _own(s)
    if s["op"] in ("loss", "step"):
        return _plain_head(s)
    if s["op"] == "norm":
        return {"norm": _plain_norm(s["grads"])}
    _plain_adamw(s)
    return _updated(s)


def work(case):
    """Inputs once, outputs once.  A step of the head: three products (logits and two gradients).  A step of the optimiser reads and
    writes weights and states, reads gradients and writes the copy."""
    c, size = case, SIZE[case["dtype"]]
    if c["op"] in ("loss", "step"):
        both = (c["rows"] + c["vocab"]) * c["dim"] * size
        graded = c["op"] == "step"
        per_row = (8 if c["wide"] else 4) + 4 + (4 if c["masked"] else 0)
        return {"bytes": both * (2 if graded else 1) + c["rows"] * per_row, "flops": c["rows"] * c["vocab"] * c["dim"] * (6 if graded else 2)}
    if c["op"] == "norm":
        return {"bytes": c["n"] * size, "flops": 2 * c["n"]}
    states = 16 if c["bits"] == 32 else 4 + 16 / BLOCK
    once = size * (2 if c["clip"] == "norm" else 1)
    return {"bytes": c["n"] * (8 + states + once + (2 if c["copy"] else 0)), "flops": 15 * c["n"]}


# ---- the definitions in 64 bits -----------------------------------------------------------

def _exact_head(c, s):
    """the loss as a function of hidden states and head, and its gradients by differentiating the logits' part by hand only"""
    w, rows = s["head"].double(), c["rows"]
    weight = torch.ones(rows, dtype=torch.float64, device=w.device) if s["weight"] is None else s["weight"].double()
    weight = torch.where(s["targets"] >= 0, weight, torch.zeros_like(weight))
    few = max(1, (1 << 27) // c["vocab"])
    loss, d_hidden, d_head = [], [], torch.zeros_like(w)
    for i in range(0, rows, few):
        h = s["hidden"][i:i + few].double()
        z = torch.matmul(h, w.t()) * c["scale"]
        t = s["targets"][i:i + few].long()
        counts = weight[i:i + few]
        z.requires_grad_(c["op"] == "step")
        q = torch.nn.functional.cross_entropy(z, torch.where(t < 0, 0, t), reduction="none") * counts
        loss.append(q.detach())
        if c["op"] == "step":
            g, = torch.autograd.grad(q.sum(), z)
            g = g * c["scale"]
            d_hidden.append(torch.matmul(g, w))
            d_head.add_(torch.matmul(g.t(), h))
    if c["op"] == "loss":
        return {"loss": torch.cat(loss)}
    return {"loss": torch.cat(loss), "d_hidden": torch.cat(d_hidden), "d_head": d_head}


def _exact_float8(y, chance, mantissa, smallest):
    """y from 0 up between two neighbouring 8-bit values: the upper one where the chance says so"""
    e = torch.floor(torch.log2(torch.clamp(y, min=smallest)))
    step = torch.exp2(e - mantissa)
    low = torch.floor(y / step) * step
    return low + torch.where((y - low) / step + chance >= 1.0, step, torch.zeros_like(step))


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] in ("loss", "step"):
        return _exact_head(c, s)
    # the values one behind the other, and where each lies among weights and among states
    sizes, dev = s["sizes"], s["grads"].device
    k = torch.as_tensor(sizes, device=dev)
    tensor = torch.repeat_interleave(torch.arange(len(sizes), device=dev), k)
    item = torch.arange(c["n"], device=dev) - (torch.cumsum(k, 0) - k)[tensor]
    place = torch.as_tensor(s["starts"], device=dev)[tensor] + item
    g = s["grads"][place].double()
    norm = torch.linalg.vector_norm(g).view(1)
    if c["op"] == "norm":
        return {"norm": norm}
    if c["clip"] != "none":
        g.mul_(torch.clamp(MOST / (norm if c["clip"] == "norm" else s["norm"].double()), max=1.0))
    held = torch.as_tensor(s["state_starts"], device=dev)[tensor] + item
    of = torch.div(held, BLOCK, rounding_mode="floor")
    p, m, v = s["params"][place].double(), s["m"][held], s["v"][held]
    if c["bits"] == 8:
        m, v = m.view(torch.float8_e4m3fn).double(), v.view(torch.float8_e5m2).double()
        m.mul_(s["scales"][:, 0].double()[of])
        v.mul_(s["scales"][:, 1].double()[of])
    m, v = torch.lerp(g, m.double(), BETA1), torch.lerp(g.square(), v.double(), BETA2)
    decay = torch.as_tensor(s["decay"], dtype=torch.float64, device=dev)[tensor]
    rate = (m / (1.0 - BETA1 ** STEP)) / ((v / (1.0 - BETA2 ** STEP)).sqrt() + EPS)
    p = p * (1.0 - LR * decay) - LR * rate
    del g, rate, decay

    def placed(x, at, like):
        return torch.zeros(like.shape, dtype=torch.float64, device=dev).index_copy_(0, at, x)

    out = {"params": placed(p, place, s["params"])}
    if c["copy"]:
        out["copies"] = out["params"]
    if c["clip"] == "norm":
        out["norm"] = norm
    if c["bits"] == 8:
        nothing = torch.zeros(len(s["scales"]), dtype=torch.float64, device=dev)
        a = nothing.scatter_reduce(0, of, m.abs(), "amax") / 448.0
        b = nothing.scatter_reduce(0, of, v, "amax") / 57344.0
        out["scales"] = torch.stack([a, b], dim=1)
        word = _random(s, dev).view(-1)[torch.as_tensor(_places(sizes, False), device=dev)[tensor] + item]
        up = ((word & 0xFFFF).double() + 0.5) / 65536.0
        m = torch.copysign(_exact_float8(m.abs() / a[of], up, 3, 2.0 ** -6), m)
        up = ((word >> 16).double() + 0.5) / 65536.0
        v = torch.where(v > 0, torch.clamp(_exact_float8(v / b[of], up, 2, 2.0 ** -14), min=2.0 ** -16), v)
    out["m"], out["v"] = placed(m, held, s["m"]), placed(v, held, s["v"])
    return out
