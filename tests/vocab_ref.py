"""Top logits, distillation and the embedding from their definitions, in 64 bits with plain tensor operations, and what the kernels' 32-bit
arithmetic may be off by."""
import math

import torch

NONE, SCALED, BUCKET = 0, 1, 2
U = 2.0 ** -24  # half a step of fp32, relative

# ln of a row's sum of exponentials.  A term's exponent (z - m) log2(e) / temperature is off by three roundings (difference, constant,
# product), U each, relative to it; a term of weight 2^-a counts a 2^-a times that, so what the row's terms can add up to is at
# most their average exponent, below log2(vocab) <= 22: 22 * 3 * ln 2 = 46 U.  The exponential itself is off by 2^-22 = 4 U, the sum by one U
# for every addition on the way: 8 of a vector, 8 vectors or the batches before, 5 of a warp, 15 warps, 7 blocks, twice that
# where sums of two maxima are joined: 80 U.  The gradient of a row of more than 262,144 words adds its further batches.
LN = 150 * U


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    """half the distance of the smallest numbers, or what 2^x flushes to zero"""
    return max(torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2, 2.0 ** -126)


def from_largest(z):
    """z less its row's largest value, so that lowest values of a type keep their differences (an empty row: as it is)"""
    m = z.amax(-1, keepdim=True)
    return z - torch.where(m > -math.inf, m, 0.0)


def top(logits, k, temperature):
    z = logits.double().cpu()
    order = torch.sort(z + 0.0, dim=1, descending=True, stable=True)
    v, ids = order.values[:, :k], order.indices[:, :k].to(torch.int32)
    x = from_largest(z) / temperature
    logp = x.gather(1, ids.long()) - torch.logsumexp(x, dim=1, keepdim=True)
    gone = v == -math.inf
    ids = torch.where(gone, -1, ids)
    logp = torch.where(gone, -math.inf, logp)
    spoiled = ~(z < math.inf).all(dim=1, keepdim=True)
    ids = torch.where(spoiled, torch.arange(k, dtype=torch.int32), ids)
    logp = torch.where(spoiled, math.nan, logp)
    logp = logp.float().double()  # what is below fp32's range is -inf
    return ids, logp, torch.where(gone, 0.0, LN + logp.abs() * 2 * U)


def distill(logits, ids, logp, rest, temperature, weight=None):
    """loss, gradient, and how far each may be off before it is rounded to the logits' type"""
    few = max(1, (1 << 24) // logits.shape[1])
    ids, logp = ids.to(logits.device), logp.to(logits.device)
    parts = [_distill_rows(logits[i:i + few], ids[i:i + few], logp[i:i + few], rest, temperature,
                           None if weight is None else weight[i:i + few]) for i in range(0, logits.shape[0], few)]
    return tuple(torch.cat(p) for p in zip(*parts))


def _distill_rows(logits, ids, logp, rest, temperature, weight):
    z, ids, lp = logits.double(), ids.long(), logp.double()
    rows, vocab = z.shape
    x = from_largest(z) / temperature
    lq = x - torch.logsumexp(x, 1, keepdim=True)
    q = lq.exp()
    at = torch.where((ids >= 0) & (ids < vocab), ids, vocab)  # one more column takes what is left out
    p = torch.zeros(rows, vocab + 1, dtype=torch.float64, device=z.device).scatter_add_(1, at, lp.exp())[:, :vocab]
    named = torch.zeros(rows, vocab + 1, dtype=torch.bool, device=z.device).scatter_(1, at, True)[:, :vocab]
    mass = p.sum(1, keepdim=True)
    if rest == SCALED:
        p = torch.where(mass == 0, 0.0, p / mass)
        mass = torch.where(mass == 0, 0.0, torch.ones_like(mass))
    L = torch.where(p == 0, 0.0, p * (p.log() - lq)).sum(1, keepdim=True)
    far = (x.amax(1, keepdim=True) - x).clamp(max=200.0) * 1.4427 * 3 * U + 8 * U  # of exp((z - reference) / temperature)
    left, pull = torch.zeros_like(mass), torch.zeros_like(q)
    if rest == BUCKET:
        some = (~named & ~(z == -math.inf)).any(1, keepdim=True)
        left = torch.where(some, (1.0 - mass).clamp(min=0.0), 0.0)
        lqr = torch.logsumexp(torch.where(named, -math.inf, lq), 1, keepdim=True)
        L = L + torch.where(left > 0, left * (left.log() - lqr), 0.0)
        pull = torch.where(named | (left == 0), 0.0, left * (lq - lqr).exp())
    b = mass + left
    w = torch.ones_like(mass) if weight is None else weight.double()[:, None]
    counts = (w != 0) & ~(z == -math.inf).all(1, keepdim=True)  # else nothing
    out = (w * L, (b * q - pull - p) * w / temperature, abs(w) * (LN * (mass + 2 * left) + 4 * U * abs(L)),
           abs(w) / temperature * ((b * q + pull) * (LN + far + 8 * U) + p * 4 * U))
    out = [torch.where(counts, o, 0.0) for o in out]
    return out[0][:, 0], out[1], out[2][:, 0], out[3]


def assert_near(got, want, tol, dtype=torch.float32, what=""):
    """equal where the definition is not finite; else within tol, rounded to dtype"""
    got, want = got.double(), want.double().to(got.device)
    assert got.shape == want.shape
    odd = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got[odd]), torch.isnan(want[odd])), what
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), what
    off = (got - want).abs()[~odd]
    tol = torch.as_tensor(tol).to(got.device).expand(want.shape)[~odd]
    most = tol * (1 + half_step(dtype)) + want[~odd].abs() * half_step(dtype) + tiny(dtype)
    bad = ~(off <= most)
    assert not bad.any(), (what, int(bad.sum()), float((off / most).max()))


def embed_grad(tokens, grad, vocab, scale, update=None):
    """the table's gradient, and how far fp32 sums of the same terms may be off"""
    t, g = tokens.cpu().long(), grad.double().cpu()
    keep = (t >= 0) & (t < vocab)
    out = torch.zeros(vocab, g.shape[1], dtype=torch.float64)
    out.index_add_(0, t[keep], g[keep])
    size = torch.zeros_like(out).index_add_(0, t[keep], g[keep].abs())
    count = torch.bincount(t[keep], minlength=vocab).double()[:, None]
    tol = abs(scale) * size * (count + 2) * U
    out = out * scale
    if update is not None:
        out = out + update.double().cpu()
        tol = torch.where(count > 0, tol + out.abs() * 2 * U, 0.0)
    return out, tol
