"""Cross entropy of hidden states against a head and its gradients from the definition, in 64 bits, and how far 16-bit operands and 32-bit sums may
be off."""
import math

import torch

U = 2.0 ** -24  # half a step of fp32, relative
LN = 150 * U    # of ln sum exp (the exponentials, 4 U each, and the additions on the way to the sum)


def sums(n, size):
    """a sum of n products made 16 at a time: a step of fp32 (the tensor cores may cut off) of the sum of sizes for each, a few more at the ends"""
    return size * 2 * U * (n / 16 + 8)


def step(hidden, head, targets, scale=1.0, weight=None, kept=False):
    """kept: the exponentials are kept in 16 bits.  In bf16 their rows' factors go into the hidden states, which are rounded too for the head's
    gradient; in fp16, where they are at most 1 in steps of 2^-24, they are multiplied and rounded once more.
    loss, d_hidden, d_head; the largest error of each before it is rounded to the operands' type, and its root mean square (the rounding of G to
    16 bits is off by a third of a half step, squared, on average)"""
    h, w = hidden.double(), head.double()
    rows, vocab, dim = h.shape[0], w.shape[0], h.shape[1]
    dtype = hidden.dtype
    u = torch.finfo(dtype).eps / 2
    wt = torch.ones(rows, dtype=torch.float64, device=h.device) if weight is None else weight.double()
    t = targets.long()
    wt = torch.where((t >= 0) & (t < vocab), wt, 0.0)
    live = wt != 0
    h = torch.where(live[:, None], h, 0.0)
    t = torch.where(live, t, 0)[:, None]
    z = h @ w.T * scale
    lse = torch.logsumexp(z, dim=1)
    q = torch.exp(z - lse[:, None])
    others, right = q.scatter(1, t, 0.0).sum(dim=1, keepdim=True), q.gather(1, t)
    # of the two forms the one in which nothing cancels (the difference is off by 2^-53 |z|, more than a loss of 1e-13 may be)
    loss = torch.where(others < right, torch.log1p(others / right.clamp(min=2.0 ** -1000)), lse[:, None] - z.gather(1, t))[:, 0]
    loss = torch.where(live, wt * loss, 0.0)
    G = q.scatter(1, t, -others) * wt[:, None]
    dz = sums(dim, h.abs() @ w.abs().T * abs(scale)) + 6 * U * z.abs()
    far = dz.amax(dim=1, keepdim=True)
    tol = {"loss": wt.abs() * (2 * far[:, 0] + LN) + loss.abs() * 4 * U}
    # a loss that is small: relative to the sum of the other words' exponentials, of which each counts as 0 below 2^-126 of the target's
    tol["loss"] = torch.minimum(tol["loss"], loss.abs() * (2 * far[:, 0].expm1() + LN + 4 * U) + wt.abs() * vocab * 2.0 ** -126 + 2.0 ** -126)
    off = G.abs() * (2 * far + LN + 4 * U)                     # the exponent
    cut = G.abs() * u * (1 + 2 * far)                         # the rounding to 16 bits
    if dtype == torch.float16:                                 # held at most 2^15 times the largest weight, in steps of 2^-24, and flushed below 2^-126
        cut = cut + 2.0 ** -39 * wt.abs().max() * 2
        if kept:
            cut = cut + G.abs() * u * 1.01 + 2.0 ** -25 * wt.abs()[:, None] * q.amax(dim=1, keepdim=True)
    cut = cut + 2.0 ** -126 * wt.abs().max()
    out = {"loss": loss, "d_hidden": G @ w * scale, "d_head": G.T @ h * scale}
    aw, ah = w.abs(), h.abs()
    tol["d_hidden"] = abs(scale) * ((off + cut) @ aw + sums(vocab, G.abs() @ aw)) + out["d_hidden"].abs() * 4 * U
    if kept and dtype == torch.bfloat16:
        cut_head, square = cut + G.abs() * u * 1.01, cut.square() + (G.abs() * u).square()
    else:
        cut_head, square = cut, cut.square()
    tol["d_head"] = abs(scale) * ((off + cut_head).T @ ah + sums(rows, G.abs().T @ ah)) + out["d_head"].abs() * 4 * U
    mean = {"d_hidden": abs(scale) * ((off @ aw + sums(vocab, G.abs() @ aw)).square() + (cut.square() / 3) @ w.square()).sqrt(),
            "d_head": abs(scale) * ((off.T @ ah + sums(rows, G.abs().T @ ah)).square() + (square.T / 3) @ h.square()).sqrt()}
    return out, tol, mean


def assert_near(got, want, tol, what="", mean=None):
    got = got.double()
    dtype_u = 0.0
    assert torch.isfinite(want).all() and torch.isfinite(got).all(), what
    err = (got - want).abs()
    bad = ~(err <= tol)
    assert not bad.any(), (what, int(bad.sum()), bad.numel(), float((err / tol.clamp(min=1e-300)).max()), dtype_u)
    if mean is not None and got.numel() >= 4096:  # of many values the root mean square error is near what is expected
        assert float(err.norm()) <= 1.5 * float(mean.norm()), (what, float(err.norm() / mean.norm()))


def check(loss, d_hidden, d_head, hidden, head, targets, scale=1.0, weight=None, pieces=1):
    vocab = head.shape[0]
    kept = vocab <= (max(-(-vocab // pieces), -(-(1 << 22) // len(targets))) + 255) // 256 * 256 and len(targets) > 128  # up to 128 rows in 32 bits
    want, tol, mean = step(hidden, head, targets, scale, weight, kept)
    assert_near(loss, want["loss"], tol["loss"] * 1.01 + want["loss"].abs() * U, "loss")
    for name, got in (("d_hidden", d_hidden), ("d_head", d_head)):
        if got is None:
            continue
        u = torch.finfo(got.dtype).eps / 2
        least = torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps / 2  # half the smallest step
        rounded = want[name].abs() * u + least
        assert_near(got, want[name], tol[name] * (1 + u) + rounded, name, torch.sqrt(mean[name].square() + (want[name].abs() * u).square() / 3 + least ** 2))
