"""One AdamW step and the norm of gradients from their definitions, on the CPU: in 64 bits, and the 8-bit states to the bit."""
import numpy as np
import torch

U = 2.0 ** -24  # half a step of fp32, relative
BLOCK = 256


def philox(counter, key):
    """Philox4x32-10 (Salmon et al., SC'11) of arrays of counters, four uint64 that hold 32 bits each"""
    low = np.uint64(0xFFFFFFFF)
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k = [np.uint64(key & 0xFFFFFFFF), np.uint64(key >> 32)]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ k[0], b & low, (a >> np.uint64(32)) ^ c[3] ^ k[1], a & low]
        k = [(k[0] + np.uint64(0x9E3779B9)) & low, (k[1] + np.uint64(0xBB67AE85)) & low]
    return c


def words(n, tensor, step, seed):
    """the random word of every value of a tensor"""
    quad = np.arange((n + 3) // 4, dtype=np.uint64)
    c = philox((quad & np.uint64(0xFFFFFFFF), quad >> np.uint64(32), np.full_like(quad, tensor), np.full_like(quad, step)), seed)
    return np.stack(c, axis=1).reshape(-1)[:n].astype(np.int64)


_TABLES = {t: torch.arange(128, dtype=torch.uint8).view(t).float().numpy() for t in (torch.float8_e4m3fn, torch.float8_e5m2)}


def held(code, dtype):
    """what bytes stand for"""
    return torch.from_numpy(code).view(dtype).float().numpy()


def round_up_or_down(y, chance, dtype):
    """y (fp32, from 0 to the type's largest value) as one of its two neighbours in the table of 8-bit values: the upper one where
    the chance (16 bits) and the part that is cut off make a whole.  What is cut off of a normal value are the low bits of its float; below the
    smallest normal value it is the distance in whole steps, of a sum that fp32 rounds."""
    lowest, cut = (np.float32(2.0 ** -6), 20) if dtype == torch.float8_e4m3fn else (np.float32(2.0 ** -14), 21)
    table = _TABLES[dtype][:127 if dtype == torch.float8_e4m3fn else 124]
    small = y < lowest
    x = np.where(small, y + lowest, y)
    part = x.view(np.int32).astype(np.int64) & ((1 << cut) - 1)
    down = x.view(np.int32) >> cut << cut
    below = np.where(small, down.astype(np.int32).view(np.float32) - lowest, down.astype(np.int32).view(np.float32))
    code = np.searchsorted(table, below)
    assert np.array_equal(table[code], below)
    return code + (part + (chance << (cut - 16)) + (1 << (cut - 17)) >= 1 << cut)


def moments(g, m, v, scale, beta1, beta2):
    """fp32, each product and sum rounded by itself"""
    f = np.float32
    x = g * f(scale)
    return f(beta1) * m + f(1.0 - beta1) * x, f(beta2) * v + f(1.0 - beta2) * (x * x)


def pack(m, v, tensor, step, seed):
    """bytes and scales of fp32 moments"""
    n = len(m)
    word = words(n, tensor, step, seed)
    of = np.arange(n) // BLOCK
    out = []
    for x, chance, dtype, most in ((m, word & 0xFFFF, torch.float8_e4m3fn, np.float32(448)), (v, word >> 16, torch.float8_e5m2, np.float32(57344))):
        largest = np.maximum.reduceat(np.abs(x), np.arange(0, n, BLOCK))
        there = largest >= np.float32(2.0 ** -100)
        with np.errstate(divide="ignore", over="ignore"):
            inverse = np.where(there, most * (np.float32(1) / largest), np.float32(0))
        y = np.minimum(np.abs(x) * inverse[of], most)
        code = round_up_or_down(y, chance, dtype)
        if dtype == torch.float8_e4m3fn:
            code = np.where((code > 0) & (x < 0), code | 128, code)
        else:
            code = np.where(y > 0, np.maximum(code, 1), 0)
        out.append((code.astype(np.uint8), np.where(there, largest * (np.float32(1) / most), np.float32(0))))
    return out[0][0], out[1][0], np.stack([out[0][1], out[1][1]], axis=1).astype(np.float32)


def step64(p, g, m, v, *, lr, decay, step, beta1, beta2, eps, scale):
    """param, m and v in 64 bits, and how far fp32 may be off: m and v by three roundings of their terms, the step by those of its factors"""
    p, g, m, v = (np.asarray(x, dtype=np.float64) for x in (p, g, m, v))
    x = g * scale
    a, b = beta1 * m, (1 - beta1) * x
    m1, v1 = a + b, beta2 * v + (1 - beta2) * x * x
    tol_m = (np.abs(a) + np.abs(b)) * 4 * U + 2.0 ** -149
    tol_v = v1 * 6 * U + 2.0 ** -148
    root = np.sqrt(v1 / (1 - beta2 ** step))
    d = root + eps
    rate = m1 / (1 - beta1 ** step) / d
    # the root: half of v's error, its factor's rounding and 2 U of its own; below it a v that fp32 holds in steps of 2^-149
    off_d = root * 8 * U + np.sqrt(2.0 ** -148 / (1 - beta2 ** step)) * (v1 < 2.0 ** -120)
    off = tol_m / (1 - beta1 ** step) / d + np.abs(rate) * (8 * U + off_d / d)
    step_ = lr * (decay * p + rate)
    return p - step_, m1, v1, lr * off + np.abs(lr * decay * p) * 4 * U + np.abs(step_) * 3 * U + np.abs(p - step_) * U, tol_m, tol_v
