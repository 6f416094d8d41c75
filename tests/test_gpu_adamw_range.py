"""States of 8 bits over all of fp32's range in one block: a second moment above 0 is never held as 0."""
import numpy as np
import pytest
import torch

import adamw_ref as R
from paper_2402_03770_b200 import binding as B

pytestmark = pytest.mark.gpu


def step(grad, v=None, scales=None, seed=0, **how):
    """one step of a tensor; weights, bytes of m and v, scales (from zeros, if not given)"""
    n, blocks = len(grad), -(-len(grad) // R.BLOCK)
    p, m = torch.ones(n, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    v = torch.zeros_like(m) if v is None else v
    scales = torch.zeros(blocks, 2, device="cuda") if scales is None else scales
    B.cvlc_adamw(B.AdamwTensors([grad], [p], [m], [v], [scales]), lr=1e-3, seed=seed, **{"step": 1, **how})
    return p, m, v, scales


@pytest.mark.parametrize("largest", [1e-15, 1e-5, 1.0, 1e10, 1.8e19])
@pytest.mark.parametrize("seed", [0, 5])
def test_second_moment_stays_above_zero(largest, seed):
    """the smallest squares that fp32 holds next to the largest; (1 - beta2) g^2 of 1e-21 is 1e-45, a step of fp32"""
    n = 700
    g = torch.logspace(-21, np.log10(largest), n, dtype=torch.float64).float().cuda()
    order = torch.randperm(n, generator=torch.Generator().manual_seed(seed)).cuda()
    g = g[order]
    p, m, v, scales = step(g, seed=seed)
    new = np.float32(1.0 - 0.999) * (g.cpu().numpy() * g.cpu().numpy())
    assert np.isfinite(new).all()
    code, held = v.cpu().numpy(), R.held(v.cpu().numpy(), torch.float8_e5m2) * scales.cpu().numpy()[np.arange(n) // R.BLOCK, 1]
    # (a block whose largest is below 2^-100 is held as zeros)
    there = np.maximum.reduceat(new, np.arange(0, n, R.BLOCK))[np.arange(n) // R.BLOCK] >= np.float32(2.0 ** -100)
    assert (code[(new > 0) & there] > 0).all()
    assert (held[(new > 0) & there] > 0).all()
    assert not code[new == 0].any() and bool(torch.isfinite(p).all())


def test_it_stays_while_it_decays():
    """a block of one large and one tiny value without gradients: both are there after many steps"""
    n = 256
    v, scales = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.tensor([[0.0, 1e30]], device="cuda")
    v[7], v[100] = 0x7B, 1  # 57344 and 2^-16
    for t in range(1, 40):
        _, _, v, scales = step(torch.zeros(n, device="cuda"), v, scales, seed=t, step=t, beta2=0.5)
        assert int(v[7]) > 0 and int(v[100]) > 0 and int((v != 0).sum()) == 2


def test_zeros_stay_zeros_and_small_blocks_are_held_as_zeros():
    g = torch.zeros(768, device="cuda")
    g[256:512] = 1e-17   # 1e-37, below 2^-100
    g[512] = 1.0
    _, m, v, scales = step(g)
    assert not bool(v[:512].any()) and not bool(scales[:2, 1].any()) and int((v[512:] != 0).sum()) == 1


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_what_is_not_finite_stays_in_its_block(bad):
    g = torch.full((600,), 1e-3, device="cuda")
    g[300] = bad
    p, m, v, scales = step(g)
    assert not bool(torch.isfinite(scales[1]).any()) and bool(torch.isfinite(scales[0]).all()) and bool(torch.isfinite(scales[2]).all())
    keep = torch.arange(600, device="cuda") != 300
    assert bool(torch.isfinite(p[keep]).all())
