"""Few logits of more than 128 rows: they go through the memory in 32 bits, so that a logit's gradient is rounded to 16 bits once, in fp16 raised by 2^15."""
import pytest
import torch

import head_ref as R
import test_gpu_head as H

pytestmark = pytest.mark.gpu


def check_rounded_once(hidden, head, t, scale=1.0, weight=None):
    rows, vocab = hidden.shape[0], head.shape[0]
    assert rows > 128 and vocab <= 8192 and rows * vocab <= 1 << 22
    alone, loss, dh, dw = H.run(hidden, head, t, scale, weight)
    want, tol, mean = R.step(hidden, head, t, scale, weight, kept=False)
    for x in (alone, loss):
        R.assert_near(x, want["loss"], tol["loss"] * 1.01 + want["loss"].abs() * R.U, "loss")
    for name, got in (("d_hidden", dh), ("d_head", dw)):
        u, least = torch.finfo(got.dtype).eps / 2, torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps / 2
        rounded = want[name].abs() * u + least
        R.assert_near(got, want[name], tol[name] * (1 + u) + rounded, name, torch.sqrt(mean[name].square() + (want[name].abs() * u).square() / 3 + least ** 2))


@pytest.mark.parametrize("dtype", [H.BF, H.HF])
@pytest.mark.parametrize("rows,dim,vocab", [(129, 64, 256), (257, 65, 513), (300, 200, 1000), (1264, 2888, 563), (5579, 104, 117), (4096, 72, 1024), (512, 64, 8192),
                                            (30000, 24, 10), (700, 1000, 1000), (2000, 4096, 70)])
def test_rounded_once(dtype, rows, dim, vocab):
    check_rounded_once(*H.make(rows, dim, vocab, dtype, seed=rows))


@pytest.mark.parametrize("dtype", [H.BF, H.HF])
@pytest.mark.parametrize("rows,dim,vocab", [(5000, 40, 12), (300, 88, 2000)])
@pytest.mark.parametrize("size", [1.0, 2.0 ** -20])
def test_rounded_once_with_weights(dtype, rows, dim, vocab, size):
    hidden, head, t = H.make(rows, dim, vocab, dtype)
    weight = (torch.rand(rows, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda") * 8 - 2) * size
    weight[::6], t[::5] = 0, -7
    check_rounded_once(hidden, head, t, 1.3, weight)


def test_fp16_gradients_are_raised():
    """no word but the rows' own is likelier than 2^-22: its G, held in fp16 as it is, would be a few steps of 2^-24 or none.  Of rows of ones d_head is the sum of
    G itself"""
    rows, dim, vocab = 512, 64, 4096
    hidden = torch.ones(rows, dim, dtype=H.HF, device="cuda")
    head = torch.zeros(vocab, dim, dtype=H.HF, device="cuda")
    head[7] = 0.25  # 16 above the others' logits: they are 2^-23 of it
    t = torch.full((rows,), 7, device="cuda")
    _, loss, dh, dw = H.run(hidden, head, t, scale=1.0)
    q = torch.softmax(hidden[:1].double() @ head.double().T, dim=1)[0]
    G = q.clone()
    G[7] = -(q.sum() - q[7])
    want = (rows * G).view(-1, 1).expand(vocab, dim)
    assert float(G[0]) < 2.0 ** -22
    # G's rounding, d_head's, and half a step of fp16 below its smallest normal value; the sums and exponentials are far below
    assert bool(((dw.double() - want).abs() <= want.abs() * (2.0 ** -11 * 2.1 + 150 * R.U) + 2.0 ** -25).all())
    other = torch.arange(vocab, device="cuda") != 7
    assert bool((dw[other] > 0).all())
