"""A logit that is infinite, at the target and elsewhere, in every way in which the logits are made: the row's loss says so, the other rows' do not."""
import math

import pytest
import torch

import test_gpu_head as H

pytestmark = pytest.mark.gpu

# few logits with 32 to 256 threads a row, one word, up to 128 rows in 32 bits, kept in 16 bits, several pieces (of each the loss alone, too)
SIZES = [(50, 64, 40, 1), (9, 72, 1023, 1), (3, 64, 8192, 1), (40, 64, 1, 1), (100, 64, 8300, 1), (300, 72, 8300, 1), (4200, 96, 3000, 3), (100, 72, 90001, 2)]


def one_far(rows, dim, vocab, dtype, other, sign):
    """hidden states of zeros but for one value of row 3 (the last one), whose product with one word, the row's target or another, is sign times 2^130"""
    hidden, head, t = H.make(rows, dim, vocab, dtype)
    at = min(3, rows - 1)
    word = int(t[at]) if not other else (int(t[at]) + 1) % vocab
    hidden.zero_()
    head[:, 0] = 0
    hidden[at, 0], head[word, 0] = 2.0 ** 15, sign * 2.0 ** 15
    return hidden, head, t, at


@pytest.mark.parametrize("dtype", [H.BF, H.HF])
@pytest.mark.parametrize("rows,dim,vocab,pieces", SIZES)
@pytest.mark.parametrize("other", [False, True])
def test_plus_infinite(dtype, rows, dim, vocab, pieces, other):
    if other and vocab == 1:
        other = False
    hidden, head, t, at = one_far(rows, dim, vocab, dtype, other, 1.0)
    alone, loss, dh, dw = H.run(hidden, head, t, scale=2.0 ** 100, pieces=pieces)
    others = torch.arange(rows, device="cuda") != at
    for x in (alone, loss):
        assert not bool(torch.isfinite(x[at])), x[at]
        # ln vocab: of logits of 0, in fp32
        assert bool(((x[others] - math.log(vocab)).abs() <= 2.0 ** -20).all())
    # the others' are numbers: 2^100 times a sum of head values / vocab, which is beyond fp16's 65504, not beyond bf16's range
    assert not bool(torch.isfinite(dh[at]).all()) and not bool(torch.isnan(dh[others]).any())
    assert dtype == H.HF or bool(torch.isfinite(dh[others]).all())
    # and a weight does not hide it
    weight = torch.full((rows,), 0.5, device="cuda")
    alone, loss, _, _ = H.run(hidden, head, t, scale=2.0 ** 100, pieces=pieces, weight=weight)
    assert not bool(torch.isfinite(alone[at])) and not bool(torch.isfinite(loss[at]))
    weight[at] = 0
    alone, loss, dh, dw = H.run(hidden, head, t, scale=2.0 ** 100, pieces=pieces, weight=weight)
    assert float(alone[at]) == 0 and float(loss[at]) == 0 and not bool(dh[at].any()) and bool(torch.isfinite(dw).all())


@pytest.mark.parametrize("dtype", [H.BF, H.HF])
@pytest.mark.parametrize("rows,dim,vocab,pieces", [s for s in SIZES if s[2] > 1])
def test_minus_infinite(dtype, rows, dim, vocab, pieces):
    """the loss of that word is infinite; of another it is what the other words make it"""
    hidden, head, t, at = one_far(rows, dim, vocab, dtype, False, -1.0)
    alone, loss, _, _ = H.run(hidden, head, t, scale=2.0 ** 100, pieces=pieces)
    others = torch.arange(rows, device="cuda") != at
    for x in (alone, loss):
        assert not bool(torch.isfinite(x[at])) and bool(torch.isfinite(x[others]).all())
    hidden, head, t, at = one_far(rows, dim, vocab, dtype, True, -1.0)
    alone, loss, _, _ = H.run(hidden, head, t, scale=2.0 ** 100, pieces=pieces)
    want = torch.full((rows,), math.log(vocab), device="cuda")
    want[at] = math.log(vocab - 1)
    for x in (alone, loss):
        assert bool(((x - want).abs() <= 2.0 ** -20).all())
