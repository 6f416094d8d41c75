"""The bounded waits inside the products: copies that never come, readers that give up while all else is at work.  Who gives up says so and leaves nothing behind:
what it had a part in is NaN, and the next call on the same workspace has its own bits."""
import pytest
import torch

import test_gpu_head as H
from paper_2402_03770_b200 import binding as B

pytestmark = pytest.mark.gpu
LIMIT = 20_000  # microseconds; a product of these takes less than 100

# rows, dim, vocab, type, pieces; the step's launches of products, of which the first makes the logits; whether hidden states' gradients are made whole
CASES = {
    "few": (300, 200, 900, H.BF, 1, 2, True),
    "few_parts": (16, 1024, 4000, H.HF, 1, 2, False),
    "few_more_tiles_than_blocks": (4000, 5120, 500, H.BF, 1, 2, True),
    "one_tile_of_rows": (100, 264, 70000, H.BF, 1, 2, False),
    "one_tile_of_rows_pieces": (100, 72, 90001, H.HF, 2, 5, False),
    "pairs_fp16": (2000, 264, 8300, H.HF, 1, 3, False),
    "pairs_pieces": (4200, 96, 3000, H.BF, 3, 10, False),
}
FAULTS = [dict(lost_copy=0), dict(lost_tile=0), dict(lost_copy=0, lost_tile=0)]


def outputs(hidden, head):
    return torch.full((hidden.shape[0],), 7.0, device="cuda"), torch.full_like(hidden, 7.0), torch.full_like(head, 7.0)


def faulty(hidden, head, t, ws, pieces=1, graded=True, **fault):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    loss, dh, dw = outputs(hidden, head)
    B.cvlc_selftest_head(hidden, head, t, loss, dh if graded else None, dw if graded else None, ws, pieces=pieces, limit_us=LIMIT, status=status, **fault)
    torch.cuda.synchronize()
    return int(status), loss, dh


def sound(hidden, head, t, ws, pieces=1):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    loss, dh, dw = outputs(hidden, head)
    B.cvlc_head_step(hidden, head, t, loss, dh, dw, ws, pieces=pieces, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    return loss, dh, dw


@pytest.mark.parametrize("name", CASES)
def test_no_fault(name):
    rows, dim, vocab, dtype, pieces, products, _ = CASES[name]
    hidden, head, t = H.make(rows, dim, vocab, dtype)
    ws = H.space(hidden, head, pieces)
    good = sound(hidden, head, t, ws, pieces)
    for product in (0, products - 1, products):  # the last one is none
        fault = dict(lost_copy=0) if product == products else {}
        status, loss, dh = faulty(hidden, head, t, ws, pieces, product=product, **fault)
        assert status == 0 and torch.equal(loss, good[0]) and torch.equal(dh, good[1])


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("graded", [False, True])
@pytest.mark.parametrize("fault", FAULTS, ids=str)
def test_logits(name, graded, fault):
    rows, dim, vocab, dtype, pieces, _, _ = CASES[name]
    hidden, head, t = H.make(rows, dim, vocab, dtype)
    ws = H.space(hidden, head, pieces)
    good = sound(hidden, head, t, ws, pieces)
    status, loss, dh = faulty(hidden, head, t, ws, pieces, graded, product=0, **fault)
    assert status == B.CVLC_ERR_DEVICE_TIMEOUT and bool(torch.isnan(loss).all())
    assert not graded or bool(torch.isnan(dh).all())
    assert all(torch.equal(x, y) for x, y in zip(sound(hidden, head, t, ws, pieces), good))


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("fault", FAULTS[:2], ids=str)
def test_gradients(name, fault):
    rows, dim, vocab, dtype, pieces, products, whole = CASES[name]
    hidden, head, t = H.make(rows, dim, vocab, dtype)
    ws = H.space(hidden, head, pieces)
    good = sound(hidden, head, t, ws, pieces)
    for product in range(1, products):
        status, loss, dh = faulty(hidden, head, t, ws, pieces, product=product, **fault)
        assert status == B.CVLC_ERR_DEVICE_TIMEOUT and torch.equal(loss, good[0]) and bool(torch.isnan(dh).all()), product
        assert all(torch.equal(x, y) for x, y in zip(sound(hidden, head, t, ws, pieces), good))


@pytest.mark.parametrize("fault", FAULTS, ids=str)
@pytest.mark.parametrize("wild", [False, True])
def test_exponentials_kept_in_bf16(fault, wild):
    """two turns of the logits, of which the second finds nothing to do without rows whose target is far below some other word"""
    hidden, head, t = H.make(2000, 264, 8300, H.BF, width=8.0 if wild else 2.0)
    if wild:
        for i in (0, 700, 1999):
            hidden[i] = (-25 * head[t[i]].float()).to(H.BF)
    ws = H.space(hidden, head, 1)
    good = sound(hidden, head, t, ws)
    for product in range(4):
        status, loss, dh = faulty(hidden, head, t, ws, product=product, **fault)
        if product == 1 and not wild:
            assert status == 0 and all(torch.equal(x, y) for x, y in zip((loss, dh), good))
        else:
            assert status == B.CVLC_ERR_DEVICE_TIMEOUT, product
            assert bool(torch.isnan(dh).all()) and (bool(torch.isnan(loss).all()) if product == 0 else True)
            assert product < 2 or torch.equal(loss, good[0])
        assert all(torch.equal(x, y) for x, y in zip(sound(hidden, head, t, ws), good))


def test_second_tiles_of_a_launch_of_both_gradients():
    """20 + 160 tiles: blocks 0 to 31 have a second one, of the head's gradient; the hidden states' is whole"""
    hidden, head, t = H.make(100, 5120, 900)
    ws = H.space(hidden, head, 1)
    good = sound(hidden, head, t, ws)
    status, loss, dh = faulty(hidden, head, t, ws, product=1, lost_tile=1)
    assert status == B.CVLC_ERR_DEVICE_TIMEOUT and torch.equal(loss, good[0]) and torch.equal(dh, good[1])
    assert all(torch.equal(x, y) for x, y in zip(sound(hidden, head, t, ws), good))


@pytest.mark.parametrize("fault", [dict(lost_tile=n) for n in (1, 2, 3)] + [dict(lost_copy=n) for n in (1, 2, 3)], ids=str)
def test_in_the_middle(fault):
    """264 tiles for 74 pairs of blocks: three or four for each"""
    for dtype in (H.BF, H.HF):
        hidden, head, t = H.make(2000, 264, 8300, dtype)
        for graded in (False, True):
            ws = H.space(hidden, head, int(graded))
            status, loss, dh = faulty(hidden, head, t, ws, graded=graded, product=0, **fault)
            assert status == B.CVLC_ERR_DEVICE_TIMEOUT and bool(torch.isnan(loss).all())
            assert not graded or bool(torch.isnan(dh).all())
    ws = H.space(hidden, head, 1)
    assert all(torch.equal(x, y) for x, y in zip(sound(hidden, head, t, ws), H.run(hidden, head, t)[1:]))
