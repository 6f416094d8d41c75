"""The two gradients of a step with places of their own: one whose rows lie on 16 bytes, which leaves by boxes, next to one whose rows begin anywhere."""
import pytest
import torch

import head_ref as R
import test_gpu_head as H
from paper_2402_03770_b200 import binding as B

pytestmark = pytest.mark.gpu
ON, ODD, SHIFTED, HALF = (0, 0), (3, 0), (0, 1), (4, 4)  # elements between rows, elements in front of the first one


def step(hidden, head, t, hidden_at, head_at, ws, times, **how):
    outs = []
    for _ in range(times):
        loss = torch.full((hidden.shape[0],), 7.0, device="cuda")
        dh, dw = (H.padded(torch.full_like(x, 7.0), *at) for x, at in ((hidden, hidden_at), (head, head_at)))
        B.cvlc_head_step(hidden, head, t, loss, dh, dw, ws, **how)
        outs.append((loss, dh, dw))
    torch.cuda.synchronize()
    return outs


# Both gradients in one launch, the hidden states' in one part, more tiles of both than SMs (20 + 160, 48 + 128, 256 + 256, 640 + 80): blocks go from a tile
# of the one to a tile of the other
@pytest.mark.parametrize("dtype", [H.BF, H.HF])
@pytest.mark.parametrize("rows,dim,vocab", [(100, 5120, 900), (300, 4096, 900), (2000, 4096, 2000), (4000, 5120, 500)])
@pytest.mark.parametrize("hidden_at,head_at", [(ON, ODD), (ON, SHIFTED), (ODD, ON), (HALF, ON), (ON, HALF)])
def test_tiles_of_both_in_a_block(dtype, rows, dim, vocab, hidden_at, head_at):
    hidden, head, t = H.make(rows, dim, vocab, dtype, seed=rows)
    ws = H.space(hidden, head, 1)
    want = step(hidden, head, t, ON, ON, ws, 1)[0]
    R.check(*want, hidden, head, t)
    for got in step(hidden, head, t, hidden_at, head_at, ws, 12):
        assert all(torch.equal(x, y) for x, y in zip(got, want))


# every other way of making them: rows and words by pairs, up to 128 rows, in pieces, joined from parts, rows that are no whole vectors
@pytest.mark.parametrize("dtype", [H.BF, H.HF])
@pytest.mark.parametrize("rows,dim,vocab,pieces", [(5, 72, 40, 1), (5579, 104, 117, 1), (16, 1024, 4000, 1), (100, 264, 8300, 1), (300, 264, 8300, 1), (4200, 96, 3000, 3),
                                                   (100, 72, 90001, 2), (300, 100, 900, 1), (300, 65, 8300, 1)])
@pytest.mark.parametrize("hidden_at,head_at", [(ON, ODD), (ODD, ON), (SHIFTED, HALF)])
def test_every_way(dtype, rows, dim, vocab, pieces, hidden_at, head_at):
    hidden, head, t = H.make(rows, dim, vocab, dtype, seed=rows)
    ws = H.space(hidden, head, pieces)
    want = step(hidden, head, t, ON, ON, ws, 1, pieces=pieces)[0]
    for got in step(hidden, head, t, hidden_at, head_at, ws, 2, pieces=pieces):
        assert all(torch.equal(x, y) for x, y in zip(got, want))
