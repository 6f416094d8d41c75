"""Cross entropy against a head and its gradients, at the sizes where tiles, pieces and alignment end."""
import math

import pytest
import torch

import head_ref as R
from paper_2402_03770_b200 import binding as B

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def padded(x, pad, shift=0):
    rows, cols = x.shape
    room = torch.zeros(rows * (cols + pad) + shift + 16, dtype=x.dtype, device="cuda")
    at = room[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    return at.copy_(x)


def make(rows, dim, vocab, dtype=BF, pad=0, shift=0, seed=1, width=2.0, wide=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    head = padded((torch.randn(vocab, dim, generator=g, device="cuda") * (width / math.sqrt(dim))).to(dtype), pad, shift)
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    lean = torch.rand(rows, 1, generator=g, device="cuda") * 2
    hidden = padded((torch.randn(rows, dim, generator=g, device="cuda") + lean * head[t].float()).to(dtype), pad, shift)
    return hidden, head, t if wide else t.int()


def space(hidden, head, pieces):
    ws = B.alloc_bytes(B.cvlc_head_workspace_bytes(hidden, head, pieces), torch.device("cuda"))
    return ws.fill_(255)


def run(hidden, head, targets, scale=1.0, weight=None, pieces=1, pad=0, shift=0, status=None):
    rows, vocab = hidden.shape[0], head.shape[0]
    loss, alone = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    dh, dw = (padded(torch.full_like(x, 7.0), pad, shift) for x in (hidden, head))
    B.cvlc_head_loss(hidden, head, targets, alone, space(hidden, head, 0), scale=scale, row_weight=weight, status=status)
    B.cvlc_head_step(hidden, head, targets, loss, dh, dw, space(hidden, head, pieces), scale=scale, row_weight=weight, pieces=pieces, status=status)
    torch.cuda.synchronize()
    return alone, loss, dh, dw


def check(hidden, head, targets, scale=1.0, weight=None, **how):
    alone, loss, dh, dw = run(hidden, head, targets, scale, weight, **how)
    R.check(loss, dh, dw, hidden, head, targets, scale, weight, how.get("pieces", 1))
    R.check(alone, None, None, hidden, head, targets, scale, weight)
    return loss, dh, dw


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,dim,vocab", [(128, 64, 256), (1, 64, 256), (129, 64, 256), (128, 128, 256), (128, 64, 257), (300, 200, 1000)])
def test_first(dtype, rows, dim, vocab):
    check(*make(rows, dim, vocab, dtype))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows", [1, 2, 16, 127, 257])
@pytest.mark.parametrize("dim", [1, 8, 63, 65, 264])
@pytest.mark.parametrize("vocab", [1, 2, 10, 255, 513, 1003])
def test_sizes(dtype, rows, dim, vocab):
    check(*make(rows, dim, vocab, dtype, seed=rows + dim + vocab, wide=rows % 2 == 0))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim,pad,shift", [(64, 8, 0), (64, 0, 8), (64, 0, 1), (64, 3, 0), (65, 0, 0), (63, 1, 0), (200, 5, 3), (7, 1, 2)])
def test_strides(dtype, dim, pad, shift):
    check(*make(200, dim, 700, dtype, pad, shift), pad=pad, shift=shift)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("vocab", [300, 2000, 2304])
@pytest.mark.parametrize("pieces", [2, 3, 8, 1000])
def test_pieces(dtype, vocab, pieces):
    check(*make(150, 96, vocab, dtype), pieces=pieces)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,dim,vocab,pieces", [(4200, 96, 3000, 3), (4200, 65, 2817, 2), (17000, 72, 600, 1000), (128, 64, 70000, 2), (100, 72, 90001, 2)])
def test_pieces_of_many_logits(dtype, rows, dim, vocab, pieces):
    hidden, head, t = make(rows, dim, vocab, dtype, pad=8 * (rows % 3), seed=rows)
    few = B.cvlc_head_workspace_bytes(hidden, head, pieces)
    assert few < B.cvlc_head_workspace_bytes(hidden, head, 1)
    t[::9] = -1
    weight = torch.rand(rows, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    weight[1::7] = 0
    hidden[1] = float("nan")
    check(hidden, head, t, scale=1.2, weight=weight, pieces=pieces)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,pieces", [(333, 1), (333, 3), (120, 1), (4400, 2)])
def test_weights_masks_and_scale(dtype, rows, pieces):
    hidden, head, t = make(rows, 72, 1500, dtype)
    g = torch.Generator(device="cuda").manual_seed(5)
    weight = torch.rand(rows, generator=g, device="cuda") * 1e-3 - 2e-4
    weight[::7] = 0
    t[::5] = -1
    t[3] = -(1 << 40)
    hidden[0] = float("nan")   # weight 0
    hidden[5] = float("inf")   # no target
    loss, dh, dw = check(hidden, head, t, scale=0.7, weight=weight, pieces=pieces)
    assert not bool(dh[::7].any()) and not bool(dh[::5].any()) and not bool(loss[::5].any())


@pytest.mark.parametrize("dtype", [BF, HF])
def test_all_rows_count_for_nothing(dtype):
    hidden, head, t = make(40, 64, 300, dtype)
    alone, loss, dh, dw = run(hidden, head, torch.full_like(t, -1))
    assert not any(bool(x.any()) for x in (alone, loss, dh, dw))
    alone, loss, dh, dw = run(hidden, head, t, weight=torch.zeros(40, device="cuda"))
    assert not any(bool(x.any()) for x in (alone, loss, dh, dw))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,dim,pad,shift", [(200, 63, 1, 0), (100, 65, 7, 0), (300, 200, 8, 8), (40, 7, 4, 3), (130, 72, 24, 0)])
@pytest.mark.parametrize("pieces", [1, 2])
def test_what_lies_between_the_rows_stays(dtype, rows, dim, pad, shift, pieces):
    hidden, head, t = make(rows, dim, 700, dtype, pad, shift)
    room = [torch.full((x.shape[0] * (dim + pad) + shift + 64,), 7.0, dtype=dtype, device="cuda") for x in (hidden, head)]
    dh, dw = (r[shift:shift + x.shape[0] * (dim + pad)].view(-1, dim + pad)[:, :dim] for r, x in zip(room, (hidden, head)))
    loss = torch.full((rows + 8,), 7.0, device="cuda")
    B.cvlc_head_step(hidden, head, t, loss[:rows], dh, dw, space(hidden, head, pieces), pieces=pieces)
    R.check(loss[:rows], dh, dw, hidden, head, t, pieces=pieces)
    dh.fill_(7.0), dw.fill_(7.0)
    assert all(bool((r == 7.0).all()) for r in room) and bool((loss[rows:] == 7.0).all())


@pytest.mark.parametrize("pieces", [1, 2])
def test_gradients_beside_what_they_belong_to(pieces):
    """hidden states and their gradient in rows of one matrix, and so the head"""
    hidden, head, t = make(150, 64, 600)
    both = [torch.zeros(x.shape[0], 128, dtype=BF, device="cuda") for x in (hidden, head)]
    for b, x in zip(both, (hidden, head)):
        b[:, :64] = x
    loss = torch.zeros(150, device="cuda")
    B.cvlc_head_step(both[0][:, :64], both[1][:, :64], t, loss, both[0][:, 64:], both[1][:, 64:], space(both[0][:, :64], both[1][:, :64], pieces), pieces=pieces)
    R.check(loss, both[0][:, 64:], both[1][:, 64:], hidden, head, t, pieces=pieces)
    assert torch.equal(both[0][:, :64], hidden) and torch.equal(both[1][:, :64], head)


def test_no_rows():
    hidden, head, t = make(4, 64, 300)
    dw = torch.ones(300, 72, dtype=BF, device="cuda")
    ws = B.alloc_bytes(256, torch.device("cuda"))
    B.cvlc_head_step(hidden[:0], head, t[:0], torch.zeros(0, device="cuda"), hidden[:0].clone(), dw[:, :64], ws)
    assert not bool(dw[:, :64].any()) and bool((dw[:, 64:] == 1).all())


@pytest.mark.parametrize("rows", [0, 1, 3])
@pytest.mark.parametrize("stride", [(1 << 30) - 8, (1 << 30) + 8, (1 << 30) + 3])
def test_rows_far_apart(rows, stride):
    """strides in bytes beyond 31 bits, and offsets of rows beyond 32"""
    hidden, head, t = make(rows, 40, 3)
    h, w, dh, dw = (torch.empty((len(x) - 1) * stride + 40 if len(x) else 0, dtype=BF, device="cuda").as_strided(x.shape, (stride, 1)) for x in (hidden, head) * 2)
    h.copy_(hidden), w.copy_(head), dh.fill_(7.0), dw.fill_(7.0)
    loss = torch.zeros(rows, device="cuda")
    B.cvlc_head_step(h, w, t, loss, dh, dw, space(h, w, 1))
    if rows:
        R.check(loss, dh, dw, hidden, head, t)
    else:
        assert not bool(dw.any())


@pytest.mark.parametrize("dtype", [BF, HF])
def test_more_logits_than_32_bits_count(dtype):
    """the exponentials' offsets pass 2^32; the oracle goes over them in rows of 2048"""
    hidden, head, t = make(16500, 24, 260500, dtype)
    assert hidden.shape[0] * head.shape[0] > 1 << 32
    loss, dh, dw = torch.empty(16500, device="cuda"), torch.empty_like(hidden), torch.empty_like(head)
    B.cvlc_head_step(hidden, head, t, loss, dh, dw, space(hidden, head, 1))
    w, total, size = head.double(), torch.zeros(head.shape, dtype=torch.float64, device="cuda"), torch.zeros(head.shape, dtype=torch.float64, device="cuda")
    u = torch.finfo(dtype).eps / 2
    for i in range(0, 16500, 2048):
        h, at = hidden[i:i + 2048].double(), t[i:i + 2048, None]
        G = h @ w.T
        far = R.sums(24, h.norm(dim=1).amax() * w.norm(dim=1).amax()) + 6 * R.U * G.abs().amax() + R.LN
        lse = torch.logsumexp(G, dim=1)
        want = lse - G.gather(1, at)[:, 0]
        R.assert_near(loss[i:i + 2048], want, 2 * far + want.abs() * 8 * R.U, "loss")
        G = G.sub_(lse[:, None]).exp_()
        least = 2.0 ** -25 * G.amax(dim=1, keepdim=True) + 2.0 ** -38 if dtype == HF else 0.0  # half steps of what is kept, and of G times 2^15
        G.scatter_add_(1, at, torch.full_like(want, -1.0)[:, None])
        total.addmm_(G.T, h)
        want, G = G @ w, G.abs_()
        # G is rounded twice, and in bf16 the hidden states for the head's gradient; its exponent and the sums (of 260500, 16 at a time)
        each = G.mul_(2.1 * u + 4 * float(far)).add_(least)
        R.assert_near(dh[i:i + 2048], want, each @ w.abs() + R.sums(260500, each @ w.abs() / (2 * u)) + want.abs() * u + 2.0 ** -25, "d_hidden")
        size.addmm_(each.T, h.abs())
    R.assert_near(dw, total, size + R.sums(16500, size / (2 * u)) + total.abs() * u + 2.0 ** -25, "d_head")


@pytest.mark.parametrize("pieces", [1, 2])
def test_words_that_are_not_there_are_reported(pieces):
    hidden, head, t = make(200, 64, 600)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    check(hidden, head, t, pieces=pieces, status=status)
    assert status.item() == 0
    t[7], t[100] = 600, 1 << 33
    check(hidden, head, t, pieces=pieces, status=status)
    assert status.item() == B.CVLC_ERR_INVALID_ARG


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("pieces", [1, 2])
@pytest.mark.parametrize("rows", [256, 128, 12000])
def test_far_logits(dtype, rows, pieces):
    """rows whose target is far below or above all others: losses of hundreds, and of next to nothing"""
    hidden, head, t = make(rows, 64, 800, dtype, width=8.0)
    hidden[:32] = (-20 * head[t[:32]].float()).to(dtype)
    hidden[64:128] = (3 * head[t[64:128]].float()).to(dtype)
    hidden[32:64] *= 12
    loss, _, _ = check(hidden, head, t, pieces=pieces)
    assert float(loss.max()) > 500 and 0 < float(loss[64:128].max()) and float(loss.min()) < 1e-30


@pytest.mark.parametrize("rows", [3, 128, 129, 700])
def test_rows_far_above_their_target(rows):
    """some word 2^60 times and more as likely as the target, in single rows, next to others of the same tiles and of others"""
    hidden, head, t = make(rows, 64, 800, width=8.0)
    weight = torch.rand(rows, generator=torch.Generator(device="cuda").manual_seed(48), device="cuda")
    for i in {0, rows // 2, rows - 1}:
        hidden[i] = (-25 * head[t[i]].float()).to(BF)
    loss, _, _ = check(hidden, head, t, scale=0.9, weight=weight)
    assert int((loss > 60 * weight).sum()) >= 1
    t[0] = -1
    check(hidden, head, t, scale=0.9, weight=weight)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("scale", [0.0, -1.5])
def test_any_scale(dtype, scale):
    check(*make(200, 64, 700, dtype), scale=scale)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows", [140, 100])
def test_not_finite(dtype, rows):
    hidden, head, t = make(rows, 64, 500, dtype)
    good = [x.clone() for x in run(hidden, head, t)]
    hidden[3, 5] = float("nan")
    alone, loss, dh, dw = run(hidden, head, t)
    others = torch.arange(rows, device="cuda") != 3
    assert bool(torch.isnan(loss[3])) and bool(torch.isnan(alone[3])) and bool(torch.isnan(dh[3]).all()) and bool(torch.isnan(dw).all(dim=1).all())
    assert torch.equal(loss[others], good[1][others]) and torch.equal(dh[others], good[2][others])


def test_same_bits_again_and_streams():
    a, b = make(300, 128, 3000, seed=1), make(200, 128, 2000, seed=2)
    first, second = run(*a), run(*b)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for (h, w, t), st in zip((a, b), streams):
        o = [torch.zeros(h.shape[0], device="cuda"), torch.zeros_like(h), torch.zeros_like(w), space(h, w, 1)]
        outs.append(o)
    torch.cuda.synchronize()
    for _ in range(5):
        for (h, w, t), st, o in zip((a, b), streams, outs):
            B.cvlc_head_step(h, w, t, o[0], o[1], o[2], o[3], stream=st)
    torch.cuda.synchronize()
    for o, x in zip(outs, (first, second)):
        assert all(torch.equal(p, q) for p, q in zip(o[:3], x[1:]))


def test_graph():
    hidden, head, t = make(130, 64, 900)
    loss, dh, dw, ws = torch.zeros(130, device="cuda"), torch.zeros_like(hidden), torch.zeros_like(head), space(hidden, head, 2)
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        B.cvlc_head_step(hidden, head, t, loss, dh, dw, ws, pieces=2, stream=stream)
    for seed in (3, 4):
        for x, y in zip((hidden, head, t), make(130, 64, 900, seed=seed)):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        want = run(hidden, head, t, pieces=2)
        assert torch.equal(loss, want[1]) and torch.equal(dh, want[2]) and torch.equal(dw, want[3])


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,dim,vocab,pieces", [(1000, 512, 20000, 1), (2500, 384, 9000, 3), (5, 1024, 50021, 1), (4097, 64, 1000, 1), (20000, 72, 130, 1)])
def test_larger(dtype, rows, dim, vocab, pieces):
    check(*make(rows, dim, vocab, dtype, seed=rows), pieces=pieces)


def test_gradients_by_differences():
    """the loss's own change along a straight way is the gradient's product with it: by the trapezium rule, of the gradients at both ends (the two ends
    are rounded to the type, so that the point they were made from is not halfway between them)"""
    hidden, head, t = make(64, 64, 400)
    weight = torch.rand(64, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(9)
    for x, at in ((hidden, 2), (head, 3)):
        way = torch.randn(x.shape, generator=g, device="cuda") * 2.0 ** -4
        up, down = (x.float() + way).to(BF), (x.float() - way).to(BF)
        moved = (up.double() - down.double())
        a = run(*((up, head) if x is hidden else (hidden, up)), t, scale=1.3, weight=weight)
        b = run(*((down, head) if x is hidden else (hidden, down)), t, scale=1.3, weight=weight)
        terms = moved * (a[at].double() + b[at].double()) / 2
        predicted = float(terms.sum())
        # what the rule leaves out (a twelfth of the third derivative, times the cube of the way) by the definition in 64 bits; the rest is the
        # gradients' rounding: 2^-8 of each of the terms
        e, f = (R.step(*((y, head) if x is hidden else (hidden, y)), t, 1.3, weight)[0] for y in (up, down))
        name = "d_hidden" if x is hidden else "d_head"
        left_out = float((e["loss"] - f["loss"]).sum() - (moved * (e[name] + f[name]) / 2).sum())
        assert abs(float(a[1].double().sum() - b[1].double().sum()) - predicted - left_out) <= 2.0 ** -8 * float(terms.norm()) * 3


# ---- more than 8192 words: the logits are not held, whatever their number ----

@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows", [1, 2, 16, 127, 129, 257])
@pytest.mark.parametrize("dim,vocab,pad,shift", [(1, 8193, 0, 0), (8, 8448, 8, 0), (63, 8449, 1, 0), (65, 8703, 0, 3), (264, 9003, 0, 8), (200, 8200, 5, 3)])
def test_many_words(dtype, rows, dim, vocab, pad, shift):
    check(*make(rows, dim, vocab, dtype, pad, shift, wide=rows % 2 == 0), pad=pad, shift=shift)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows", [120, 333])
def test_many_words_weights_masks_and_scale(dtype, rows):
    hidden, head, t = make(rows, 96, 8300, dtype, pad=8)
    g = torch.Generator(device="cuda").manual_seed(7)
    weight = torch.rand(rows, generator=g, device="cuda") * 1e-3 - 2e-4
    weight[::7] = 0
    t[::5] = -1
    hidden[0], hidden[5] = float("nan"), float("inf")
    loss, dh, _ = check(hidden, head, t, scale=0.7, weight=weight)
    assert not bool(loss[::7].any()) and not bool(dh[::5].any())
    loss, dh, _ = check(hidden, head, t, scale=-0.7, weight=weight)
    weight[:] = 0
    _, loss, dh, dw = run(hidden, head, t, weight=weight)
    assert not any(bool(x.any()) for x in (loss, dh, dw))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows", [3, 128, 129, 700])
def test_many_words_far_logits(dtype, rows):
    """some word 2^60 times and more as likely as the target, in single rows, next to others of the same tiles and of others"""
    hidden, head, t = make(rows, 64, 8200, dtype, width=8.0)
    weight = torch.rand(rows, generator=torch.Generator(device="cuda").manual_seed(48), device="cuda")
    for i in {0, rows // 2, rows - 1}:
        hidden[i] = (-25 * head[t[i]].float()).to(dtype)
    hidden[1] = (3 * head[t[1]].float()).to(dtype)
    loss, _, _ = check(hidden, head, t, scale=0.9, weight=weight)
    assert int((loss > 60 * weight).sum()) >= 1
    t[0] = -1
    check(hidden, head, t, scale=0.9, weight=weight)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows", [140, 100])
def test_many_words_not_finite(dtype, rows):
    hidden, head, t = make(rows, 64, 8300, dtype)
    good = [x.clone() for x in run(hidden, head, t)]
    hidden[3, 5] = float("nan")
    alone, loss, dh, dw = run(hidden, head, t)
    others = torch.arange(rows, device="cuda") != 3
    assert bool(torch.isnan(loss[3])) and bool(torch.isnan(alone[3])) and bool(torch.isnan(dh[3]).all()) and bool(torch.isnan(dw).all(dim=1).all())
    assert torch.equal(loss[others], good[1][others]) and torch.equal(dh[others], good[2][others])


@pytest.mark.parametrize("rows", [100, 200])
def test_many_words_in_a_graph(rows):
    hidden, head, t = make(rows, 64, 8300)
    loss, dh, dw, ws = torch.zeros(rows, device="cuda"), torch.zeros_like(hidden), torch.zeros_like(head), space(hidden, head, 1)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        B.cvlc_head_step(hidden, head, t, loss, dh, dw, ws, stream=stream)
    for seed in (3, 4):
        for x, y in zip((hidden, head, t), make(rows, 64, 8300, seed=seed)):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        want = run(hidden, head, t)
        assert torch.equal(loss, want[1]) and torch.equal(dh, want[2]) and torch.equal(dw, want[3])


# ---- few logits: where warps, blocks, parts of sums and what is held end ----

@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,dim,vocab", [(1, 5000, 3), (7, 4096, 32), (129, 2049, 33), (40, 640, 127), (9, 72, 1023), (9, 72, 1024), (9, 72, 1025), (3, 640, 2049),
                                            (500, 64, 8191), (512, 64, 8192), (513, 64, 8192), (127, 64, 8193), (4096, 72, 1024), (4097, 72, 1024), (1024, 64, 1024),
                                            (1025, 64, 1024), (30000, 24, 10), (65000, 16, 64), (2000, 2048, 70), (700, 1000, 1000)])
def test_few_logits(dtype, rows, dim, vocab):
    check(*make(rows, dim, vocab, dtype, seed=rows))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,dim,vocab", [(5000, 40, 12), (300, 88, 2000)])
def test_few_logits_weights_masks_and_strides(dtype, rows, dim, vocab):
    hidden, head, t = make(rows, dim, vocab, dtype, pad=11, shift=3)
    weight = torch.rand(rows, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda") * 8 - 2
    weight[::6], t[::5] = 0, -7
    hidden[0], hidden[6] = float("nan"), float("-inf")
    loss, dh, _ = check(hidden, head, t, scale=1.3, weight=weight, pad=11, shift=3)
    assert not bool(loss[::5].any()) and not bool(dh[::6].any())


@pytest.mark.parametrize("rows,dim,vocab,pad", [(5000, 41, 12, 7), (5000, 40, 12, 8), (60, 33, 700, 1)])
def test_few_logits_leave_what_lies_between_the_rows(rows, dim, vocab, pad):
    hidden, head, t = make(rows, dim, vocab, pad=pad)
    room = [torch.full((x.shape[0], dim + pad), 7.0, dtype=BF, device="cuda") for x in (hidden, head)]
    loss = torch.full((rows + 8,), 7.0, device="cuda")
    B.cvlc_head_step(hidden, head, t, loss[:rows], room[0][:, :dim], room[1][:, :dim], space(hidden, head, 1))
    R.check(loss[:rows], room[0][:, :dim], room[1][:, :dim], hidden, head, t)
    assert all(bool((r[:, dim:] == 7.0).all()) for r in room) and bool((loss[rows:] == 7.0).all())


@pytest.mark.parametrize("dtype", [BF, HF])
def test_few_logits_ignored_rows_of_any_weight(dtype):
    hidden, head, t = make(50, 64, 40, dtype)
    weight = torch.ones(50, device="cuda")
    weight[::5], t[::5] = float("nan"), -1
    _, loss, dh, dw = run(hidden, head, t, weight=weight)
    live = torch.arange(50, device="cuda") % 5 != 0
    assert not bool(loss[~live].any()) and not bool(dh[~live].any())
    weight[::5] = 0
    R.check(loss, dh, dw, hidden, head, t, 1.0, weight)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("pieces", [1, 2])
def test_many_rows_in_graphs_of_two_streams(dtype, pieces):
    """two captured steps of sizes of their own, replayed at once, again and again with other inputs"""
    sizes = ((4200, 64, 2100), (2300, 72, 4000))
    cases = [[*make(*n, dtype, seed=1)] for n in sizes]
    outs = [(torch.zeros(h.shape[0], device="cuda"), torch.zeros_like(h), torch.zeros_like(w), space(h, w, pieces)) for h, w, _ in cases]
    graphs, streams = [], [torch.cuda.Stream() for _ in sizes]
    for (h, w, t), (loss, dh, dw, ws), stream in zip(cases, outs, streams):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            B.cvlc_head_step(h, w, t, loss, dh, dw, ws, pieces=pieces, stream=stream)
    for seed in (3, 4):
        for case, n in zip(cases, sizes):
            for x, y in zip(case, make(*n, dtype, seed=seed)):
                x.copy_(y)
        torch.cuda.synchronize()
        for _ in range(3):
            for graph, stream in zip(graphs, streams):
                with torch.cuda.stream(stream):
                    graph.replay()
        torch.cuda.synchronize()
        for (h, w, t), out in zip(cases, outs):
            want = run(h, w, t, pieces=pieces)
            assert all(torch.equal(x, y) for x, y in zip(out[:3], want[1:]))
