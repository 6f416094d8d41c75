"""Top logits and distillation on the GPU against their definitions in 64 bits."""
import math

import pytest
import torch

import vocab_ref as R

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16, torch.float32]


def binding():
    from paper_2402_03770_b200 import binding as B
    B.cvlc_set_device(0)
    return B


def rows_of(values, dtype, pad=0, lead=0, guard=7.0):
    """the values as rows with `pad` guarded elements behind each and `lead` before the first"""
    rows, vocab = values.shape
    flat = torch.full((lead + rows * (vocab + pad) + 8,), guard, dtype=dtype, device="cuda")
    m = flat[lead:lead + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    m.copy_(values)
    return m, flat


def logits_of(rows, vocab, dtype, seed, kind="normal", pad=0, lead=0):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(rows, vocab, generator=g) * 3
    if kind == "ties":
        z = (z * 2).round() / 2
    elif kind == "equal":
        z = torch.full((rows, vocab), 1.5)
    elif kind == "masked":
        z[torch.rand(rows, vocab, generator=g) < 0.6] = -math.inf
        z[0] = -math.inf
        z[-1, vocab // 2 + 1:] = -math.inf
    elif kind == "lowest":
        z[torch.rand(rows, vocab, generator=g) < 0.5] = torch.finfo(dtype).min
        z[0] = torch.finfo(dtype).min
    elif kind == "zeros":
        z = torch.where(torch.rand(rows, vocab, generator=g) < 0.5, 0.0, -0.0)
    elif kind == "far":
        z = z + 3.0e4 * (1 if dtype == torch.float16 else 1e3)
    elif kind == "crowd":  # many equal ones at the top, in few 16 bytes
        z = z.round().clamp(max=2)
        z[:, 100:100 + min(12000, vocab // 3)] = 5
    elif kind == "front":  # the large ones lie together
        z[:, :max(1, vocab // 50)] += 30
    return rows_of(z.to(dtype), dtype, pad, lead)


SHAPES = [(1, 1, 1), (3, 2, 2), (2, 7, 5), (4, 100, 10), (3, 1000, 256), (5, 4099, 64), (2, 33000, 100), (1, 70001, 256), (3, 131072, 50),
          (300, 2500, 20)]


def check_top(B, z, k, tau):
    ids = torch.full((z.shape[0] + 1, k), -7, dtype=torch.int32, device="cuda")
    logp = torch.full((z.shape[0] + 1, k), 99.0, device="cuda")
    B.cvlc_top_logits(z, ids[:-1], logp[:-1], temperature=tau)
    want_ids, want, tol = R.top(z, k, tau)
    assert (ids[-1] == -7).all() and (logp[-1] == 99).all()
    assert torch.equal(ids[:-1].cpu(), want_ids)
    R.assert_near(logp[:-1], want, tol)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab,k", SHAPES)
def test_top_logits(dtype, rows, vocab, k):
    B = binding()
    z, _ = logits_of(rows, vocab, dtype, seed=vocab)
    check_top(B, z, k, 1.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["ties", "equal", "masked", "lowest", "zeros", "far", "front"])
@pytest.mark.parametrize("rows,vocab,k", [(3, 5, 5), (3, 300, 40), (4, 9001, 256), (2, 40007, 64)])
def test_top_logits_of_odd_rows(dtype, kind, rows, vocab, k):
    B = binding()
    z, _ = logits_of(rows, vocab, dtype, seed=k, kind=kind)
    check_top(B, z, k, 0.5)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lead", [1, 3, 5])
@pytest.mark.parametrize("pad", [0, 1, 6])
def test_top_logits_of_rows_anywhere(dtype, lead, pad):
    B = binding()
    z, _ = logits_of(5, 3001, dtype, seed=lead, pad=pad, lead=lead)
    check_top(B, z, 33, 2.0)


@pytest.mark.parametrize("dtype", DTYPES)
def test_top_logits_spoiled_rows(dtype):
    B = binding()
    z, _ = logits_of(4, 5000, dtype, seed=1)
    z[0, 17] = math.nan
    z[1, 4999] = math.inf
    z[2] = math.nan
    check_top(B, z, 20, 1.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind,lead,pad,k", [("normal", 0, 0, 64), ("ties", 1, 1, 256), ("equal", 0, 3, 20), ("masked", 3, 0, 100), ("lowest", 0, 8, 256),
                                             ("zeros", 5, 0, 33), ("far", 0, 1, 1), ("front", 1, 0, 200), ("crowd", 1, 1, 256), ("crowd", 0, 0, 3)])
def test_top_logits_of_many_long_rows(dtype, kind, lead, pad, k):
    """more rows than blocks, each of several stages"""
    B = binding()
    z, _ = logits_of(610, 35000 // torch.finfo(dtype).bits * 16 + 7, dtype, seed=k, kind=kind, pad=pad, lead=lead)
    if kind == "normal":
        z[3, 5], z[4, 7], z[300] = math.nan, math.inf, -math.inf
    check_top(B, z, k, 0.7)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["normal", "equal"])
def test_top_logits_of_more_words_than_a_cluster_keeps(dtype, kind):
    B = binding()
    z, _ = logits_of(2, 300007, dtype, seed=3, kind=kind, lead=1, pad=1)
    check_top(B, z, 100, 1.0)


# ---- distillation -------------------------------------------------------------------------------

def records(z, k, tau, seed, kind="top"):
    """a teacher near the student, and its k records; `kind`: how they are laid out"""
    g = torch.Generator().manual_seed(seed)
    rows, vocab = z.shape
    t = torch.nan_to_num(z.double(), neginf=-40.0).clamp(-40, 40) + torch.randn(rows, vocab, generator=g).to(z.device)
    lp = torch.log_softmax(t / tau, 1)
    if kind == "any":  # words drawn with repetition
        ids = torch.randint(0, vocab, (rows, k), generator=g)
        lp = torch.log_softmax(torch.randn(rows, k, generator=g), 1)
    else:
        lp, ids = [r.cpu() for r in torch.topk(lp, k, dim=1)]
    if kind == "twice":  # two clients' lists
        ids = torch.cat([ids, ids.flip(1)], 1)
        lp = torch.cat([lp + math.log(0.25), lp.flip(1) + math.log(0.75)], 1)
    if kind == "absent":
        ids[torch.rand(rows, k, generator=g) < 0.4] = -1
        ids[0] = -1
    return ids.to(torch.int32).cuda(), lp.float().cuda()


def check_distill(B, z, flat, ids, lp, rest, tau, weight=None, in_place=True):
    rows, vocab = z.shape
    dtype = z.dtype
    want, want_g, tol, tol_g = R.distill(z, ids, lp, rest, tau, weight)
    how = dict(rest=rest, temperature=tau, row_weight=weight)
    loss, stats = torch.full((rows,), 5.0, device="cuda"), torch.zeros(rows, B.DISTILL_STATS, device="cuda")
    B.cvlc_distill_loss(z, ids, lp, loss, **how)
    R.assert_near(loss, want, tol, what="loss")
    again = torch.full((rows,), 5.0, device="cuda")
    B.cvlc_distill_loss(z, ids, lp, again, stats, **how)
    assert torch.equal(again.nan_to_num(), loss.nan_to_num())
    g, guard = rows_of(torch.zeros(rows, vocab), dtype, pad=3, lead=2)
    B.cvlc_distill_grad(z, ids, lp, stats, g, **how)
    R.assert_near(g, want_g, tol_g, dtype, "grad")
    h, _ = rows_of(torch.zeros(rows, vocab), dtype, pad=16 // z.element_size())
    B.cvlc_distill_step(z, ids, lp, again, h, **how)
    R.assert_near(again, want, tol, what="step loss")
    R.assert_near(h, want_g, tol_g, dtype, "step grad")
    outside = torch.ones_like(guard, dtype=torch.bool)
    outside[2:2 + rows * (vocab + 3)].view(rows, vocab + 3)[:, :vocab] = False
    assert (guard[outside] == 7).all(), "written outside the rows"
    if in_place:
        kept = flat.clone()
        z_copy = z.clone()
        z.fill_(7)
        beside = flat == 7
        z.copy_(z_copy)
        B.cvlc_distill_step(z, ids, lp, again, z, **how)
        assert torch.equal(z.nan_to_num(), h.nan_to_num())
        z.fill_(7)
        assert torch.equal(flat == 7, beside) and flat.shape == kept.shape
    return loss


@pytest.mark.parametrize("rest", [R.NONE, R.SCALED, R.BUCKET])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (3, 2, 1), (2, 7, 5), (4, 100, 10), (3, 1000, 200), (5, 4099, 64), (2, 33000, 100),
                                          (2, 70001, 256), (3, 131072, 50), (300, 700, 20)])
def test_distill(rest, dtype, rows, vocab, k):
    B = binding()
    z, flat = logits_of(rows, vocab, dtype, seed=vocab)
    ids, lp = records(z, k, 1.0, seed=k)
    check_distill(B, z, flat, ids, lp, rest, 1.0)


@pytest.mark.parametrize("rest", [R.NONE, R.SCALED, R.BUCKET])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["twice", "absent", "any"])
@pytest.mark.parametrize("vocab,k", [(50, 40), (6001, 100), (40007, 512)])
def test_distill_of_lists(rest, dtype, kind, vocab, k):
    B = binding()
    z, flat = logits_of(4, vocab, dtype, seed=vocab, pad=1, lead=1)
    ids, lp = records(z, k, 2.0, seed=k, kind=kind)
    weight = torch.tensor([1.0, 0.25, 0.0, -2.0], device="cuda")
    check_distill(B, z, flat, ids, lp, rest, 2.0, weight)


@pytest.mark.parametrize("rest", [R.NONE, R.SCALED, R.BUCKET])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["masked", "lowest", "equal", "far", "front"])
def test_distill_of_odd_rows(rest, dtype, kind):
    B = binding()
    z, flat = logits_of(4, 3001, dtype, seed=5, kind=kind, pad=2)
    ids, lp = records(z, 30, 0.5, seed=2)
    check_distill(B, z, flat, ids, lp, rest, 0.5)


@pytest.mark.parametrize("rest", [R.NONE, R.SCALED, R.BUCKET])
def test_distill_where_every_word_is_listed(rest):
    B = binding()
    for vocab in (1, 3, 40):
        z, flat = logits_of(3, vocab, torch.float32, seed=vocab)
        ids, lp = records(z, vocab, 1.0, seed=1)
        check_distill(B, z, flat, ids, lp, rest, 1.0)
    # ... and where those that are not listed are masked
    z, flat = logits_of(3, 100, torch.float32, seed=9)
    z[:, 20:] = -math.inf
    ids, lp = records(z, 20, 1.0, seed=1)
    check_distill(B, z, flat, ids, lp, rest, 1.0)


@pytest.mark.parametrize("rest", [R.NONE, R.SCALED, R.BUCKET])
def test_distill_without_records(rest):
    B = binding()
    z, flat = logits_of(3, 500, torch.bfloat16, seed=9)
    ids, lp = torch.zeros(3, 0, dtype=torch.int32, device="cuda"), torch.zeros(3, 0, device="cuda")
    check_distill(B, z, flat, ids, lp, rest, 1.0)


@pytest.mark.parametrize("rest", [R.NONE, R.SCALED, R.BUCKET])
def test_distill_of_a_sure_student(rest):
    """the unlisted words' share is far below what one minus a sum holds in 32 bits"""
    B = binding()
    z = torch.randn(3, 2000, generator=torch.Generator().manual_seed(0))
    z[:, 7] += torch.tensor([20.0, 60.0, 150.0])
    z, flat = rows_of(z, torch.float32)
    ids, lp = records(torch.zeros(3, 2000), 10, 1.0, seed=4)
    ids[:, 0] = 7
    ids[:, 1:] = torch.arange(20, 29, dtype=torch.int32, device="cuda")
    check_distill(B, z, flat, ids, lp, rest, 1.0)


def test_distill_masked_word_in_the_list():
    B = binding()
    z, flat = logits_of(2, 300, torch.float32, seed=9)
    ids, lp = records(z, 10, 1.0, seed=1)
    z[0, int(ids[0, 3])] = -math.inf
    for rest in (R.NONE, R.SCALED, R.BUCKET):
        loss = check_distill(B, z, flat, ids, lp, rest, 1.0, in_place=False)
        assert loss[0] == math.inf and torch.isfinite(loss[1])


@pytest.mark.parametrize("dtype", DTYPES)
def test_distill_spoiled_rows(dtype):
    """a NaN spoils its own row; without weight it spoils nothing"""
    B = binding()
    z, _ = logits_of(5, 3000, dtype, seed=2)
    clean = z.clone()
    z[1, 100] = math.nan
    z[2, 100] = math.inf
    z[3] = math.nan
    ids, lp = records(clean, 20, 1.0, seed=1)
    weight = torch.tensor([1.0, 1.0, 1.0, 0.0, 1.0], device="cuda")
    loss, g = torch.zeros(5, device="cuda"), torch.zeros_like(z)
    B.cvlc_distill_step(z, ids, lp, loss, g, row_weight=weight)
    ref, h = torch.zeros(5, device="cuda"), torch.zeros_like(z)
    B.cvlc_distill_step(clean, ids, lp, ref, h)
    assert torch.isnan(loss[1:3]).all() and torch.isnan(g[1]).all() and loss[3] == 0 and (g[3] == 0).all()
    for r in (0, 4):
        assert loss[r] == ref[r] and torch.equal(g[r], h[r])


def test_distill_reports_words_outside():
    B = binding()
    z, _ = logits_of(3, 1000, torch.bfloat16, seed=2)
    ids, lp = records(z, 20, 1.0, seed=1)
    loss, status = torch.zeros(3, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.cvlc_distill_loss(z, ids, lp, loss, status=status)
    assert int(status) == 0
    ids[1, 4] = 1000
    B.cvlc_distill_loss(z, ids, lp, loss, status=status)
    assert int(status) == B.CVLC_ERR_INVALID_ARG
    want, _, tol, _ = R.distill(z, ids, lp, R.BUCKET, 1.0)
    R.assert_near(loss, want, tol)
    B.cvlc_distill_loss(z, ids, lp, loss)


@pytest.mark.parametrize("rest", [R.NONE, R.SCALED, R.BUCKET])
def test_distill_of_more_words_than_a_cluster_keeps(rest):
    B = binding()
    for dtype in (torch.float32, torch.bfloat16):
        z, flat = logits_of(2, 300007, dtype, seed=3, lead=1, pad=1)
        ids, lp = records(z, 100, 1.0, seed=1, kind="twice")
        check_distill(B, z, flat, ids, lp, rest, 1.0)


@pytest.mark.parametrize("rows,vocab,dtype", [(300, 900_001, torch.bfloat16), (300, 530_000, torch.float32), (1, 1 << 22, torch.float32),
                                              (2, (1 << 22) - 3, torch.float16)])
def test_distill_of_the_longest_rows(rows, vocab, dtype):
    B = binding()
    g = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn(rows, vocab, generator=g, device="cuda").mul_(2).to(dtype)
    ids = torch.randint(0, vocab, (rows, 40), generator=g, device="cuda", dtype=torch.int32)
    lp = torch.log_softmax(torch.randn(rows, 41, generator=g, device="cuda"), 1)[:, :40].contiguous()
    check_distill(B, z, z.flatten(), ids, lp, R.BUCKET, 1.0, in_place=False)
    if rows < 3:
        check_top(B, z, 256, 1.0)


@pytest.mark.parametrize("rest", [R.NONE, R.SCALED, R.BUCKET])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind,lists,lead,pad", [("normal", "top", 0, 0), ("normal", "twice", 1, 1), ("masked", "absent", 3, 2), ("lowest", "any", 0, 8),
                                                 ("front", "twice", 5, 0), ("far", "top", 0, 3)])
def test_distill_of_many_long_rows(rest, dtype, kind, lists, lead, pad):
    """more rows than blocks, each of several stages; some without weight, in a row and apart"""
    B = binding()
    rows, vocab = 610, 35000 // torch.finfo(dtype).bits * 16 + 7
    z, flat = logits_of(rows, vocab, dtype, seed=vocab, kind=kind, pad=pad, lead=lead)
    ids, lp = records(z, 70, 1.5, seed=3, kind=lists)
    weight = torch.rand(rows, generator=torch.Generator().manual_seed(1))
    weight[torch.rand(rows, generator=torch.Generator().manual_seed(2)) < 0.2] = 0.0
    weight[297:305] = 0.0
    check_distill(B, z, flat, ids, lp, rest, 1.5, weight.cuda() if lists != "top" else None)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("k", [0, 1, 1024])
def test_distill_of_many_long_rows_records(dtype, k):
    B = binding()
    z, flat = logits_of(160, 40000, dtype, seed=k, lead=2)
    if k:
        ids, lp = records(z, k, 1.0, seed=3, kind="any")
        ids[5], ids[6, 1:] = 39999, ids[6, :1]
    else:
        ids, lp = torch.zeros(160, 0, dtype=torch.int32, device="cuda"), torch.zeros(160, 0, device="cuda")
    check_distill(B, z, flat, ids, lp, R.BUCKET, 1.0)


def test_distill_spoiled_among_many_long_rows():
    B = binding()
    z, _ = logits_of(310, 20000, torch.bfloat16, seed=2)
    clean = z.clone()
    z[1, 100] = math.nan
    z[297] = math.inf
    ids, lp = records(clean, 20, 1.0, seed=1)
    loss, g, ref, h = torch.zeros(310, device="cuda"), torch.zeros_like(z), torch.zeros(310, device="cuda"), torch.zeros_like(z)
    B.cvlc_distill_step(z, ids, lp, loss, g)
    B.cvlc_distill_step(clean, ids, lp, ref, h)
    assert torch.isnan(loss[[1, 297]]).all() and torch.isnan(g[[1, 297]]).all()
    keep = torch.ones(310, dtype=torch.bool)
    keep[[1, 297]] = False
    assert torch.equal(loss[keep.cuda()], ref[keep.cuda()]) and torch.equal(g[keep.cuda()], h[keep.cuda()])


@pytest.mark.parametrize("rest", [R.NONE, R.SCALED, R.BUCKET])
def test_distill_gradient_by_differences(rest):
    """the gradient against differences of the loss in 64 bits, by central differences of step h: off by h^2 / 6 times a third derivative
    below 2 (|w| / tau^3) and by twice the loss's rounding over 2 h"""
    B = binding()
    tau, h = 1.5, 1e-4
    z, _ = logits_of(2, 30, torch.float32, seed=2)
    ids, lp = records(z, 8, tau, seed=1, kind="any")
    loss, g = torch.zeros(2, device="cuda"), torch.zeros_like(z)
    B.cvlc_distill_step(z, ids, lp, loss, g, rest=rest, temperature=tau)
    z64 = z.double().cpu()
    num = torch.zeros_like(z64)
    for j in range(30):
        up, down = z64.clone(), z64.clone()
        up[:, j] += h
        down[:, j] -= h
        num[:, j] = (R.distill(up, ids, lp, rest, tau)[0] - R.distill(down, ids, lp, rest, tau)[0]) / (2 * h)
    assert (g.cpu().double() - num).abs().max() < 2 * h * h + 1e-14 / h + R.LN * 4


# ---- how they are called -------------------------------------------------------------------------

@pytest.mark.parametrize("rows,vocab", [(20, 9001), (310, 20001)])
def test_rows_on_another_stream_and_in_a_graph(rows, vocab):
    B = binding()
    z, _ = logits_of(rows, vocab, torch.bfloat16, seed=4)
    side = torch.cuda.Stream()
    ids, lp = torch.zeros(rows, 40, dtype=torch.int32, device="cuda"), torch.zeros(rows, 40, device="cuda")
    loss, g = torch.zeros(rows, device="cuda"), torch.zeros_like(z)
    torch.cuda.synchronize()
    B.cvlc_top_logits(z, ids, lp, stream=side)
    B.cvlc_distill_step(z, ids, lp, loss, g, stream=side)
    side.synchronize()
    want = [t.clone() for t in (ids, lp, loss, g)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.cvlc_top_logits(z, ids, lp)
        B.cvlc_distill_step(z, ids, lp, loss, g)
    for _ in range(2):
        for t in (ids, lp, loss, g):
            t.zero_()
        graph.replay()
        for t, w in zip((ids, lp, loss, g), want):
            assert torch.equal(t, w)
    other, _ = logits_of(rows, vocab, torch.bfloat16, seed=5)
    z.copy_(other)
    graph.replay()
    check_ids, _, _ = R.top(z, 40, 1.0)
    assert torch.equal(ids.cpu(), check_ids)


def test_two_calls_at_once():
    """two streams, each with rows for all SMs: equal bits to one after the other"""
    B = binding()
    zs = [logits_of(330, 20000, torch.bfloat16, seed=s)[0] for s in (1, 2)]
    recs = [records(z, 30, 1.0, seed=4) for z in zs]
    loss, g = [torch.zeros(330, device="cuda") for _ in zs], [torch.zeros_like(z) for z in zs]
    for i in (0, 1):
        B.cvlc_distill_step(zs[i], *recs[i], loss[i], g[i])
    want = [t.clone() for t in loss + g]
    streams = [torch.cuda.Stream() for _ in zs]
    torch.cuda.synchronize()
    for _ in range(5):
        for i in (0, 1):
            B.cvlc_distill_step(zs[i], *recs[i], loss[i], g[i], stream=streams[i])
    torch.cuda.synchronize()
    for t, w in zip(loss + g, want):
        assert torch.equal(t, w)


@pytest.mark.parametrize("rows,vocab", [(6, 3000), (310, 18000)])
def test_gradient_with_weights_of_its_own(rows, vocab):
    """what the loss keeps holds for every row, also for those that its own weights left out"""
    B = binding()
    z, _ = logits_of(rows, vocab, torch.float32, seed=8)
    ids, lp = records(z, 25, 1.0, seed=4)
    early = torch.zeros(rows, device="cuda")
    early[::2] = 1.0
    late = torch.rand(rows, generator=torch.Generator().manual_seed(2)).cuda()
    late[3] = 0.0
    loss, stats, g = torch.zeros(rows, device="cuda"), torch.zeros(rows, B.DISTILL_STATS, device="cuda"), torch.ones_like(z)
    B.cvlc_distill_loss(z, ids, lp, loss, stats, row_weight=early)
    assert (loss[1::2] == 0).all()
    B.cvlc_distill_grad(z, ids, lp, stats, g, row_weight=late)
    _, want, _, tol = R.distill(z, ids, lp, R.BUCKET, 1.0, late)
    R.assert_near(g, want, tol)


@pytest.mark.parametrize("rows,vocab,stride", [(3, 5003, (1 << 31) + 5), (3, 140001, (1 << 31) + 8), (160, 20001, 27_000_003)])
def test_rows_far_apart(rows, vocab, stride):
    """rows behind 2^32 elements, by their strides"""
    B = binding()
    flat = torch.empty((rows - 1) * stride + vocab + 8, dtype=torch.bfloat16, device="cuda")
    z = flat.as_strided((rows, vocab), (stride, 1), 3)
    z.copy_(torch.randn(rows, vocab, generator=torch.Generator().manual_seed(rows)) * 3)
    check_top(B, z, 40, 0.7)
    ids, lp = records(z, 40, 1.0, seed=2)
    want, want_g, tol, tol_g = R.distill(z, ids, lp, R.BUCKET, 1.0)
    loss, stats = torch.zeros(rows, device="cuda"), torch.zeros(rows, B.DISTILL_STATS, device="cuda")
    B.cvlc_distill_loss(z, ids, lp, loss, stats)
    R.assert_near(loss, want, tol)
    g = torch.zeros_like(z.contiguous())
    B.cvlc_distill_grad(z, ids, lp, stats, g)
    R.assert_near(g, want_g, tol_g, z.dtype)
    B.cvlc_distill_step(z, ids, lp, loss, z)  # in the logits' place
    R.assert_near(loss, want, tol)
    R.assert_near(z, want_g, tol_g, z.dtype)


def test_no_rows():
    B = binding()
    z, ids, lp = torch.zeros(0, 100, device="cuda"), torch.zeros(0, 5, dtype=torch.int32, device="cuda"), torch.zeros(0, 5, device="cuda")
    loss, stats, g = torch.zeros(0, device="cuda"), torch.zeros(0, B.DISTILL_STATS, device="cuda"), torch.zeros(0, 100, device="cuda")
    B.cvlc_top_logits(z, ids, lp)
    B.cvlc_distill_loss(z, ids, lp, loss, stats)
    B.cvlc_distill_grad(z, ids, lp, stats, g)
    B.cvlc_distill_step(z, ids, lp, loss, g)


def test_launches_are_counted():
    B = binding()
    z, _ = logits_of(2, 100, torch.float32, seed=4)
    ids, lp = torch.zeros(2, 4, dtype=torch.int32, device="cuda"), torch.zeros(2, 4, device="cuda")
    names = ["k_top_logits", "k_distill_loss", "k_distill_grad", "k_distill_step"]
    before = [B.cvlc_launch_count(n) for n in names]
    loss, stats, g = torch.zeros(2, device="cuda"), torch.zeros(2, B.DISTILL_STATS, device="cuda"), torch.zeros_like(z)
    B.cvlc_top_logits(z, ids, lp)
    B.cvlc_distill_loss(z, ids, lp, loss, stats)
    B.cvlc_distill_grad(z, ids, lp, stats, g)
    B.cvlc_distill_step(z, ids, lp, loss, g)
    assert [B.cvlc_launch_count(n) - b for n, b in zip(names, before)] == [1, 1, 1, 1]


def test_binding_refuses_what_it_cannot_pass_on():
    B = binding()
    z, _ = logits_of(2, 100, torch.float32, seed=4)
    ids, lp = torch.zeros(2, 4, dtype=torch.int32, device="cuda"), torch.zeros(2, 4, device="cuda")
    loss = torch.zeros(2, device="cuda")
    for bad in (lambda: B.cvlc_top_logits(z.t(), ids, lp), lambda: B.cvlc_top_logits(z, ids.long(), lp), lambda: B.cvlc_top_logits(z.cpu(), ids, lp),
                lambda: B.cvlc_distill_loss(z, ids, lp[:, :3], loss), lambda: B.cvlc_distill_loss(z, ids[:1], lp[:1], loss),
                lambda: B.cvlc_distill_step(z, ids, lp, loss, z.half())):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(B.CvlcError):
        B.cvlc_top_logits(z[:1].expand(2, 100), ids, lp)
