"""Rows of logits at the ends of what the definitions allow: lists of any mass, temperatures, values and sizes far apart."""
import math

import pytest
import torch

import vocab_ref as R
from test_gpu_vocab_rows import binding, check_top, logits_of, records, rows_of

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
FORMS = [(4, 6001), (160, 36007)]  # rows cut over a cluster; more long rows than blocks, which go from row to row


def moved_to_one(ids, lp, vocab):
    """log-probabilities less their row's largest: SCALED stays what it is"""
    there = (ids >= 0) & (ids < vocab)
    top = torch.where(there, lp.double(), -math.inf).amax(1, keepdim=True)
    return torch.where(there, lp.double() - torch.where(top > -math.inf, top, 0.0), -math.inf)


def check(B, z, ids, lp, rest, tau, weight, want):
    """the loss, the gradient behind it and both in one call against loss, gradient and what each may be off by"""
    loss64, grad64, tol, tol_g = want
    loss64, grad64 = loss64.float().double(), grad64.float().double()  # what is beyond fp32's range is infinite
    # an exponential below 2^-126 is 0, and the gradient is that times up to twice |weight| / temperature (the student's share and the bucket's)
    # the bucket's share is one less a sum whose terms have relative errors of 2^-36 (their definition in 64 bits has 2^-53): what is left of
    # a list that holds nearly everything is off by that much of one
    per = (1.0 if weight is None else weight.double().abs()[:, None]) / tau
    tol_g = tol_g + (2 * 2.0 ** -126 + (2.0 ** -36 if rest == R.BUCKET else 0.0)) * per
    rows, vocab = z.shape
    how = dict(rest=rest, temperature=tau, row_weight=weight)
    loss, stats = torch.full((rows,), 5.0, device="cuda"), torch.zeros(rows, B.DISTILL_STATS, device="cuda")
    B.cvlc_distill_loss(z, ids, lp, loss, stats, **how)
    R.assert_near(loss, loss64, tol, what="loss")
    g, _ = rows_of(torch.zeros(rows, vocab), z.dtype, pad=3, lead=2)
    B.cvlc_distill_grad(z, ids, lp, stats, g, **how)
    R.assert_near(g, grad64, tol_g, z.dtype, "grad")
    loss.fill_(5.0)
    h = torch.zeros_like(z)
    B.cvlc_distill_step(z, ids, lp, loss, h, **how)
    R.assert_near(loss, loss64, tol, what="step loss")
    R.assert_near(h, grad64, tol_g, z.dtype, "step grad")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", FORMS)
@pytest.mark.parametrize("kind", ["top", "twice", "absent"])
@pytest.mark.parametrize("by", [-88.0, -95.0, -110.0, -300.0, -800.0, -1e5, 90.0, 900.0])
def test_scaled_lists_of_any_mass(dtype, rows, vocab, kind, by):
    """p / P does not change when a list's weight does, whatever a number holds of p and P"""
    B = binding()
    z, _ = logits_of(rows, vocab, dtype, seed=vocab, pad=1, lead=1)
    ids, lp = records(z, 30, 1.5, seed=7, kind=kind)
    lp += by
    weight = torch.ones(rows, device="cuda")
    weight[2] = 0.0
    check(B, z, ids, lp, R.SCALED, 1.5, weight, R.distill(z, ids, moved_to_one(ids, lp, vocab), R.SCALED, 1.5, weight))


@pytest.mark.parametrize("rows,vocab", FORMS)
def test_scaled_lists_with_a_word_outside(rows, vocab):
    """what is left out has no part in the list's mass"""
    B = binding()
    z, _ = logits_of(rows, vocab, torch.float32, seed=3)
    ids, lp = records(z, 20, 1.0, seed=7)
    lp -= 400.0
    ids[1, 0], lp[1, 0] = vocab, 0.0
    ids[2, 3], lp[2, 3] = -1, 50.0
    lp[3] = -math.inf  # no mass: nothing
    want = R.distill(z, ids, moved_to_one(ids, lp, vocab), R.SCALED, 1.0)
    assert want[0][3] == 0 and (want[1][3] == 0).all()
    check(B, z, ids, lp, R.SCALED, 1.0, None, want)


@pytest.mark.parametrize("rest", [R.NONE, R.SCALED, R.BUCKET])
@pytest.mark.parametrize("rows,vocab", FORMS)
def test_rare_words_far_from_the_student(rest, rows, vocab):
    """a probability below fp32's smallest number counts where the word's logit is as far away"""
    B = binding()
    tau = 1e-6
    z, _ = logits_of(rows, vocab, torch.float32, seed=3)
    z.div_(1e7)
    ids = torch.arange(1, 9, dtype=torch.int32, device="cuda").repeat(rows, 1) * 37
    lp = torch.tensor([-1.0, -2.0, -2.5, -90.0, -100.0, -106.0, -110.0, -110.5], device="cuda").repeat(rows, 1)
    for i in (3, 4, 5, 6, 7):
        z[i % rows, int(ids[0, i])] = torch.finfo(torch.float32).min
    weight = torch.full((rows,), tau, device="cuda")
    check(B, z, ids, lp, rest, tau, weight, R.distill(z, ids, lp, rest, tau, weight))


@pytest.mark.parametrize("rest", [R.NONE, R.SCALED, R.BUCKET])
@pytest.mark.parametrize("rows,vocab", FORMS)
def test_a_masked_word_listed_at_any_probability(rest, rows, vocab):
    """its loss is infinite as long as its log-probability is a number"""
    B = binding()
    z, _ = logits_of(rows, vocab, torch.float32, seed=3)
    ids, lp = records(z, 20, 1.0, seed=1)
    z.scatter_(1, ids[:, 5:6].long(), -math.inf)
    lp[0, 5], lp[1, 5], lp[2, 5], lp[3, 5] = -601.0, -740.0, -1e30, -math.inf
    loss, g = torch.zeros(rows, device="cuda"), torch.zeros_like(z)
    for call in (lambda: B.cvlc_distill_loss(z, ids, lp, loss, rest=rest), lambda: B.cvlc_distill_step(z, ids, lp, loss, g, rest=rest)):
        loss.zero_()
        call()
        assert (loss[:3] == math.inf).all() and (loss[4:] == math.inf).all() and torch.isfinite(loss[3])
    assert torch.isfinite(g).all()


@pytest.mark.parametrize("rows,vocab,dtype", [(80, 1 << 22, torch.float32), (39, 1 << 22, torch.float32), (39, (1 << 22) - 5, torch.bfloat16),
                                              (160, 100_003, torch.float32)])
def test_sums_of_many_equal_terms(rows, vocab, dtype):
    """all logits of a row but the first ones, of which every thread has some, are the same, so that additions round alike.  A term's exponent v log2(e) is off by three roundings, twice
    where sums of two maxima meet (6 |v| U), each power of two by 4 U and a product, and the sum by one for every addition that a term goes
    through: at most 16 of a batch or stage, 32 of the stages that are summed together, 32 of those sums, 5 + 5 of warps and 3 of blocks.
    The logarithm and its difference from the logit are rounded last."""
    B = binding()
    v = -0.25 * (torch.arange(rows, device="cuda") % 39 + 1)
    z = v[:, None].to(dtype).expand(rows, vocab).contiguous()
    first = min(32768, vocab // 4)
    z[:, :first] = 0.0
    ids, logp = torch.ones(rows, 1, dtype=torch.int32, device="cuda"), torch.zeros(rows, 1, device="cuda")
    B.cvlc_top_logits(z, ids, logp)
    assert (ids == 0).all()
    ln = torch.log(first + (vocab - first) * torch.exp(v.double()))
    tol = (6 * v.double().abs() + 10 + 93) * R.U
    R.assert_near(logp[:, 0], -ln, tol + 2 * R.U * ln)
    loss = torch.zeros(rows, device="cuda")
    B.cvlc_distill_loss(z, ids, torch.zeros_like(logp), loss, rest=R.NONE)
    R.assert_near(loss, ln, tol + 2 * R.U * ln)
    g = torch.zeros_like(z)
    B.cvlc_distill_step(z, ids, torch.zeros_like(logp), loss, g, rest=R.NONE)
    R.assert_near(loss, ln, tol + 2 * R.U * ln)


TEMPERATURES = [1e-6, 1e-3, 1e3, 1e6]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", FORMS)
@pytest.mark.parametrize("kind", ["normal", "lowest", "masked", "ties"])
@pytest.mark.parametrize("tau", TEMPERATURES)
def test_top_logits_at_the_ends_of_the_temperature(dtype, rows, vocab, kind, tau):
    B = binding()
    z, _ = logits_of(rows, vocab, dtype, seed=vocab, kind=kind, pad=1)
    check_top(B, z, 60, tau)


@pytest.mark.parametrize("rest", [R.NONE, R.SCALED, R.BUCKET])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", FORMS)
@pytest.mark.parametrize("kind,lists", [("normal", "top"), ("lowest", "top"), ("lowest", "any"), ("masked", "top"), ("normal", "twice")])
@pytest.mark.parametrize("tau", TEMPERATURES)
def test_distill_at_the_ends_of_the_temperature(rest, dtype, rows, vocab, kind, lists, tau):
    """with weights of the temperature, which keep the gradient in the type's range, and without"""
    B = binding()
    z, _ = logits_of(rows, vocab, dtype, seed=vocab, kind=kind, pad=1, lead=1)
    ids, lp = records(z, 40, tau, seed=3, kind=lists)
    seen = lp if rest != R.SCALED else moved_to_one(ids, lp, vocab)
    weight = torch.full((rows,), tau, device="cuda")
    check(B, z, ids, lp, rest, tau, weight, R.distill(z, ids, seen, rest, tau, weight))
    if dtype != torch.float16:
        check(B, z, ids, lp, rest, tau, None, R.distill(z, ids, seen, rest, tau))


@pytest.mark.parametrize("rows,vocab", FORMS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_top_logits_of_rows_wider_than_the_type(rows, vocab, dtype):
    """differences beyond the type's range, which a high temperature brings back"""
    B = binding()
    z, _ = logits_of(rows, vocab, dtype, seed=vocab)
    z[:, ::7] = torch.finfo(dtype).min
    z[:, 5] = torch.finfo(dtype).max
    z[:, 200:] = torch.finfo(dtype).min  # fewer than k others
    check_top(B, z, 256, 1e6)
    check_top(B, z, 256, 1.0)


@pytest.mark.parametrize("rows,vocab", FORMS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("gap,first", [(0, "logits"), (3, "logits"), (5, "grad")])
def test_gradient_between_the_rows_of_the_logits(rows, vocab, dtype, gap, first):
    B = binding()
    both = torch.full((rows, 2 * vocab + 2 * gap), 7.0, dtype=dtype, device="cuda")
    a, b = both[:, :vocab], both[:, vocab + gap:2 * vocab + gap]
    z, g = (a, b) if first == "logits" else (b, a)
    z.copy_(logits_of(rows, vocab, dtype, seed=vocab)[0])
    ids, lp = records(z, 30, 1.0, seed=7)
    copy = both.clone()  # logits that lie alike against 16 bytes, whose sums are grouped alike
    apart = copy[:, :vocab] if first == "logits" else copy[:, vocab + gap:2 * vocab + gap]
    want, want_g = torch.zeros(rows, device="cuda"), torch.zeros(rows, vocab, dtype=dtype, device="cuda")
    B.cvlc_distill_step(apart, ids, lp, want, want_g)
    loss, stats = torch.zeros(rows, device="cuda"), torch.zeros(rows, B.DISTILL_STATS, device="cuda")
    B.cvlc_distill_step(z, ids, lp, loss, g)
    assert torch.equal(loss, want) and torch.equal(g, want_g) and torch.equal(z, apart)
    g.zero_()
    B.cvlc_distill_loss(z, ids, lp, loss, stats)
    B.cvlc_distill_grad(z, ids, lp, stats, g)
    B.cvlc_distill_grad(apart, ids, lp, stats, want_g)
    assert torch.equal(g, want_g) and torch.equal(z, apart)
    assert (both[:, vocab:vocab + gap] == 7).all() and (both[:, 2 * vocab + gap:] == 7).all()


def test_one_row_in_the_logits_place_whatever_the_strides():
    B = binding()
    flat = torch.randn(4096, generator=torch.Generator().manual_seed(1)).cuda()
    z, g = flat.as_strided((1, 500), (2000, 1)), flat.as_strided((1, 500), (700, 1))
    ids, lp = records(z, 9, 1.0, seed=7)
    loss, want, want_g = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(1, 500, device="cuda")
    B.cvlc_distill_step(z, ids, lp, want, want_g)
    B.cvlc_distill_step(z, ids, lp, loss, g)
    assert torch.equal(loss, want) and torch.equal(g, want_g)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind,lead,pad,k", [("normal", 0, 0, 64), ("ties", 1, 1, 256), ("crowd", 3, 0, 100), ("masked", 0, 2, 7), ("front masked", 5, 1, 96)])
def test_top_logits_of_many_rows_of_many_stages(dtype, kind, lead, pad, k):
    """more than 32 stages a row, which are summed 32 at a time; with the front masked the list of what reaches the bound overflows"""
    B = binding()
    rows, vocab = 82, 140_003 if dtype == torch.float32 else 270_005
    z, _ = logits_of(rows, vocab, dtype, seed=k, kind="normal" if kind == "front masked" else kind, lead=lead, pad=pad)
    if kind == "front masked":
        z[:, :vocab // 4] = -math.inf
    if kind == "normal":
        z[3, 5], z[4, vocab - 1], z[5] = math.nan, math.inf, -math.inf
    check_top(B, z, k, 0.7)
