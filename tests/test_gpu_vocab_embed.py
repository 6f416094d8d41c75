"""The embedding's lookup and gradient on the GPU against their definitions in 64 bits, and a client's round with both ends."""
import math

import numpy as np
import pytest
import torch

import vocab_ref as R

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16, torch.float32]


def binding():
    from paper_2402_03770_b200 import binding as B
    B.cvlc_set_device(0)
    return B


def tokens_of(n, vocab, kind, wide, seed=0):
    g = torch.Generator().manual_seed(seed)
    if kind == "one":
        t = torch.full((n,), vocab - 1)
    elif kind == "padding":
        t = torch.full((n,), -1)
    elif kind == "zipf":
        t = torch.exp(torch.rand(n, generator=g) * math.log(vocab + 1)).long().sub(1).clamp(0, vocab - 1)
    elif kind == "few":
        t = torch.randint(0, min(3, vocab), (n,), generator=g)
    else:
        t = torch.randint(-1, vocab, (n,), generator=g)
    return t.to(torch.int64 if wide else torch.int32).cuda()


def matrix(rows, dim, dtype, seed, pad=0, lead=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((lead + rows * (dim + pad) + 4,), 3.0, dtype=dtype, device="cuda")
    m = flat[lead:lead + rows * (dim + pad)].view(rows, dim + pad)[:, :dim]
    m.copy_(torch.randn(rows, dim, generator=g, device="cuda"))
    return m, flat


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,dim,vocab", [(1, 1, 1), (1, 1024, 500), (5, 8, 3), (100, 33, 70), (33, 4096, 40), (1000, 130, 5000), (7, 9000, 11)])
@pytest.mark.parametrize("layout", [(0, 0), (1, 1), (8, 0)])
def test_embed(dtype, n, dim, vocab, layout):
    B = binding()
    pad, lead = layout
    table, _ = matrix(vocab, dim, dtype, 1, pad, lead)
    out, flat = matrix(n, dim, dtype, 2, pad, lead)
    for wide in (False, True):
        t = tokens_of(n, vocab, "any", wide, seed=n)
        before = flat.clone()
        out.zero_()
        B.cvlc_embed(table, t, out, scale=1.7)
        want = torch.where(t[:, None] >= 0, table[t.long().clamp(min=0)].double() * float(np.float32(1.7)), 0.0)
        # one product in 32 bits, then the rounding to the table's type
        R.assert_near(out, want.cpu(), want.abs().cpu() * R.U, dtype)
        gap = torch.ones_like(flat, dtype=torch.bool)
        gap[lead:lead + n * (dim + pad)].view(n, dim + pad)[:, :dim] = False
        assert torch.equal(flat[gap], before[gap])


def test_embed_reports_tokens_outside():
    B = binding()
    table, _ = matrix(10, 16, torch.float32, 1)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    t = torch.tensor([3, -5, 9], device="cuda")
    out = torch.ones(3, 16, device="cuda")
    B.cvlc_embed(table, t, out, status=status)
    assert int(status) == 0
    t[0] = 10
    B.cvlc_embed(table, t, out, status=status)
    assert int(status) == B.CVLC_ERR_INVALID_ARG
    assert (out[:2] == 0).all() and torch.equal(out[2], table[9])
    t[0] = 1 << 40
    B.cvlc_embed(table, t, out)
    assert (out[0] == 0).all()


def check_grad(B, t, g, vocab, scale, accumulate, pad=0, lead=0, status=0):
    n, dim = g.shape
    u, flat = matrix(vocab, dim, torch.float32, 3, pad, lead)
    before, flat_before = u.clone(), flat.clone()
    need = B.cvlc_embed_grad_workspace_bytes(n, dim, vocab)
    ws = torch.full((need + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    B.cvlc_embed_grad(t, g, u, ws[:need], scale=scale, accumulate=accumulate)
    assert B.cvlc_read_status(ws) == status
    assert (ws[need:] == 0xA5).all()
    want, tol = R.embed_grad(t, g, vocab, float(np.float32(scale)), before if accumulate else None)
    R.assert_near(u, want, tol)
    gap = torch.ones_like(flat, dtype=torch.bool)
    gap[lead:lead + vocab * (dim + pad)].view(vocab, dim + pad)[:, :dim] = False
    assert torch.equal(flat[gap], flat_before[gap])
    absent = torch.ones(vocab, dtype=torch.bool)
    tc = t.cpu().long()
    absent[tc[(tc >= 0) & (tc < vocab)]] = False
    assert torch.equal(u[absent.cuda()], before[absent.cuda()] if accumulate else torch.zeros_like(before[absent.cuda()]))
    # equal inputs, equal bits, whatever the workspace held
    first = u.clone()
    u.copy_(before)
    B.cvlc_embed_grad(t, g, u, ws[:need], scale=scale, accumulate=accumulate)
    assert torch.equal(u, first)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["any", "zipf", "one", "few", "padding"])
@pytest.mark.parametrize("n,dim,vocab", [(1, 1, 1), (2, 64, 9), (31, 3, 600), (100, 129, 50), (2048, 16, 513), (2049, 8, 100000), (5000, 40, 300)])
def test_embed_grad(accumulate, dtype, kind, n, dim, vocab):
    B = binding()
    g, _ = matrix(n, dim, dtype, n)
    check_grad(B, tokens_of(n, vocab, kind, n % 2 == 0, seed=n), g, vocab, 0.3, accumulate)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", [(1, 0), (0, 1), (8, 0), (3, 5)])
def test_embed_grad_of_rows_anywhere(dtype, layout):
    B = binding()
    pad, lead = layout
    g, _ = matrix(700, 72, dtype, 8, pad, lead)
    check_grad(B, tokens_of(700, 90, "zipf", False), g, 90, 1.0, True, pad, lead)
    check_grad(B, tokens_of(700, 90, "zipf", True), g, 90, -1.0, False, pad, lead)


@pytest.mark.parametrize("kind", ["zipf", "one", "any"])
def test_embed_grad_of_many_tokens(kind):
    B = binding()
    g, _ = matrix(150_001, 24, torch.bfloat16, 8)
    check_grad(B, tokens_of(150_001, 70_000, kind, True), g, 70_000, 1.0, True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["zipf", "few"])
@pytest.mark.parametrize("dim", [1, 8, 17, 32, 64, 200])
def test_embed_grad_of_many_short_rows(dim, kind, dtype):
    """several chunks in a block, the last of which has no position"""
    B = binding()
    for n, vocab in ((70_001, 5000), (33_000, 400)):
        g, _ = matrix(n, dim, dtype, 8)
        check_grad(B, tokens_of(n, vocab, kind, False), g, vocab, 1.0, kind == "few")


def test_embed_of_rows_far_apart():
    """rows behind 2^32 elements, by their strides"""
    B = binding()
    stride = (1 << 31) + 16
    flat = torch.empty(2 * stride + 1024, dtype=torch.bfloat16, device="cuda")
    table, out = flat.as_strided((3, 256), (stride, 1)), flat.as_strided((3, 200), (stride, 1), 512)
    table.copy_(torch.randn(3, 256, generator=torch.Generator().manual_seed(1)))
    t = torch.tensor([2, 0, 2], device="cuda")
    B.cvlc_embed(table[:, :200], t, out)
    assert torch.equal(out, table[t, :200])
    far = flat.as_strided((3, 256), (stride, 1), 768)
    far.copy_(table)
    got = torch.empty(3, 256, dtype=torch.bfloat16, device="cuda")
    B.cvlc_embed(far, t, got)
    assert torch.equal(got, table[t])
    check_grad(B, t, far, 3, 1.0, False)


def test_embed_grad_of_a_wide_row():
    B = binding()
    g, _ = matrix(40, 8192, torch.float16, 8)
    check_grad(B, tokens_of(40, 30, "zipf", True), g, 30, 1.0, False)


def test_embed_grad_of_a_large_vocabulary():
    """words of more than 27 bits: four digits; rows behind 2^32 elements"""
    B = binding()
    vocab, dim = 200_000_000, 24
    u = torch.zeros(vocab, dim, device="cuda")
    t = torch.tensor([5, vocab - 1, -1, 5, 178_956_971, vocab - 1], dtype=torch.int64, device="cuda")
    g, _ = matrix(6, dim, torch.float32, 8)
    ws = B.alloc_bytes(B.cvlc_embed_grad_workspace_bytes(6, dim, vocab), u.device)
    B.cvlc_embed_grad(t, g, u, ws, accumulate=True)
    assert torch.equal(u[5], g[0] + g[3]) and torch.equal(u[vocab - 1], g[1] + g[5]) and torch.equal(u[178_956_971], g[4])
    assert int((u != 0).any(1).sum()) == 3


def test_embed_grad_without_tokens():
    B = binding()
    u = torch.ones(10, 8, device="cuda")
    ws = B.alloc_bytes(B.cvlc_embed_grad_workspace_bytes(0, 8, 10), u.device)
    t, g = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, 8, device="cuda")
    B.cvlc_embed_grad(t, g, u, ws, accumulate=True)
    assert (u == 1).all()
    B.cvlc_embed_grad(t, g, u, ws)
    assert (u == 0).all()


def test_embed_grad_reports_tokens_outside():
    B = binding()
    for n in (50, 6000):
        t = tokens_of(n, 100, "any", True)
        t[n // 2] = 100
        t[n // 3] = 1 << 33
        g, _ = matrix(n, 16, torch.float32, 8)
        check_grad(B, t, g, 100, 1.0, True, status=B.CVLC_ERR_INVALID_ARG)


def test_embed_on_another_stream_and_in_a_graph():
    B = binding()
    table, _ = matrix(500, 64, torch.bfloat16, 1)
    t = tokens_of(3000, 500, "zipf", False)
    out, u = torch.zeros(3000, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(500, 64, device="cuda")
    ws = B.alloc_bytes(B.cvlc_embed_grad_workspace_bytes(3000, 64, 500), u.device)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    B.cvlc_embed(table, t, out, stream=side)
    B.cvlc_embed_grad(t, out, u, ws, stream=side)
    side.synchronize()
    want_out, want = out.clone(), u.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.cvlc_embed(table, t, out)
        B.cvlc_embed_grad(t, out, u, ws)
    out.zero_(), u.zero_()
    for _ in range(2):
        graph.replay()
    assert torch.equal(out, want_out) and torch.equal(u, want)


def test_a_clients_round_with_both_ends_of_the_vocabulary():
    """Teacher's answers, two local steps of a small language model, the update of its table (and of its output matrix) compressed, sent
    and applied: gradients against automatic differentiation in 64 bits, the table after the round against the decoded update."""
    B = binding()
    torch.manual_seed(3)
    vocab, dim, n, k, lr, tau = 1100, 32, 96, 12, 0.5, 2.0
    dev = torch.device("cuda:0")
    table, head = torch.randn(vocab, dim, device=dev) * 0.3, torch.randn(dim, vocab, device=dev) * 0.3
    d = 2 * vocab * dim
    update = torch.zeros(d, device=dev)
    of_table, of_head = update[:vocab * dim].view(vocab, dim), update[vocab * dim:].view(dim, vocab)
    answers = torch.randn(2, n, vocab, device=dev) * 2
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    ws = B.alloc_bytes(B.cvlc_embed_grad_workspace_bytes(n, dim, vocab), dev)
    ids, logp = torch.zeros(n, k, dtype=torch.int32, device=dev), torch.zeros(n, k, device=dev)
    loss, weight = torch.zeros(n, device=dev), torch.full((n,), tau * tau / n, device=dev)
    want_table, want_head = table.double(), head.double()
    for step in range(2):
        tokens = torch.randint(-1, vocab, (n,), device=dev)
        x = torch.zeros(n, dim, device=dev)
        now = table - of_table, head - of_head
        B.cvlc_embed(now[0], tokens, x, scale=math.sqrt(dim), status=status)
        z = x @ now[1]
        B.cvlc_top_logits(answers[step], ids, logp, temperature=tau)
        B.cvlc_distill_step(z, ids, logp, loss, z, temperature=tau, row_weight=weight, status=status)
        dx = z @ now[1].t()
        of_head.add_(x.t() @ z, alpha=lr)
        B.cvlc_embed_grad(tokens, dx, of_table, ws, scale=lr * math.sqrt(dim), accumulate=True)
        assert B.cvlc_read_status(ws) == 0 and int(status) == 0
        # the same step in 64 bits
        W, H = want_table.clone().requires_grad_(True), want_head.clone().requires_grad_(True)
        keep = (tokens >= 0)[:, None]
        rows = torch.where(keep, W[tokens.clamp(min=0)] * math.sqrt(dim), 0.0)
        lq = torch.log_softmax(rows @ H / tau, 1)
        p = logp.double().exp()
        named = torch.zeros(n, vocab, dtype=torch.bool, device=dev).scatter_(1, ids.long(), True)
        left = 1 - p.sum(1)
        want = (p * (p.log() - lq.gather(1, ids.long()))).sum(1) + left * (left.log() - lq.masked_fill(named, -math.inf).logsumexp(1))
        total = (want * weight.double()).sum()
        total.backward()
        # products of 32 terms in fp32 on both sides of the loss: 1e-5 of the largest value is 160 roundings
        assert (loss.double() - want.detach() * weight.double()).abs().max() < 1e-5 * float(want.detach().max() * weight[0])
        want_table, want_head = want_table - lr * W.grad, want_head - lr * H.grad
        assert ((table.double() - of_table.double()) - want_table).abs().max() < 1e-5 * want_table.abs().max()
        assert ((head.double() - of_head.double()) - want_head).abs().max() < 1e-5 * want_head.abs().max()
    untouched = (of_table == 0).all(1)
    assert 800 < int(untouched.sum()) < vocab
    # the update is what the codec takes
    p = B.make_params(d, 2 * d, seed=5)
    enc = B.ClientEncoder(p, dev)
    stream = enc.run(update)
    assert enc.status() == B.CVLC_OK
    agg = B.Aggregator(1, d, dev)
    agg.set_clients([stream], torch.ones(1))
    model, decoded = torch.cat([table.flatten(), head.flatten()]), torch.zeros(d, device=dev)
    before = model.clone()
    agg.apply(1, model, decoded)
    assert agg.status() == B.CVLC_OK
    assert torch.equal(model, before - decoded)
    import oracle as O
    po = O.make_params(d, 2 * d, seed=5)
    u = update.cpu().numpy()
    assert (stream.cpu().numpy() == O.encode(u, po, O.plan(u, po))).all()
