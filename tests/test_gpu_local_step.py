"""A client's local steps from tokens to the stream it sends, and the server's step with what it decodes: embedding, training loss and its gradients, their
norm, AdamW with states of 8 bits, the update, compression, aggregation, AdamW at the server.  Every link against its definition."""
import numpy as np
import pytest
import torch

import adamw_ref as A
import gpu_util as G
import head_ref as H
import vocab_ref as V
from paper_2402_03770_b200 import binding as B

pytestmark = pytest.mark.gpu
VOCAB, DIM, TOKENS = 503, 72, 300
HOW = dict(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8)


def f32(t):
    return t.detach().float().cpu().numpy()


class Client:
    """table and head as blocks of one vector, with 16-bit copies that the products read"""

    def __init__(self, w0, seed):
        self.seed = seed
        n = VOCAB * DIM
        self.w = w0.clone()
        self.table, self.head = (self.w[i * n:(i + 1) * n].view(VOCAB, DIM) for i in (0, 1))
        self.copies = [x.bfloat16() for x in (self.table, self.head)]
        self.d_table = torch.zeros(VOCAB, DIM, device="cuda")
        self.d_head = torch.zeros(VOCAB, DIM, dtype=torch.bfloat16, device="cuda")
        blocks = -(-n // B.STATE_BLOCK)
        self.states = [[torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2)] + [torch.zeros(blocks, 2, device="cuda")] for _ in range(2)]
        self.lists = [B.AdamwTensors([g], [p.view(-1)], [s[0]], [s[1]], [s[2]], [c], weight_decay=0.1) for g, p, s, c in
                      zip((self.d_table, self.d_head), (self.table, self.head), self.states, self.copies)]
        self.ws = B.alloc_bytes(B.cvlc_embed_grad_workspace_bytes(TOKENS, DIM, VOCAB), torch.device("cuda"))
        self.norm_ws = B.alloc_bytes(B.cvlc_grad_norm_workspace_bytes(self.lists[0]), torch.device("cuda"))
        self.norms = [torch.zeros(1, device="cuda") for _ in range(2)]
        self.hidden, self.d_hidden = (torch.zeros(TOKENS, DIM, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.loss = torch.zeros(TOKENS, device="cuda")
        self.weight = torch.full((TOKENS,), 1.0 / TOKENS, device="cuda")
        self.head_ws = B.alloc_bytes(B.cvlc_head_workspace_bytes(self.hidden, self.copies[1]), torch.device("cuda"))

    def step(self, tokens, targets, t):
        B.cvlc_embed(self.copies[0], tokens, self.hidden, scale=8.0)
        B.cvlc_head_step(self.hidden, self.copies[1], targets, self.loss, self.d_hidden, self.d_head, self.head_ws, row_weight=self.weight)
        B.cvlc_embed_grad(tokens, self.d_hidden, self.d_table, self.ws, scale=8.0)
        for x, n in zip(self.lists, self.norms):
            B.cvlc_grad_norm(x, n, self.norm_ws)
        norm = torch.hypot(*self.norms)
        for i, x in enumerate(self.lists):
            B.cvlc_adamw(x, step=t, norm=norm, max_norm=0.5, seed=self.seed + i, **HOW)
        return norm


def test_round():
    g = torch.Generator(device="cuda").manual_seed(11)
    d = 2 * VOCAB * DIM
    w0 = torch.randn(d, generator=g, device="cuda") * 0.1
    streams, scales = [], []
    params = []
    for c in range(2):
        client = Client(w0, 100 * c)
        for t in (1, 2, 3):
            tokens = torch.randint(0, VOCAB, (TOKENS,), generator=g, device="cuda")
            targets = torch.randint(-30, VOCAB, (TOKENS,), generator=g, device="cuda")
            table, head = (x.clone() for x in client.copies)
            before = [f32(x).reshape(-1).copy() for x in (client.table, client.head)]
            held = []
            for s in client.states:
                sc, of = f32(s[2]), np.arange(VOCAB * DIM) // B.STATE_BLOCK
                held.append((A.held(s[0].cpu().numpy(), torch.float8_e4m3fn) * sc[of, 0], A.held(s[1].cpu().numpy(), torch.float8_e5m2) * sc[of, 1]))
            norm = client.step(tokens, targets, t)
            torch.cuda.synchronize()
            # the embedding, the loss and its gradients
            assert torch.equal(client.hidden, (table.float() * 8.0).bfloat16()[tokens])
            H.check(client.loss, client.d_hidden, client.d_head, client.hidden, head, targets, 1.0, client.weight)
            want, tol = V.embed_grad(tokens, client.d_hidden, VOCAB, 8.0)
            V.assert_near(client.d_table.cpu(), want, tol)
            grads = [f32(x).reshape(-1) for x in (client.d_table, client.d_head)]
            size = np.sqrt(sum(float((x.astype(np.float64) ** 2).sum()) for x in grads))
            assert abs(norm.item() - size) <= size * 16 * A.U
            # the step
            clip = np.float32(1.0) if norm.item() <= 0.5 else np.float32(0.5) / np.float32(norm.item())
            for p, x, (m, v), grad, copy in zip((client.table, client.head), before, held, grads, client.copies):
                want, _, _, tol, _, _ = A.step64(x, grad, m, v, decay=0.1, step=t, scale=float(clip), **HOW)
                assert (np.abs(f32(p).reshape(-1) - want) <= tol).all()
                assert torch.equal(copy, p.bfloat16())
        # the update, compressed: the stream is the oracle's
        update = w0 - client.w
        pd = G.params_dict(d, 2 * d, seed=c, client_id=c)
        enc = B.ClientEncoder(G.gpu_params(pd), torch.device("cuda"))
        out = enc.run(update)
        assert enc.status() == B.CVLC_OK
        _, ref = G.oracle_plan_encode(f32(update), pd)
        assert np.array_equal(out.cpu().numpy(), ref)
        streams.append(out)
    # the server: the aggregate is the gradient
    agg = B.Aggregator(2, d, torch.device("cuda"))
    agg.set_clients(streams, torch.tensor([1.0, 3.0]))
    mean = torch.empty(d, device="cuda")
    agg.run(2, mean)
    assert agg.status() == B.CVLC_OK and bool((mean != 0).any())
    model, m, v = w0.clone(), torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
    B.cvlc_adamw(B.AdamwTensors([mean], [model], [m], [v]), lr=0.1, step=1, beta1=0.9, beta2=0.99, eps=1e-3)
    want, m1, v1, tol, tol_m, tol_v = A.step64(f32(w0), f32(mean), 0.0, 0.0, lr=float(np.float32(0.1)), decay=0.0, step=1, beta1=0.9, beta2=0.99, eps=1e-3, scale=1.0)
    assert (np.abs(f32(model) - want) <= tol).all() and (np.abs(f32(m) - m1) <= tol_m).all() and (np.abs(f32(v) - v1) <= tol_v).all()
