"""The workspace of the embedding's gradient: what serves a call serves every smaller one."""
import pytest

from paper_2402_03770_b200 import binding as B

EDGES = [0, 1, 16, 17, 2047, 2048, 2049, 32767, 32768, 32769, 40000, 65535, 65536, 65537, 131072, 131073, 262144, 262145, 524288, 524289, 600000,
         1 << 20, (1 << 20) + 1, (1 << 20) + 513, 1 << 21, (1 << 31) - 1]


@pytest.mark.parametrize("dim", [1, 64, 2048, 1 << 20])
def test_the_workspace_grows_with_the_tokens(dim):
    need = [B.cvlc_embed_grad_workspace_bytes(n, dim, 1000) for n in EDGES]
    assert need == sorted(need)


def test_the_workspace_grows_by_every_token():
    need = [B.cvlc_embed_grad_workspace_bytes(n, 256, 1000) for n in list(range(0, 3000)) + list(range(32000, 34000)) + list(range(524000, 526000))]
    assert need == sorted(need)


def test_the_workspace_grows_with_columns_and_words():
    need = [B.cvlc_embed_grad_workspace_bytes(40000, dim, 1000) for dim in (1, 2, 3, 8, 100, 4096, 1 << 20)]
    assert need == sorted(need)
    need = [B.cvlc_embed_grad_workspace_bytes(40000, 64, vocab) for vocab in (1, 2, 511, 512, 1 << 20, (1 << 31) - 1)]
    assert need == sorted(need)


@pytest.mark.gpu
@pytest.mark.parametrize("most,n", [(40000, 32768), (65537, 65536), (530000, 524288), (40000, 1)])
def test_a_workspace_for_more_tokens(most, n):
    import torch

    import vocab_ref as R
    dim, vocab = 40, 700
    gen = torch.Generator(device="cuda").manual_seed(n)
    tokens = torch.randint(-1, vocab, (n,), generator=gen, device="cuda", dtype=torch.int32)
    grad = torch.randn(n, dim, generator=gen, device="cuda")
    u = torch.zeros(vocab, dim, device="cuda")
    ws = torch.full((B.cvlc_embed_grad_workspace_bytes(most, dim, vocab),), 0xA5, dtype=torch.uint8, device="cuda")
    B.cvlc_embed_grad(tokens, grad, u, ws)
    R.assert_near(u, *R.embed_grad(tokens, grad, vocab, 1.0))
