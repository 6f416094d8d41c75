"""AdamW over many tensors and the norm of their gradients against the definitions."""
import numpy as np
import pytest
import torch

import adamw_ref as R
from paper_2402_03770_b200 import binding as B

pytestmark = pytest.mark.gpu
F = {torch.float32: np.float32, torch.float16: np.float16}
HOW = dict(lr=2e-3, step=7, beta1=0.9, beta2=0.999, eps=1e-8)


def numbers(t):
    return t.detach().float().cpu().numpy()


def make(sizes, param=torch.float32, grad=torch.float32, bits=32, copy=None, shift=0, seed=1, fresh=False):
    """tensors of these sizes, `shift` elements behind an aligned place"""
    g = torch.Generator().manual_seed(seed)

    def place(x):
        room = torch.zeros(x.numel() + shift + 16, dtype=x.dtype, device="cuda")
        at = room[shift:shift + x.numel()]
        at.copy_(x)
        return at

    s = {"sizes": sizes, "decay": [0.1 * (i % 3) for i in range(len(sizes))], "rates": [1.0 + 0.5 * (i % 2) for i in range(len(sizes))]}
    width = [10.0 ** (i % 5 - 4) for i in range(len(sizes))]
    s["grads"] = [place((torch.randn(n, generator=g) * w).to(grad)) for n, w in zip(sizes, width)]
    s["params"] = [place(torch.randn(n, generator=g).to(param)) for n in sizes]
    m = [torch.randn(n, generator=g) * w * 0.3 * (not fresh) for n, w in zip(sizes, width)]
    v = [(torch.rand(n, generator=g) * w) ** 2 * 0.01 * (not fresh) for n, w in zip(sizes, width)]
    s["scales"] = s["copies"] = None
    if bits == 32:
        s["m"], s["v"] = [place(x) for x in m], [place(x) for x in v]
    else:
        packed = [R.pack(a.numpy(), b.numpy(), 100, 1, 3) for a, b in zip(m, v)]
        s["m"], s["v"] = ([place(torch.from_numpy(x[k])) for x in packed] for k in (0, 1))
        s["scales"] = [torch.from_numpy(x[2]).cuda() for x in packed]
    if copy is not None:
        s["copies"] = [place(torch.zeros(n, dtype=copy)) for n in sizes]
    s["list"] = B.AdamwTensors(s["grads"], s["params"], s["m"], s["v"], s["scales"], s["copies"], lr=s["rates"], weight_decay=s["decay"])
    return s


def states(s, i):
    if s["scales"] is None:
        return numbers(s["m"][i]), numbers(s["v"][i])
    sc = numbers(s["scales"][i])
    of = np.arange(s["sizes"][i]) // R.BLOCK
    m, v = s["m"][i].cpu().numpy(), s["v"][i].cpu().numpy()
    return R.held(m, torch.float8_e4m3fn) * sc[of, 0], R.held(v, torch.float8_e5m2) * sc[of, 1]


def check(s, scale=1.0, seed=0, **how):
    """runs a step and compares all that it writes"""
    how = {**HOW, **how}
    before = [(numbers(s["params"][i]), numbers(s["grads"][i]), *states(s, i)) for i in range(len(s["sizes"]))]
    more = {k: how.pop(k) for k in ("norm", "max_norm", "grad_scale", "lr_dev", "step_dev", "status") if k in how}
    call = dict(how)
    if "step_dev" in more:
        call["step"] = 0
    B.cvlc_adamw(s["list"], seed=seed, **call, **more)
    torch.cuda.synchronize()
    lr = np.float32(how.pop("lr"))
    if "lr_dev" in more:
        lr = lr * np.float32(more["lr_dev"].item())
    for i, (p, g, m, v) in enumerate(before):
        n = s["sizes"][i]
        if n == 0:
            continue
        want, m1, v1, tol, tol_m, tol_v = R.step64(p, g, m, v, lr=float(lr * np.float32(s["rates"][i])), decay=s["decay"][i], scale=scale, **how)
        got = numbers(s["params"][i]).astype(np.float64)
        dtype = s["params"][i].dtype
        tol = tol * (1 + torch.finfo(dtype).eps) + (np.abs(want) * torch.finfo(dtype).eps / 2 if dtype != torch.float32 else 0.0) + 2.0 ** -25 * (dtype == torch.float16)
        assert (np.abs(got - want) <= tol).all(), (i, n, np.max(np.abs(got - want) / tol))
        if s["scales"] is None:
            a, b = states(s, i)
            assert (np.abs(a - m1) <= tol_m).all() and (np.abs(b - v1) <= tol_v).all(), (i, n)
        else:
            a, b = R.moments(g, m, v, scale, how["beta1"], how["beta2"])
            cm, cv, sc = R.pack(a, b, i, how["step"], seed)
            assert np.array_equal(numbers(s["scales"][i]), sc), i
            assert np.array_equal(s["m"][i].cpu().numpy(), cm) and np.array_equal(s["v"][i].cpu().numpy(), cv), (i, n)
        if s["copies"] is not None:
            assert torch.equal(s["copies"][i], s["params"][i].to(s["copies"][i].dtype))


SIZES = [1, 255, 256, 257, 0, 8, 7, 2048, 4097, 70001]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad,copy", [(torch.float32, torch.float32, None), (torch.float32, torch.bfloat16, torch.bfloat16),
                                             (torch.float32, torch.float16, torch.float16), (torch.bfloat16, torch.bfloat16, None),
                                             (torch.float16, torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("shift", [0, 1, 5])
def test_step(bits, param, grad, copy, shift):
    check(make(SIZES, param, grad, bits, copy, shift), seed=0x123456789ABC)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n", [9, 65, 441, 900])
def test_many_tensors(bits, n):
    check(make([(7 * i) % 300 for i in range(n)], bits=bits, shift=n % 3), seed=n)


@pytest.mark.parametrize("bits", [32, 8])
def test_long(bits):
    check(make([3_000_001, 12, 1_500_000], grad=torch.bfloat16, bits=bits, copy=torch.bfloat16))


@pytest.mark.parametrize("bits", [32, 8])
def test_first_steps_from_zeros(bits):
    s = make([1000, 300], bits=bits, fresh=True)
    for t in (1, 2, 3):
        check(s, step=t, seed=5)
    assert float(s["v"][0].float().min()) > 0


@pytest.mark.parametrize("bits", [32, 8])
def test_clip_and_scale(bits):
    s = make([5000, 77], bits=bits)
    norm = torch.zeros(1, device="cuda")
    ws = B.alloc_bytes(B.cvlc_grad_norm_workspace_bytes(s["list"]), torch.device("cuda"))
    B.cvlc_grad_norm(s["list"], norm, ws, grad_scale=0.25)
    want = 0.25 * np.sqrt(sum(float((x.double() ** 2).sum()) for x in s["grads"]))
    assert abs(norm.item() - want) <= want * 2 * R.U * 8
    clip = np.float32(0.25) * (np.float32(1e-3) / np.float32(norm.item()))
    check(s, scale=float(clip), grad_scale=0.25, norm=norm, max_norm=1e-3)
    check(s, scale=0.25, grad_scale=0.25, norm=norm, max_norm=1e9, step=8)


@pytest.mark.parametrize("bits", [32, 8])
def test_values_from_device_words(bits):
    s = make([5000, 77], bits=bits)
    check(s, lr_dev=torch.tensor([0.3], device="cuda"), step_dev=torch.tensor([12345], dtype=torch.int32, device="cuda"), step=12345)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("norm", [float("inf"), float("nan")])
def test_no_step_behind_a_norm_that_is_not_finite(bits, norm):
    s = make([5000, 77], bits=bits, copy=torch.bfloat16)
    before = [[x.clone() for x in s[k]] for k in ("params", "m", "v", "copies")]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.cvlc_adamw(s["list"], norm=torch.tensor([norm], device="cuda"), status=status, **HOW)
    assert status.item() == B.CVLC_ERR_NONFINITE_INPUT
    for k, b in zip(("params", "m", "v", "copies"), before):
        assert all(torch.equal(x, y) for x, y in zip(s[k], b))


def test_no_step_of_number_0():
    s = make([5000, 77], bits=8)
    before = [[x.clone() for x in s[k]] for k in ("params", "m", "v", "scales")]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.cvlc_adamw(s["list"], lr=1e-3, step=5, step_dev=torch.zeros(1, dtype=torch.int32, device="cuda"), status=status)
    assert status.item() == B.CVLC_ERR_INVALID_ARG
    for k, b in zip(("params", "m", "v", "scales"), before):
        assert all(torch.equal(x, y) for x, y in zip(s[k], b))


def test_streams_at_once():
    """two lists in two streams, and their norms, are what they are alone"""
    a, b = (make([300_000, 77, 4001], bits=bits, seed=bits, shift=1) for bits in (8, 32))
    c, d = (make([300_000, 77, 4001], bits=bits, seed=bits, shift=1) for bits in (8, 32))
    streams = [torch.cuda.Stream() for _ in range(2)]
    norms = [torch.zeros(1, device="cuda") for _ in range(4)]
    ws = [B.alloc_bytes(B.cvlc_grad_norm_workspace_bytes(x["list"]), torch.device("cuda")) for x in (a, b, c, d)]
    torch.cuda.synchronize()
    for t in range(1, 6):
        for x, n, w, st in zip((a, b), norms, ws, streams):
            B.cvlc_grad_norm(x["list"], n, w, stream=st)
            B.cvlc_adamw(x["list"], lr=1e-3, step=t, norm=n, seed=t, stream=st)
    torch.cuda.synchronize()
    for x, n, w in zip((c, d), norms[2:], ws[2:]):
        for t in range(1, 6):
            B.cvlc_grad_norm(x["list"], n, w)
            B.cvlc_adamw(x["list"], lr=1e-3, step=t, norm=n, seed=t)
    for x, y in ((a, c), (b, d)):
        assert all(torch.equal(p, q) for k in ("params", "m", "v") for p, q in zip(x[k], y[k]))


def test_nan_stays_in_its_block():
    s = make([600], bits=8)
    s["grads"][0][300] = float("nan")
    B.cvlc_adamw(s["list"], **HOW)
    m, v = states(s, 0)
    assert np.isnan(m[256:512]).all() and np.isnan(v[256:512]).all() and np.isfinite(m[:256]).all() and np.isfinite(v[512:]).all()
    assert bool(torch.isnan(s["params"][0][300])) and int(torch.isnan(s["params"][0]).sum()) == 1


def test_gradients_of_zero_and_tiny_blocks():
    s = make([512, 300], bits=8)
    for k in ("m", "v", "scales"):
        s[k][0].zero_()
    s["grads"][0].zero_()
    s["grads"][0][256:].fill_(1e-32)  # squares below what is held
    p = s["params"][0].clone()
    check(s, seed=3)
    assert torch.equal(s["scales"][0][0], torch.zeros(2, device="cuda")) and not bool(s["m"][0][:256].any())
    assert torch.equal(s["params"][0][:256], p[:256] - 0.0)


def test_bytes_keep_the_average():
    """the mean of what is held, over many seeds, is the value: within six deviations of a step that is taken or not"""
    n, seeds = 256, 400
    total_m, total_v = np.zeros(n), np.zeros(n)
    for seed in range(seeds):
        s = make([n], bits=8, seed=4)
        g, (m, v) = numbers(s["grads"][0]), states(s, 0)
        B.cvlc_adamw(s["list"], seed=seed, **HOW)
        a, b = states(s, 0)
        total_m += a
        total_v += b
    m1, v1 = R.moments(g, m, v, 1.0, 0.9, 0.999)
    step_m, step_v = np.abs(m1).max() * 2.0 ** -9 / 0.875 + np.abs(m1) / 8, v1.max() * 2.0 ** -30 + v1 / 4
    assert (np.abs(total_m / seeds - m1) <= 6 * 0.5 * step_m / np.sqrt(seeds)).all()
    big = v1 > v1.max() * 1e-8
    assert (np.abs(total_v / seeds - v1) <= 6 * 0.5 * step_v / np.sqrt(seeds))[big].all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("sizes,shift", [([1], 0), ([0, 5], 1), ([257, 1000, 3], 3), ([10_000_019, 1], 1), ([100 + i % 900 for i in range(950)], 0)])
def test_norm(dtype, sizes, shift):
    g = torch.Generator(device="cuda").manual_seed(3)
    grads = [torch.randn(n + shift, generator=g, device="cuda").to(dtype)[shift:] for n in sizes]
    t = B.AdamwTensors(grads)
    norm, ws = torch.zeros(1, device="cuda"), B.alloc_bytes(B.cvlc_grad_norm_workspace_bytes(t), torch.device("cuda"))
    ws.fill_(255)
    B.cvlc_grad_norm(t, norm, ws, grad_scale=-2.0)
    want = 2.0 * np.sqrt(sum(float((x.double() ** 2).sum()) for x in grads))
    # eight squares and sums in 32 bits, U each, halved by the root, then one rounding
    assert abs(norm.item() - want) <= want * (8 * R.U / 2 + R.U) * 1.01
    first = norm.clone()
    B.cvlc_grad_norm(t, norm, ws, grad_scale=-2.0)
    assert torch.equal(first, norm)


def test_norm_of_nothing_and_of_what_is_not_finite():
    t = B.AdamwTensors([])
    norm, ws = torch.ones(1, device="cuda"), B.alloc_bytes(B.cvlc_grad_norm_workspace_bytes(t), torch.device("cuda"))
    B.cvlc_grad_norm(t, norm, ws)
    assert norm.item() == 0.0
    for x in (float("inf"), float("nan"), 3e19):
        g = torch.ones(5000, device="cuda")
        g[4321] = x
        B.cvlc_grad_norm(B.AdamwTensors([g]), norm, ws)
        assert not np.isfinite(norm.item())


def test_graph_of_several_steps():
    """a captured step with its number and rate in device words, replayed, is the steps one by one"""
    a, b = (make([5000, 300], grad=torch.bfloat16, bits=8, copy=torch.bfloat16) for _ in range(2))
    t, rate, norm = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.ones(1, device="cuda"), torch.zeros(1, device="cuda")
    ws = B.alloc_bytes(B.cvlc_grad_norm_workspace_bytes(a["list"]), torch.device("cuda"))
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        t += 1
        rate *= 0.5
        B.cvlc_grad_norm(a["list"], norm, ws, stream=stream)
        B.cvlc_adamw(a["list"], lr=1e-2, step=0, step_dev=t, lr_dev=rate, norm=norm, max_norm=0.5, seed=9, stream=stream)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for k in (1, 2, 3):
        B.cvlc_grad_norm(b["list"], norm, ws)
        B.cvlc_adamw(b["list"], lr=1e-2, step=k, step_dev=torch.tensor([k], dtype=torch.int32, device="cuda"),
                     lr_dev=torch.tensor([0.5 ** k], device="cuda"), norm=norm, max_norm=0.5, seed=9)
    for k in ("params", "m", "v", "scales", "copies"):
        assert all(torch.equal(x, y) for x, y in zip(a[k], b[k])), k


def test_neighbours_are_left_alone():
    """tensors that lie in one vector: what is between them stays"""
    room = {k: torch.full((4000,), 7.0, device="cuda") for k in "pgmv"}
    cuts = [(3, 500), (505, 1), (507, 1000), (2000, 1999)]
    at = {k: [x[a:a + n] for a, n in cuts] for k, x in room.items()}
    B.cvlc_adamw(B.AdamwTensors(at["g"], at["p"], at["m"], at["v"]), **HOW)
    inside = torch.zeros(4000, dtype=torch.bool, device="cuda")
    for a, n in cuts:
        inside[a:a + n] = True
    for k in "pmv":
        assert bool((room[k][~inside] == 7.0).all()) and bool((room[k][inside] != 7.0).all()), k
    assert bool((room["g"] == 7.0).all())


def test_binding_refuses():
    p = torch.zeros(10, device="cuda")
    with pytest.raises(AssertionError):
        B.AdamwTensors([p], [p[:5]], [p], [p])
    with pytest.raises(AssertionError):
        B.AdamwTensors([p], [p], [p.half()], [p])
    with pytest.raises(AssertionError):
        B.cvlc_adamw(B.AdamwTensors([p]), **HOW)
    with pytest.raises(AssertionError):
        B.AdamwTensors([p.cpu()], [p], [p], [p])
