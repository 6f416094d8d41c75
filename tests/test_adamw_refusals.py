"""What the optimiser's entry points refuse, without a GPU: every check is made before anything is launched."""
import ctypes as C
import math

import pytest
import torch

from paper_2402_03770_b200 import binding as B

BAD = B.CVLC_ERR_INVALID_ARG
AT = 1 << 20  # an address that nothing reads


def args(**kw):
    a = dict(param_dtype=B.CVLC_F32, grad_dtype=B.CVLC_F32, copy_dtype=B.CVLC_BF16, state_bits=32, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, seed=0, step=1,
             grad_scale=1.0, max_norm=1.0, reserved=0, norm_dev=None, lr_dev=None, step_dev=None, status_dev=None)
    a.update(kw)
    return B.CvlcAdamwArgs(**a)


def tensor(**kw):
    a = dict(n=10, grad_dev=AT, param_dev=AT, m_dev=AT, v_dev=AT, scale_dev=None, copy_dev=None, lr=1.0, weight_decay=0.0)
    a.update(kw)
    return B.CvlcAdamwTensor(**a)


def step(tensors, a):
    return B.lib().cvlc_adamw((B.CvlcAdamwTensor * max(1, len(tensors)))(*tensors), len(tensors), C.byref(a), None)


@pytest.mark.parametrize("kw", [
    dict(param_dtype=3), dict(grad_dtype=9), dict(state_bits=16), dict(lr=math.nan), dict(lr=math.inf), dict(lr=1e39), dict(beta1=1.0), dict(beta1=-0.1),
    dict(beta2=1.0), dict(beta2=math.nan), dict(eps=0.0), dict(eps=-1.0), dict(eps=1e-31), dict(eps=math.inf), dict(step=0), dict(grad_scale=math.inf),
    dict(norm_dev=AT, max_norm=0.0), dict(norm_dev=AT, max_norm=math.nan), dict(norm_dev=AT + 2), dict(lr_dev=AT + 1), dict(step_dev=AT + 2),
    dict(status_dev=AT + 2)])
def test_adamw_refuses(kw):
    assert step([tensor(scale_dev=AT)], args(**kw)) == BAD


@pytest.mark.parametrize("kw,a", [
    (dict(n=(1 << 40) + 1), {}), (dict(grad_dev=None), {}), (dict(param_dev=None), {}), (dict(m_dev=None), {}), (dict(v_dev=None), {}), (dict(grad_dev=AT + 2), {}),
    (dict(param_dev=AT + 1), dict(param_dtype=B.CVLC_BF16)), (dict(m_dev=AT + 2), {}), (dict(scale_dev=None), dict(state_bits=8)),
    (dict(scale_dev=AT + 4), dict(state_bits=8)), (dict(copy_dev=AT + 1), {}), (dict(copy_dev=AT), dict(copy_dtype=B.CVLC_F32)), (dict(lr=math.nan), {}),
    (dict(weight_decay=math.inf), {})])
def test_adamw_refuses_tensors(kw, a):
    assert step([tensor(), tensor(**kw)], args(**a)) == BAD


def test_nothing_to_do():
    assert step([], args()) == B.CVLC_OK
    assert step([tensor(n=0, grad_dev=None, param_dev=None, m_dev=None, v_dev=None)], args()) == B.CVLC_OK
    assert B.lib().cvlc_adamw(None, 1, C.byref(args()), None) == BAD and B.lib().cvlc_adamw(None, 0, None, None) == BAD


def test_all_tensors_count():
    assert step([tensor(n=1 << 39), tensor(n=(1 << 39) + 1)], args()) == BAD


@pytest.mark.parametrize("kw", [dict(dtype=3), dict(scale=math.nan), dict(norm=None), dict(norm=AT + 2), dict(ws=None), dict(ws=AT + 128)])
def test_norm_refuses(kw):
    a = dict(dtype=B.CVLC_F32, scale=1.0, norm=AT, ws=AT)
    a.update(kw)
    t = tensor()
    assert B.lib().cvlc_grad_norm(C.byref(t), 1, a["dtype"], a["scale"], a["norm"], a["ws"], 1 << 20, None) == BAD


def test_norm_workspace():
    need = B.lib().cvlc_grad_norm_workspace_bytes(1)
    assert need > 0 and need % 256 == 0 and B.lib().cvlc_grad_norm_workspace_bytes(2000) > need and B.lib().cvlc_grad_norm_workspace_bytes(0) == need
    t = tensor()
    assert B.lib().cvlc_grad_norm(C.byref(t), 1, 0, 1.0, AT, AT, need - 1, None) == B.CVLC_ERR_WORKSPACE_TOO_SMALL
    t = tensor(grad_dev=AT + 2)
    assert B.lib().cvlc_grad_norm(C.byref(t), 1, 0, 1.0, AT, AT, need, None) == BAD
    assert C.sizeof(B.CvlcAdamwTensor) == 64 and C.sizeof(B.CvlcAdamwArgs) == 104


def test_binding_refuses_what_overlaps():
    p, q, g, m, v, w, x, c = (torch.zeros(300) for _ in range(8))
    half = torch.zeros(300, dtype=torch.bfloat16)
    B.AdamwTensors([g, g], [p, q], [m, w], [v, x], copies=[half, None])  # gradients alone may be shared
    B.AdamwTensors([g, g])
    byte, scales = torch.zeros(4, 300, dtype=torch.uint8), torch.zeros(2, 2, 2)
    B.AdamwTensors([g[:0], g], [p[:0], p], [byte[0][:0], byte[1]], [byte[2][:0], byte[3]], scales=[scales[0][:0], scales[1]])
    for how in (([g, c], [p, p], [m, w], [v, x]), ([g, c], [g, q], [m, w], [v, x]), ([g, c], [p, q], [m, m], [v, x]), ([g, c], [p, q], [m, w], [w, x]), ([g, p], [p, q], [m, w], [v, x]),
                ([g[:100], c[:100]], [p[:100], p[99:199]], [m[:100], w[:100]], [v[:100], x[:100]])):
        with pytest.raises(AssertionError, match="overlap"):
            B.AdamwTensors(*how)
    with pytest.raises(AssertionError, match="overlap"):
        B.AdamwTensors([g, c], [p, q], [m, w], [v, x], copies=[half, half])
    with pytest.raises(AssertionError, match="overlap"):
        B.AdamwTensors([g, c], [p, q], [byte[0], byte[1]], [byte[2], byte[3]], scales=[scales[0], scales[0]])


def test_binding_takes_rows_of_one_tensor():
    g, p, m, v = torch.zeros(4, 3, 512).unbind()
    byte, copies = torch.zeros(2, 3, 512, dtype=torch.uint8), torch.zeros(3, 512, dtype=torch.bfloat16)
    t = B.AdamwTensors(g, p, byte[0], byte[1], scales=torch.zeros(3, 2, 2), copies=copies)
    assert t.n == 3 and t.array[1].copy_dev == copies[1].data_ptr() and t.array[2].m_dev == byte[0, 2].data_ptr()
    assert B.AdamwTensors(g, p, m, v).array[1].v_dev == v[1].data_ptr()
