"""What the head's entry points refuse, without a GPU: every check is made before anything is launched."""
import ctypes as C
import math

import pytest

from paper_2402_03770_b200 import binding as B

BAD = B.CVLC_ERR_INVALID_ARG
AT = 1 << 30  # an address that nothing reads
FAR = 1 << 32


def head(**kw):
    a = dict(hidden_dev=AT, head_dev=AT + FAR, targets_dev=AT, row_weight_dev=None, status_dev=None, rows=10, hidden_stride=64, head_stride=64, vocab=500, dim=64,
             dtype=B.CVLC_BF16, token_bytes=4, scale=1.0, pieces=1)
    a.update(kw)
    return B.CvlcHead(**a)


def loss(a, loss=AT, ws=AT, ws_bytes=1 << 40):
    return B.lib().cvlc_head_loss(C.byref(a), loss, ws, ws_bytes, None)


def step(a, loss=AT, dh=AT + 2 * FAR, dh_stride=64, dw=AT + 3 * FAR, dw_stride=64, ws=AT, ws_bytes=1 << 40):
    return B.lib().cvlc_head_step(C.byref(a), loss, dh, dh_stride, dw, dw_stride, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [loss, step])
@pytest.mark.parametrize("kw", [
    dict(dtype=B.CVLC_F32), dict(dtype=3), dict(vocab=0), dict(vocab=B.MAX_VOCAB + 1), dict(dim=0), dict(dim=65537, hidden_stride=1 << 17, head_stride=1 << 17),
    dict(rows=(1 << 24) + 1), dict(hidden_stride=63), dict(head_stride=63), dict(hidden_stride=1 << 33), dict(head_stride=1 << 33), dict(scale=math.nan),
    dict(scale=math.inf), dict(pieces=0), dict(token_bytes=2), dict(token_bytes=8, targets_dev=AT + 4), dict(hidden_dev=None), dict(hidden_dev=AT + 1),
    dict(head_dev=None), dict(head_dev=AT + FAR + 1), dict(targets_dev=None), dict(row_weight_dev=AT + 2), dict(status_dev=AT + 1)])
def test_refuses(call, kw):
    assert call(head(**kw)) == BAD


@pytest.mark.parametrize("call", [loss, step])
@pytest.mark.parametrize("kw", [dict(loss=None), dict(loss=AT + 2), dict(ws=None), dict(ws=AT + 128)])
def test_refuses_outputs(call, kw):
    assert call(head(), **kw) == BAD


@pytest.mark.parametrize("kw", [
    dict(dh=None), dict(dh=AT + 1), dict(dw=None), dict(dw=AT + 3), dict(dh_stride=63), dict(dw_stride=63), dict(dw_stride=1 << 33), dict(dh=AT), dict(dh=AT + 2 * 639),
    dict(dw=AT + FAR), dict(dw=AT + FAR - 2), dict(dh=AT + FAR + 128), dict(dw=AT - 500 * 128 + 2), dict(dh=AT + 3 * FAR + 64), dict(dh=AT + 64, dh_stride=128),
    dict(dh=AT + 64, dh_stride=64)])
def test_refuses_gradients(kw):
    assert step(head(), **kw) == BAD


def test_workspace():
    L = B.lib()
    a = head()
    small, large = (L.cvlc_head_workspace_bytes(C.byref(a), k) for k in (0, 1))
    assert 0 < small < large and small % 256 == 0 and large % 256 == 0
    assert loss(a, ws_bytes=small - 1) == B.CVLC_ERR_WORKSPACE_TOO_SMALL and step(a, ws_bytes=large - 1) == B.CVLC_ERR_WORKSPACE_TOO_SMALL
    b = head(vocab=100000, rows=1000, pieces=1)
    c = head(vocab=100000, rows=1000, pieces=10)
    assert L.cvlc_head_workspace_bytes(C.byref(b), 1) > 5 * L.cvlc_head_workspace_bytes(C.byref(c), 1)
    d = head(hidden_dev=AT + 2)  # rows that have to be copied
    assert L.cvlc_head_workspace_bytes(C.byref(d), 0) > small
    assert L.cvlc_head_workspace_bytes(None, 0) == 0 and L.cvlc_head_workspace_bytes(C.byref(head(dim=0)), 0) == 0
    assert C.sizeof(B.CvlcHead) == 88


def test_no_rows_is_no_loss():
    assert loss(head(rows=0, hidden_dev=None, targets_dev=None), loss=None, ws=None, ws_bytes=0) == B.CVLC_OK
    assert B.lib().cvlc_head_loss(None, AT, AT, 0, None) == BAD
