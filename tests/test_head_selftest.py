"""What the self-test of the head's products refuses, without a GPU: every check is made before anything is launched."""
import ctypes as C
import math

import pytest

from paper_2402_03770_b200 import binding as B
from test_head_refusals import AT, BAD, FAR, head


def call(a, loss=AT, dh=AT + 2 * FAR, dw=AT + 3 * FAR, ws=AT, ws_bytes=1 << 40, limit_us=1000):
    return B.lib().cvlc_selftest_head(C.byref(a), loss, dh, 64, dw, 64, 0, 0, 0, limit_us, ws, ws_bytes, None)


@pytest.mark.parametrize("kw", [dict(limit_us=1_000_001), dict(loss=None), dict(dh=None), dict(dw=AT + FAR), dict(dh=AT), dict(ws=AT + 128)])
@pytest.mark.parametrize("graded", [True, False])
def test_refuses(kw, graded):
    if not graded:
        kw = {k: v for k, v in kw.items() if k not in ("dh", "dw")} or dict(loss=AT + 2)
        kw["dw"] = None
    assert call(head(), **kw) == BAD


@pytest.mark.parametrize("kw", [dict(dtype=B.CVLC_F32), dict(scale=math.nan), dict(vocab=0), dict(pieces=0)])
@pytest.mark.parametrize("dw", [AT + 3 * FAR, None])
def test_refuses_heads(kw, dw):
    assert call(head(**kw), dw=dw) == BAD
    assert call(head(), dw=dw, ws_bytes=256) == B.CVLC_ERR_WORKSPACE_TOO_SMALL
