"""What the vocabulary entry points refuse, without a GPU: every check is made before anything is launched."""
import ctypes as C
import math

import pytest

from paper_2402_03770_b200 import binding as B

BAD = B.CVLC_ERR_INVALID_ARG
AT = 1 << 20  # an address that nothing reads


def top(**kw):
    a = dict(logits=AT, dtype=B.CVLC_BF16, rows=4, vocab=100, stride=100, k=10, temperature=1.0, ids=AT, logp=AT)
    a.update(kw)
    return B.lib().cvlc_top_logits(a["logits"], a["dtype"], a["rows"], a["vocab"], a["stride"], a["k"], a["temperature"], a["ids"], a["logp"], None)


@pytest.mark.parametrize("kw", [
    dict(logits=None), dict(logits=AT + 1), dict(logits=AT + 2, dtype=B.CVLC_F32), dict(dtype=3), dict(rows=(1 << 27) + 1),
    dict(vocab=0, stride=0, k=1), dict(vocab=B.MAX_VOCAB + 1, stride=B.MAX_VOCAB + 1), dict(stride=99), dict(stride=1 << 33), dict(k=0),
    dict(k=101), dict(vocab=1000, stride=1000, k=257), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=9e-7), dict(temperature=1.1e6), dict(temperature=math.inf),
    dict(temperature=math.nan), dict(ids=None), dict(ids=AT + 2), dict(logp=None), dict(logp=AT + 1)])
def test_top_logits_refuses(kw):
    assert top(**kw) == BAD


def test_no_rows_is_nothing():
    assert top(rows=0) == B.CVLC_OK
    assert top(rows=0, logits=None, ids=None, logp=None) == B.CVLC_OK
    assert distill("step", rows=0, logits=None, ids=None, logp=None, loss=None, grad=None) == B.CVLC_OK
    assert embed(n=0, tokens=None, out=None) == B.CVLC_OK


def distill(call, **kw):
    a = dict(logits=AT, dtype=B.CVLC_BF16, rows=4, vocab=100, stride=100, k=10, temperature=1.0, ids=AT, logp=AT, rest=B.CVLC_REST_BUCKET,
             weight=None, status=None, loss=AT, stats=AT, grad=AT << 4, grad_stride=100)
    a.update(kw)
    d = B.CvlcDistill(a["logits"], a["rows"], a["stride"], a["vocab"], a["dtype"], a["ids"], a["logp"], a["k"], a["rest"], a["temperature"], 0,
                      a["weight"], a["status"])
    L = B.lib()
    if call == "loss":
        return L.cvlc_distill_loss(C.byref(d), a["loss"], a["stats"], None)
    if call == "grad":
        return L.cvlc_distill_grad(C.byref(d), a["stats"], a["grad"], a["grad_stride"], None)
    return L.cvlc_distill_step(C.byref(d), a["loss"], a["grad"], a["grad_stride"], None)


@pytest.mark.parametrize("call", ["loss", "grad", "step"])
@pytest.mark.parametrize("kw", [
    dict(logits=None), dict(logits=AT + 1), dict(dtype=7), dict(vocab=0, stride=0), dict(stride=99), dict(k=B.MAX_RECORDS + 1), dict(rest=3),
    dict(temperature=0.0), dict(temperature=math.nan), dict(ids=None), dict(logp=AT + 2), dict(weight=AT + 2), dict(status=AT + 1)])
def test_distill_refuses(call, kw):
    assert distill(call, **kw) == BAD


@pytest.mark.parametrize("call,kw", [
    ("loss", dict(loss=None)), ("loss", dict(loss=AT + 2)), ("loss", dict(stats=AT + 4)), ("grad", dict(stats=None)), ("grad", dict(stats=AT + 8)),
    ("grad", dict(grad=None)), ("grad", dict(grad=AT + 1)), ("step", dict(loss=None)), ("step", dict(grad_stride=99)), ("step", dict(grad=None)),
    ("step", dict(grad=AT + 2)), ("step", dict(grad=AT, grad_stride=101)), ("grad", dict(grad=AT + 2 * 399)), ("grad", dict(grad=AT - 2 * 399))])
def test_distill_refuses_outputs(call, kw):
    assert distill(call, **kw) == BAD


def embed(**kw):
    a = dict(table=AT, dtype=B.CVLC_F32, vocab=100, dim=8, stride=8, tokens=AT, size=4, n=5, out=AT, out_stride=8, status=None)
    a.update(kw)
    return B.lib().cvlc_embed(a["table"], a["dtype"], a["vocab"], a["dim"], a["stride"], a["tokens"], a["size"], a["n"], 1.0, a["out"],
                              a["out_stride"], a["status"], None)


@pytest.mark.parametrize("kw", [
    dict(table=None), dict(table=AT + 2), dict(dtype=3), dict(vocab=0), dict(vocab=1 << 31), dict(dim=0), dict(dim=(1 << 20) + 1, stride=1 << 21),
    dict(stride=7), dict(tokens=None), dict(tokens=AT + 4, size=8), dict(size=2), dict(n=1 << 31), dict(out=None), dict(out=AT + 1),
    dict(out_stride=7), dict(status=AT + 2)])
def test_embed_refuses(kw):
    assert embed(**kw) == BAD


def embed_grad(**kw):
    a = dict(tokens=AT, size=4, n=5, grad=AT, dtype=B.CVLC_F32, dim=8, stride=8, vocab=100, update=AT, update_stride=8, accumulate=0, ws=AT,
             ws_bytes=1 << 30)
    a.update(kw)
    return B.lib().cvlc_embed_grad(a["tokens"], a["size"], a["n"], a["grad"], a["dtype"], a["dim"], a["stride"], a["vocab"], 1.0, a["update"],
                                   a["update_stride"], a["accumulate"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw", [
    dict(tokens=None), dict(tokens=AT + 4, size=8), dict(size=1), dict(n=1 << 31), dict(grad=None), dict(grad=AT + 2), dict(dtype=9), dict(dim=0),
    dict(stride=7), dict(vocab=0), dict(vocab=1 << 31), dict(update=None), dict(update=AT + 2), dict(update_stride=7), dict(accumulate=2),
    dict(ws=None), dict(ws=AT + 128)])
def test_embed_grad_refuses(kw):
    assert embed_grad(**kw) == BAD


def test_embed_grad_workspace():
    need = B.cvlc_embed_grad_workspace_bytes(5, 8, 100)
    assert need > 0 and need % 256 == 0
    assert embed_grad(ws_bytes=need - 1) == B.CVLC_ERR_WORKSPACE_TOO_SMALL
    assert B.cvlc_embed_grad_workspace_bytes(5, 0, 100) == 0 and B.cvlc_embed_grad_workspace_bytes(5, 8, 0) == 0
    assert B.cvlc_embed_grad_workspace_bytes(1 << 31, 8, 100) == 0
    assert C.sizeof(B.CvlcDistill) == 80
