"""Gradients that overlap what they are made of, or each other, are refused before anything is launched, also where there are no rows: zeros would be written."""
import pytest

from paper_2402_03770_b200 import binding as B
from test_head_refusals import AT, BAD, FAR, head, step


# head: 500 rows of 128 bytes from AT + FAR on
@pytest.mark.parametrize("rows", [0, 1, 10])
@pytest.mark.parametrize("dw,dw_stride", [(AT + FAR, 64), (AT + FAR + 64, 64), (AT + FAR + 499 * 128 + 126, 64), (AT + FAR - 499 * 128 - 126, 64), (AT + FAR, 128),
                                          (AT + FAR - 2, 64)])
def test_head_and_its_gradient(rows, dw, dw_stride):
    assert step(head(rows=rows), dw=dw, dw_stride=dw_stride) == BAD


@pytest.mark.parametrize("kw", [dict(dtype=B.CVLC_F32), dict(head_dev=None), dict(pieces=0)])
def test_no_rows_refuses(kw):
    assert step(head(rows=0, **kw)) == BAD
