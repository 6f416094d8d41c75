"""Which gradients the distillation calls refuse because they overlap the logits, without a GPU."""
import pytest

from paper_2402_03770_b200 import binding as B
from test_vocab_refusals import AT, BAD, distill


# rows of 100 elements of 2 bytes, 4 of them; the logits begin at AT
@pytest.mark.parametrize("call", ["grad", "step"])
@pytest.mark.parametrize("stride,grad,grad_stride", [
    (250, AT + 2 * 99, 250),        # a row's end
    (250, AT + 2 * 151, 250),       # the next row's beginning
    (250, AT - 2 * 99, 250),
    (250, AT - 2 * 151, 250),
    (250, AT + 2 * (500 + 99), 250),
    (250, AT - 2 * (500 + 151), 250),
    (250, AT + 2 * 120, 251),       # between the rows, but not as far apart
    (199, AT + 2 * 100, 199),       # no room for a row
    (100, AT + 2 * 100, 100)])
def test_overlaps_are_refused(call, stride, grad, grad_stride):
    assert distill(call, stride=stride, grad=grad, grad_stride=grad_stride) == BAD


def test_one_row_overlaps_itself():
    assert distill("step", rows=1, grad=AT + 2 * 99, stride=100) == BAD
    assert distill("step", rows=1, grad=AT - 2 * 99, stride=500, grad_stride=250) == BAD
    assert B.CVLC_OK == distill("step", rows=0, grad=AT + 2)
