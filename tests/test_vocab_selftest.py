"""What the self-test of the ring refuses, without a GPU: every check is made before anything is launched."""
import pytest

from paper_2402_03770_b200 import binding as B

AT = 1 << 20  # an address that nothing reads


@pytest.mark.parametrize("kw", [dict(row=None), dict(row=AT + 4), dict(stages=0), dict(stages=257), dict(limit_us=1_000_001), dict(status=None), dict(status=AT + 2),
                                dict(seen=None), dict(seen=AT + 8)])
def test_ring_refuses(kw):
    a = dict(row=AT, stages=3, limit_us=1000, status=AT, seen=AT)
    a.update(kw)
    assert B.lib().cvlc_selftest_ring(a["row"], a["stages"], 1, a["limit_us"], a["status"], a["seen"], None) == B.CVLC_ERR_INVALID_ARG
