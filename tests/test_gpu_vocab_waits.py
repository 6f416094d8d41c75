"""The ring through which rows of logits are copied: a wait that runs out stops the copies, is reported, and overwrites nothing."""
import pytest
import torch

pytestmark = pytest.mark.gpu
STAGE = 4096


@pytest.mark.parametrize("stages", [1, 2, 3, 7, 64])
@pytest.mark.parametrize("give_back", [True, False])
def test_ring(stages, give_back):
    from paper_2402_03770_b200 import binding as B
    B.cvlc_set_device(0)
    row = torch.arange(stages * STAGE, dtype=torch.float32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    seen = torch.full((2 * STAGE,), -1.0, device="cuda")
    B.cvlc_selftest_ring(row, give_back, 1000, status, seen)
    cuts = row.view(stages, STAGE)
    # given back, a place holds the last stage that came to it; else the first
    for place in range(min(2, stages)):
        last = stages - 1 - (stages - 1 - place) % 2
        assert torch.equal(seen[place * STAGE:][:STAGE], cuts[last if give_back else place])
    # that stages are not given back is noticed by who waits for it: for the next copy, or, at the end, for all of them
    assert int(status) == (B.CVLC_OK if give_back else B.CVLC_ERR_DEVICE_TIMEOUT)
    status.fill_(B.CVLC_ERR_INVALID_ARG)
    B.cvlc_selftest_ring(row, give_back, 0, status, seen)
    assert int(status) == B.CVLC_ERR_INVALID_ARG  # the first error stays
