"""The binding's vocabulary calls pass on only tensors of the current device, without a GPU: tensors that say where they are."""
import pytest
import torch

from paper_2402_03770_b200 import binding as B


class On:
    """a contiguous tensor on a device"""
    is_cuda = True

    def __init__(self, device, dtype, *shape):
        self.device, self.dtype, self.shape = device, dtype, shape

    def get_device(self):
        return self.device

    def dim(self):
        return len(self.shape)

    def numel(self):
        return torch.Size(self.shape).numel()

    def element_size(self):
        return torch.empty(0, dtype=self.dtype).element_size()

    def stride(self):
        return (self.shape[1], 1) if len(self.shape) == 2 else (1,)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


class Calls:
    """in the library's place"""

    def __init__(self):
        self.names = []

    def __getattr__(self, name):
        return lambda *a: self.names.append(name) or 0


F, I = torch.float32, torch.int32
CALLS = {
    "cvlc_top_logits": [(F, 4, 9), (I, 4, 3), (F, 4, 3)],
    "cvlc_distill_loss": [(F, 4, 9), (I, 4, 3), (F, 4, 3), (F, 4)],
    "cvlc_distill_grad": [(F, 4, 9), (I, 4, 3), (F, 4, 3), (F, 4, B.DISTILL_STATS), (F, 4, 9)],
    "cvlc_distill_step": [(F, 4, 9), (I, 4, 3), (F, 4, 3), (F, 4), (F, 4, 9)],
    "cvlc_embed": [(F, 20, 9), (I, 4), (F, 4, 9)],
    "cvlc_embed_grad": [(I, 4), (F, 4, 9), (F, 20, 9), (torch.uint8, 4096)],
}


@pytest.mark.parametrize("name", CALLS)
def test_tensors_of_another_device_are_refused(name, monkeypatch):
    calls = Calls()
    monkeypatch.setattr(B, "lib", lambda: calls)
    monkeypatch.setattr(B, "_device", lambda: 0)
    monkeypatch.setattr(B, "_stream_on", lambda stream, device: 0)
    args = [On(0, *a) for a in CALLS[name]]
    getattr(B, name)(*args)
    assert calls.names == [name]
    for i, a in enumerate(CALLS[name]):
        with pytest.raises(AssertionError):
            getattr(B, name)(*args[:i], On(1, *a), *args[i + 1:])
    assert calls.names == [name]
