"""What the owners of the token operators check by themselves, without a device."""
import pytest
import torch

from paper_2406_02052_amd import Attention, Coupling, HeadNorm, VocabLoss
from paper_2406_02052_amd.ops import _Owner


class Stream:
    """What the owners look at of a stream; default streams of all devices have the handle 0."""

    def __init__(self, index, handle=0):
        self.device_index, self.cuda_stream = index, handle


@pytest.mark.parametrize("handle", [0, 64])
def test_owners_refuse_streams_of_another_device(handle):
    owner = _Owner()
    owner.workspace, owner.streams = torch.empty(4), {0, 64}   # (on no device: -1)
    assert owner._on(Stream(-1, handle)) == handle and owner._on(handle) == handle
    with pytest.raises(ValueError, match="stream of the owner's device"):
        owner._on(Stream(1, handle))


def test_calls_without_a_workspace_refuse_them_too():
    head = torch.zeros(1, 2, 2, 64)
    with pytest.raises(ValueError, match="stream of the owner's device"):
        HeadNorm(1, 2, 2, 2, 64, "fp32", norm=None, device="cpu").forward(head, head, head, head, stream=Stream(1))
    with pytest.raises(ValueError, match="stream of the owner's device"):
        Coupling(4, 64, "fp32", device="cpu").forward(None, stream=Stream(1))


def test_owners_have_streams_of_their_own():
    for op in (Attention(1, 2, 2, 1, 1, 64, device="cpu"), VocabLoss(4, 8, 8, "fp32", device="cpu")):
        assert op.streams == set()   # (on no device there are none)
        with pytest.raises(ValueError, match="stream of the owner's device"):
            op._on(Stream(0))
