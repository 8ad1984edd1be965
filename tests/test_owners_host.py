"""What the owners of the token operators check by themselves, without a device."""
import pytest
import torch

from paper_2406_02052_amd import AdamW, Attention, Coupling, HeadNorm, VocabLoss
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


def adamw(count, copies=False):
    """An owner of tensors on the host, as it is once they are laid out."""
    op = AdamW.__new__(AdamW)
    op.params, op.grads = ([torch.zeros(5 + i) for i in range(count)] for _ in range(2))
    op.copies = [torch.zeros(5 + i, dtype=torch.bfloat16) if copies else None for i in range(count)]
    op.m, op.v, op.m_scale, op.v_scale = torch.zeros(64), torch.zeros(64), None, None
    op.lr, op.steps = torch.zeros(1), torch.zeros(1, dtype=torch.int64)
    op.workspace, op.table = torch.empty(4), torch.empty(4)
    op._keep()
    return op


@pytest.mark.parametrize("what", ["params", "grads", "copies"])
@pytest.mark.parametrize("count,at", [(1, 0), (5, 4), (40, 33)])
def test_adamw_refuses_tensors_of_other_memory(count, at, what):
    """In the turn of the one that moved, and from then on; what was laid out stays as long as the owner."""
    op = adamw(count, copies=True)
    turns = -(-3 * count // 8)
    for _ in range(2 * turns):
        op._need_laid()
    t = getattr(op, what)[at]
    t.fill_(3.0)
    old = t.data_ptr()
    t.data = torch.zeros_like(t)
    kept = [x for x in op._owned() if x.data_ptr() == old]
    assert len(kept) == 1 and (kept[0] == 3).all()
    passed = 0
    with pytest.raises(ValueError, match=rf"{what}\[{at}\]: its memory"):
        for passed in range(turns + 1):
            op._need_laid()
    assert passed <= turns
    for _ in range(3):
        with pytest.raises(ValueError, match="its memory"):
            op._need_laid()


def test_adamw_refuses_replaced_states():
    for name in ("m", "v", "m_scale"):
        op = adamw(2)
        op._need_laid()
        setattr(op, name, torch.zeros(64))
        with pytest.raises(ValueError, match=f"{name}: has been replaced"):
            op._need_laid()
        assert sum(t.numel() == 64 for t in op._owned()) == 2   # the memory of those laid out stays


def test_adamw_without_elements():
    op = adamw(1)
    op.params, op.grads = [torch.empty(0)], [torch.empty(0)]
    op._keep()
    for _ in range(3):
        op._need_laid()


def test_adamw_eps_has_a_finite_reciprocal():
    from paper_2406_02052_amd import _lib as L

    for eps, ok in ((2.0 ** -126, True), (2.0 ** -127, False), (1e-45, False), (0.0, False)):
        desc = L.AdamwDesc(0.9, 0.999, eps, L.PETRA_FP32, L.PETRA_FP32, 0)
        if ok:
            L.petra_adamw_query(desc, None, 0)
        else:
            with pytest.raises(L.PetraError, match="eps"):
                L.petra_adamw_query(desc, None, 0)


def test_vocab_scale_is_finite_with_its_logarithm():
    from paper_2406_02052_amd import _lib as L

    for scale, ok in ((2.0 ** 126, True), (2.0 ** 127, False), (3e38, False), (1e-44, True)):
        if ok:
            VocabLoss(4, 8, 8, scale=scale, device="cpu")
        else:
            with pytest.raises(L.PetraError, match="scale"):
                VocabLoss(4, 8, 8, scale=scale, device="cpu")
