"""What an AdamW step refuses on a device, and that it goes on afterwards."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def owner(**more):
    from paper_2406_02052_amd import AdamW

    theta, grad = torch.ones(300, device="cuda"), torch.ones(300, device="cuda")
    return AdamW([theta], [grad], lr=0.5, weight_decay=0.0, **more), theta, grad


@pytest.mark.parametrize("name,wrong", [
    ("steps", lambda: torch.zeros(1, dtype=torch.int64)), ("steps", lambda: torch.zeros(1, dtype=torch.int32, device="cuda")),
    ("steps", lambda: torch.zeros(2, dtype=torch.int64, device="cuda")), ("lr", lambda: torch.zeros(1)),
    ("m", lambda: torch.zeros(320, device="cuda")), ("v", lambda: torch.zeros(320, device="cuda"))])
def test_adamw_refuses_what_its_table_does_not_know(name, wrong):
    op, theta, _ = owner()
    right = getattr(op, name)
    setattr(op, name, wrong())
    with pytest.raises(ValueError, match=name):
        op.step()
    assert (theta == 1).all() and op.steps.sum() == 0
    setattr(op, name, right)
    op.step()
    assert (theta == 0.5).all() and op.steps == 1


def test_adamw_refuses_moved_tensors():
    op, theta, grad = owner()
    op.step()
    new = theta.clone()
    theta.data = new
    with pytest.raises(ValueError, match="params"):
        op.step()
    assert (new == 0.5).all()
    op, theta, grad = owner()
    grad.data = torch.zeros(300, device="cuda")
    with pytest.raises(ValueError, match="grads"):
        op.step()
    assert (theta == 1).all()


def test_adamw_with_replaced_lr_and_steps_on_another_stream():
    """Both may be the caller's own, and the owner may be dropped at once."""
    side = torch.cuda.Stream()
    for i in range(2):
        op, theta, _ = owner()
        op.step(stream=side if i else None)
        torch.cuda.synchronize()
        op.lr, op.steps = torch.full((1,), 0.25, device="cuda"), torch.full((1,), 9, dtype=torch.int64, device="cuda")
        steps = op.steps
        side.wait_stream(torch.cuda.current_stream())
        op.step(stream=side)
        del op
        junk = [torch.full((1,), 1e30, device="cuda") for _ in range(64)]
        side.synchronize()
        # the second step as the tenth, of gradients of 1; fp32 throughout
        want = 0.5 - 0.25 * 0.19 / (1 - 0.9 ** 10) / math.sqrt(0.001999 / (1 - 0.999 ** 10))
        assert steps == 10 and ((theta - want).abs() < 1e-6).all()
        del junk


@pytest.mark.parametrize("states", ["fp32", "fp8"])
def test_adamw_least_eps_leaves_parameters_without_gradients(states):
    op, theta, grad = owner(states=states, eps=2.0 ** -126)
    grad[:100] = 0.0
    op.step(rng=torch.tensor([1, 2], device="cuda"))
    assert (theta[:100] == 1).all() and ((theta[100:] - 0.5).abs() < 1e-6).all()


def test_vocab_largest_scale():
    from paper_2406_02052_amd import VocabLoss

    x, w, t = torch.zeros(4, 8, device="cuda"), torch.ones(5, 8, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    loss, lse, dx, dw = torch.empty(4, device="cuda"), torch.empty(4, device="cuda"), torch.empty_like(x), torch.empty_like(w)
    VocabLoss(4, 8, 5, "fp32", scale=2.0 ** 126).gradient(x, w, t, loss, lse, dx, dw)
    assert ((loss - math.log(5)).abs() < 1e-6).all() and torch.isfinite(dx).all()
