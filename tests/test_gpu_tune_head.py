"""The policy loss of a head's windows with an advantage for every position: the loss's gradient and the head's gradients from it."""
import pytest
import torch

from paper_2511_11346_b200 import inputs as I
from paper_2511_11346_b200 import runner as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("by_sequence", [False, True])
def test_window_policy_backward_by_position(by_sequence):
    T = 90
    wl = I.make_workload("by position", I.HeadShape(I.CP, 4, 8, 256, 128), T, seed=5, weight_std=0.1)
    dh = R.DeviceHead(wl)
    g = torch.Generator(device="cuda").manual_seed(6)
    logp = dh.window_logprob()
    old, a = logp + 0.2 * torch.randn(T, device="cuda", generator=g), torch.randn(T, device="cuda", generator=g)
    offsets = torch.tensor([0, 20, 20, 77, 90], dtype=torch.int32, device="cuda")
    out = dh.window_policy_backward(old, None, a, offsets, by_sequence=by_sequence, by_position=True)
    want = R.policy_loss(logp, old, None, a, offsets, by_sequence=by_sequence, by_position=True)
    assert all(torch.equal(out[key], want[key]) for key in ("loss", "stats", "d_logp"))
    back = dh.window_logprob_backward(want["d_logp"])
    assert all(torch.equal(out[key], back[key]) for key in ("dh", "dW_emit", "dW_sum"))
    # an advantage that is the same all over a sequence is that sequence's
    same = torch.repeat_interleave(a[:4], torch.tensor([20, 0, 57, 13], device="cuda"))
    x, y = dh.window_policy_backward(old, None, same, offsets, by_position=True), dh.window_policy_backward(old, None, a[:4].contiguous(), offsets)
    assert torch.equal(x["d_logp"], y["d_logp"]) and torch.equal(x["loss"], y["loss"]) and dh.head.mtpc_get_status() == 0
    dh.close()
