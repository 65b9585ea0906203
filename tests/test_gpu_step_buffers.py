"""A training call that writes the buffers of an earlier one again, with clipping: against a call that has buffers of its own."""
import pytest
import torch

from paper_2511_11346_b200 import binding as B
from paper_2511_11346_b200 import inputs as I
from paper_2511_11346_b200 import runner as R

pytestmark = pytest.mark.gpu

N, L = 2, 12


def head(family=I.HMM, seed=3):
    wl = I.make_workload("buffers", I.HeadShape(family, 4, 8, 64, 64), N * L, seed=seed, weight_std=0.1)
    dh = R.DeviceHead(wl)
    hidden, targets = dh.hidden_device(), torch.from_numpy(wl.targets).cuda()
    return dh, lambda gamma=0.9, **kw: dh.window_loss_backward(N, L, gamma, hidden=hidden, targets=targets, **kw)


def test_buffers_of_another_type_or_place_are_refused():
    dh, call = head()
    for key, other in (("dW_emit", lambda t: t.bfloat16()), ("dW_sum", lambda t: t.cpu()), ("dh", lambda t: t.t().contiguous().t()), ("slot_loss", lambda t: None)):
        out = call()
        out[key] = other(out[key])
        with pytest.raises(B.MtpcError):
            call(out=out)
    dh.close()


@pytest.mark.parametrize("key", ["dW_emit", "dW_sum", "dT_static"])
def test_a_buffer_that_is_not_the_lists_is_refused(key):
    """The list of a dict holds the addresses that it was made of. Another buffer in its place would be written, but not be clipped."""
    dh, call = head()
    out = call(max_norm=1e-3)
    kept = {k: t.clone() for k, t in out.items() if isinstance(t, torch.Tensor)}
    old, new = out[key], torch.full_like(out[key], 7.0)
    out[key] = new
    with pytest.raises(B.MtpcError):
        call(0.5, out=out, max_norm=1e-3)
    torch.cuda.synchronize()
    assert (new == 7).all() and torch.equal(old, kept[key]) and all(torch.equal(out[k], t) for k, t in kept.items() if k != key)       # nothing was written
    # without the list they are buffers as any others
    fresh = call(0.5, out={k: t for k, t in out.items() if k not in ("gradients", "grad_norm")}, max_norm=1e-3)
    want = call(0.5, max_norm=1e-3)
    assert fresh[key] is new and torch.equal(fresh["grad_norm"], want["grad_norm"]) and fresh["grad_norm"].item() > 1e-3
    assert all(torch.equal(fresh[k], want[k]) for k in ("dW_emit", "dW_sum", "dT_static"))
    # back in its place: the list's again; another tensor on the same memory is the same buffer
    out[key] = old.view(old.shape)
    assert call(0.5, out=out, max_norm=1e-3) is out and torch.equal(out[key], want[key]) and torch.equal(out["grad_norm"], want["grad_norm"])
    dh.close()


def test_the_norm_of_an_earlier_step_does_not_stay():
    dh, call = head(I.CP)
    out = call(max_norm=1e-3)
    norm = out["grad_norm"]
    assert norm.item() > 1e-3
    assert call(0.5, out=out) is out and "grad_norm" not in out
    want = call(0.5, max_norm=1e-3)
    plain = call(0.5)
    assert all(torch.equal(out[k], plain[k]) for k in ("dW_emit", "dW_sum", "dh", "loss"))
    assert call(0.5, out=out, max_norm=1e-3)["grad_norm"] is norm and torch.equal(norm, want["grad_norm"])       # (a graph that writes it still does)
    dh.close()


def test_a_captured_step_with_clipping():
    """The list is made by an eager step; a graph of the next one serves every step after it, whatever eager steps do to the dict in between."""
    dh, _ = head()
    g = torch.Generator(device="cuda").manual_seed(1)
    hidden, targets = torch.randn(N * L, 64, device="cuda", generator=g).bfloat16(), torch.randint(0, 64, (N * L, 4), device="cuda", generator=g, dtype=torch.int32)
    hidden = hidden.to(dh.hidden_device().dtype)
    call = lambda **kw: dh.window_loss_backward(N, L, 0.9, hidden=hidden, targets=targets, **kw)  # noqa: E731
    out = call(max_norm=1e-3)
    norm = out["grad_norm"]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out=out, max_norm=1e-3)
    call(out=out)
    spare = [torch.full((1,), 5.0, device="cuda") for _ in range(64)]      # where a buffer that was let go would lie
    for turn in range(3):
        hidden.copy_(torch.randn(N * L, 64, device="cuda", generator=g))
        for k in ("dW_emit", "dW_sum", "dT_static", "dh"):
            out[k].fill_(7.0)
        norm.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = {k: t.clone() for k, t in out.items() if isinstance(t, torch.Tensor)}
        want = call(max_norm=1e-3)
        assert all(torch.equal(got[k], want[k]) for k in got) and torch.equal(norm, want["grad_norm"]) and norm.item() > 1e-3
    assert all(s.item() == 5.0 for s in spare)
    dh.close()
