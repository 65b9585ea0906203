"""The calls that fit a model to tasks together with the head, as a training and a decoding step use them.
Training: activations -> dropout -> adapted projection (its adaptors read the dropped-out rows) -> residual norm -> the head's window log-likelihood -> policy or preference
loss -> the head's gradients -> the norm's -> the projection's -> the dropout's -> clipping. Every stage is compared with the fp64 oracle on that stage's own inputs as
the device holds them; the head's gradients as a whole by the bar of their own test (relative L2 error 5e-3).
Decoding: adapted projection -> norm -> draft, some rows without adaptor; eager and replayed from a graph."""
import numpy as np
import pytest
import torch

from oracle import mtpc_oracle as orc
from oracle import mtpc_oracle_grad as og
from oracle import mtpc_oracle_tune as tu
from paper_2511_11346_b200 import binding as B
from paper_2511_11346_b200 import inputs as I
from paper_2511_11346_b200 import runner as R

pytestmark = pytest.mark.gpu


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def near(got, want, rel):
    got, want = host(got).reshape(want.shape), want
    assert np.linalg.norm(got - want) <= rel * np.linalg.norm(want) + 1e-30


@pytest.mark.parametrize("family,n,r,v,d,loss", [(I.CP, 4, 8, 256, 256, "policy"), (I.HMM, 3, 4, 320, 128, "preference")])
def test_training_step(family, n, r, v, d, loss):
    lengths, wide, k, S = [41, 60, 1, 38], 192, 12, 2
    T = sum(lengths)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device="cuda")
    wl = I.make_workload("tune", I.HeadShape(family, n, r, v, d), T, seed=91 + d, weight_std=0.1)
    dh = R.DeviceHead(wl)
    g = torch.Generator(device="cuda").manual_seed(6)
    new = lambda *s, std=1.0: (torch.randn(s, device="cuda", generator=g) * std).bfloat16()  # noqa: E731
    x, W, A, Bf, trunk = new(T, wide), new(d, wide, std=0.1), new(S, d, k, std=0.1), new(S, k, wide, std=0.1), new(T, d)
    scale, weight = torch.tensor([0.5, 2.0], device="cuda"), 1 + 0.1 * torch.randn(d, device="cuda", generator=g)
    task = torch.repeat_interleave(torch.tensor([0, 1, -1, 0], device="cuda"), torch.tensor(lengths, device="cuda")).to(torch.int32)
    rng = torch.tensor([77, 3], dtype=torch.int64, device="cuda")
    targets = torch.from_numpy(wl.targets).cuda()
    mask = torch.rand(T, device="cuda", generator=g) < 0.8

    x_low = R.dropout(x, 0.25, rng, offset=1)
    y, low = R.adapted_projection(x, W, A, Bf, scale, task, x_low=x_low)
    hidden, total = R.residual_rmsnorm(y, trunk, weight)
    logp = dh.window_logprob(hidden=hidden, targets=targets)
    ref = logp + 0.1 * torch.randn(T, device="cuda", generator=g)
    if loss == "policy":
        old, a = logp + 0.2 * torch.randn(T, device="cuda", generator=g), torch.randn(4, device="cuda", generator=g)
        out = dh.window_policy_backward(old, ref, a, offsets, 0.2, 0.28, beta=0.05, mask=mask, by_sequence=True, hidden=hidden, targets=targets)
        f = lambda z: float(np.float32(z))  # noqa: E731
        want, stats, d_logp, _ = tu.policy_loss(host(logp), host(old), host(ref), host(a), offsets.tolist(), f(0.2), f(0.28), f(0.05), mask.cpu().numpy(), True)
        near(out["stats"], stats, 1e-5)
    else:
        out = dh.window_preference_backward(ref, offsets, beta=0.4, smoothing=0.1, mask=mask, hidden=hidden, targets=targets)
        want, h, d_logp = tu.preference_loss(host(logp), host(ref), offsets.tolist(), float(np.float32(0.4)), float(np.float32(0.1)), mask.cpu().numpy())
        near(out["h"], h, 1e-6)
    assert dh.head.mtpc_get_status() == 0 and abs(out["loss"].item() - want) <= 1e-5 * (1 + abs(want))
    near(out["d_logp"], d_logp, 1e-5)
    d_y, d_weight = R.residual_rmsnorm_backward(total, weight, out["dh"], dtype=torch.bfloat16)
    back = R.adapted_projection_backward(x, W, A, Bf, low, d_y, scale, task, x_low=x_low)
    d_x = R.dropout(back["d_x_low"], 0.25, rng, offset=1, residual=back["d_x"])

    assert np.array_equal(host(x_low) != 0, tu.dropout_kept(T, wide, 0.25, 77, 4) & (host(x) != 0))
    y_ref, low_ref, _, _ = tu.adapted_projection(host(x), host(W), host(A), host(Bf), host(scale), task.cpu().numpy(), host(x_low))
    near(y, y_ref, 3e-3)
    near(low, low_ref, 1e-5)
    lp = orc.window_logprob(family, host(hidden), wl.W_emit_q, wl.W_sum_q, wl.T_static, wl.targets)
    assert np.abs(host(logp) - lp).max() <= 2e-3
    ref_grads = og.window_logprob_grad(family, host(hidden), wl.W_emit_q, wl.W_sum_q, wl.T_static, wl.targets, host(out["d_logp"]).astype(np.float32))
    for key in ("dh", "dW_emit", "dW_sum"):
        near(out[key], ref_grads[key], 5e-3)
    r_ = tu.adapted_projection_grad(host(x_low), host(W), host(A), host(Bf), host(scale), task.cpu().numpy(), host(low), host(d_y))
    near(back["d_x"], r_["d_x_base"], 3e-3)
    near(back["d_x_low"], r_["d_x_low"], 3e-3)
    near(back["dA"], r_["dA"], 1e-5)
    near(back["dB"], r_["dB"], 1e-5)
    near(d_x, tu.dropout(host(back["d_x_low"]), 0.25, 77, 4, host(back["d_x"])), 3e-3)
    norm = torch.empty(1, device="cuda")
    grads = [back["dA"], back["dB"], d_weight, out["dW_emit"], out["dW_sum"]]
    size = float(sum((t.double() ** 2).sum() for t in grads)) ** 0.5
    B.GradientList(grads).mtpc_clip_gradients(0.5 * size, norm)
    assert abs(norm.item() - size) <= 1e-6 * size
    dh.close()


def test_the_whole_step_by_differences():
    """The loss of the step above moves along a direction of A and B as their gradients say: central differences of whole steps. The directions are steps of the
    factors' own grid (bf16) large enough that the roundings of the activations (2^-9 of them, of random sign, through some hundred positions) stay below a tenth of them."""
    n, r, v, d, T, k, S = 4, 8, 256, 256, 120, 8, 2
    wl = I.make_workload("tune", I.HeadShape(I.CP, n, r, v, d), T, seed=17, weight_std=0.1)
    dh = R.DeviceHead(wl)
    g = torch.Generator(device="cuda").manual_seed(4)
    new = lambda *s, std=1.0: (torch.randn(s, device="cuda", generator=g) * std).bfloat16()  # noqa: E731
    x, W, A, Bf = new(T, 128), new(d, 128, std=0.09), new(S, d, k, std=0.125), new(S, k, 128, std=0.125)
    task = (torch.arange(T, device="cuda") // 30 % 2).to(torch.int32)
    offsets = torch.tensor([0, 30, 60, 90, 120], dtype=torch.int32, device="cuda")
    weight, targets = torch.ones(d, device="cuda"), torch.from_numpy(wl.targets).cuda()

    def step(A_, B_):
        y, low = R.adapted_projection(x, W, A_, B_, None, task)
        hidden, total = R.residual_rmsnorm(y, None, weight)
        return y, low, hidden, total, dh.window_logprob(hidden=hidden, targets=targets)
    y, low, hidden, total, logp = step(A, Bf)
    ref = logp.clone()
    out = dh.window_preference_backward(ref, offsets, beta=0.05, hidden=hidden, targets=targets)
    d_y, _ = R.residual_rmsnorm_backward(total, weight, out["dh"], dtype=torch.bfloat16)
    back = R.adapted_projection_backward(x, W, A, Bf, low, d_y, None, task)

    def loss(A_, B_):
        value = tu.preference_loss(host(step(A_, B_)[4]), host(ref), offsets.tolist(), 0.05)[0]
        return value
    for name, t, grad in (("A", A, back["dA"]), ("B", Bf, back["dB"])):
        by = torch.sign(grad) * 2.0 ** -6                    # along the gradient: the largest change for its size
        up, down = (t.float() + by).bfloat16(), (t.float() - by).bfloat16()
        moved = (up.double() - down.double())
        said = float((grad.double() * moved).sum())
        args = (lambda z: (z, Bf)) if name == "A" else (lambda z: (A, z))
        seen = loss(*args(up)) - loss(*args(down))
        assert said > 0 and abs(seen - said) <= 0.25 * said, (name, seen, said)
    dh.close()


def test_decoding_steps_eager_and_from_a_graph():
    n, r, v, d, P, S, k = 4, 8, 320, 256, 6, 4, 16
    wl = I.make_workload("decode", I.HeadShape(I.CP, n, r, v, d), P, seed=31, weight_std=0.1)
    dh = R.DeviceHead(wl, max_positions=P, max_wpp=1)
    g = torch.Generator(device="cuda").manual_seed(8)
    new = lambda *s, std=1.0: (torch.randn(s, device="cuda", generator=g) * std).bfloat16()  # noqa: E731
    W, A, Bf, x = new(d, d, std=0.06), new(S, d, k, std=0.1), new(S, k, d, std=0.06), new(P, d)
    task = torch.tensor([2, -1, 0, 3, 3, -1], dtype=torch.int32, device="cuda")
    u, weight = torch.rand(P, 2 * n, device="cuda", generator=g), torch.ones(d, device="cuda")
    y, hidden = torch.empty_like(x), torch.empty_like(x)
    drafted, prefix = torch.empty(P, n, dtype=torch.int32, device="cuda"), torch.empty(P, n, device="cuda")

    def step():
        B.mtpc_adapted_projection(x, W, A, Bf, None, task, y)
        B.mtpc_residual_rmsnorm(y, x, weight, 1e-5, hidden)
        dh.head.mtpc_draft_sample_prefix(hidden, 1, u, drafted, prefix)
    step()
    want = [t.clone() for t in (y, hidden, drafted, prefix)]
    near(y, tu.adapted_projection(host(x), host(W), host(A), host(Bf), None, task.cpu().numpy())[0], 3e-3)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in (y, hidden, drafted, prefix):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((y, hidden, drafted, prefix), want)) and dh.head.mtpc_get_status() == 0
    # rows without adaptor are those of the verifier: as with no adaptors at all
    plain = torch.empty_like(y)
    B.mtpc_adapted_projection(x, W, A, Bf, None, torch.full_like(task, -1), plain)
    assert torch.equal(plain[task < 0], y[task < 0]) and not torch.equal(plain[task >= 0], y[task >= 0])
    dh.close()


def test_the_first_calls_of_a_process_may_be_captured():
    """(in a process of its own: nothing has run before)"""
    import subprocess
    import sys
    code = """
import torch
from paper_2511_11346_b200 import binding as B
bf = torch.bfloat16
g = torch.Generator(device="cuda").manual_seed(1)
new = lambda *s: torch.randn(s, device="cuda", generator=g).to(bf)
W, A, Bf, rng = new(96, 64), new(2, 96, 16), new(2, 16, 64), torch.tensor([1, 2], device="cuda")
sets = []
for T in (1, 20, 300):
    sets.append((new(T, 64), new(T, 96), (torch.arange(T, device="cuda") % 3 - 1).int(), torch.zeros(T, 96, device="cuda", dtype=bf), torch.zeros(T, 16, device="cuda"),
                 torch.zeros(T, 64, device="cuda", dtype=bf), torch.zeros(2, 96, 16, device="cuda"), torch.zeros(2, 16, 64, device="cuda")))
logp, offsets = -torch.rand(70000, device="cuda", generator=g), torch.tensor([0, 30, 500, 600, 700, 70000, 70000], dtype=torch.int32, device="cuda")
losses, grads = torch.zeros(4, device="cuda"), torch.zeros(4, 70000, device="cuda")

def calls():
    for x, d_out, which, out, low, d_x, dA, dB in sets:
        B.mtpc_adapted_projection(x, W, A, Bf, None, which, out, out_low=low)
        B.mtpc_adapted_projection_backward(x, W, A, Bf, None, which, low, d_out, d_x, dA, dB)
        B.mtpc_dropout(d_x, d_x, 0.5, rng)
    for i, n in enumerate((700, 70000)):
        of = offsets if n == 70000 else offsets[:5]
        B.mtpc_policy_loss(logp[:n], logp[:n] - 0.1, None, torch.ones(of.numel() - 1, device="cuda"), of, 0.2, 0.2, 0.0, losses[2 * i:2 * i + 1], grads[2 * i][:n])
        B.mtpc_preference_loss(logp[:n], logp[:n] * 0.9, of, 0.1, losses[2 * i + 1:2 * i + 2], grads[2 * i + 1][:n])
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    calls()
graph.replay()
torch.cuda.synchronize()
first = [t.clone() for s in sets for t in s[3:]] + [losses.clone(), grads.clone()]
calls()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(first, [t for s in sets for t in s[3:]] + [losses, grads]))
# the one row of the first set has no adaptor: its low, dA and dB are zeros by definition
assert [bool(t.any()) for t in first] == [True, False, True, False, False] + [True] * 12
"""
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


def test_calls_on_three_streams_at_once():
    """Few rows, tiles and gradients beside each other, again and again: every call gives what it gives alone."""
    g = torch.Generator(device="cuda").manual_seed(8)
    new = lambda *s: torch.randn(s, device="cuda", generator=g).bfloat16()  # noqa: E731
    d, m, S = 1024, 768, 4
    jobs = []
    for T, k in ((1, 16), (40, 64), (700, 16), (1500, 64)):
        x, W, A, Bf, d_out = new(T, d), new(m, d), new(S, m, k), new(S, k, d), new(T, m)
        which = (torch.arange(T, device="cuda") % (S + 1) - 1).int()
        low = torch.randn(T, k, device="cuda", generator=g)

        def job(x=x, W=W, A=A, Bf=Bf, d_out=d_out, which=which, low=low):
            out, kept = R.adapted_projection(x, W, A, Bf, None, which)
            return [out, kept, *(t for t in R.adapted_projection_backward(x, W, A, Bf, low, d_out, None, which).values() if t is not None)]
        jobs.append((job, job()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for i in range(48):
        with torch.cuda.stream(streams[i % 3]):
            got.append((i % 4, jobs[i % 4][0]()))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for which, results in got for a, b in zip(results, jobs[which][1]))
