"""The calls beside the head together with it, as a training and a decoding step use them.
Training: bytes -> embedding -> residual norm -> the head's loss and gradients -> the norm's gradient -> the embedding's -> clipping. Every stage is
compared with the fp64 oracle on that stage's own inputs as the device holds them, by the stage's own bars (the embedding's, norm's and
clipping's in their test files, the head's gradients as a whole in test_gpu_backward.py: relative L2 error 5e-3).
Decoding: draft -> acceptance -> the accepted byte's embedding -> residual norm -> the next draft; eager and replayed from a graph."""
import numpy as np
import pytest
import torch

from oracle import mtpc_oracle_grad as og
from oracle import mtpc_oracle_step as st
from paper_2511_11346_b200 import binding as B
from paper_2511_11346_b200 import inputs as I
from paper_2511_11346_b200 import runner as R

pytestmark = pytest.mark.gpu

U32, EPS = 2.0 ** -24, 1e-5


def host(t):
    return t.detach().double().cpu().numpy()


def near(got, want, size, units):
    assert (np.abs(host(got) - want) <= units * U32 * size + 2.0 ** -133).all()


@pytest.mark.parametrize("family,n,r,v,d,N,L", [(I.CP, 4, 8, 256, 256, 3, 41), (I.HMM, 3, 4, 320, 128, 1, 150), (I.BTREE, 4, 4, 64, 64, 2, 33)])
def test_training_step(family, n, r, v, d, N, L):
    wl = I.make_workload("chain", I.HeadShape(family, n, r, v, d), N * L, seed=77 + d, weight_std=0.1)
    dh = R.DeviceHead(wl)
    g = torch.Generator(device="cuda").manual_seed(5)
    T = N * L
    tokens = torch.randint(0, v, (T,), device="cuda", generator=g, dtype=torch.int32)
    tokens[L - 3:L] = -1                                                   # padding behind the first text
    table = torch.randn(v, d, device="cuda", generator=g).bfloat16()
    trunk = torch.randn(T, d, device="cuda", generator=g).bfloat16()       # what the layers before the last addition gave
    weight = 1 + 0.1 * torch.randn(d, device="cuda", generator=g)
    targets = torch.from_numpy(wl.targets).cuda()
    targets[L - 3:L] = -1
    out = None
    for max_norm in (1e-2, 1e6):                                           # the second step writes the first one's buffers
        x = R.embed(tokens, table, scale=d ** 0.5)
        hidden, total = R.residual_rmsnorm(x, trunk, weight, eps=EPS)
        out = dh.window_loss_backward(N, L, 0.9, hidden=hidden, targets=targets, out=out, max_norm=max_norm)
        d_x, d_weight = R.residual_rmsnorm_backward(total, weight, out["dh"], d_total=None, eps=EPS, dtype=torch.float32)
        d_table = R.embed_backward(tokens, d_x, v, scale=d ** 0.5)
        assert dh.head.mtpc_get_status() == 0

        assert (np.abs(host(x) - st.embed(tokens.cpu().numpy(), host(table), float(np.float32(d ** 0.5)))) <= 2.0 ** -8 * 1.001 * np.abs(host(x))).all()
        s_ref, h_ref = st.rmsnorm(host(x), host(trunk), host(weight), float(np.float32(EPS)))
        assert (np.abs(host(total) - s_ref) <= 2.0 ** -8 * 1.001 * np.abs(s_ref)).all()
        assert (np.abs(host(hidden) - h_ref) <= (2.0 ** -8 + 33 * U32) * np.abs(h_ref)).all()
        ref = og.composite_loss_grad(family, host(hidden), wl.W_emit_q, wl.W_sum_q, wl.T_static, targets.cpu().numpy(), N, 0.9)
        assert abs(float(out["loss"].cpu()[0]) - ref["loss"]) <= 2e-3 * n
        names = ["dW_emit", "dW_sum"] + (["dT_static"] if family == I.HMM else [])
        norm = float(np.sqrt(sum((ref[k] ** 2).sum() for k in names)))
        by = min(1.0, max_norm / norm)
        assert abs(float(out["grad_norm"].cpu()[0]) - norm) <= 5e-3 * norm
        for k in ["dh"] + names:
            want = ref[k] * (1.0 if k == "dh" else by)
            got = host(out[k]).reshape(want.shape)
            assert np.linalg.norm(got - want) <= (5e-3 if by == 1.0 or k == "dh" else 1e-2) * np.linalg.norm(want), k
        dx_ref, dw_ref, size, size_w = st.rmsnorm_grad(host(total), host(weight), float(np.float32(EPS)), host(out["dh"]))
        near(d_x, dx_ref, size, 141)
        near(d_weight, dw_ref, size_w, -(-T // 148) + 110)
        t_ref, t_size = st.embed_grad(tokens.cpu().numpy(), host(d_x), float(np.float32(d ** 0.5)), v)
        near(d_table, t_ref, t_size, T + 3)
    dh.close()


def test_buffers_of_a_call_with_other_sizes_are_refused():
    wl = I.make_workload("chain", I.HeadShape(I.CP, 4, 8, 256, 256), 24, seed=3, weight_std=0.1)
    dh = R.DeviceHead(wl)
    hidden, targets = dh.hidden_device(), torch.from_numpy(wl.targets).cuda()
    out = dh.window_loss_backward(2, 8, 0.9, hidden=hidden[:16], targets=targets[:16], max_norm=1.0)
    with pytest.raises(B.MtpcError):
        dh.window_loss_backward(3, 8, 0.9, hidden=hidden, targets=targets, out=out, max_norm=1.0)
    again = dh.window_loss_backward(2, 8, 0.9, hidden=hidden[8:], targets=targets[8:], out=out, max_norm=1.0)
    assert again is out
    dh.close()


def test_training_step_of_a_factored_head_with_a_tied_table():
    n, r, v, d, k, N, L = 3, 4, 320, 128, 16, 2, 60
    T = N * L
    wl = I.make_workload("tied", I.HeadShape(I.CP, n, r, v, d), T, seed=9, weight_std=0.1)
    Wb, A, Bm = I.lowrank_parameters(n, r, v, d, k, seed=10, weight_std=0.1, adaptor_std=0.1)
    dh = R.DeviceHead(wl, lowrank=(Wb, A, Bm))
    table = dh.lowrank[0][0]                                               # the embedding is the first slot's unembedding
    tokens = torch.randint(0, v, (T,), device="cuda", dtype=torch.int32)
    weight, targets = torch.ones(d, device="cuda"), torch.from_numpy(wl.targets).cuda()
    hidden, total = R.residual_rmsnorm(R.embed(tokens, table, scale=3.0), None, weight)
    f32 = dict(dtype=torch.float32, device="cuda")
    dW_base, dA, dB = torch.empty((n, v, d), **f32), torch.empty((n, r, v, k), **f32), torch.empty((n, r, k, d), **f32)
    d_hidden, dW_sum, slot, loss, norm = torch.empty((T, d), **f32), torch.empty((r, d), **f32), torch.empty(n, **f32), torch.empty(1, **f32), torch.empty(1, **f32)
    dh.head.mtpc_lowrank_window_loss_backward(hidden, targets, N, L, 0.9, slot, loss, d_hidden, dW_base, dA, dB, dW_sum)
    d_x, d_weight = R.residual_rmsnorm_backward(total, weight, d_hidden, dtype=torch.float32)
    own = dW_base.clone()
    R.embed_backward(tokens, d_x, v, scale=3.0, into=dW_base[0])
    want, size = st.embed_grad(tokens.cpu().numpy(), host(d_x), 3.0, v, start=host(own[0]))
    near(dW_base[0], want, size, T + 3)
    assert torch.equal(dW_base[1:], own[1:])
    grads = [dW_base, dA, dB, dW_sum, d_weight]
    before = [host(x) for x in grads]
    B.GradientList(grads).mtpc_clip_gradients(0.05, norm)
    ref, scaled = st.clip(before, float(np.float32(0.05)))
    assert ref > 0.05 and abs(norm.item() - ref) <= U32 * ref * 1.001
    for x, y in zip(grads, scaled):
        assert (np.abs(host(x) - y) <= 3 * U32 * np.abs(y) + 2.0 ** -150).all()
    assert dh.head.mtpc_get_status() == 0
    dh.close()


def test_decoding_steps_eager_and_from_a_graph():
    n, r, v, d, P, steps = 4, 8, 320, 256, 5, 6
    wl = I.make_workload("decode", I.HeadShape(I.CP, n, r, v, d), P, seed=31, weight_std=0.1)
    dh = R.DeviceHead(wl, max_positions=P, max_wpp=1)
    g = torch.Generator(device="cuda").manual_seed(7)
    table = torch.randn(v, d, device="cuda", generator=g).bfloat16()
    weight = 1 + 0.1 * torch.randn(d, device="cuda", generator=g)
    draws = [(torch.rand(P, 2 * n, device="cuda", generator=g), torch.rand(P, n + 1, device="cuda", generator=g),
              torch.softmax(2 * torch.randn(P, n + 1, v, device="cuda", generator=g), dim=-1)) for _ in range(steps)]
    start = torch.randn(P, d, device="cuda", generator=g).bfloat16()
    u, au, target = (x.clone() for x in draws[0])
    stream, hidden, x = start.clone(), torch.empty_like(start), torch.empty_like(start)
    drafted, prefix = torch.empty(P, n, dtype=torch.int32, device="cuda"), torch.empty(P, n, device="cuda")
    accepted, nxt, status = (torch.zeros(k, dtype=torch.int32, device="cuda") for k in (P, P, 1))

    def step():
        B.mtpc_residual_rmsnorm(stream, None, weight, EPS, hidden)
        dh.head.mtpc_draft_sample_prefix(hidden, 1, u, drafted, prefix)
        dh.head.mtpc_speculative_accept(P, 1, drafted, prefix, target, au, accepted, nxt)
        B.mtpc_embed(nxt, table, x, scale=0.5, out_status=status)
        B.mtpc_residual_rmsnorm(x, stream, weight, EPS, hidden, out_sum=stream)            # in place: the stream goes on

    def run(call):
        stream.copy_(start)
        seen = []
        for a, b, c in draws:
            u.copy_(a)
            au.copy_(b)
            target.copy_(c)
            call()
            seen.append((drafted.clone(), accepted.clone(), nxt.clone(), hidden.clone(), stream.clone()))
        torch.cuda.synchronize()
        return seen
    eager = run(step)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    replayed = run(graph.replay)
    assert all(torch.equal(a, b) for p, q in zip(eager, replayed) for a, b in zip(p, q))
    assert status.item() == 0 and dh.head.mtpc_get_status() == 0
    assert len({tuple(s[2].tolist()) for s in eager}) > 1
    # the last step's stream is its last addition
    s_ref = host(eager[-2][4]) + host(table)[eager[-1][2].cpu().numpy()] * 0.5
    assert (np.abs(host(eager[-1][4]) - s_ref) <= 2 * 2.0 ** -8 * 1.001 * (np.abs(s_ref) + np.abs(host(table)[eager[-1][2].cpu().numpy()]))).all()
    dh.close()
