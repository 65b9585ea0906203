"""The adaptors' gradients where their sum over the rows is cut into runs whose parts are added up at the end. Errors as for the gradients of few runs: low's three
terms are within 2^-26; an accumulator takes 512 rows at most, 64 V (V = 2^-23: a tensor core's accumulation is cut off); all fp32 additions of chunks and runs together are
fewer than T / 512 + 40, each u = 2^-24: (72 + T / 256) V of the terms' magnitudes. dB: v's error, (72 + m / 64) V, beside it."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import mtpc_oracle_tune as tu
from paper_2511_11346_b200 import binding as B

pytestmark = pytest.mark.gpu

V = 2.0 ** -23


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def runs_of(T, d, m, k, S):
    """How many runs a call is cut into, from the workspace that it asks for: behind the terms and the bitmaps lie the parts of all runs (0: one run, no parts)."""
    need, up = ctypes.c_size_t(0), lambda x: -(-x // 256) * 256
    assert B.lib().mtpc_adapted_projection_backward_workspace_bytes(T, d, m, k, S, 1, ctypes.byref(need)) == 0
    k16, blocks, tiles = -(-k // 16) * 16, -(-T // 64), -(-d // 128) + -(-m // 128)
    rest = need.value - up(T * -(-k // 32) * 128) - 2 * up(T * 3 * k16 * 2) - up(-(-blocks // 32) * S * 8)
    return rest // (S * tiles * 128 * k16 * 4)


@pytest.mark.parametrize("T,d,m,k,S", [(2001, 72, 67, 16, 2), (3001, 131, 72, 12, 1), (4001, 72, 130, 16, 1), (5003, 200, 264, 40, 1), (6005, 130, 67, 12, 1), (8001, 264, 136, 64, 1),
                                       (10001, 130, 70, 24, 3)])
@pytest.mark.parametrize("kind", ["one", "runs", "mixed", "none"])
def test_gradients_cut_into_runs(T, d, m, k, S, kind):
    assert runs_of(T, d, m, k, S) > 1
    g = torch.Generator(device="cuda").manual_seed(T + k)
    new = lambda *s, std: (torch.randn(s, device="cuda", generator=g) * std).bfloat16()  # noqa: E731
    x, W, A, Bf, d_out = new(T, d, std=1.0), new(m, d, std=0.1), new(S, m, k, std=0.1), new(S, k, d, std=0.1), new(T, m, std=0.1)
    low, scale = torch.randn(T, k, device="cuda", generator=g), 0.5 + torch.rand(S, device="cuda", generator=g)
    which = {"one": None, "none": torch.full((T,), -1, device="cuda"), "runs": torch.arange(T, device="cuda") * (S + 1) // T - 1,
             "mixed": torch.randint(-1, S, (T,), device="cuda", generator=g)}[kind]
    which = None if which is None else which.int()

    def call(want_a=True, want_b=True):
        dA, dB = (torch.full(s, 7.0, device="cuda") if wanted else None for s, wanted in (((S, m, k), want_a), ((S, k, d), want_b)))
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.mtpc_adapted_projection_backward(x if want_b else None, W, A, Bf, scale, which, low if want_a else None, d_out, None, dA, dB, out_status=status)
        assert status.item() == 0
        return dA, dB
    dA, dB = call()
    r = tu.adapted_projection_grad(host(x), host(W), host(A), host(Bf), host(scale), None if which is None else which.cpu().numpy(), host(low), host(d_out))
    assert (np.abs(host(dA) - r["dA"]) <= (72 + T / 256) * V * r["dA_size"] + 1e-30).all()
    assert (np.abs(host(dB) - r["dB"]) <= ((72 + T / 256) * V + (72 + m / 64) * V) * r["dB_size"] + 1e-30).all()
    again = call()
    assert torch.equal(dA, again[0]) and torch.equal(dB, again[1])                         # the runs are added up in their order
    assert torch.equal(call(want_b=False)[0], dA) and torch.equal(call(want_a=False)[1], dB)
    if kind == "none":
        assert not dA.any() and not dB.any()


def test_nothing_of_one_request_reaches_another_in_runs():
    """Rows of adaptor 1 and of none hold infinities and NaN: the gradients of the others are as without."""
    T, d, m, k, S = 4003, 72, 67, 16, 3
    assert runs_of(T, d, m, k, S) > 1
    g = torch.Generator(device="cuda").manual_seed(2)
    new = lambda *s: (torch.randn(s, device="cuda", generator=g) * 0.2).bfloat16()  # noqa: E731
    x, W, A, Bf, d_out, low = new(T, d), new(m, d), new(S, m, k), new(S, k, d), new(T, m), torch.randn(T, k, device="cuda", generator=g)
    which = (torch.arange(T, device="cuda") * 7 // 5 % 4 - 1).int()
    out = [torch.empty(S, m, k, device="cuda"), torch.empty(S, k, d, device="cuda")]
    B.mtpc_adapted_projection_backward(x, W, A, Bf, None, which, low, d_out, None, *out)
    other = (which == 0) | (which == 2)
    x2, g2, low2 = x.clone(), d_out.clone(), low.clone()
    x2[~other], g2[~other], low2[~other] = float("nan"), float("inf"), float("nan")
    got = [torch.empty_like(t) for t in out]
    B.mtpc_adapted_projection_backward(x2, W, A, Bf, None, which, low2, g2, None, *got)
    for i in (0, 2):
        assert all(torch.equal(a[i], b[i]) for a, b in zip(got, out))
    assert not torch.isfinite(got[0][1]).any()


def test_runs_in_a_replayed_graph():
    T, d, m, k, S = 4003, 72, 67, 16, 3
    g = torch.Generator(device="cuda").manual_seed(3)
    new = lambda *s: (torch.randn(s, device="cuda", generator=g) * 0.2).bfloat16()  # noqa: E731
    x, W, A, Bf, d_out, low = new(T, d), new(m, d), new(S, m, k), new(S, k, d), new(T, m), torch.randn(T, k, device="cuda", generator=g)
    which = (torch.arange(T, device="cuda") % 4 - 1).int()
    out = [torch.empty_like(x), torch.empty(S, m, k, device="cuda"), torch.empty(S, k, d, device="cuda")]

    def step():
        B.mtpc_adapted_projection_backward(x, W, A, Bf, None, which, low, d_out, *out)
    step()
    want = [t.clone() for t in out]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
        step()
    for t in out:
        t.fill_(7)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
