"""The norm of many gradients and clipping against the fp64 oracle. Squares and sums are fp64 (2^-53 relative each, a million times less than what follows):
the norm is rounded to fp32 once, U32 = 2^-24. A scaled gradient is the product with a ratio rounded to fp32, rounded once itself: 2 u, and the output's
half step; below the normal range half the smallest step instead."""
import numpy as np
import pytest
import torch

from oracle import mtpc_oracle_step as st
from paper_2511_11346_b200 import binding as B

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
SLACK = 1 + 2.0 ** -20
F, H = torch.float32, torch.bfloat16


def host(t):
    return t.detach().double().cpu().numpy().reshape(-1)


def check(grads, outs, max_norm):
    given = [host(g) for g in grads]
    plan = B.GradientList(grads, outs)
    norm = torch.full((1,), float("nan"), device="cuda")
    plan.mtpc_clip_gradients(max_norm, norm)
    want, scaled = st.clip(given, float(np.float32(max_norm)))
    if want > 3.4028236e38:                                                # what fp32 cannot hold is infinity
        assert norm.item() == float("inf")
    else:
        assert abs(norm.item() - want) <= U32 * want * SLACK + 2.0 ** -150
    for g, x, before, y in zip(grads, grads if outs is None else outs, given, scaled):
        if x is None:
            assert (host(g) == before).all()
            continue
        u, tiny = torch.finfo(x.dtype).eps / 2, (2.0 ** -134 if x.dtype is H else 2.0 ** -150)
        first = 0.0 if want <= float(np.float32(max_norm)) else 2 * U32                # not scaled: copied
        assert (np.abs(host(x) - y) <= (first + u) * np.abs(y) * SLACK + tiny).all()
    return norm.item()


def tensors(sizes, dtypes, std=1.0, off=0):
    return [(torch.randn(s + off, device="cuda") * std).to(t)[off:] for s, t in zip(sizes, dtypes * len(sizes))]


@pytest.mark.parametrize("sizes", [[1], [8], [7, 9], [8192], [8193], [8200, 1, 16384], [100003, 3, 0, 5], [1] * 700, [3000000, 17]])
@pytest.mark.parametrize("types", [[F], [H], [F, H]])
@pytest.mark.parametrize("off", [0, 1, 3])
def test_clipping(sizes, types, off):
    torch.manual_seed(sum(sizes) + off)
    grads = tensors(sizes, types, off=off)
    count = sum(sizes)
    for max_norm in (0.5 * count ** 0.5, 4.0 * count ** 0.5, float("inf")):
        check(grads, [torch.empty_like(g) for g in grads], max_norm)                       # elsewhere
        check(grads, [torch.empty(g.numel() + 1, device="cuda")[1:] for g in grads], max_norm)      # as fp32, differently aligned
        check(grads, [torch.empty(g.numel(), dtype=H, device="cuda") for g in grads], max_norm)
        check([g.clone() for g in grads], None, max_norm)                                  # in place
    check(grads, [None] * len(grads), 1.0)
    check(grads, [None if i % 2 else torch.empty_like(g) for i, g in enumerate(grads)], 1.0)


def test_packed_tensors_leave_what_is_beside_them():
    torch.manual_seed(1)
    sizes = [1 + (i * 7919) % 4099 for i in range(200)]
    for t in (F, H):
        flat = torch.randn(sum(sizes) + 20, device="cuda").to(t)
        out = torch.full_like(flat, 7.0)
        inner = flat[3:3 + sum(sizes)], out[3:3 + sum(sizes)]
        check(list(torch.split(inner[0], sizes)), list(torch.split(inner[1], sizes)), 1.0)
        assert (out[:3] == 7).all() and (out[3 + sum(sizes):] == 7).all()
        copy = flat.clone()
        check(list(torch.split(copy[3:3 + sum(sizes)], sizes)), None, 1.0)
        assert torch.equal(copy[:3], flat[:3]) and torch.equal(copy[3 + sum(sizes):], flat[3 + sum(sizes):])


def test_matrices_and_the_same_gradient_twice():
    g = torch.randn(30, 50, device="cuda")
    check([g, g], [torch.empty_like(g), None], 2.0)                        # counted twice, written once
    with pytest.raises(B.MtpcError):
        B.GradientList([g, g])                                             # in place twice
    with pytest.raises(B.MtpcError):
        B.GradientList([g.t()])
    with pytest.raises(B.MtpcError):
        B.GradientList([g], [torch.empty(31, 50, device="cuda")])
    with pytest.raises(B.MtpcError):
        B.GradientList([g.double()])
    with pytest.raises(B.MtpcError):
        B.GradientList([g, g.cpu()])
    plan = B.GradientList([g])
    for bad in (0.0, -1.0, float("nan")):
        with pytest.raises(B.MtpcError):
            plan.mtpc_clip_gradients(bad, torch.empty(1, device="cuda"))
    with pytest.raises(B.MtpcError):
        plan.mtpc_clip_gradients(1.0, torch.empty(2, device="cuda"))


def test_extreme_values():
    big = [torch.full((5000,), 1e38, device="cuda"), torch.full((3,), -3e38, device="cuda")]      # the norm exceeds fp32
    norm = torch.zeros(1, device="cuda")
    outs = [torch.empty_like(g) for g in big]
    B.GradientList(big, outs).mtpc_clip_gradients(1e-3, norm)
    want, scaled = st.clip([host(g) for g in big], float(np.float32(1e-3)))
    assert torch.isinf(norm).all() and want > 3.4e38
    assert all((np.abs(host(o) - y) <= 3 * U32 * np.abs(y) * SLACK).all() for o, y in zip(outs, scaled))
    check([torch.full((100,), 1e38, device="cuda")], None, 1.0)
    check([torch.full((100,), 1e-30, device="cuda")], None, 1.0)            # squares below fp32's range
    check([torch.full((100,), 1e-30, device="cuda")], None, 1e-30)
    check([torch.zeros(100, device="cuda"), torch.zeros(9, dtype=H, device="cuda")], None, 1.0)
    check([torch.zeros(0, device="cuda")], None, 1.0)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_norm_that_is_no_number_scales_nothing(bad):
    g = [torch.randn(20000, device="cuda"), torch.randn(77, device="cuda").to(H)]
    g[0][12345] = bad
    before = [x.clone() for x in g]
    out, norm = [torch.empty_like(x) for x in g], torch.zeros(1, device="cuda")
    B.GradientList(g, out).mtpc_clip_gradients(1.0, norm)
    assert not torch.isfinite(norm).any()
    B.GradientList(g).mtpc_clip_gradients(1.0, norm)
    assert all(torch.equal(torch.nan_to_num(x, nan=3.0), torch.nan_to_num(y, nan=3.0)) for a in (g, out) for x, y in zip(a, before))


def test_same_bits_call_after_call_on_streams_and_in_graphs():
    torch.manual_seed(2)
    grads = tensors([200000, 33, 70001], [F, H, F])
    outs = [torch.empty_like(g) for g in grads]
    plan, norm = B.GradientList(grads, outs), torch.zeros(1, device="cuda")
    plan.mtpc_clip_gradients(1.0, norm)
    want = [o.clone() for o in outs] + [norm.clone()]
    others = [(B.GradientList(grads, o), o, torch.zeros(1, device="cuda"), torch.cuda.Stream()) for o in ([torch.empty_like(g) for g in grads] for _ in range(3))]
    torch.cuda.synchronize()
    for _ in range(5):                                                   # three lists of the same gradients at once
        for p, o, nrm, s in others:
            p.mtpc_clip_gradients(1.0, nrm, stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for _, o, nrm, _ in others for a, b in zip(o + [nrm], want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.mtpc_clip_gradients(1.0, norm)
    for _ in range(3):
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs + [norm], want))


def test_a_tensor_of_more_than_32_bits():
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GB")
    g = torch.zeros(2 ** 32 + 9, dtype=H, device="cuda")
    g[0], g[2 ** 31], g[2 ** 32 + 8] = 2.0, 4.0, 4.0
    norm = torch.zeros(1, device="cuda")
    B.GradientList([g]).mtpc_clip_gradients(3.0, norm)
    assert norm.item() == 6.0 and g[0] == 1.0 and g[2 ** 31] == 2.0 and g[2 ** 32 + 8] == 2.0 and g.count_nonzero() == 3
