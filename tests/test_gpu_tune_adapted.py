"""The projection with adaptors and its gradients against the fp64 oracle. With u = 2^-24 and V = 2^-23 (a tensor core's accumulation is cut off, not rounded):
low, v. A chunk of 512 terms is 32 accumulations of 16 products, the products' own alignment counted as one more each: 64 V of the terms' magnitudes; at most
d / 512 fp32 additions of chunks and the scale: (64 V + (d / 512 + 2) u); few rows: d / 128 + 8 fp32 multiply-adds. Both below (72 + d / 64) V =: L(d).
out. (d / 16) accumulations, twice, and the adaptors' 8: (d / 8 + 16) V of all terms; low's error counts with A, and its two terms are within 2^-17 of it: (L + 2^-17)
of the adaptors' terms; one rounding to bf16: 2^-8 of the value.
dA. low's three terms are within 2^-26; 512 rows an accumulator: 64 V, their sums and the splits' below (T / 512 + 40) u: (72 + T / 256) V. dB: v's error beside it."""
import numpy as np
import pytest
import torch

from oracle import mtpc_oracle_tune as tu
from paper_2511_11346_b200 import binding as B
from paper_2511_11346_b200 import runner as R

pytestmark = pytest.mark.gpu

V, BF16 = 2.0 ** -23, 2.0 ** -8


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def low_units(d):
    return (72 + d / 64) * V


def which_of(kind, T, S, g):
    if kind == "one":
        return None
    if kind == "runs":
        w = (torch.arange(T, device="cuda") * (S + 1) // max(T, 1)) - 1
    elif kind == "none":
        w = torch.full((T,), -1, device="cuda")
    else:
        w = torch.randint(-1, S, (T,), device="cuda", generator=g)
    return w.to(torch.int32)


def make(T, d, m, k, S, kind, seed, off=0, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rows(n, c, std):
        return (torch.randn(n * (c + pad) + off, device="cuda", generator=g) * std).bfloat16()[off:].view(n, c + pad)[:, :c]
    x, W = rows(T, d, 1.0), rows(m, d, 0.1)
    A = (torch.randn(S * m * k + off, device="cuda", generator=g) * 0.1).bfloat16()[off:].view(S, m, k)
    Bf = (torch.randn(S * k * d + off, device="cuda", generator=g) * d ** -0.5).bfloat16()[off:].view(S, k, d)
    return x, W, A, Bf, 0.5 + torch.rand(S, device="cuda", generator=g), which_of(kind, T, S, g), g


def check_forward(x, W, A, Bf, scale, which, x_low=None, pad=0):
    T, d, m, k = x.shape[0], x.shape[1], W.shape[0], A.shape[2]
    out, low = torch.full((T, m + pad), 7.0, device="cuda").bfloat16(), torch.full((T, k), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.mtpc_adapted_projection(x, W, A, Bf, scale, which, out[:, :m], out_low=low, x_low=x_low, out_status=status)
    want, want_low, size, low_size = tu.adapted_projection(host(x), host(W), host(A), host(Bf), host(scale), None if which is None else which.cpu().numpy(), host(x_low))
    assert status.item() == 0 and (out[:, m:] == 7).all()
    assert (np.abs(host(low) - want_low) <= low_units(d) * low_size + 1e-30).all()
    assert (np.abs(host(out[:, :m]) - want) <= ((d / 8 + 16) * V + low_units(d) + 2.0 ** -17) * size + BF16 * np.abs(want) * 1.01 + 1e-30).all()
    return out[:, :m], low


def check_backward(x, W, A, Bf, scale, which, low, d_out, apart=False):
    T, d, m, k, S = x.shape[0], x.shape[1], W.shape[0], A.shape[2], A.shape[0]
    d_x, dA, dB = torch.empty(T, d, dtype=x.dtype, device="cuda"), torch.full((S, m, k), 7.0, device="cuda"), torch.full((S, k, d), 7.0, device="cuda")
    d_low = torch.empty_like(d_x) if apart else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.mtpc_adapted_projection_backward(x, W, A, Bf, scale, which, low, d_out, d_x, dA, dB, d_x_low=d_low, out_status=status)
    assert status.item() == 0
    r = tu.adapted_projection_grad(host(x), host(W), host(A), host(Bf), host(scale), None if which is None else which.cpu().numpy(), host(low), host(d_out))
    unit = (m / 8 + 16) * V + low_units(m) + 2.0 ** -17
    for got, name in ((d_x, "d_x_base" if apart else "d_x"), (d_low, "d_x_low")):
        if got is not None:
            assert (np.abs(host(got) - r[name]) <= unit * r[name + "_size"] + BF16 * np.abs(r[name]) * 1.01 + 1e-30).all(), name
    assert (np.abs(host(dA) - r["dA"]) <= (72 + T / 256) * V * r["dA_size"] + 1e-30).all()
    assert (np.abs(host(dB) - r["dB"]) <= ((72 + T / 256) * V + low_units(m)) * r["dB_size"] + 1e-30).all()
    return d_x, dA, dB


SIZES = [(1, 64, 128, 16, 1), (1, 8, 1, 1, 3), (3, 200, 96, 16, 2), (16, 512, 256, 8, 5), (17, 576, 130, 32, 4), (64, 1024, 384, 64, 30), (128, 320, 200, 40, 7),
         (129, 64, 64, 16, 2), (200, 136, 72, 24, 3), (300, 512, 256, 64, 4), (513, 1000, 520, 16, 3), (640, 72, 300, 48, 6)]


@pytest.mark.parametrize("T,d,m,k,S", SIZES)
@pytest.mark.parametrize("kind", ["one", "runs", "mixed", "none"])
def test_forward(T, d, m, k, S, kind):
    x, W, A, Bf, scale, which, g = make(T, d, m, k, S, kind, T + d)
    out, low = check_forward(x, W, A, Bf, scale, which, pad=8)
    if kind == "none":
        assert not low.any()
    again = torch.empty_like(out)
    B.mtpc_adapted_projection(x, W, A, Bf, None, which, again)
    check_forward(x, W, A, Bf, None, which, x_low=torch.randn(T, d, device="cuda", generator=g).bfloat16())


@pytest.mark.parametrize("T,d,m,k,S", [(1, 33, 5, 3, 2), (7, 101, 67, 5, 3), (64, 129, 130, 12, 9), (150, 77, 61, 7, 3), (260, 201, 131, 33, 2)])
@pytest.mark.parametrize("off,pad", [(0, 0), (1, 0), (0, 3), (8, 8)])
def test_odd_widths_strides_and_addresses(T, d, m, k, S, off, pad):
    x, W, A, Bf, scale, which, g = make(T, d, m, k, S, "mixed", T + off, off, pad)
    _, low = check_forward(x, W, A, Bf, scale, which, pad=pad)
    d_out = (torch.randn(T, m + pad, device="cuda", generator=g) * 0.1).bfloat16()[:, :m]
    check_backward(x, W, A, Bf, scale, which, low, d_out)


@pytest.mark.parametrize("T,d,m,k,S", SIZES + [(1500, 264, 136, 16, 2)])
@pytest.mark.parametrize("kind", ["one", "runs", "mixed", "none"])
def test_backward(T, d, m, k, S, kind):
    x, W, A, Bf, scale, which, g = make(T, d, m, k, S, kind, T + m)
    low = torch.randn(T, k, device="cuda", generator=g)
    d_out = (torch.randn(T, m, device="cuda", generator=g) * 0.1).bfloat16()
    first = check_backward(x, W, A, Bf, scale, which, low, d_out)
    check_backward(x, W, A, Bf, None, which, low, d_out, apart=True)
    again = [torch.empty_like(t) for t in first]
    B.mtpc_adapted_projection_backward(x, W, A, Bf, scale, which, low, d_out, *again)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("T,d,m,k,S,kind", [(2100, 192, 1100, 20, 5, "runs"), (2100, 192, 1100, 20, 5, "mixed"), (1300, 136, 2072, 64, 2, "one"), (2500, 70, 515, 9, 3, "runs")])
def test_many_rows_in_pairs(T, d, m, k, S, kind):
    x, W, A, Bf, scale, which, g = make(T, d, m, k, S, kind, T + d)
    _, low = check_forward(x, W, A, Bf, scale, which)
    d_out = (torch.randn(T, m, device="cuda", generator=g) * 0.1).bfloat16()
    check_backward(x, W, A, Bf, scale, which, low, d_out)
    check_backward(x, W, A, Bf, scale, which, low, d_out, apart=True)


@pytest.mark.parametrize("T", [2, 40, 100, 300])
def test_many_adaptors(T):
    x, W, A, Bf, scale, which, g = make(T, 128, 96, 16, 64, "mixed", T)
    _, low = check_forward(x, W, A, Bf, scale, which)
    check_backward(x, W, A, Bf, scale, which, low, (torch.randn(T, 96, device="cuda", generator=g) * 0.1).bfloat16())


@pytest.mark.parametrize("T,k", [(2, 16), (40, 16), (300, 16), (300, 40), (1200, 16)])
def test_nothing_of_one_request_reaches_another(T, k):
    """Adaptor 1's factors, and the rows of adaptor 1 and of none, hold infinities and NaN: every result of the others is as without."""
    d, m, S = 200, 136, 3
    x, W, A, Bf, scale, _, g = make(T, d, m, k, S, "one", T + k)
    which = (torch.arange(T, device="cuda") * 7 // 5 % 4 - 1).to(torch.int32)
    if T == 2:
        which = torch.tensor([1, 2], dtype=torch.int32, device="cuda")
    d_out = (torch.randn(T, m, device="cuda", generator=g) * 0.1).bfloat16()
    out, low = check_forward(x, W, A, Bf, scale, which)
    d_x, dA, dB = check_backward(x, W, A, Bf, scale, which, low, d_out)
    A2, B2, x2, g2, low2 = A.clone(), Bf.clone(), x.clone(), d_out.clone(), low.clone()
    A2[1, ::2], A2[1, 1::2] = float("nan"), float("inf")
    B2[1, :, ::2], B2[1, :, 1::2] = float("-inf"), torch.finfo(torch.bfloat16).min
    other = (which == 0) | (which == 2)
    x2[~other], g2[~other], low2[~other] = float("nan"), float("inf"), float("nan")
    out2, l2 = torch.empty_like(out), torch.empty_like(low)
    B.mtpc_adapted_projection(x2, W, A2, B2, scale, which, out2, out_low=l2)
    assert torch.equal(out2[other], out[other]) and torch.equal(l2[other], low[other]) and not torch.isfinite(out2[~other].float()).any()
    d_x2, dA2, dB2 = torch.empty_like(d_x), torch.empty_like(dA), torch.empty_like(dB)
    B.mtpc_adapted_projection_backward(x2, W, A2, B2, scale, which, low2, g2, d_x2, dA2, dB2)
    assert torch.equal(d_x2[other], d_x[other]) and not torch.isfinite(d_x2[~other].float()).any()
    for i in (0, 2):
        assert torch.equal(dA2[i], dA[i]) and torch.equal(dB2[i], dB[i])
    # rows of W reach only their own columns
    W2 = W.clone()
    W2[5] = float("nan")
    B.mtpc_adapted_projection(x, W2, A, Bf, scale, which, out2)
    assert torch.isnan(out2[:, 5].float()).all() and torch.equal(out2[:, 6:], out[:, 6:])


@pytest.mark.parametrize("T", [1, 3, 90, 200, 1100])
def test_adaptors_that_do_not_exist(T):
    d, m, k, S = 96, 88, 16, 2
    x, W, A, Bf, scale, _, g = make(T, d, m, k, S, "one", T)
    which = (torch.arange(T, device="cuda") % 4 - 1).to(torch.int32)      # -1, 0, 1, 2
    which[0] = 2
    ok = which < S
    out, low, status = torch.empty(T, m, device="cuda").bfloat16(), torch.empty(T, k, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.mtpc_adapted_projection(x, W, A, Bf, scale, which, out, out_low=low, out_status=status)
    assert status.item() == B.STATUS_BAD_ADAPTOR
    want = tu.adapted_projection(host(x), host(W), host(A), host(Bf), host(scale), which.cpu().numpy())[0]
    assert torch.isnan(out[~ok].float()).all() and torch.isnan(low[~ok]).all() and np.abs(host(out)[host(ok) > 0] - want[host(ok) > 0]).max(initial=0) < 0.1
    status.zero_()
    d_out = (torch.randn(T, m, device="cuda", generator=g) * 0.1).bfloat16()
    d_x, dA, dB = torch.empty_like(x), torch.empty(S, m, k, device="cuda"), torch.empty(S, k, d, device="cuda")
    B.mtpc_adapted_projection_backward(x, W, A, Bf, scale, which, low, d_out, d_x, dA, dB, out_status=status)
    assert status.item() == B.STATUS_BAD_ADAPTOR and torch.isnan(d_x[~ok].float()).all() and torch.isfinite(d_x[ok].float()).all()
    kept = torch.where(ok, which, -1).to(torch.int32)
    dA2, dB2 = torch.empty_like(dA), torch.empty_like(dB)
    B.mtpc_adapted_projection_backward(x, W, A, Bf, scale, kept, low, d_out, None, dA2, dB2)
    assert torch.equal(dA, dA2) and torch.equal(dB, dB2)
    far = torch.full((T,), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    B.mtpc_adapted_projection(x, W, A, Bf, scale, far, out)
    assert torch.isnan(out.float()).all()
    B.mtpc_adapted_projection(x, W, A, Bf, scale, torch.full_like(far, -2 ** 31), out)
    assert torch.isfinite(out.float()).all()


def test_parts_of_the_gradient_alone():
    x, W, A, Bf, scale, which, g = make(333, 120, 72, 24, 3, "mixed", 5)
    low, d_out = torch.randn(333, 24, device="cuda", generator=g), (torch.randn(333, 72, device="cuda", generator=g) * 0.1).bfloat16()
    d_x, dA, dB = check_backward(x, W, A, Bf, scale, which, low, d_out)
    a, b, c = torch.empty_like(d_x), torch.empty_like(dA), torch.empty_like(dB)
    B.mtpc_adapted_projection_backward(None, W, A, Bf, scale, which, None, d_out, a)
    B.mtpc_adapted_projection_backward(None, W, A, Bf, scale, which, low, d_out, None, b)
    B.mtpc_adapted_projection_backward(x, W, A, Bf, scale, which, None, d_out, None, None, c)
    assert torch.equal(a, d_x) and torch.equal(b, dA) and torch.equal(c, dB)
    B.mtpc_adapted_projection_backward(None, W, A, Bf, scale, which, None, d_out, None)      # nothing is wanted
    e = torch.empty_like(d_x)
    B.mtpc_adapted_projection_backward(None, W, A, Bf, scale, which, None, d_out, None, d_x_low=e)
    with pytest.raises(B.MtpcError):
        B.mtpc_adapted_projection_backward(x, W, A, Bf, scale, which, None, d_out, a, b, c)
    with pytest.raises(B.MtpcError):
        B.mtpc_adapted_projection_backward(None, W, A, Bf, scale, which, low, d_out, a, b, c)
    z = torch.zeros(0, dtype=torch.int32, device="cuda")
    B.mtpc_adapted_projection_backward(x[:0], W, A, Bf, scale, z, low[:0], d_out[:0], d_x[:0], b, c)
    assert not b.any() and not c.any()
    B.mtpc_adapted_projection(x[:0], W, A, Bf, scale, z, torch.empty(0, 72, dtype=x.dtype, device="cuda"))


def test_rows_that_are_all_the_same_and_rows_far_apart():
    for T in (50, 300):
        x, W, A, Bf, scale, which, g = make(T, 104, 80, 16, 3, "mixed", T)
        one = x[:1].expand(T, 104)
        check_forward(one, W, A, Bf, scale, which, x_low=x)
        check_forward(x, W, A, Bf, scale, which, x_low=one)
        _, low = check_forward(one, W[:1].expand(80, 104), A, Bf, scale, which)
        check_backward(one, W, A, Bf, scale, which, low, (torch.randn(1, 80, device="cuda", generator=g)).bfloat16().expand(T, 80))


def test_offsets_that_pass_32_bits():
    T, d, m = 1 << 20, 64, 2064
    x, W, A, Bf, scale, _, g = make(64, d, m, 16, 2, "one", 3)
    many = x.repeat(T // 64, 1)
    which = torch.zeros(T, dtype=torch.int32, device="cuda")
    which[T // 2:] = 1
    out = torch.empty(T, m, dtype=x.dtype, device="cuda")
    B.mtpc_adapted_projection(many, W, A, Bf, scale, which, out)
    ref = torch.empty(256, m, dtype=x.dtype, device="cuda")
    B.mtpc_adapted_projection(many[:256], W, A, Bf, scale, which[:256], ref)
    assert torch.equal(out[:256], ref)
    B.mtpc_adapted_projection(many[-256:], W, A, Bf, scale, which[-256:], ref)
    assert torch.equal(out[-256:], ref) and out.numel() > 2 ** 31


@pytest.mark.parametrize("T", [2, 60, 700])
def test_graphs_streams_and_calls_side_by_side(T):
    x, W, A, Bf, scale, which, g = make(T, 256, 192, 16, 3, "runs", T)
    d_out = (torch.randn(T, 192, device="cuda", generator=g) * 0.1).bfloat16()
    out, low = torch.empty(T, 192, dtype=x.dtype, device="cuda"), torch.empty(T, 16, device="cuda")
    grads = [torch.empty_like(x), torch.empty(3, 192, 16, device="cuda"), torch.empty(3, 16, 256, device="cuda")]

    def step(stream=None):
        B.mtpc_adapted_projection(x, W, A, Bf, scale, which, out, out_low=low, stream=stream)
        B.mtpc_adapted_projection_backward(x, W, A, Bf, scale, which, low, d_out, *grads, stream=stream)
    step()
    want = [t.clone() for t in (out, low, *grads)]

    def cleared():
        for t in (out, low, *grads):
            t.fill_(7)
        torch.cuda.synchronize()
    graphs = []
    for _ in range(2):                                       # an eager call between the captures; replays in turn and on another stream
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step()
        step()
    side = torch.cuda.Stream()
    for graph, stream in ((graphs[0], torch.cuda.current_stream()), (graphs[1], side), (graphs[0], side)):
        cleared()
        with torch.cuda.stream(stream):
            graph.replay()
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, low, *grads), want))
    cleared()
    step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((out, low, *grads), want))
    # many calls on two streams at once, each with results of its own
    outs = [torch.empty_like(out) for _ in range(8)]
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        B.mtpc_adapted_projection(x, W, A, Bf, scale, which, o, stream=side if i % 2 else None)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[0]) for o in outs)


def test_results_do_not_depend_on_the_workspace():
    x, W, A, Bf, scale, which, g = make(400, 264, 136, 16, 3, "mixed", 9)
    a, b = torch.empty(400, 136, dtype=x.dtype, device="cuda"), torch.empty(400, 136, dtype=x.dtype, device="cuda")
    need = 1 << 22
    for fill, out in ((0, a), (255, b)):                     # 255: NaN wherever it is read
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        B.mtpc_adapted_projection(x, W, A, Bf, scale, which, out, workspace=ws)
    assert torch.equal(a, b)
    low, d_out = torch.randn(400, 16, device="cuda"), torch.randn(400, 136, device="cuda").bfloat16()
    got = []
    for fill in (0, 255):
        ws = torch.full((1 << 23,), fill, dtype=torch.uint8, device="cuda")
        r = [torch.empty_like(x), torch.empty(3, 136, 16, device="cuda"), torch.empty(3, 16, 264, device="cuda")]
        B.mtpc_adapted_projection_backward(x, W, A, Bf, scale, which, low, d_out, *r, workspace=ws)
        got.append(r)
    assert all(torch.equal(p, q) for p, q in zip(*got))


def test_calls_that_are_refused():
    x, W, A, Bf, scale, which, _ = make(20, 64, 48, 16, 2, "mixed", 1)
    out, low = torch.empty(20, 48, dtype=x.dtype, device="cuda"), torch.empty(20, 16, device="cuda")
    f = B.mtpc_adapted_projection
    for call in (lambda: f(x.float(), W, A, Bf, scale, which, out), lambda: f(x, W.float(), A, Bf, scale, which, out), lambda: f(x, W, A.float(), Bf, scale, which, out),
                 lambda: f(x, W[:, :32], A, Bf, scale, which, out), lambda: f(x, W, A[:1], Bf, scale, which, out), lambda: f(x, W, A.transpose(0, 1), Bf, scale, which, out),
                 lambda: f(x, W, A, Bf, scale.double(), which, out), lambda: f(x, W, A, Bf, scale, which.long(), out), lambda: f(x, W, A, Bf, scale[:1], which, out),
                 lambda: f(x, W, A, Bf, scale, which[:3], out), lambda: f(x, W, A, Bf, scale, which, out.float()), lambda: f(x, W, A, Bf, scale, which, out[:3]),
                 lambda: f(x, W, A, Bf, scale, which, out, out_low=low.t().contiguous().t()), lambda: f(x, W, A, Bf, scale, which, out, out_low=low.bfloat16()),
                 lambda: f(x, W, A, Bf, scale, which, out, x_low=x[:3]), lambda: f(x.t().contiguous().t(), W, A, Bf, scale, which, out),
                 lambda: f(x, W, A.cpu(), Bf, scale, which, out), lambda: f(x, W, A, Bf, scale, which.cpu(), out),
                 lambda: f(x, W, A, Bf, scale, which, out, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")),
                 lambda: f(x, W, A, Bf, scale, which, out, workspace=torch.empty(1 << 20, device="cuda"))):
        with pytest.raises(B.MtpcError):
            call()
    wide = torch.zeros(1, 65, 64, device="cuda").bfloat16(), torch.zeros(1, 48, 65, device="cuda").bfloat16()
    with pytest.raises(B.MtpcError):
        f(x, W, wide[1], wide[0], None, None, out)


@pytest.mark.parametrize("T", [2, 9, 33, 70, 128])
@pytest.mark.parametrize("d,m,k,S", [(64, 300, 64, 16), (40, 19100, 3, 16), (200, 9700, 16, 20), (300, 1100, 24, 16), (1024, 136, 64, 16), (2000, 130, 9, 12)])
def test_few_rows_in_every_cluster_size(T, d, m, k, S):
    x, W, A, Bf, scale, which, g = make(T, d, m, k, S, "mixed", T + m)
    out, low = check_forward(x, W, A, Bf, scale, which, pad=T % 3)
    # rows by themselves and rows of a longer batch (tiles) agree within their errors, and a row does not depend on the others
    alone = torch.empty(T, m, dtype=x.dtype, device="cuda")
    for t in range(0, T, 31):
        B.mtpc_adapted_projection(x[t:t + 1], W, A, Bf, scale, which[t:t + 1], alone[t:t + 1])
        assert (alone[t].double() - out[t].double()).abs().max().item() <= 0.05 * out[t].double().abs().max().item() + 1e-3


@pytest.mark.parametrize("T,d,m,k,S", [(300, 576, 576, 16, 3), (300, 1088, 72, 40, 2), (700, 300, 330, 16, 4), (520, 2112, 64, 8, 2), (140, 2500, 1100, 64, 3)])
def test_low_of_chunks_of_every_length(T, d, m, k, S):
    x, W, A, Bf, scale, which, g = make(T, d, m, k, S, "runs", T + d)
    _, low = check_forward(x, W, A, Bf, scale, which)
    d_out = (torch.randn(T, m, device="cuda", generator=g) * 0.1).bfloat16()
    check_backward(x, W, A, Bf, scale, which, low, d_out)
    check_backward(x, W, A, Bf, scale, which, low, d_out, apart=True)
