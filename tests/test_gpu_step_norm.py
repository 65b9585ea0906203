"""Residual norm and its gradients against the fp64 oracle. With u = 2^-24 and U half a step of the output's type:
forward. s is one fp32 addition (u relative). Its squares' sum has terms of one sign; each passes at most 32 + 10 additions and its own rounding, and s's
error counts twice: 45 u relative; the mean and eps add 2 u; the inverse root halves that and is itself within 2 units (4 u):
rstd is within 28 u. out = s rstd weight: with s and two products 31 u, taken as 32 u.
8 bits. The scale is the quotient of such a value: within 33 u. A code is the nearest to a quotient within 66 u of the exact one, so it lies between the
codes of the exact quotient times 1 -+ 67 u.
gradients. unit = s rstd within 29 u; each term of mean(weight d_out s rstd) passes 42 additions and 3 products beside rstd's 28 u: 75 u of the terms'
magnitudes; unit * mean: 105 u, times step: 135 u, the subtractions 2 u: taken as 140 u of rstd (|weight d_out| + |unit| mean|weight d_out unit|) + |d_sum|.
d_weight: a block adds up ceil(T / 148) terms at most, 74 blocks' parts per warp, then 5 more additions; every term is within 31 u."""
import numpy as np
import pytest
import torch

from oracle import mtpc_oracle_step as st
from paper_2511_11346_b200 import binding as B

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
TINY = 2.0 ** -133                      # half the smallest step of bf16 (and more than fp32's): values below the normal range
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def half_step(t):
    return torch.finfo(t).eps / 2


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def rows(T, d, t, off=0, pad=0, std=1.0):
    return (torch.randn(T * (d + pad) + off, device="cuda") * std).to(t)[off:].view(T, d + pad)[:, :d]


def check_forward(x, residual, weight, out, out_sum, q=None, scale=None, group=0, eps=EPS):
    given = host(x), host(residual), host(weight)
    B.mtpc_residual_rmsnorm(x, residual, weight, eps, out, out_sum=out_sum, out_q=q, out_scale=scale, scale_group=group)
    s, y = st.rmsnorm(*given, np.float64(np.float32(eps)))
    t = x.dtype
    if out_sum is not None:
        assert (np.abs(host(out_sum) - s) <= (U32 + half_step(t)) * np.abs(s) * (1 + U32) + TINY).all()
    if out is not None:
        assert (np.abs(host(out) - y) <= (32 * U32 + half_step(t)) * np.abs(y) * (1 + U32) + TINY).all()
    if q is not None:
        want = st.code_scales(y, group)
        assert (np.abs(host(scale) - want) <= 33 * U32 * want).all()
        exact = (st.in_groups(y, group) / want[:, :, None]).reshape(y.shape[0], -1)[:, :y.shape[1]]
        got = host(q.view(torch.float8_e4m3fn))
        ends = st.e4m3(exact * (1 - 67 * U32)), st.e4m3(exact * (1 + 67 * U32))
        assert (got >= np.minimum(*ends)).all() and (got <= np.maximum(*ends)).all()


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("T,d,off,pad", [(1, 4096, 0, 0), (2, 8, 0, 0), (77, 256, 0, 0), (13, 512, 0, 8), (40, 520, 0, 0), (9, 1024, 0, 16), (5, 8192, 0, 0),
                                         (3, 8200, 0, 0), (2, 32768, 0, 0), (2, 32761, 0, 0), (31, 1001, 0, 0), (7, 1, 0, 0), (6, 4097, 0, 3), (33, 264, 1, 0),
                                         (600, 64, 0, 0), (3, 31, 0, 1)])
def test_forward(io, T, d, off, pad):
    t = TYPES[io]
    torch.manual_seed(T + d)
    x, res = rows(T, d, t, off, pad), rows(T, d, t, off, pad, 3.0)
    weight = 1 + 0.2 * torch.randn(d, device="cuda")
    new = lambda: torch.full((T, d + pad), 5.0, dtype=t, device="cuda")  # noqa: E731
    out, total = new(), new()
    check_forward(x, res, weight.to(t), out[:, :d], total[:, :d])
    assert (out[:, d:] == 5).all() and (total[:, d:] == 5).all()
    check_forward(x, None, weight, out[:, :d], None)
    check_forward(x, res, None, out[:, :d], None)
    for group in (0, 32, 64, 128):
        scale = torch.empty(T, -(-d // group) if group else 1, device="cuda")
        q = torch.full((T, d + pad), 1.0, device="cuda").to(torch.float8_e4m3fn)
        check_forward(x, res, weight.to(t), None if group else out[:, :d], total[:, :d], q[:, :d], scale, group)
        assert (q[:, d:].float() == 1).all()


def test_same_bits_for_any_alignment_of_codes_and_weights():
    T, d = 20, 1024
    x, res, weight = rows(T, d, torch.bfloat16), rows(T, d, torch.bfloat16), torch.randn(d + 1, device="cuda")
    want = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    for w in (weight[:d], weight[1:]):                                    # the second is not on a vector's boundary
        check_forward(x, res, w, want, None)
    q, scale = torch.empty(T * d + 1, dtype=torch.uint8, device="cuda"), torch.empty(T, 8, device="cuda")
    check_forward(x, res, weight[:d], None, None, q[1:].view(T, d), scale, 128)


def test_in_place_and_broadcast_rows():
    torch.manual_seed(3)
    for t, d in ((torch.bfloat16, 4096), (torch.float32, 300), (torch.float32, 77)):
        x, res, w = rows(9, d, t), rows(9, d, t), torch.randn(d, device="cuda")
        check_forward(x.clone(), res, w, torch.empty_like(x), None)
        for place in ("x", "residual"):
            a, b = x.clone(), res.clone()
            target = a if place == "x" else b
            check_forward(a, b, w, torch.empty_like(x), target)          # the sum over one of its terms
            a, b = x.clone(), res.clone()
            check_forward(a, b, w, a if place == "x" else b, None)       # the output over one of them
        check_forward(x, res[:1].expand(9, d), w, torch.empty_like(x), None)
        check_forward(x[:1].expand(9, d), res, w, torch.empty_like(x), None)


def test_rows_of_zeros_of_extremes_and_of_what_is_no_number():
    d = 512
    for t in (torch.float32, torch.bfloat16):
        x = torch.zeros(8, d, dtype=t, device="cuda")
        x[1] = torch.randn(d, device="cuda") * 3e37                         # squares beyond fp32
        x[2] = torch.randn(d, device="cuda") * 1e-30                        # squares below it: eps alone counts
        x[3, 5] = torch.finfo(t).max
        x[4] = torch.finfo(t).min / 4                                      # a mask's lowest value (a quarter: the sum stays finite)
        x[5, 7] = 1e19
        x[5, 8] = 1.0
        x[6, 0] = 2.0 ** 64
        w = torch.randn(d, device="cuda")
        out, total = torch.empty_like(x), torch.empty_like(x)
        q, scale = torch.empty(8, d, dtype=torch.uint8, device="cuda"), torch.empty(8, 4, device="cuda")
        check_forward(x, None, w, out, total, q, scale, 128)
        assert not out[0].any() and not q[0].view(torch.float8_e4m3fn).float().any() and (scale[0] == 1).all()
        check_forward(x, torch.zeros_like(x), w, out, total, q, scale[:, :1].contiguous(), 0)
        clean = out.clone()
        x[0, 3], x[7, 9] = float("nan"), float("inf")
        scale = torch.empty(8, 4, device="cuda")
        B.mtpc_residual_rmsnorm(x, None, w, EPS, out, out_sum=total, out_q=q, out_scale=scale, scale_group=128)
        assert torch.isnan(out[0]).all() and torch.equal(out[1:7], clean[1:7])            # other rows are as they were
        assert torch.isnan(out[7, 9]) and torch.isnan(scale[7, 0]) and not torch.isnan(scale[7, 1:]).any() and torch.isnan(scale[0]).all()
        assert torch.isnan(q[0].view(torch.float8_e4m3fn).float()).all()
        # gradients: finite rows only
        x[0], x[7] = 0, 0
        dy, dx, dw = torch.randn(8, d, device="cuda"), torch.empty(8, d, device="cuda"), torch.empty(d, device="cuda")
        check_backward(x, w, dy, None, dx, dw)


@pytest.mark.parametrize("d,where", [(77, 0), (77, 76), (77, 40), (5, 2), (1003, 1002), (4099, 0)])
def test_what_is_no_number_beside_the_vectors(d, where):
    for t in (torch.float32, torch.bfloat16):
        x = torch.randn(9, d, device="cuda").to(t)
        clean = torch.empty(9, d, dtype=t, device="cuda")
        q, scale, q2, scale2 = (f(9) for f in (lambda n: torch.empty(n, d, dtype=torch.uint8, device="cuda"), lambda n: torch.empty(n, 1, device="cuda")) * 2)
        check_forward(x, None, None, clean, None, q, scale)
        x[3, where], x[6, where] = float("nan"), float("-inf")
        out = torch.empty_like(clean)
        B.mtpc_residual_rmsnorm(x, None, None, EPS, out, out_q=q2, out_scale=scale2)
        others = [0, 1, 2, 4, 5, 7, 8]
        assert torch.equal(out[others], clean[others]) and torch.equal(q2[others], q[others]) and torch.equal(scale2[others], scale[others])
        assert torch.isnan(out[3]).all() and torch.isnan(scale2[3]) and torch.isnan(q2[3].view(torch.float8_e4m3fn).float()).all()
        assert torch.isnan(out[6, where]) and torch.isnan(scale2[6])
        x[3, where], x[6, where] = 0, 0
        x[3, where] = torch.finfo(t).max                                    # a single element beyond what fp32 can square
        check_forward(x, None, None, out, None, q2, scale2)


def check_backward(s, weight, dy, more, dx, dw, eps=EPS):
    given = host(s), host(weight), host(dy), host(more)
    B.mtpc_residual_rmsnorm_backward(s, weight, eps, dy, more, dx, dw)
    want, want_w, size, size_w = st.rmsnorm_grad(given[0], given[1], np.float64(np.float32(eps)), given[2], given[3])
    T = s.shape[0]
    assert (np.abs(host(dx) - want) <= 140 * U32 * size + half_step(dx.dtype) * np.abs(want) + TINY).all()
    if dw is not None:
        assert (np.abs(host(dw) - want_w) <= (-(-T // 148) + 74 + 5 + 31) * U32 * size_w + TINY).all()


@pytest.mark.parametrize("io,dy,dx", [(a, b, c) for a in TYPES for b in TYPES for c in TYPES])
@pytest.mark.parametrize("T,d", [(1, 4096), (700, 256), (300, 2048), (20, 1001), (3, 8200), (2, 32768), (2, 20001), (5000, 8), (450, 72), (4, 1)])
def test_backward(io, dy, dx, T, d):
    torch.manual_seed(T + d)
    s, up = rows(T, d, TYPES[io], std=2.0), rows(T, d, TYPES[dy])
    more = rows(T, d, TYPES[dx])
    weight = 1 + 0.2 * torch.randn(d, device="cuda")
    out = torch.empty(T, d, dtype=TYPES[dx], device="cuda")
    dw = torch.full((d,), float("nan"), device="cuda")
    check_backward(s, weight.to(TYPES[io]), up, more, out, dw)
    check_backward(s, weight, up, None, out, dw)
    check_backward(s, None, up, more, out, None)


@pytest.mark.parametrize("off,pad", [(0, 8), (0, 3), (1, 0)])
def test_backward_of_strided_rows_and_in_place(off, pad):
    torch.manual_seed(off + pad)
    T, d = 170, 640
    s, up, more = rows(T, d, torch.float32, off, pad), rows(T, d, torch.float32, off, pad), rows(T, d, torch.float32, off, pad)
    w, dw = torch.randn(d, device="cuda"), torch.empty(d, device="cuda")
    whole = torch.full((T * (d + pad) + off,), 5.0, device="cuda")
    out = whole[off:].view(T, d + pad)
    check_backward(s, w, up, more, out[:, :d], dw)
    assert (out[:, d:] == 5).all() and (whole[:off] == 5).all()
    for which in range(3):
        a = [s.clone(), up.clone(), more.clone()]
        check_backward(a[0], w, a[1], a[2], a[which], dw)
    check_backward(s[:1].expand(T, d), w, up, None, out[:, :d], dw)
    check_backward(s, w, up[:1].expand(T, d), more[:1].expand(T, d), out[:, :d], dw)


@pytest.mark.parametrize("T,d,off", [(300, 520, 1), (300, 2048, 3), (5, 8200, 0), (3, 20001, 0), (300, 64, 5)])
def test_backward_in_place_of_rows_that_are_not_alike_or_wide(T, d, off):
    torch.manual_seed(T + d)
    s, more, w, dw = rows(T, d, torch.float32), rows(T, d, torch.float32), torch.randn(d, device="cuda"), torch.empty(d, device="cuda")
    up = rows(T, d, torch.float32, off)
    for which in range(3):
        a = [s.clone(), torch.cat([torch.zeros(off, device="cuda"), up.flatten()])[off:].view(T, d), more.clone()]
        check_backward(a[0], w, a[1], a[2], a[which], dw)
    x, res = rows(T, d, torch.bfloat16), rows(T, d, torch.bfloat16, off)
    for which in range(2):
        a = [x.clone(), torch.cat([torch.zeros(off, device="cuda").bfloat16(), res.flatten()])[off:].view(T, d)]
        check_forward(a[0], a[1], w, torch.empty_like(x), a[which])


# Rows that start off their vectors, alike in all matrices and not; more of them than blocks, of which 144 at least take part in d weight here.
@pytest.mark.parametrize("T,d,off,pad", [(700, 1001, 0, 0), (400, 2047, 3, 0), (310, 4099, 5, 4), (20, 8191, 0, 0), (500, 5, 1, 0), (500, 13, 0, 1), (300, 520, 3, 8),
                                         (9, 9, 0, 0)])
@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_rows_off_their_vectors(io, T, d, off, pad):
    torch.manual_seed(T + d)
    t, other = TYPES[io], torch.bfloat16 if io == "f32" else torch.float32
    x, res, weight = rows(T, d, t, off, pad), rows(T, d, t, off + 8, pad, 2.0), 1 + 0.2 * torch.randn(d, device="cuda")
    whole = torch.full((T * (d + pad) + off,), 5.0, dtype=t, device="cuda")
    out = whole[off:].view(T, d + pad)
    codes = torch.full((T * (d + pad) + off,), 1, dtype=torch.uint8, device="cuda")
    q, scale = codes[off:].view(T, d + pad), torch.empty(T, 1, device="cuda")
    check_forward(x, res, weight.to(t), out[:, :d], None, q[:, :d], scale)
    kept = out.clone(), q.clone()
    assert (out[:, d:] == 5).all() and (whole[:off] == 5).all() and (q[:, d:] == 1).all() and (codes[:off] == 1).all()
    check_forward(x.clone(), res, weight.to(t), out[:, :d], torch.empty(T, d, dtype=t, device="cuda"), q[:, :d], scale)       # a sum elsewhere, one kernel or the other
    check_forward(x, res, weight, out[:, :d], res, q[:, :d], scale)                                                          # over its term
    check_forward(x, None, None, out[:, :d], None)
    assert torch.equal(kept[1][:, d:], q[:, d:])
    up, more = rows(T, d, other, off, pad), rows(T, d, t, off, pad)
    dw = torch.empty(d, device="cuda")
    for grads in ((up, more), (up, None), (rows(T, d, other, off + 1, pad), more)):
        check_backward(x, weight, grads[0], grads[1], out[:, :d], dw)
        assert (out[:, d:] == 5).all() and (whole[:off] == 5).all()
    check_backward(x, weight.to(t), up, more, more, dw)
    big = x.clone()
    big[0] = torch.randn(d, device="cuda") * 3e37                              # squares beyond fp32
    check_backward(big, weight, up, None, out[:, :d], dw)
    check_forward(big, None, weight, out[:, :d], None, q[:, :d], scale)


def test_gradients_are_the_norms_differences():
    """Directional derivatives of the forward call (fp32) by central differences. With h the step, each difference quotient is off by its curvature, below
    50 h^2 of the terms' magnitudes here, and by the outputs' roundings, 32 u of theirs divided by h: h = 2^-8 keeps both below 1.5e-3."""
    torch.manual_seed(11)
    T, d, h = 40, 384, 2.0 ** -8
    x, res, w, up = (torch.randn(T, d, device="cuda") for _ in range(2)), None, 1 + 0.1 * torch.randn(d, device="cuda"), torch.randn(T, d, device="cuda")
    x, res = x
    total, out, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty_like(w)
    B.mtpc_residual_rmsnorm(x, res, w, EPS, out, out_sum=total)
    B.mtpc_residual_rmsnorm_backward(total, w, EPS, up, None, dx, dw)

    def value(x, w):
        B.mtpc_residual_rmsnorm(x, res, w, EPS, out)
        return (out.double() * up.double()).sum().item()
    size = (out.abs() * up.abs()).double().sum().item()
    v, vw = torch.randn_like(x), torch.randn_like(w)
    assert abs((value(x + h * v, w) - value(x - h * v, w)) / (2 * h) - (dx.double() * v.double()).sum().item()) <= 1.5e-3 * size
    assert abs((value(x, w + h * vw) - value(x, w - h * vw)) / (2 * h) - (dw.double() * vw.double()).sum().item()) <= 1.5e-3 * size


def test_no_rows():
    x = torch.zeros(0, 64, device="cuda")
    w, dw = torch.ones(64, device="cuda"), torch.full((64,), 3.0, device="cuda")
    B.mtpc_residual_rmsnorm(x, x, w, EPS, x)
    B.mtpc_residual_rmsnorm_backward(x, w, EPS, x, None, x, dw)
    assert not dw.any()


def test_same_bits_on_streams_and_in_graphs():
    torch.manual_seed(12)
    T, d = 1000, 1024
    sets = [(rows(T, d, torch.bfloat16), rows(T, d, torch.float32)) for _ in range(3)]
    w = torch.randn(d, device="cuda")

    def run(s, up, stream=None):
        out, dx, dw = torch.zeros_like(s), torch.zeros_like(s), torch.zeros(d, device="cuda")
        torch.cuda.synchronize()
        B.mtpc_residual_rmsnorm(s, None, w, EPS, out, stream=stream)
        B.mtpc_residual_rmsnorm_backward(s, w, EPS, up, s, dx, dw, stream=stream)
        return out, dx, dw
    want = [run(*x) for x in sets]
    side = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        got = [run(*x, stream=s) for x, s in zip(sets, side)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))
    s, up = sets[0][0].clone(), sets[0][1].clone()
    out, dx, dw = torch.zeros_like(s), torch.zeros_like(s), torch.zeros(d, device="cuda")
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.mtpc_residual_rmsnorm(s, None, w, EPS, out)
            B.mtpc_residual_rmsnorm_backward(s, w, EPS, up, s, dx, dw)
        graphs.append(graph)
    for i in range(6):
        s.copy_(sets[i % 3][0])
        up.copy_(sets[i % 3][1])
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, dx, dw), want[i % 3]))


def test_offsets_beyond_32_bits():
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    T, d = 70000, 32768
    x = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    at = [0, 1, 65535, 65536, T - 1]
    x[at] = torch.randn(len(at), d, device="cuda").bfloat16()
    out = torch.empty_like(x)
    B.mtpc_residual_rmsnorm(x, None, None, EPS, out)
    small = torch.empty(len(at), d, dtype=torch.bfloat16, device="cuda")
    B.mtpc_residual_rmsnorm(x[at], None, None, EPS, small)
    assert torch.equal(out[at], small)
    B.mtpc_residual_rmsnorm_backward(x, None, EPS, x, None, out)
    B.mtpc_residual_rmsnorm_backward(x[at], None, EPS, x[at], None, small)
    assert torch.equal(out[at], small)
