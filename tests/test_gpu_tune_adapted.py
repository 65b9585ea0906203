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
NAMES = ("d_x", "dA", "dB")


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
