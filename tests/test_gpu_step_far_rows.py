"""Norms of rows far from one, in fp32, against the definition in 64 bits. The bars are those of test_gpu_step_norm.py (forward 32 units of 2^-24 and half a
step of the output, gradient 140 units of its terms' magnitudes), and half the smallest step that they allow, 2^-133."""
import numpy as np
import pytest
import torch

from oracle import mtpc_oracle_step as st
from paper_2511_11346_b200 import binding as B

pytestmark = pytest.mark.gpu

U32, TINY = 2.0 ** -24, 2.0 ** -133


def host(t):
    return t.detach().double().cpu().numpy()


def layouts(values):
    """The same rows as vectors, between vectors and (beside an output that is not alike) element by element: (x, out)."""
    T, d = values.shape
    yield values.clone(), torch.empty_like(values)
    yield torch.cat([values, values[:, :1]], 1)[:, :d], torch.empty(T, d + 1, device="cuda")[:, :d]
    yield values.clone(), torch.empty(T * d + 1, device="cuda")[1:].view(T, d)


def check(values, eps, backward=True):
    eps64 = float(np.float32(eps))
    for x, out in layouts(values):
        B.mtpc_residual_rmsnorm(x, None, None, eps, out)
        want = st.rmsnorm(host(x), None, None, eps64)[1]
        assert (np.abs(host(out) - want) <= 33 * U32 * np.abs(want) * (1 + U32) + TINY).all()
        if backward:
            up = torch.empty(x.shape[0], x.stride(0), device="cuda")[:, :x.shape[1]].copy_(torch.sin(torch.arange(x.numel(), device="cuda")).view(x.shape))
            B.mtpc_residual_rmsnorm_backward(x, None, eps, up, None, out)
            grad, _, size, _ = st.rmsnorm_grad(host(x), None, eps64, host(up))
            assert (np.abs(host(out) - grad) <= 140 * U32 * size + U32 * np.abs(grad) + TINY).all()


def normal(T, d, *stds):
    g = torch.Generator(device="cuda").manual_seed(d)
    return torch.randn(T, d, device="cuda", generator=g) * torch.tensor(stds, device="cuda").repeat(T // len(stds))[:, None]


@pytest.mark.parametrize("d", [64, 520, 4096, 9000])
@pytest.mark.parametrize("eps", [1e-5, 1e34, 1e36, 1e38, 3e38])
def test_eps_beside_squares_beyond_the_range(d, eps):
    check(normal(6, d, 1e17, 1e18, 1e19), eps)


@pytest.mark.parametrize("d", [64, 520, 4096, 9000])
def test_small_elements_beside_squares_beyond_the_range(d):
    """(what the largest element's square does to the rest)"""
    x = normal(6, d, 1e-6, 1e-12, 1e-18)
    x[:3, d // 3], x[3:, d // 2] = 1e20, -3e38
    check(x, 1e-5, backward=False)


@pytest.mark.parametrize("d", [64, 520, 4096, 9000])
@pytest.mark.parametrize("eps", [1e-45, 1e-42, 1e-39, 1e-36, 1e-30])
def test_squares_below_the_range_beside_as_small_an_eps(d, eps):
    check(normal(6, d, 1e-17, 1e-20, 1e-22), eps)
