"""Clipping where max_norm / norm is far below what fp32 holds: a scaled gradient is the product with the ratio, rounded once (2^-24, and 2^-24 of the ratio;
below the normal range half the smallest step)."""
import numpy as np
import pytest
import torch

from oracle import mtpc_oracle_step as st
from paper_2511_11346_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_norm", [1e-8, 1e-16, 1e-20, 1e-23, 1e-26, 1e-30, 1e-36, 1e-38])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ratios_below_the_range_of_fp32(max_norm, dtype):
    g = torch.Generator(device="cuda").manual_seed(3)
    grads = [(torch.randn(n, device="cuda", generator=g) * 3e37).to(dtype) for n in (3 * 2048 * 4, 77, 2049)]
    outs = [torch.empty(x.shape, device="cuda") for x in grads]
    given, norm = [x.double().cpu().numpy() for x in grads], torch.empty(1, device="cuda")
    want, scaled = st.clip(given, float(np.float32(max_norm)))
    B.GradientList(grads, outs).mtpc_clip_gradients(max_norm, norm)
    for x, y in zip(outs, scaled):
        assert (np.abs(x.double().cpu().numpy() - y) <= 2.001 * 2.0 ** -24 * np.abs(y) + 1.001 * 2.0 ** -150).all()
    B.GradientList(grads).mtpc_clip_gradients(max_norm, norm)
    for x, y in zip(grads, scaled):
        assert (np.abs(x.double().cpu().numpy() - y) <= (2.0 ** -24 + torch.finfo(dtype).eps / 2) * 1.001 * np.abs(y) + (2.0 ** -134 if dtype is torch.bfloat16 else 1.001 * 2.0 ** -150)).all()
