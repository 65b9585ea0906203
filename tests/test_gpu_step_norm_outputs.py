"""Where the norm's outputs may lie: over x and over residual, each over one of them, but not both over the same."""
import pytest
import torch

from paper_2511_11346_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,d", [(1, 512), (9, 4096), (5, 77)])
def test_both_outputs_over_the_inputs(T, d):
    g = torch.Generator(device="cuda").manual_seed(d)
    x, res = (torch.randn(T, d, device="cuda", generator=g).bfloat16() for _ in range(2))
    out, total = torch.empty_like(x), torch.empty_like(x)
    B.mtpc_residual_rmsnorm(x, res, None, 1e-5, out, out_sum=total)
    for swap in (False, True):
        a, b = x.clone(), res.clone()
        B.mtpc_residual_rmsnorm(a, b, None, 1e-5, b if swap else a, out_sum=a if swap else b)
        assert torch.equal(b if swap else a, out) and torch.equal(a if swap else b, total)
    for same in (torch.empty_like(x), x, res):
        before = same.clone()
        with pytest.raises(B.MtpcError):
            B.mtpc_residual_rmsnorm(x, res, None, 1e-5, same, out_sum=same)
        assert torch.equal(same.view(torch.int16), before.view(torch.int16))
