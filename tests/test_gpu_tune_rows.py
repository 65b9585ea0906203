"""Few rows beside a W of many rows, by rank: what decides how many CTAs share K and how many of a thread's factor rows are on their way at once. With u = 2^-24, V = 2^-23 (a tensor
core's accumulation is cut off): (d / 16) accumulations and as much for the products' own alignment, (d / 8) V of all terms; low in fp32 by d / 128 + 8 multiply-adds, below d / 64 + 72 V;
its product with A k multiply-adds, k u; the parts' sums 9 u; one rounding to bf16, 2^-8 of the value."""
import pytest
import torch

from paper_2511_11346_b200 import binding as B

pytestmark = pytest.mark.gpu

V = 2.0 ** -23


@pytest.mark.parametrize("T", [33, 43, 64, 65, 97, 128])
@pytest.mark.parametrize("m,d,k", [(4096, 576, 16), (4001, 576, 24), (4096, 1100, 33), (3800, 640, 48), (4096, 576, 64), (2300, 1030, 64)])
def test_few_rows_beside_many_rows_of_W(T, m, d, k):
    S = 48
    assert T <= min(128, 640 // k + 8 * S)
    g = torch.Generator(device="cuda").manual_seed(T + k)
    new = lambda *s, std: (torch.randn(s, device="cuda", generator=g) * std).bfloat16()  # noqa: E731
    x, W, A, Bf = new(T, d, std=1.0), new(m, d, std=0.1), new(S, m, k, std=0.1), new(S, k, d, std=d ** -0.5)
    which = torch.randint(-1, S, (T,), device="cuda", generator=g).int()
    out, status = torch.full((T, m), 7.0, device="cuda").bfloat16(), torch.zeros(1, dtype=torch.int32, device="cuda")
    low, again = torch.empty(T, k, device="cuda"), torch.empty(T, m, dtype=x.dtype, device="cuda")
    B.mtpc_adapted_projection(x, W, A, Bf, None, which, out, out_low=low, out_status=status)
    B.mtpc_adapted_projection(x, W, A, Bf, None, which, again)
    any_, i = (which >= 0).double()[:, None], which.clamp_min(0).long()
    xd, Bd, Ad = x.double(), Bf.double()[i], A.double()[i]
    want_low = any_ * torch.einsum("tkd,td->tk", Bd, xd)
    low_size = any_ * torch.einsum("tkd,td->tk", Bd.abs(), xd.abs())
    want = xd @ W.double().T + torch.einsum("tmk,tk->tm", Ad, want_low)
    size = xd.abs() @ W.double().abs().T + torch.einsum("tmk,tk->tm", Ad.abs(), low_size)
    unit = (72 + d / 64) * V
    assert status.item() == 0 and torch.equal(out, again) and ((low.double() - want_low).abs() <= unit * low_size + 1e-30).all()
    assert ((out.double() - want).abs() <= ((d / 8 + k / 2 + 5) * V + unit) * size + 1.01 * 2.0 ** -8 * want.abs() + 1e-30).all()
