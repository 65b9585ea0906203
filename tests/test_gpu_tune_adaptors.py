"""Adaptors that do not exist are reported by every call that asks for something, whichever of the gradients it asks for."""
import pytest
import torch

from paper_2511_11346_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 90, 200, 1100, 4001])
@pytest.mark.parametrize("wanted", [("dA",), ("dB",), ("d_x",), ("d_x_low",), ("dA", "dB"), ("d_x", "d_x_low"), ("dA", "d_x")])
@pytest.mark.parametrize("at", [0, -1])
def test_adaptors_that_do_not_exist(T, wanted, at):
    d, m, k, S = 96, 88, 16, 2
    g = torch.Generator(device="cuda").manual_seed(T)
    new = lambda *s: (torch.randn(s, device="cuda", generator=g) * 0.2).bfloat16()  # noqa: E731
    x, W, A, Bf, d_out, low = new(T, d), new(m, d), new(S, m, k), new(S, k, d), new(T, m), torch.randn(T, k, device="cuda", generator=g)
    which = (torch.arange(T, device="cuda") % 3 - 1).int()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = dict(d_x=torch.empty_like(x), d_x_low=torch.empty_like(x), dA=torch.empty(S, m, k, device="cuda"), dB=torch.empty(S, k, d, device="cuda"))

    def call():
        status.zero_()
        o = {key: t if key in wanted else None for key, t in out.items()}
        B.mtpc_adapted_projection_backward(x, W, A, Bf, None, which, low, d_out, o["d_x"], o["dA"], o["dB"], d_x_low=o["d_x_low"], out_status=status)
        return status.item()
    assert call() == 0
    which[at] = S
    assert call() == B.STATUS_BAD_ADAPTOR
    which[at] = 2 ** 31 - 1
    assert call() == B.STATUS_BAD_ADAPTOR
