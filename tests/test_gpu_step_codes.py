"""The norm's 8-bit output by its definition: scale = largest |out| of the group / 448 (1 if that is 0), code = out / scale rounded to the nearest e4m3.
fp32 rows return `out` as it is before it is coded, so both are formed here from it, by an fp32 division each and the conversion of the CPU, and have to be
equal bit for bit: nothing is rounded but those quotients."""
import pytest
import torch

from paper_2511_11346_b200 import binding as B

pytestmark = pytest.mark.gpu


def coded(out, group):
    T, d = out.shape
    parts = torch.nn.functional.pad(out, (0, -d % (group or d))).view(T, -1, group or d)
    scale = parts.abs().amax(2) / 448.0
    scale = torch.where(scale == 0, 1.0, scale)
    q = (parts / scale[:, :, None]).clamp(-448.0, 448.0).reshape(T, -1)[:, :d]
    return scale, q.to(torch.float8_e4m3fn).view(torch.uint8)


def check(x, residual, weight, group, q):
    T, d = x.shape
    out, scale = torch.empty(T, d, device="cuda"), torch.full((T, -(-d // group) if group else 1), 7.0, device="cuda")
    B.mtpc_residual_rmsnorm(x, residual, weight, 1e-5, out, out_q=q, out_scale=scale, scale_group=group)
    want_scale, want = coded(out.cpu(), group)
    assert torch.equal(scale.cpu(), want_scale)
    # (a zero of either sign stands for the same value)
    got = q.cpu()
    assert torch.equal(torch.where(got == 128, 0, got), torch.where(want == 128, 0, want))


# rows of vectors (a warp's, a block's, all builds), of single elements (odd widths with groups), between vectors (odd widths, a scale a row)
@pytest.mark.parametrize("T,d", [(4000, 64), (1500, 256), (900, 512), (400, 1024), (300, 4096), (60, 8192), (20, 8200), (6, 32768), (1200, 77), (400, 1001),
                                 (90, 4099), (10, 20001)])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
def test_codes_and_scales_are_the_quotients(T, d, group):
    g = torch.Generator(device="cuda").manual_seed(T + d + group)
    x, res = (torch.randn(T, d, device="cuda", generator=g) for _ in range(2))
    x *= 1 + 15 * (torch.rand(d, device="cuda", generator=g) < 0.01)
    weight = 1 + 0.1 * torch.randn(d, device="cuda", generator=g)
    check(x, res, weight, group, torch.empty(T, d, dtype=torch.uint8, device="cuda"))
    check(x, None, None, group, torch.empty(T * d + 1, dtype=torch.uint8, device="cuda")[1:].view(T, d))


# weights that take the scales to both ends of fp32's range (scales below the normal range have few digits, and codes then end at 448)
@pytest.mark.parametrize("size", [1e-45, 1e-42, 1e-39, 1e-36, 1e-33, 1e-31, 1e-29, 1e-25, 1e-19, 1e-17, 1e20, 1e35])
@pytest.mark.parametrize("d,group", [(1024, 0), (1024, 32), (1001, 0), (1001, 128)])
def test_codes_at_the_ends_of_the_range(size, d, group):
    g = torch.Generator(device="cuda").manual_seed(d + group)
    x = torch.randn(64, d, device="cuda", generator=g)
    x[5], x[6, :40] = 0.0, 0.0
    weight = (1 + 0.3 * torch.randn(d, device="cuda", generator=g)) * size
    check(x, None, weight, group, torch.empty(64, d, dtype=torch.uint8, device="cuda"))
