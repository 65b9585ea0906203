"""The mean of a row is its sum divided by its width. Rows of one value c of five bits: the squares' sum is a whole number of 2^-8 below 2^24 of them, so it is
exact in any order, its quotient by the width is c^2 exactly, and eps = 2^-40 rounds away beside it. So every width gives the bits of a width that is a
power of two, where nothing is rounded either way; the same holds for the gradient's mean of weight d_out s with a d_out of one value of four bits."""
import pytest
import torch

from paper_2511_11346_b200 import binding as B

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -40
VECTORS = [24, 40, 56, 88, 200, 264, 328, 520, 1000, 1032, 2000, 4088, 5000, 8200, 12000, 16376]
OTHERS = [41, 47, 77, 83, 333, 1001, 2047, 4099, 10001, 16383]


def rows(d, off=0, pad=0):
    """[16, d] of 16/16 .. 31/16, one value a row, `off` elements off a vector's boundary and `pad` further apart than wide."""
    whole = torch.zeros(16 * (d + pad) + off, device="cuda")
    x = whole[off:].view(16, d + pad)[:, :d]
    x[:] = (torch.arange(16, 32, device="cuda") / 16.0)[:, None]
    return x


def forward(d, off=0, pad=0):
    x, out = rows(d, off, pad), rows(d, 0, pad)
    B.mtpc_residual_rmsnorm(x, None, None, EPS, out)
    return out


def backward(d, value, off=0, pad=0):
    x, up, dx = rows(d, off, pad), rows(d, 0, pad), rows(d, 0, pad)
    up[:] = value
    B.mtpc_residual_rmsnorm_backward(x, None, EPS, up, None, dx)
    return dx


# alike: vectors, or (from the second row on) vectors between single elements; not alike: single elements
@pytest.mark.parametrize("widths,power,off,pad", [(VECTORS, 64, 0, 0), (OTHERS, 64, 0, 1), (VECTORS + OTHERS, 64, 1, 0)])
def test_every_width_has_the_bits_of_a_power_of_two(widths, power, off, pad):
    want = forward(power, off, pad)[:, power // 2]
    for d in widths:
        own_pad = pad if d % 2 == 0 else 0
        got = forward(d, off, own_pad)
        assert torch.equal(got, want[:, None].expand(16, d)), d


@pytest.mark.parametrize("widths,power,off,pad", [(VECTORS[:13], 64, 0, 0), (VECTORS[13:], 16384, 0, 0), (OTHERS[:8], 64, 0, 1), (VECTORS + OTHERS, 64, 1, 0)])
def test_the_gradients_mean(widths, power, off, pad):
    for value in (1.0, 1.375, 1.875):
        want = backward(power, value, off, pad)[:, power // 2]
        for d in widths:
            got = backward(d, value, off, pad if d % 2 == 0 else 0)[:, 8:d - 15]           # (the elements beside the vectors are added up in another order)
            assert torch.equal(got, want[:, None].expand(16, got.shape[1])), (d, value)
