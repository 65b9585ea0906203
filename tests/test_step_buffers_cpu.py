"""Buffers of an earlier training call that are written again: what the call would write past, or elsewhere, is refused before anything is launched."""
import pytest
import torch

from paper_2511_11346_b200 import binding as B
from paper_2511_11346_b200 import runner as R

SHAPES = dict(loss=(1,), dW=(3, 4), dT_static=None)
HERE = torch.device("cpu")


def buffers(**other):
    return dict(dict(loss=torch.zeros(1), dW=torch.zeros(3, 4), dT_static=None), **other)


def test_buffers_of_the_same_call_serve_again():
    for out in (buffers(), buffers(grad_norm=torch.zeros(1)), {k: v for k, v in buffers().items() if k != "dT_static"}):
        assert R._written_again("call", SHAPES, HERE, out) is out


@pytest.mark.parametrize("other", [
    dict(dW=torch.zeros(3, 4, dtype=torch.bfloat16)), dict(dW=torch.zeros(3, 4, dtype=torch.float64)), dict(dW=torch.zeros(4, 3).t()),
    dict(dW=torch.zeros(3, 8)[:, ::2]), dict(dW=torch.zeros(3, 1).expand(3, 4)), dict(dW=torch.zeros(3, 5)), dict(dW=torch.zeros(12)),
    dict(dW=torch.zeros(3, 4, device="meta")), dict(dW=None), dict(dW=[0.0] * 12), dict(loss=torch.zeros(())), dict(dT_static=torch.zeros(1, 2, 2)),
])
def test_other_buffers_are_refused(other):
    with pytest.raises(B.MtpcError):
        R._written_again("call", SHAPES, HERE, buffers(**other))


def test_missing_buffers_are_refused():
    with pytest.raises(B.MtpcError):
        R._written_again("call", SHAPES, HERE, dict(loss=torch.zeros(1)))
