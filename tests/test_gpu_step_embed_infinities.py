"""Positions of the embedding gradient that hold infinities and NaN: exactly the elements of the table that add them up are not finite, by each of the
gradient's ways (one launch, the one-launch sort, digits; columns by fours and one by one), written and added."""
import numpy as np
import pytest
import torch

from paper_2511_11346_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,v,d", [(100, 30, 64), (900, 30, 64), (900, 30, 63), (5000, 700, 40), (20000, 300, 36), (40000, 3000, 20)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_infinities_reach_their_elements_and_no_others(T, v, d, accumulate):
    rng = np.random.default_rng(T + d)
    tokens = rng.integers(0, v, T)
    tokens[[11, 12, T - 1]] = 7, v - 1, 19                                  # apart, so that each can be told
    d_out = torch.randn(T, d, device="cuda")
    d_out[11] = float("inf")
    d_out[12, 5] = float("nan")
    d_out[T - 1, d - 1] = float("-inf")
    away = np.where(tokens == 3)[0]
    tokens[away] = np.where(np.arange(len(away)) % 2, -1, v + 2)           # padding and no token: never looked at
    d_out[torch.from_numpy(away).cuda()] = float("nan")
    table = torch.ones(v, d, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.mtpc_embed_backward(torch.from_numpy(tokens.astype(np.int32)).cuda(), d_out, table, accumulate=accumulate, out_status=status)
    want = torch.zeros(v, d, dtype=torch.bool, device="cuda")
    want[7], want[v - 1, 5], want[19, d - 1] = True, True, True
    assert torch.equal(~torch.isfinite(table), want)
    assert (table[7] == float("inf")).all() and torch.isnan(table[v - 1, 5]) and table[19, d - 1] == float("-inf")
    assert (table[3] == (1 if accumulate else 0)).all() and status.item() == (B.STATUS_BAD_TOKEN if len(away) else 0)
