"""Offsets that are refused cost a call no more than the header says: min(S, 4736) T positions, not S T."""
import math

import pytest
import torch

from paper_2511_11346_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,S", [(1 << 20, 1 << 20), (1 << 20, 4736), (60000, 1 << 14), (1 << 20, 300)])
@pytest.mark.parametrize("masked", [False, True])
def test_sequences_that_all_name_every_position(T, S, masked):
    """Every other sequence is [0, T). In S T positions the first of these would be 2^40, ten seconds; a warp takes T of them at most, 20 ms in all."""
    logp = -torch.rand(T + 8, device="cuda")
    mask = (torch.arange(T + 8, device="cuda") % 3 > 0)[:T] if masked else None
    offsets = torch.zeros(S + 1, dtype=torch.int32, device="cuda")
    offsets[1::2] = T
    a, status, loss = torch.ones(S, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda")
    d = torch.full((T + 8,), 9.0, device="cuda")
    calls = [lambda w=w: B.mtpc_policy_loss(logp[:T], logp[:T], logp[:T], a, offsets, 0.2, 0.2, 0.1, loss, d[:T], mask=mask, by_sequence=w, out_status=status) for w in (False, True)]
    calls.append(lambda: B.mtpc_preference_loss(logp[:T], logp[:T], offsets, 0.1, loss, d[:T], mask=mask, out_status=status))
    for call in calls:
        status.zero_(), loss.zero_()
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        call()
        end.record()
        torch.cuda.synchronize()
        assert status.item() == B.STATUS_BAD_OFFSET and math.isnan(loss.item()) and (d[T:] == 9).all()
        assert start.elapsed_time(end) < 1000
    # and what follows is as if nothing had been
    good = torch.tensor([0, T // 2, T], dtype=torch.int32, device="cuda")
    B.mtpc_policy_loss(logp[:T], logp[:T], None, torch.ones(2, device="cuda"), good, 0.2, 0.2, 0.0, loss, d[:T])
    assert abs(loss.item() + 1) < 1e-6 and torch.allclose(d[:T] * T, torch.tensor(-1.0, device="cuda"))
