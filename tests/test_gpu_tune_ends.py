"""What the losses of sequences give at the ends of their range: windows without probability, terms whose factor is zero, differences and sums that lose nothing."""
import math

import pytest
import torch

from paper_2511_11346_b200 import binding as B

pytestmark = pytest.mark.gpu

INF = math.inf


def packed(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def preference(lengths, holes, beta=0.5, smoothing=0.0):
    """A batch of sequences of equal log-likelihoods (h = 0) but for windows without probability at `holes` -> (loss, h, gradient)."""
    offsets, T = packed(lengths), sum(lengths)
    logp = torch.full((T,), -1.0, device="cuda")
    ref = torch.full((T,), -1.0, device="cuda")
    logp[holes] = -INF
    d, loss, h = torch.full((T,), 9.0, device="cuda"), torch.empty(1, device="cuda"), torch.empty(len(lengths) // 2, device="cuda")
    B.mtpc_preference_loss(logp, ref, offsets, beta, loss, d, smoothing=smoothing, out_h=h)
    return loss.item(), h, d


# one cluster; pairs formed by whoever needs them; pairs in a launch of their own
@pytest.mark.parametrize("lengths", [[6, 5, 4, 3], [40000, 30000, 4, 3] + [9] * 252, [40000, 30000, 4, 3], [300, 300, 2, 1] + [60] * 1196])
def test_preference_of_windows_without_probability(lengths):
    pairs, n = len(lengths) // 2, sum(lengths)
    rest = (pairs - 1) / pairs * math.log(2)                      # the other pairs have h = 0
    first, second = slice(0, lengths[0]), slice(lengths[0], lengths[0] + lengths[1])
    # the rejected one has such a window: the pair is decided, it costs nothing and has no gradient
    loss, h, d = preference(lengths, [lengths[0] + 1])
    assert h[0].item() == INF and not h[1:].any() and abs(loss - rest) <= 1e-6 and not d[:second.stop].any()
    assert (d[second.stop:].abs() > 0).all() and torch.isfinite(d).all() and d.numel() == n
    # the preferred one: the loss has no bound, the slope is -beta
    loss, h, d = preference(lengths, [1])
    assert h[0].item() == -INF and loss == INF
    assert torch.allclose(d[first], torch.tensor(-0.5 / pairs, device="cuda")) and torch.allclose(d[second], torch.tensor(0.5 / pairs, device="cuda"))
    # smoothing 1 turns the two about; between 0 and 1 both cost
    loss, h, d = preference(lengths, [1], smoothing=1.0)
    assert h[0].item() == -INF and abs(loss - rest) <= 1e-6 and not d[:second.stop].any()
    for hole in (1, lengths[0] + 1):
        loss, h, d = preference(lengths, [hole], smoothing=0.25)
        assert loss == INF and torch.isfinite(d).all()
    # beta 0 leaves nothing of the sums
    loss, h, d = preference(lengths, [1], beta=0.0)
    assert abs(loss - math.log(2)) <= 1e-6 and not h.any() and not d.any()
    # both have one: nothing can be said of the pair
    loss, h, d = preference(lengths, [1, lengths[0] + 1])
    assert math.isnan(loss) and math.isnan(h[0].item()) and not h[1:].any()
