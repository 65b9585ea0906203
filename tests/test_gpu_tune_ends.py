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


def policy(logp, old, ref, advantage, offsets, beta, low=0.2, high=0.2, by_position=False):
    d, loss, stats = torch.full_like(logp, 9.0), torch.empty(1, device="cuda"), torch.empty(3, device="cuda")
    B.mtpc_policy_loss(logp, old, ref, advantage, offsets, low, high, beta, loss, d, out_stats=stats, by_position=by_position)
    return d, loss.item(), stats


@pytest.mark.parametrize("T", [16, 70000])
def test_kl_term_of_windows_without_probability(T):
    """q = ref - logp without a bound: e^q - 1 - q is infinite whichever way, and its slope beta (1 - e^q) what it tends to."""
    one, offsets, a = torch.full((T,), -1.0, device="cuda"), packed([T // 2, T - T // 2]), torch.ones(2, device="cuda")
    holes = [1, T // 2 + 2, T - 1]
    bad = one.clone()
    bad[holes] = -INF
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[holes] = False
    d, loss, stats = policy(bad, one, one, a, offsets, 0.5)                       # the policy gives a window no probability, the reference does: q = inf
    assert loss == INF and stats[1].item() == INF and (d[holes] == -INF).all() and math.isfinite(stats[0].item())
    assert torch.equal(d[keep], torch.full_like(d[keep], -1.0 / T))
    d, loss, stats = policy(one, one, bad, a, offsets, 0.5)                       # the other way about: q = -inf, e^q = 0
    assert loss == INF and stats[1].item() == INF and (d[holes] == (0.5 - 1.0) / T).all() and torch.equal(d[keep], torch.full_like(d[keep], -1.0 / T))
    # so large that only e^q overflows fp32
    far = one.clone()
    far[holes] = -1001.0
    d, loss, stats = policy(far, one, one, a, offsets, 0.5)
    assert loss == INF and (d[holes] == -INF).all() and not torch.isnan(stats).any()


@pytest.mark.parametrize("T", [64, 70000])
def test_differences_of_log_likelihoods_lose_nothing(T):
    """Log-likelihoods whose difference does not fit fp32: rounded, it would move a ratio by up to |diff| u = 80 u (u = 2^-24). Without: expf and expm1f are within
    2 units in the last place (4 u), the rest of the difference, the product with the advantage, the weight and its product u each: 8 u; e^q - 1 - q one more."""
    u = 2.0 ** -24
    g = torch.Generator(device="cuda").manual_seed(T)
    near, far = -torch.rand(T, device="cuda", generator=g), -50 - 30 * torch.rand(T, device="cuda", generator=g)
    offsets = packed([T // 2, T - T // 2])
    d, loss, stats = policy(near, far, None, torch.full((2,), -1.0, device="cuda"), offsets, 0.0)       # a ratio above the upper end counts where the advantage is negative
    want = torch.exp(near.double() - far.double()) / T
    assert ((d.double() - want).abs() <= 8 * u * want).all() and (want > d.double()).any() and (want < d.double()).any()
    assert abs(loss - float(want.sum())) <= 8 * u * float(want.sum()) and stats[2].item() == 0
    d, loss, stats = policy(far, far, near, torch.zeros(2, device="cuda"), offsets, 1.0)                # the KL term alone
    q = near.double() - far.double()
    assert ((d.double() + torch.expm1(q) / T).abs() <= 9 * u * torch.expm1(q) / T).all()
    want = float((torch.expm1(q) - q).sum()) / T
    assert abs(loss - want) <= 9 * u * want


@pytest.mark.parametrize("T", [64, 70000])
def test_sums_of_terms_that_cancel(T):
    """Terms of 2^25 and 1 whose large ones cancel: exact in fp64, lost where fp32 adds them up. Ratios are 1 here, the terms the advantages with their signs turned."""
    logp, a = torch.full((T,), -3.0, device="cuda"), torch.tensor([2.0 ** 25, 1.0, -2.0 ** 25, 1.0], device="cuda").repeat(T // 4)
    d, loss, stats = policy(logp, logp, None, a, packed([T]), 0.0, by_position=True)
    assert loss == -0.5 and stats[0].item() == -0.5 and torch.allclose(d * T, -a, rtol=2.0 ** -23, atol=0)


@pytest.mark.parametrize("lo,hi", [(0.499, 0.4999999), (-0.4999999, -0.499), (0.48, 0.4999)])
def test_series_of_the_kl_term(lo, hi):
    """What the series of e^q - 1 - q leaves out at its end, |q| = 1/2: 2 q^8 / 10! = 2^-28.8 of q^2 / 2 (with one coefficient less 2^-24.5). A value's own roundings hide that; here
    the terms' mean is less an advantage that is nearly it, so that the loss is what they are off together: the roundings of 2^17 different q (within 3 u each, u = 2^-24, of either
    sign) average out to below u / 100, those of the coefficients (u / 2 of 1/6 and the ones behind it, of 1/2 nothing) stay below u q / 6 + u q^2 / 12 < u / 8. 2^-26 is a quarter of u."""
    T = 1 << 17
    logp = -(lo + (hi - lo) * torch.rand(T, device="cuda", dtype=torch.float64, generator=torch.Generator(device="cuda").manual_seed(3))).float()
    q = -logp.double()
    want = float((torch.expm1(q) - q).mean())
    a = torch.tensor([want], dtype=torch.float32, device="cuda")
    _, loss, _ = policy(logp, logp, torch.zeros(T, device="cuda"), a, packed([T]), 1.0)
    assert abs(loss - (want - a.double().item())) <= 2.0 ** -26 * want
