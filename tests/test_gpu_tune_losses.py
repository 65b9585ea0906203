"""The losses of sequences against the fp64 oracle, with u = 2^-24.
policy: a position's difference of log-likelihoods is exact in fp64; rounded to fp32 it moves r by |diff| u <= 2 u (|diff| <= 2 here), expf is within 2 units in
the last place (4 u), the product with the advantage rounds once: |r a| within 7 u, the ends' within 2 u. e^q - 1 is within 1 unit of expm1f and |q| u of q's rounding
(|q| <= 2: 6 u, taken relative to e^q - 1 + |q|); e^q - 1 - q by eight terms within 12 u of itself near zero, within 10 u of e^q elsewhere. Sums are fp64; the weight is
rounded once and multiplied (2 u), the sums once to fp32. Taken together: gradients within 12 u of w (|r a| + beta (|e^q - 1| + |q|)), the loss within 12 u of
the weighted terms' magnitudes and beta w (e^q) and u of itself.
preference: h and the loss are fp64 throughout, rounded once; slopes too."""
import math

import numpy as np
import pytest
import torch

from oracle import mtpc_oracle_tune as tu
from paper_2511_11346_b200 import binding as B

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def batch(lengths, seed, masked, behind=3, off=0):
    """Packed sequences of these lengths with `behind` positions after the last; values off the vectors' boundaries with off."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    T = sum(lengths) + behind
    new = lambda std: torch.randn(T + off, device="cuda", generator=g)[off:] * std  # noqa: E731
    logp = -11 * torch.rand(T + off, device="cuda", generator=g)[off:]
    old, ref = logp + new(0.3), logp + new(0.2)
    mask = (torch.rand(T + off, device="cuda", generator=g) < 0.7)[off:] if masked else None
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device="cuda")
    return logp, old, ref, mask, offsets


def check_policy(logp, old, ref, mask, offsets, advantage, beta, by_sequence=False, by_position=False, low=0.2, high=0.28):
    T = logp.numel()
    d, loss, stats = torch.full_like(logp, 9.0), torch.empty(1, device="cuda"), torch.empty(3, device="cuda")
    B.mtpc_policy_loss(logp, old, ref, advantage, offsets, low, high, beta, loss, d, mask=mask, by_sequence=by_sequence, by_position=by_position, out_stats=stats)
    f = lambda x: float(np.float32(x))  # noqa: E731
    lp, ol, rf, of = host(logp), host(old), host(ref), offsets.tolist()
    want, want_stats, grad, size = tu.policy_loss(lp, ol, rf, host(advantage), of, f(low), f(high), f(beta), None if mask is None else mask.cpu().numpy(),
                                                  by_sequence, by_position)
    got, inside = host(d), ~np.isnan(grad)
    assert (got[~inside] == 9.0).all() and inside.sum() == of[-1] - of[0]
    valid = inside if mask is None else inside & mask.cpu().numpy()
    assert (got[inside & ~valid] == 0).all()
    if valid.any():
        w = np.zeros(T)
        for s in range(len(of) - 1):
            here = valid[of[s]:of[s + 1]].sum()
            w[of[s]:of[s + 1]] = 1 / (max(1, here) * (len(of) - 1)) if by_sequence else 1 / valid.sum()
        a = host(advantage) if by_position else np.concatenate([np.repeat(host(advantage), np.diff(of)), np.zeros(T - of[-1])])
        q = (rf - lp) * (1.0 if beta else 0.0)
        with np.errstate(all="ignore"):
            bar = 12 * U32 * w * (np.exp(lp - ol) * np.abs(a) + beta * (np.abs(np.expm1(q)) + np.abs(q)))
            assert (np.abs(got - grad)[valid] <= bar[valid] + 1e-40).all()
            extra = beta * (w * np.exp(q))[valid].sum()
        assert abs(loss.item() - want) <= 12 * U32 * (size + extra) + U32 * abs(want)
        assert abs(stats[0].item() - want_stats[0]) <= 12 * U32 * size + U32 * abs(want_stats[0])
        assert abs(stats[1].item() - want_stats[1]) <= 12 * U32 * (want_stats[1] + (w * np.exp(q))[valid].sum())
        assert abs(stats[2].item() - want_stats[2]) <= 2 * U32 * want_stats[2] + 1e-15
    else:
        assert loss.item() == 0 and not stats.any()


@pytest.mark.parametrize("lengths", [[1], [0, 5, 0], [3, 1, 64, 17, 2], [700, 1, 90], [5] * 300, [4000, 60], [0]])
@pytest.mark.parametrize("masked,off", [(False, 0), (True, 0), (True, 1)])
def test_policy(lengths, masked, off):
    logp, old, ref, mask, offsets = batch(lengths, sum(lengths) + off, masked, off=off)
    a = torch.randn(len(lengths), device="cuda")
    per = torch.randn(logp.numel() + off, device="cuda")[off:]
    for by_sequence in (False, True):
        check_policy(logp, old, ref, mask, offsets, a, 0.05, by_sequence)
        check_policy(logp, old, ref, mask, offsets, a, 0.0, by_sequence)
        check_policy(logp, old, ref, mask, offsets, per, 0.5, by_sequence, by_position=True)


def test_policy_of_many_positions():
    """Beyond what one cluster does: the launches of each phase, against the same in vectors of fp64."""
    lengths = [50000, 1, 0, 30001, 2, 9000] + [37] * 100
    for masked in (False, True):
        logp, old, ref, mask, offsets = batch(lengths, 3, masked, behind=5)
        T, S = logp.numel(), len(lengths)
        a = torch.randn(S, device="cuda")
        a[3] = 0.0
        of = torch.repeat_interleave(torch.arange(S, device="cuda"), torch.tensor(lengths, device="cuda"))
        n = len(of)
        valid = torch.ones(n, dtype=torch.bool, device="cuda") if mask is None else mask[:n]
        for by_sequence in (False, True):
            d, loss, stats = torch.full_like(logp, 9.0), torch.empty(1, device="cuda"), torch.empty(3, device="cuda")
            B.mtpc_policy_loss(logp, old, ref, a, offsets, 0.25, 0.25, 0.125, loss, d, mask=mask, by_sequence=by_sequence, out_stats=stats)
            again, loss2 = torch.full_like(logp, 9.0), torch.empty(1, device="cuda")
            B.mtpc_policy_loss(logp, old, ref, a, offsets, 0.25, 0.25, 0.125, loss2, again, mask=mask, by_sequence=by_sequence)
            assert torch.equal(d, again) and torch.equal(loss, loss2) and (d[n:] == 9).all()
            count = torch.zeros(S, device="cuda", dtype=torch.float64).index_add_(0, of, valid.double())
            w = torch.where(valid, 1 / (S * count.clamp_min(1))[of] if by_sequence else 1 / count.sum(), 0.0)
            r, adv, q = torch.exp(logp[:n].double() - old[:n].double()), a.double()[of], ref[:n].double() - logp[:n].double()
            held = r.clamp(0.75, 1.25) * adv
            first, kl = -torch.minimum(r * adv, held), torch.expm1(q) - q
            grad = w * (torch.where(held < r * adv, 0.0, -r * adv) - 0.125 * torch.expm1(q))
            bar = 12 * U32 * w * (r * adv.abs() + 0.125 * (torch.expm1(q).abs() + q.abs()))
            assert ((d[:n].double() - grad).abs() <= bar + 1e-40).all()
            want = float((w * (first + 0.125 * kl)).sum())
            assert abs(loss.item() - want) <= 12 * U32 * float((w * (first.abs() + 0.125 * (kl + torch.exp(q)))).sum()) + U32 * abs(want)
            assert abs(stats[2].item() - float((w * (held < r * adv)).sum())) <= 1e-6


@pytest.mark.parametrize("lengths", [[1, 1], [0, 0], [5, 0], [3, 1, 64, 17], [700, 1, 90, 3], [5] * 300, [4000, 60], [60000, 20000, 3, 0, 1, 9]])
@pytest.mark.parametrize("masked,off", [(False, 0), (True, 0), (True, 3)])
def test_preference(lengths, masked, off):
    logp, _, ref, mask, offsets = batch(lengths, sum(lengths), masked, off=off)
    S = len(lengths)
    for beta, smoothing in ((0.1, 0.0), (0.4, 0.2), (0.0, 0.0), (0.1, 1.0)):
        d, loss, h = torch.full_like(logp, 9.0), torch.empty(1, device="cuda"), torch.empty(S // 2, device="cuda")
        B.mtpc_preference_loss(logp, ref, offsets, beta, loss, d, mask=mask, smoothing=smoothing, out_h=h)
        want, want_h, grad = tu.preference_loss(host(logp), host(ref), offsets.tolist(), float(np.float32(beta)), float(np.float32(smoothing)),
                                                None if mask is None else mask.cpu().numpy())
        inside = ~np.isnan(grad)
        assert (host(d)[~inside] == 9).all()
        assert (np.abs(host(d) - grad)[inside] <= 1.01 * U32 * np.abs(grad[inside]) + 1e-44).all()
        assert (np.abs(host(h) - want_h) <= 1.01 * U32 * np.abs(want_h) + 1e-12).all()
        assert abs(loss.item() - want) <= 1.01 * U32 * want
    B.mtpc_preference_loss(logp, ref, offsets, 0.1, loss, d, mask=mask)


def test_far_apart_pairs_and_long_sums():
    """h in the thousands: no exponential overflows, the loss is |h| or nothing. And sums of 2^17 terms whose differences are small beside them."""
    logp = torch.full((8,), -1e4, device="cuda")
    ref = torch.zeros(8, device="cuda")
    ref[4:] = -2e4
    offsets = torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda")
    d, loss, h = torch.empty_like(logp), torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    B.mtpc_preference_loss(logp, ref, offsets, 1.0, loss, d, out_h=h)
    assert h.item() == -8e4 and loss.item() == 8e4 and (d[:4] == -1).all() and (d[4:] == 1).all()
    B.mtpc_preference_loss(logp.flip(0).contiguous(), ref.flip(0).contiguous(), offsets, 1.0, loss, d, out_h=h)
    assert h.item() == 8e4 and loss.item() == 0 and not d.any()
    n = 1 << 17
    logp = -100 * torch.rand(2 * n, device="cuda")
    ref = logp + 1e-5 * torch.randn(2 * n, device="cuda")
    offsets = torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda")
    d = torch.empty_like(logp)
    B.mtpc_preference_loss(logp, ref, offsets, 0.5, loss, d, out_h=h)
    r = logp.double() - ref.double()
    want = 0.5 * float(r[:n].sum() - r[n:].sum())
    assert abs(h.item() - want) <= 1.01 * U32 * abs(want) + 1e-12


def test_masked_positions_may_hold_anything_and_ends_are_sharp():
    low, high = 0.25, 0.25
    edge = math.log1p(high)
    old = torch.zeros(16, device="cuda")
    logp = torch.tensor([edge] * 16, device="cuda")                       # fp32 beside the logarithm of the end: which side is known exactly
    side = float(logp[0].double()) > edge
    mask = torch.ones(16, dtype=torch.uint8, device="cuda")
    mask[3], mask[7], mask[9], mask[12] = 0, 0, 0, 0
    bad = logp.clone()
    bad[3], bad[7], bad[9], bad[12] = float("nan"), float("inf"), float("-inf"), torch.finfo(torch.float32).min
    offsets = torch.tensor([0, 8, 16], dtype=torch.int32, device="cuda")
    a = torch.tensor([1.0, -1.0], device="cuda")
    for values in (logp, bad):
        d, loss, stats = torch.empty(16, device="cuda"), torch.empty(1, device="cuda"), torch.empty(3, device="cuda")
        B.mtpc_policy_loss(values, old, values, a, offsets, low, high, 0.1, loss, d, mask=mask, out_stats=stats)
        keep = mask.bool()
        assert torch.isfinite(d).all() and torch.isfinite(loss).all() and not d[~keep].any()
        assert (d[:8][keep[:8]] == 0).all() == side and (d[8:][keep[8:]] > 0).all()
        assert abs(stats[2].item() - (0.5 if side else 0.0)) < 1e-6 and stats[1].item() == 0
        B.mtpc_preference_loss(values, old, offsets, 0.1, loss, d, mask=mask)
        assert torch.isfinite(d).all() and torch.isfinite(loss).all() and not d[~keep].any()
    # a window without probability now: its ratio is zero, its gradient too
    logp = torch.tensor([-math.inf, -1.0], device="cuda")
    d = torch.empty(2, device="cuda")
    B.mtpc_policy_loss(logp, torch.full((2,), -1.0, device="cuda"), None, a[:1], torch.tensor([0, 2], dtype=torch.int32, device="cuda"), 0.2, 0.2, 0.0, loss, d)
    assert d[0].item() == 0 and d[1].item() == -0.5 and loss.item() == -0.5
    # with a negative advantage it is beyond the lower end: the end's value, clipped
    stats = torch.empty(3, device="cuda")
    B.mtpc_policy_loss(logp, torch.full((2,), -1.0, device="cuda"), None, a[1:], torch.tensor([0, 2], dtype=torch.int32, device="cuda"), 0.25, 0.25, 0.0, loss, d,
                       out_stats=stats)
    assert d[0].item() == 0 and d[1].item() == 0.5 and loss.item() == 0.875 and stats[2].item() == 0.5
    # what an end at zero, or none, does: ratios of 1 are not beyond it, all others are; a clip_low of 1 or more never clips
    two, zero = torch.full((2,), -1.0, device="cuda"), torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    for sign in (1.0, -1.0):
        adv = torch.tensor([sign], device="cuda")
        for step, clipped in ((0.0, 0.0), (2.0 ** -23, 1.0), (0.5, 1.0)):
            B.mtpc_policy_loss(two + sign * step, two, None, adv, zero, 0.0, 0.0, 0.0, loss, d, out_stats=stats)
            assert stats[2].item() == clipped and (d.abs() > 0).all() == (clipped == 0)
    B.mtpc_policy_loss(two - 50, two, None, a[1:], zero, 1.0, 0.2, 0.0, loss, d, out_stats=stats)
    assert stats[2].item() == 0 and loss.item() >= 0


def test_offsets_that_are_refused_stay_within_the_buffers():
    logp, old, ref, mask, _ = batch([40, 40], 5, True, behind=0)
    a, status = torch.ones(2, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for bad in ([0, 50, 40], [-5, 20, 80], [0, 40, 81], [0, -2 ** 31, 2 ** 31 - 1], [90, 95, 99]):
        offsets = torch.tensor(bad, dtype=torch.int32, device="cuda")
        d, loss, status[:] = torch.empty(80, device="cuda"), torch.empty(1, device="cuda"), 0
        B.mtpc_policy_loss(logp, old, ref, a, offsets, 0.2, 0.2, 0.1, loss, d, mask=mask, out_status=status)
        assert math.isnan(loss.item()) and status.item() == B.STATUS_BAD_OFFSET
        status[:], loss[:] = 0, 0
        B.mtpc_preference_loss(logp, ref, offsets, 0.1, loss, d, mask=mask, out_status=status)
        assert math.isnan(loss.item()) and status.item() == B.STATUS_BAD_OFFSET
    B.mtpc_preference_loss(logp, ref, torch.tensor([0, 40, 80], dtype=torch.int32, device="cuda"), 0.1, loss, d)
    assert not math.isnan(loss.item())


def test_streams_and_graphs():
    logp, old, ref, mask, offsets = batch([300, 200, 100, 77], 8, True)
    a = torch.randn(4, device="cuda")
    outs = [torch.zeros_like(logp) for _ in range(4)]
    losses = torch.zeros(4, device="cuda")

    def calls(i, stream=None):
        B.mtpc_policy_loss(logp, old, ref, a, offsets, 0.2, 0.2, 0.1, losses[i:i + 1], outs[i], mask=mask, stream=stream)
        B.mtpc_preference_loss(logp, ref, offsets, 0.1, losses[i + 1:i + 2], outs[i + 1], mask=mask, stream=stream)
    calls(0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph.replay()
    side.synchronize()
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3]) and torch.equal(losses[:2], losses[2:])
    side.wait_stream(torch.cuda.current_stream())
    outs[0].zero_()
    side.wait_stream(torch.cuda.current_stream())
    calls(0, stream=side)
    side.synchronize()
    assert torch.equal(outs[0], outs[2])
