"""The losses of sequences in the forms that long batches take, against the same in vectors of fp64 (u = 2^-24). The warps' slices of a sequence, here `parts_of`, decide the form.
policy: expf is within 2 units in the last place (4 u), what rounding leaves of a difference of log-likelihoods is taken in within u, the product with the advantage, the weight and its
product u each; the KL term's e^q - 1 as much of |e^q - 1| + |q|, e^q - 1 - q within 12 u of e^q: 12 u of the terms' magnitudes, as in the test of short batches. preference: fp64, rounded once."""
import numpy as np
import pytest
import torch

from paper_2511_11346_b200 import binding as B

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24


def parts_of(T, S):
    """Slices of a sequence and whether one cluster does the call."""
    short = T <= 1 << 16
    parts = max(1, min(-(-T // (S * 128)), (1024 if short else 148 * 2 * 16) // S))
    return parts, short and S * parts <= 1024


def lengths_of(T, S, seed):
    """S lengths, uneven, some of them zero, that add up to T."""
    rng = np.random.default_rng(seed)
    share = rng.exponential(size=S) * (rng.random(S) < 0.9)
    n = np.floor(share / max(share.sum(), 1e-9) * T).astype(int)
    n[rng.integers(S)] += T - n.sum()
    return n


def batch(T, S, masked, off, seed, behind=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lengths_of(T - behind, S, seed)
    new = lambda std: torch.randn(T + off, device="cuda", generator=g)[off:] * std  # noqa: E731
    logp = -11 * torch.rand(T + off, device="cuda", generator=g)[off:]
    old, ref = logp + new(0.3), logp + new(0.2)
    mask = (torch.rand(T + off, device="cuda", generator=g) < 0.7)[off:] if masked else None
    of = torch.repeat_interleave(torch.arange(S, device="cuda"), torch.tensor(n, device="cuda"))
    return logp, old, ref, mask, torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32, device="cuda"), of, g


@pytest.mark.parametrize("masked,off", [(False, 0), (True, 0), (True, 1), (False, 1)])
@pytest.mark.parametrize("T,S,parts,small", [
    (65000, 50, 11, True), (64001, 40, 13, True), (65536, 1024, 1, True),      # one cluster: blocks that share two or three sequences, one slice each
    (60000, 2, 235, True), (60003, 3, 157, True),                              # longer than a warp counts by itself
    (400001, 300, 11, False), (600000, 320, 14, False),                        # a launch for each phase
    (200000, 256, 7, False), (80000, 2, 313, False), (100001, 6000, 1, False)])
def test_policy(T, S, parts, small, masked, off):
    assert parts_of(T, S) == (parts, small)
    logp, old, ref, mask, offsets, of, g = batch(T, S, masked, off, T + S)
    n = len(of)
    valid = torch.ones(n, dtype=torch.bool, device="cuda") if mask is None else mask[:n]
    by_s, by_t = torch.randn(S, device="cuda", generator=g), torch.randn(T + off, device="cuda", generator=g)[off:]
    count = torch.zeros(S, device="cuda", dtype=torch.float64).index_add_(0, of, valid.double())
    for by_sequence, by_position, beta in ((True, False, 0.125), (False, False, 0.0), (True, True, 0.0), (False, True, 0.125)):
        d, loss, stats = torch.full_like(logp, 9.0), torch.empty(1, device="cuda"), torch.empty(3, device="cuda")
        again, loss2 = torch.full_like(logp, 9.0), torch.empty(1, device="cuda")
        for to, value, extra in ((d, loss, stats), (again, loss2, None)):
            B.mtpc_policy_loss(logp, old, ref if beta else None, by_t if by_position else by_s, offsets, 0.25, 0.25, beta, value, to, mask=mask, by_sequence=by_sequence,
                               by_position=by_position, out_stats=extra)
        assert torch.equal(d, again) and torch.equal(loss, loss2) and (d[n:] == 9).all() and not d[:n][~valid].any()
        w = torch.where(valid, 1 / (S * count.clamp_min(1))[of] if by_sequence else 1 / count.sum(), 0.0)
        adv = by_t[:n].double() if by_position else by_s.double()[of]
        r, q = torch.exp(logp[:n].double() - old[:n].double()), ref[:n].double() - logp[:n].double()
        held = r.clamp(0.75, 1.25) * adv
        first, kl = -torch.minimum(r * adv, held), torch.expm1(q) - q
        grad = w * (torch.where(held < r * adv, 0.0, -r * adv) - beta * torch.expm1(q))
        bar = 12 * U32 * w * (r * adv.abs() + beta * (torch.expm1(q).abs() + q.abs()))
        assert ((d[:n].double() - grad).abs() <= bar + 1e-40).all()
        want, size = float((w * (first + beta * kl)).sum()), float((w * (first.abs() + beta * (kl + torch.exp(q)))).sum())
        assert abs(loss.item() - want) <= 12 * U32 * size + U32 * abs(want)
        assert abs(stats[0].item() - float((w * first).sum())) <= 13 * U32 * float((w * first.abs()).sum())
        assert abs(stats[1].item() - (float((w * kl).sum()) if beta else 0.0)) <= 13 * U32 * float((w * torch.exp(q)).sum())
        clipped = float((w * (held < r * adv)).sum())
        assert abs(stats[2].item() - clipped) <= 2 * U32 * clipped + 1e-12


@pytest.mark.parametrize("masked,off", [(False, 0), (True, 0), (True, 1), (False, 1)])
@pytest.mark.parametrize("T,S,parts,small", [
    (200000, 256, 7, False), (70000, 1024, 1, False), (1000003, 128, 37, False),       # pairs formed by whoever needs them
    (200000, 1200, 2, False), (200000, 2, 782, False), (100001, 6000, 1, False),   # in a launch of their own
    (65000, 50, 11, True), (30000, 1024, 1, True), (3000, 2000, 1, False)])
def test_preference(T, S, parts, small, masked, off):
    assert parts_of(T, S) == (parts, small)
    logp, _, ref, mask, offsets, of, _ = batch(T, S, masked, off, T + S)
    n = len(of)
    valid = torch.ones(n, dtype=torch.bool, device="cuda") if mask is None else mask[:n]
    for beta, smoothing in ((0.1, 0.0), (0.02, 0.2), (0.1, 1.0)):
        d, loss, h = torch.full_like(logp, 9.0), torch.empty(1, device="cuda"), torch.empty(S // 2, device="cuda")
        again, loss2 = torch.full_like(logp, 9.0), torch.empty(1, device="cuda")
        B.mtpc_preference_loss(logp, ref, offsets, beta, loss, d, mask=mask, smoothing=smoothing, out_h=h)
        B.mtpc_preference_loss(logp, ref, offsets, beta, loss2, again, mask=mask, smoothing=smoothing)
        assert torch.equal(d, again) and torch.equal(loss, loss2) and (d[n:] == 9).all() and not d[:n][~valid].any()
        b, s = float(np.float32(beta)), float(np.float32(smoothing))
        total = torch.zeros(S, device="cuda", dtype=torch.float64).index_add_(0, of, torch.where(valid, logp[:n].double() - ref[:n].double(), 0.0))
        want_h = b * (total[0::2] - total[1::2])
        want = float((-(1 - s) * torch.nn.functional.logsigmoid(want_h) - s * torch.nn.functional.logsigmoid(-want_h)).mean())
        slope = b * (s - torch.sigmoid(-want_h)) / (S // 2)
        grad = torch.where(valid, torch.stack([slope, -slope], 1).reshape(-1)[of], 0.0)
        # fp64 sums in another order: some 1e-13 of the terms' magnitudes, beside one rounding
        assert ((h.double() - want_h).abs() <= 1.01 * U32 * want_h.abs() + 1e-9).all()
        assert ((d[:n].double() - grad).abs() <= 1.01 * U32 * grad.abs() + 1e-9 * b / S).all()
        assert abs(loss.item() - want) <= 1.01 * U32 * want + 1e-9
