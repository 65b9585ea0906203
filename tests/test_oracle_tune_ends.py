"""Pins of the oracle of the losses of sequences at the ends of their range, where the values are known without it."""
import math

import numpy as np

from oracle import mtpc_oracle_tune as tu


def test_preference_of_windows_without_probability():
    logp, ref = np.full(8, -1.0), np.full(8, -1.0)
    for hole, smoothing, want in ((5, 0.0, 0.5 * math.log(2)), (1, 1.0, 0.5 * math.log(2)), (1, 0.0, math.inf), (5, 0.25, math.inf), (1, 0.25, math.inf)):
        x = logp.copy()
        x[hole if hole < 2 else 2] = -math.inf                        # of the preferred or of the rejected sequence of the first pair
        loss, h, grad = tu.preference_loss(x, ref, [0, 2, 4, 6, 8], 0.5, smoothing)
        assert loss == want and h[0] == (-math.inf if hole < 2 else math.inf) and h[1] == 0 and np.isfinite(grad).all()
        assert not grad[:4].any() or want == math.inf
    loss, h, grad = tu.preference_loss(x, ref, [0, 2, 4, 6, 8], 0.0)
    assert loss == math.log(2) and not h.any() and not grad.any()


def test_kl_term_of_windows_without_probability():
    one, bad = np.full(4, -1.0), np.array([-1.0, -math.inf, -1.0, -1.0])
    with np.errstate(all="raise"):
        loss, stats, grad, _ = tu.policy_loss(bad, one, one, [1.0, 1.0], [0, 2, 4], 0.2, 0.2, 0.5)
        assert loss == stats[1] == math.inf and stats[0] == -0.75 and grad[1] == -math.inf and (np.delete(grad, 1) == -0.25).all()
        loss, stats, grad, _ = tu.policy_loss(one, one, bad, [1.0, 1.0], [0, 2, 4], 0.2, 0.2, 0.5)
        assert loss == stats[1] == math.inf and stats[0] == -1 and grad[1] == -0.125
