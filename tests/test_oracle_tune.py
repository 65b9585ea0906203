"""Pins of the oracle of dropout and the losses of sequences."""
import numpy as np
import pytest

from oracle import mtpc_oracle_tune as tu


def test_philox_equals_the_published_known_answers():
    # kat_vectors of the authors' Random123 distribution, philox4x32 with ten rounds
    assert tu.philox4x32([0, 0, 0, 0], [0, 0]) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert tu.philox4x32([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert tu.philox4x32([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_dropout_keeps_the_mean_and_its_share():
    x = np.ones((64, 257))
    y = tu.dropout(x, 0.25, 99, 3)
    kept = (y != 0).mean()
    assert abs(kept - 0.75) < 5 * np.sqrt(0.75 * 0.25 / x.size) and np.allclose(y[y != 0], 4 / 3)
    assert (tu.dropout(x, 0.25, 99, 4) != y).any() and (tu.dropout(x, 0.25, 100, 3) != y).any()
    assert (tu.dropout(x, 0.0, 99, 3) == x).all() and tu.dropout_cut(0.999999) == 65535
    # a place's draw does not depend on the rows' width
    assert (tu.dropout_kept(64, 257, 0.25, 99, 3).ravel() == tu.dropout_kept(257, 64, 0.25, 99, 3).ravel()).all()


@pytest.mark.parametrize("by_sequence", [False, True])
@pytest.mark.parametrize("beta", [0.0, 0.3])
@pytest.mark.parametrize("by_position", [False, True])
def test_policy_gradient_by_differences(by_sequence, beta, by_position):
    rng = np.random.default_rng(5)
    offsets = [0, 4, 4, 9, 15]
    logp = -5 * rng.random(17)
    old, ref, a = logp + 0.3 * rng.standard_normal(17), logp + 0.3 * rng.standard_normal(17), rng.standard_normal(17 if by_position else 4)
    mask = rng.random(17) < 0.8
    call = lambda lp: tu.policy_loss(lp, old, ref, a, offsets, 0.2, 0.28, beta, mask, by_sequence, by_position)  # noqa: E731
    grad, eps = call(logp)[2], 1e-6
    assert np.isnan(grad[15:]).all()
    for t in range(15):
        up, down = logp.copy(), logp.copy()
        up[t] += eps
        down[t] -= eps
        assert abs((call(up)[0] - call(down)[0]) / (2 * eps) - grad[t]) < 1e-8
    assert (grad[:15][~mask[:15]] == 0).all()


def test_policy_by_hand():
    # ratios 1, 2, 1/2, 2 with advantages 1, 1, -1, -1; clipped to [0.8, 1.25]
    logp, old = np.log([1, 2, 1, 2]), np.log([1, 1, 2, 1])
    loss, stats, grad, _ = tu.policy_loss(logp, old, logp, [1, -1], [0, 2, 4], 0.2, 0.25, 0.0)
    assert np.allclose(loss, (-1 - 1.25 + 0.8 + 2) / 4) and np.allclose(stats[2], 0.5) and np.allclose(grad, np.array([-1, 0, 0, 2]) / 4)


@pytest.mark.parametrize("smoothing", [0.0, 0.2, 1.0])
def test_preference_gradient_by_differences(smoothing):
    rng = np.random.default_rng(6)
    offsets = [0, 3, 8, 8, 12, 14, 15]
    logp = -5 * rng.random(16)
    ref, mask = logp + rng.standard_normal(16), rng.random(16) < 0.8
    call = lambda lp: tu.preference_loss(lp, ref, offsets, 0.7, smoothing, mask)  # noqa: E731
    loss, h, grad = call(logp)
    assert np.isnan(grad[15]) and len(h) == 3
    for t in range(15):
        up, down = logp.copy(), logp.copy()
        up[t] += 1e-6
        down[t] -= 1e-6
        assert abs((call(up)[0] - call(down)[0]) / 2e-6 - grad[t]) < 1e-8
    assert np.allclose(tu.preference_loss(logp, logp, offsets, 0.7)[0], np.log(2))


def test_adapted_projection_is_the_composed_matrix():
    rng = np.random.default_rng(7)
    T, d, m, k, S = 6, 5, 4, 2, 3
    x, W, A, B = (rng.standard_normal(s) for s in ((T, d), (m, d), (S, m, k), (S, k, d)))
    scale, which = rng.random(S), np.array([0, 2, -1, 2, 1, 3])
    out, low, size, _ = tu.adapted_projection(x, W, A, B, scale, which)
    for t in (0, 1, 3, 4):
        i = which[t]
        assert np.allclose(out[t], (W + scale[i] * A[i] @ B[i]) @ x[t]) and np.allclose(A[i] @ low[t], out[t] - W @ x[t])
    assert np.allclose(out[2], W @ x[2]) and not low[2].any() and np.isnan(out[5]).all() and (np.abs(out[:5]) <= size[:5]).all()
    other = rng.standard_normal((T, d))
    assert np.allclose(tu.adapted_projection(x, W, A, B, None, None, other)[0], x @ W.T + other @ (A[0] @ B[0]).T)


def test_adapted_projection_gradients_by_differences():
    rng = np.random.default_rng(8)
    T, d, m, k, S = 5, 4, 3, 2, 2
    given = dict(x=rng.standard_normal((T, d)), x_low=rng.standard_normal((T, d)), A=rng.standard_normal((S, m, k)), B=rng.standard_normal((S, k, d)))
    W, scale, which, g = rng.standard_normal((m, d)), rng.random(S), np.array([1, -1, 0, 1, 1]), rng.standard_normal((T, m))
    value = lambda v: float((tu.adapted_projection(v["x"], W, v["A"], v["B"], scale, which, v["x_low"])[0] * g).sum())  # noqa: E731
    low = tu.adapted_projection(given["x"], W, given["A"], given["B"], scale, which, given["x_low"])[1]
    got = tu.adapted_projection_grad(given["x_low"], W, given["A"], given["B"], scale, which, low, g)
    assert np.allclose(got["d_x"], got["d_x_base"] + got["d_x_low"])
    for name, grad in (("x", "d_x_base"), ("x_low", "d_x_low"), ("A", "dA"), ("B", "dB")):
        for at in np.ndindex(given[name].shape):
            up, down = dict(given), dict(given)
            up[name], down[name] = given[name].copy(), given[name].copy()
            up[name][at] += 1e-6
            down[name][at] -= 1e-6
            assert abs((value(up) - value(down)) / 2e-6 - got[grad][at]) < 1e-7
