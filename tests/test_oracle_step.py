"""Pins of oracle/mtpc_oracle_step.py: gradients against central differences of its forward functions, e4m3 against the table of its values."""
import numpy as np

from oracle import mtpc_oracle_step as st


def differences(f, x, h=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        g[i] = (f(up) - f(down)) / (2 * h)
    return g


def test_embedding_gradient_is_the_lookups():
    rng = np.random.default_rng(1)
    table, out = rng.normal(size=(5, 3)), rng.normal(size=(9, 3))
    tokens = np.array([0, 4, 4, -1, 2, 0, 4, 7, 2])
    weight = out * (tokens < 5)[:, None]                                  # a row that is no token has no gradient
    f = lambda x: float((np.nan_to_num(st.embed(tokens, x, 1.5)) * weight).sum())  # noqa: E731
    grad, size = st.embed_grad(tokens, out, 1.5, 5)
    assert np.abs(grad - differences(f, table)).max() < 1e-9
    assert (size >= np.abs(grad)).all() and not grad[[1, 3]].any()
    again, _ = st.embed_grad(tokens, out, 1.5, 5, start=table)
    assert np.abs(again - grad - table).max() < 1e-15
    assert np.isnan(st.embed(tokens, table, 1.5)[7]).all() and not st.embed(tokens, table, 1.5)[3].any()


def test_norm_gradients_are_the_norms():
    rng = np.random.default_rng(2)
    x, res, w, dy, more = (rng.normal(size=(3, 7)), rng.normal(size=(3, 7)), rng.normal(size=7), rng.normal(size=(3, 7)), rng.normal(size=(3, 7)))
    f = lambda x, r, w: float((st.rmsnorm(x, r, w, 0.1)[1] * dy).sum() + ((x + r) * more).sum())  # noqa: E731
    s, _ = st.rmsnorm(x, res, w, 0.1)
    dx, dw, _, _ = st.rmsnorm_grad(s, w, 0.1, dy, more)
    assert np.abs(dx - differences(lambda y: f(y, res, w), x)).max() < 1e-8
    assert np.abs(dx - differences(lambda y: f(x, y, w), res)).max() < 1e-8
    assert np.abs(dw - differences(lambda y: f(x, res, y), w)).max() < 1e-8
    s, out = st.rmsnorm(x, None, None, 1e-12)
    assert (s == x).all() and np.abs((out * out).mean(1) - 1).max() < 1e-9


def test_e4m3_is_the_nearest_of_its_values():
    values = sorted({m * 2.0 ** -9 for m in range(8)} | {(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8) if (1 + m / 8) * 2.0 ** e <= 448})
    values = np.array([-x for x in values[:0:-1]] + values)
    x = np.random.default_rng(3).normal(size=4000) * np.exp(np.random.default_rng(4).uniform(-8, 7, size=4000))
    near = values[np.abs(x[:, None] - values[None, :]).argmin(1)]
    got = st.e4m3(x)
    assert (np.abs(got - x) == np.abs(near - x)).all() and np.isin(got, values).all()
    assert (st.e4m3(values) == values).all() and st.e4m3(1.0625) == 1.0 and st.e4m3(1.1875) == 1.25 and st.e4m3(1e9) == 448


def test_clipped_gradients_have_the_norm():
    g = [np.random.default_rng(5).normal(size=s) for s in (3, 1, 50)]
    norm, out = st.clip(g, 0.5)
    assert abs(np.sqrt(sum((x ** 2).sum() for x in out)) - 0.5) < 1e-12 and norm > 0.5
    assert all((x == y).all() for x, y in zip(g, st.clip(g, 100.0)[1]))
