"""Dropout against the fp64 oracle, with u = 2^-24 and U half a step of the output's type. x * scale: scale is within u of 65536 / (65536 - cut), the
product rounds once (2 u of it); the residual's addition rounds once (u of the sum); the result to its type."""
import numpy as np
import pytest
import torch

from oracle import mtpc_oracle_tune as tu
from paper_2511_11346_b200 import binding as B
from paper_2511_11346_b200 import runner as R

pytestmark = pytest.mark.gpu

U32, TINY = 2.0 ** -24, 2.0 ** -133
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def state(seed, step):
    wrap = lambda v: (v + 2 ** 63) % 2 ** 64 - 2 ** 63  # noqa: E731
    return torch.tensor([wrap(seed), wrap(step)], dtype=torch.int64, device="cuda")


def check(x, out, p, seed, step, offset=0, residual=None):
    given, res = host(x), host(residual)
    B.mtpc_dropout(x, out, p, state(seed, step), offset=offset, residual=residual)
    want = tu.dropout(given, p, seed, (step + offset) % 2 ** 64, res)
    size = np.abs(tu.dropout(given, p, seed, (step + offset) % 2 ** 64)) * 2 * U32 + np.abs(want) * (U32 + torch.finfo(out.dtype).eps / 2)
    assert (np.abs(host(out) - want) <= size * (1 + 8 * U32) + TINY).all()
    return want


@pytest.mark.parametrize("T,d,off,pad", [(1, 1, 0, 0), (1, 7, 0, 0), (3, 8, 0, 0), (5, 13, 0, 0), (5, 13, 1, 0), (4, 24, 0, 8), (4, 24, 0, 3), (2, 1000, 0, 0), (7, 33, 0, 7),
                                         (1, 2053, 0, 0), (40, 264, 0, 0)])
def test_sizes_types_and_strides(T, d, off, pad):
    torch.manual_seed(T * d)
    for ti in TYPES.values():
        for to in TYPES.values():
            x = torch.randn(T * (d + pad) + off, device="cuda").to(ti)[off:].view(T, d + pad)[:, :d]
            res = torch.randn(T * (d + pad) + off, device="cuda").to(to)[off:].view(T, d + pad)[:, :d]
            out = torch.full((T, d + pad), 7.0, dtype=to, device="cuda")
            check(x, out[:, :d], 0.3, 2 ** 63 + 5, 11)
            check(x, out[:, :d], 0.5, -3 % 2 ** 64, 2 ** 64 - 2, offset=5, residual=res)
            check(x, out[:, :d], 0.0, 1, 2 ** 40, residual=res)
            assert (out[:, d:] == 7).all()


def test_many_elements():
    """Blocks of draws two to a thread, odd and even numbers of them: all equal to the many rows' one by one."""
    for T, d in ((2400, 1024), (2401, 1032), (1, 2500001)):
        x = torch.randn(T, d, device="cuda").bfloat16()
        out, plain = torch.empty_like(x), torch.empty(T, d + 1, dtype=x.dtype, device="cuda")[:, :d]
        rng = state(17, 3)
        B.mtpc_dropout(x, out, 0.1, rng)
        spread = torch.empty(T, d + 1, dtype=x.dtype, device="cuda")[:, :d]
        spread.copy_(x)
        if T > 1:
            B.mtpc_dropout(spread, plain, 0.1, rng)
            assert torch.equal(out, plain)
        rows = min(T, 3)
        want = tu.dropout(host(x.view(-1)[:4096]).reshape(1, -1), 0.1, 17, 3)
        assert (np.abs(host(out.view(-1)[:4096]) - want[0]) <= np.abs(want[0]) * (2.0 ** -8 + 3 * U32)).all() and rows
        kept = (out != 0).double().mean().item()
        assert abs(kept - (1 - tu.dropout_cut(0.1) / 65536)) < 6 * (0.09 / x.numel()) ** 0.5
        assert (out.view(-1)[-9:] != 0).any()


def test_in_place_broadcast_and_gradient():
    T, d = 6, 40
    x, res, rng = torch.randn(T, d, device="cuda"), torch.randn(T, d, device="cuda"), state(5, 6)
    want = torch.empty_like(x)
    B.mtpc_dropout(x, want, 0.4, rng, residual=res)
    for target in ("x", "residual"):
        a, b = x.clone(), res.clone()
        B.mtpc_dropout(a, a if target == "x" else b, 0.4, rng, residual=b)
        assert torch.equal(a if target == "x" else b, want)
    same = torch.empty_like(x)
    B.mtpc_dropout(x[:1].expand(T, d), same, 0.4, rng)
    assert torch.equal(same != 0, (torch.tensor(tu.dropout_kept(T, d, 0.4, 5, 6), device="cuda")))
    # <d_out, dropout(x)> has the gradient dropout(d_out) in x
    d_out, d_x, y = torch.randn(T, d, device="cuda"), torch.empty_like(x), torch.empty_like(x)
    B.mtpc_dropout(d_out, d_x, 0.4, rng)
    B.mtpc_dropout(x, y, 0.4, rng)
    for t, c in ((0, 0), (3, 17), (5, 39)):
        up = x.clone()
        up[t, c] += 1.0
        z = torch.empty_like(x)
        B.mtpc_dropout(up, z, 0.4, rng)
        assert abs(float(((z - y).double() * d_out.double()).sum()) - d_x[t, c].item()) <= 1e-5


def test_dropped_places_may_hold_anything():
    x = torch.full((4, 64), float("nan"), device="cuda")
    kept = torch.tensor(tu.dropout_kept(4, 64, 0.5, 8, 9), device="cuda")
    x[kept] = 1.0
    out = torch.empty_like(x)
    B.mtpc_dropout(x, out, 0.5, state(8, 9))
    assert torch.equal(out, kept.float() * 2)


def test_replayed_graphs_draw_anew():
    x, rng = torch.ones(32, 128, device="cuda"), state(3, 0)
    y, g = torch.empty_like(x), torch.empty_like(x)
    R.dropout(x, 0.5, rng)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rng[1] += 1
        B.mtpc_dropout(x, y, 0.5, rng, offset=2)
        B.mtpc_dropout(x, g, 0.5, rng, offset=2)
    seen = []
    for step in range(1, 4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, g)
        assert torch.equal(y != 0, torch.tensor(tu.dropout_kept(32, 128, 0.5, 3, step + 2), device="cuda"))
        seen.append(y.clone())
    assert not torch.equal(seen[0], seen[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.mtpc_dropout(x, g, 0.5, rng, offset=2, stream=side)
    side.synchronize()
    assert torch.equal(y, g)


def test_calls_that_are_refused():
    x, rng = torch.ones(4, 8, device="cuda"), state(1, 1)
    out = torch.empty_like(x)
    for call in (lambda: B.mtpc_dropout(x, out[:3], 0.5, rng), lambda: B.mtpc_dropout(x.double(), out, 0.5, rng), lambda: B.mtpc_dropout(x, out, 1.0, rng),
                 lambda: B.mtpc_dropout(x, out, -0.1, rng), lambda: B.mtpc_dropout(x, out, 0.5, rng.int()), lambda: B.mtpc_dropout(x, out, 0.5, rng[:1]),
                 lambda: B.mtpc_dropout(x, out, 0.5, rng.cpu()), lambda: B.mtpc_dropout(x, out, 0.5, rng, residual=x.bfloat16()),
                 lambda: B.mtpc_dropout(x, out[:1].expand(4, 8), 0.5, rng), lambda: B.mtpc_dropout(x, out.t().contiguous().t(), 0.5, rng)):
        with pytest.raises(B.MtpcError):
            call()
    B.mtpc_dropout(x[:0], out[:0], 0.5, rng)


def test_places_beyond_32_bits():
    n = 2 ** 31 + 4096 + 3
    x = torch.ones(3, n // 3, dtype=torch.bfloat16, device="cuda")         # (a row has 2^30 elements at most)
    out = torch.empty_like(x)
    assert x.numel() == n
    B.mtpc_dropout(x, out, 0.5, state(21, 2))
    first = (n // 8 - 64)
    draws = []
    for block in range(first, -(-n // 8)):
        words = tu.philox4x32([block & tu.MASK32, block >> 32, 2, 0], [21, 0])
        draws += [part for w in words for part in (w & 0xFFFF, w >> 16)]
    want = np.array(draws[:n - 8 * first]) >= 32768
    assert np.array_equal(host(out.view(-1)[8 * first:]) != 0, want)
