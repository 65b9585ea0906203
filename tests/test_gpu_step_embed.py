"""Byte embeddings and their gradient against the fp64 oracle. With u = 2^-24 (fp32) and U half a step of the output's type:
lookup: one fp32 product, one rounding: |error| <= (u + U) |value| (1 + u).
gradient: a sum of m terms in fp32, cut into chunks and joined: every term passes m additions at most, the product with the scale and, accumulating,
one more addition: |error| <= (m + 3) u * sum of the terms' magnitudes."""
import numpy as np
import pytest
import torch

from oracle import mtpc_oracle_step as st
from paper_2511_11346_b200 import binding as B

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def half_step(t):
    return torch.finfo(t).eps / 2


def host(t):
    return t.detach().double().cpu().numpy()


def tokens_of(kind, T, v, rng):
    if kind == "zipf":
        p = 1.0 / np.arange(1, v + 1) ** 1.1
        t = rng.permutation(v)[rng.choice(v, size=T, p=p / p.sum())]
        t[rng.random(T) < 0.05] = -1
    elif kind == "one":
        t = np.full(T, v - 1)
    elif kind == "runs":                       # runs that end on, before and behind every cut
        t = np.repeat(np.arange(T), rng.integers(1, 60, size=T))[:T] % v
        t = rng.permutation(t)
    elif kind == "padding":
        t = np.full(T, -1)
    elif kind == "bad":
        t = rng.integers(0, v, size=T)
        t[::7] = v + rng.integers(0, 1000, size=len(t[::7]))
        t[::11] = -5
        t[0] = 2 ** 31 - 1
    else:
        t = rng.integers(0, v, size=T)
    return t.astype(np.int32)


@pytest.mark.parametrize("table,out", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("T,v,d,off,pad", [(1, 320, 4096, 0, 0), (64, 320, 4096, 0, 0), (5000, 320, 512, 0, 0), (333, 268, 1001, 0, 0), (17, 5, 8, 0, 8),
                                           (100, 1000, 64, 1, 3), (4800, 256, 72, 0, 8), (3, 1, 1, 0, 0), (70000, 31, 24, 0, 0)])
def test_lookup(table, out, T, v, d, off, pad):
    rng = np.random.default_rng(T + d)
    tokens = tokens_of("zipf" if T > 1 else "any", T, v, rng)
    tab = torch.randn(v * (d + pad) + off, dtype=torch.float32, device="cuda").to(TYPES[table])[off:].view(v, d + pad)[:, :d]
    whole = torch.full((T + 1, d + pad), 7.0, dtype=TYPES[out], device="cuda")
    B.mtpc_embed(torch.from_numpy(tokens).cuda(), tab, whole[:T, :d], scale=1.7)
    want = st.embed(tokens, host(tab), float(np.float32(1.7)))
    assert (np.abs(host(whole[:T, :d]) - want) <= (U32 + half_step(TYPES[out])) * np.abs(want) * (1 + U32)).all()
    assert (whole[T] == 7).all() and (whole[:, d:] == 7).all()                     # what lies beside and behind stays as it was


def test_lookup_of_bad_tokens_and_special_values():
    tokens = torch.tensor([0, -1, 7, 2 ** 31 - 1, -2 ** 31, 6, 1], dtype=torch.int32, device="cuda")
    table = torch.randn(7, 40, device="cuda")
    table[1, 3], table[0, 5], table[6, 0], table[6, 1] = float("nan"), float("inf"), -3.4e38, 1e-45
    out, status = torch.empty(7, 40, device="cuda"), torch.tensor([1], dtype=torch.int32, device="cuda")
    B.mtpc_embed(tokens, table, out, scale=1.0, out_status=status)
    assert status.item() == 1 | B.STATUS_BAD_TOKEN
    want = torch.zeros(7, 40, device="cuda")
    want[0], want[5], want[6] = table[0], table[6], table[1]
    want[2], want[3] = float("nan"), float("nan")
    assert torch.equal(torch.nan_to_num(out, nan=5.0), torch.nan_to_num(want, nan=5.0))
    status.zero_()
    B.mtpc_embed(tokens[:2], table, out[:2], out_status=status)
    B.mtpc_embed(tokens[:0], table, out[:0], out_status=status)
    assert status.item() == 0
    B.mtpc_embed(torch.zeros(5, dtype=torch.int32, device="cuda"), table[2:3].expand(3, 40), out[:5], scale=2.0)     # one row for every token
    assert torch.equal(out[:5], 2 * table[2].expand(5, 40))


def check_gradient(tokens, d_out, v, d_table, scale, start=None, status=None):
    B.mtpc_embed_backward(torch.from_numpy(tokens).cuda(), d_out, d_table, scale=scale, accumulate=start is not None, out_status=status)
    want, size = st.embed_grad(tokens, host(d_out), float(np.float32(scale)), v, None if start is None else host(start))
    m = np.bincount(tokens[(tokens >= 0) & (tokens < v)], minlength=v)[:, None]
    got = host(d_table)
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= (m + 3) * U32 * size).all(), np.abs(got - want).max()


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("kind,T,v,d", [
    ("any", 1, 320, 4096), ("zipf", 8192, 320, 512), ("zipf", 8192, 320, 1000), ("one", 5000, 320, 256), ("one", 16385, 3, 64), ("runs", 3000, 400, 96),
    ("runs", 16384, 511, 40), ("runs", 4097, 512, 1001), ("padding", 100, 10, 64), ("bad", 2000, 77, 64), ("any", 2005, 32768, 128), ("any", 17, 300000, 8),
    ("zipf", 40000, 320, 72), ("any", 33000, 5000, 33), ("any", 20000, 300000, 4), ("one", 70001, 1, 16), ("runs", 70000, 900, 12), ("any", 16, 4, 20000),
    ("any", 2, 2, 1), ("runs", 300000, 700, 3), ("any", 100, 32768, 300), ("bad", 128, 33000, 257), ("any", 1, 40000, 256),
])
def test_gradient(grad, kind, T, v, d):
    rng = np.random.default_rng(T + v)
    tokens = tokens_of(kind, T, v, rng)
    d_out = torch.randn(T, d, device="cuda").to(TYPES[grad])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    check_gradient(tokens, d_out, v, torch.full((v, d), float("nan"), device="cuda"), 0.7, status=status)
    assert status.item() == (B.STATUS_BAD_TOKEN if kind == "bad" else 0)


@pytest.mark.parametrize("kind,T,v,d", [("zipf", 3000, 320, 256), ("any", 5, 40, 33), ("one", 400, 3, 64), ("zipf", 20000, 320, 24),
                                        ("any", 100, 32769, 12), ("any", 100, 32768, 12)])
def test_gradient_added_to_a_tied_table(kind, T, v, d):
    rng = np.random.default_rng(9 + T)
    start = torch.randn(v, d, device="cuda")
    check_gradient(tokens_of(kind, T, v, rng), torch.randn(T, d, device="cuda"), v, start.clone(), 2.0, start=start)


@pytest.mark.parametrize("off,pad", [(0, 4), (1, 0), (2, 6), (0, 3)])
def test_gradient_of_strided_rows(off, pad):
    T, v, d = 700, 50, 132
    rng = np.random.default_rng(off + 10 * pad)
    for t in (torch.float32, torch.bfloat16):
        d_out = torch.randn(T * (d + pad) + off, device="cuda").to(t)[off:].view(T, d + pad)[:, :d]
        whole = torch.full((v * (d + pad) + off,), 3.0, device="cuda")
        table = whole[off:].view(v, d + pad)
        check_gradient(tokens_of("zipf", T, v, rng), d_out, v, table[:, :d], 1.0)
        assert (table[:, d:] == 3).all() and (whole[:off] == 3).all()
    one = torch.randn(1, d, device="cuda")
    check_gradient(tokens_of("any", T, v, rng), one.expand(T, d), v, torch.empty(v, d, device="cuda"), 1.0)      # the same row at every position


# The one launch of few positions, the sort in one, the digits' sort: on both sides of where one takes over.
@pytest.mark.parametrize("T", [127, 128, 129, 16384, 16385, 32768, 32769, 310000])
@pytest.mark.parametrize("kind,v,d", [("any", 1, 1), ("bad", 300, 37), ("bad", 511, 4), ("zipf", 512, 3), ("any", 300000, 2), ("zipf", 320, 64), ("padding", 7, 260)])
def test_gradient_where_the_kernels_change(kind, T, v, d):
    rng = np.random.default_rng(T)
    tokens = tokens_of(kind, T, v, rng)
    for t in (torch.float32, torch.bfloat16):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        d_out, start = torch.randn(T, d, device="cuda").to(t), torch.randn(v, d, device="cuda")
        check_gradient(tokens, d_out, v, torch.full((v, d), float("nan"), device="cuda"), 0.7, status=status)
        assert status.item() == (B.STATUS_BAD_TOKEN if kind == "bad" else 0)
        check_gradient(tokens, d_out, v, start.clone(), 0.7, start=start)


def test_few_positions_keep_infinities_in_their_rows_and_the_same_bits():
    rng = np.random.default_rng(3)
    tokens = tokens_of("zipf", 128, 20, rng)
    d_out = torch.randn(128, 300, device="cuda")
    d_out[5, 7], d_out[90] = float("inf"), float("nan")
    first, again = torch.empty(20, 300, device="cuda"), torch.empty(20, 300, device="cuda")
    where = torch.from_numpy(tokens).cuda()
    B.mtpc_embed_backward(where, d_out, first)
    for _ in range(20):
        B.mtpc_embed_backward(where, d_out, again)
        assert torch.equal(first.view(torch.int32), again.view(torch.int32))
    touched = {int(tokens[5]), int(tokens[90])}
    bad = set(torch.nonzero(~torch.isfinite(first).all(1)).flatten().tolist())
    assert bad == {b for b in touched if 0 <= b < 20}


def test_gradient_without_positions():
    table = torch.ones(300, 50, device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    B.mtpc_embed_backward(none, torch.zeros(0, 50, device="cuda"), table, accumulate=True)
    assert (table == 1).all()
    B.mtpc_embed_backward(none, torch.zeros(0, 50, device="cuda"), table)
    assert not table.any()


def test_infinities_stay_in_their_rows():
    T, v, d = 900, 30, 64
    tokens = tokens_of("any", T, v, np.random.default_rng(3))
    d_out = torch.randn(T, d, device="cuda")
    d_out[11] = float("inf")
    d_out[12, 5] = float("nan")
    pad = np.where(tokens == 7)[0]
    tokens[pad] = -1
    d_out[torch.from_numpy(pad).cuda()] = float("nan")                     # behind padding: never looked at
    table = torch.empty(v, d, device="cuda")
    B.mtpc_embed_backward(torch.from_numpy(tokens).cuda(), d_out, table)
    bad = ~torch.isfinite(table)
    rows = {int(tokens[i]) for i in (11, 12) if tokens[i] >= 0}
    assert set(torch.nonzero(bad.any(1)).flatten().tolist()) <= rows and not table[7].any()


def test_gradient_is_the_lookups():
    """<embed(table), out> differentiated by the formula is what the gradient call returns: the two calls are adjoint."""
    T, v, d = 1500, 100, 200
    rng = np.random.default_rng(5)
    tokens = torch.from_numpy(tokens_of("zipf", T, v, rng)).cuda()
    table, out, up = torch.randn(v, d, device="cuda"), torch.empty(T, d, device="cuda"), torch.randn(T, d, device="cuda")
    grad = torch.empty(v, d, device="cuda")
    B.mtpc_embed(tokens, table, out, scale=3.0)
    B.mtpc_embed_backward(tokens, up, grad, scale=3.0)
    left, right = (out.double() * up.double()).sum().item(), (table.double() * grad.double()).sum().item()
    # either side is a sum of T d products whose factors are rounded as above (at most T + 3 roundings each)
    assert abs(left - right) <= (T + 5) * U32 * (out.double() * up.double()).abs().sum().item()


def test_same_bits_on_streams_in_graphs_and_with_a_kept_workspace():
    T, v, d = 9000, 320, 256
    tokens = torch.from_numpy(tokens_of("zipf", T, v, np.random.default_rng(6))).cuda()
    ups = [torch.randn(T, d, device="cuda") for _ in range(3)]
    want = []
    for up in ups:
        g = torch.empty(v, d, device="cuda")
        B.mtpc_embed_backward(tokens, up, g)
        want.append(g)
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in range(3)]
    for turn in range(5):                                                # three calls at once
        got = [torch.zeros(v, d, device="cuda") for _ in ups]
        torch.cuda.synchronize()
        for s, up, g in zip(side, ups, got):
            B.mtpc_embed_backward(tokens, up, g, stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    up, g, out, table = ups[0].clone(), torch.zeros(v, d, device="cuda"), torch.zeros(T, d, device="cuda"), torch.randn(v, d, device="cuda")
    ws = torch.empty(B.mtpc_embed_backward_workspace_bytes(T, v, d), dtype=torch.uint8, device="cuda")
    graphs = []
    for kept in (None, ws):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.mtpc_embed(tokens, table, out)
            B.mtpc_embed_backward(tokens, up, g, workspace=kept)
        graphs.append(graph)
    for i, graph in enumerate(graphs + graphs[::-1]):
        up.copy_(ups[i % 3])
        g.fill_(9.0)
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(g, want[i % 3])
        assert torch.equal(out, torch.where(tokens[:, None] < 0, 0.0, table[tokens.clamp_min(0).long()]))


def test_offsets_beyond_32_bits():
    T, v, d = 40000, 300, 65536                                            # 2.6 G elements of bf16
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GB")
    tokens = tokens_of("any", T, v, np.random.default_rng(8))
    dev = torch.from_numpy(tokens).cuda()
    table = torch.randn(v, d, device="cuda").bfloat16()
    out = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    B.mtpc_embed(dev, table, out)
    for at in (0, 32767, 32768, 32769, T - 1):
        assert torch.equal(out[at], table[tokens[at]])
    grad = torch.empty(v, d, device="cuda")
    B.mtpc_embed_backward(dev, out, grad)
    count = torch.bincount(dev.long(), minlength=v)[:, None]
    want = count.double() * table.double()                               # count equal terms: (count + 3) u relative
    assert ((grad.double() - want).abs() <= (count + 3) * U32 * want.abs()).all()
