"""Waits of the adapted projection and of its gradients that expire: with a limit of 50 ns, shorter than any copy, the kernels give up on their own, say so in the status word and
return; the next calls are what they were. (Nothing is withheld from a kernel: its copies land, and it waits for them before it ends.)"""
import pytest
import torch

from paper_2511_11346_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture
def limit():
    yield B.mtpc_debug_set_adapted_wait_limit_ns
    torch.cuda.synchronize()
    B.mtpc_debug_set_adapted_wait_limit_ns(0)


def equal(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


# one row with low in the same launch; few rows in clusters of one, four and eight; tiles of 64 and of 128 columns; pairs; odd rows, which are copied first
@pytest.mark.parametrize("T,d,m,k,S", [(1, 1024, 256, 16, 2), (2, 64, 200, 16, 2), (40, 512, 256, 16, 8), (40, 64, 128, 16, 8), (40, 256, 19100, 16, 8), (100, 1024, 136, 64, 16), (300, 512, 256, 64, 4), (700, 1024, 1300, 16, 3),
                                       (2100, 192, 1100, 20, 5), (1300, 136, 2072, 64, 2), (260, 201, 131, 33, 2)])
def test_calls_give_up_and_recover(T, d, m, k, S, limit):
    g = torch.Generator(device="cuda").manual_seed(T)
    new = lambda *s: (torch.randn(s, device="cuda", generator=g) * 0.2).bfloat16()  # noqa: E731
    x, W, A, Bf, d_out, low = new(T, d), new(m, d), new(S, m, k), new(S, k, d), new(T, m), torch.randn(T, k, device="cuda", generator=g)
    which = (torch.arange(T, device="cuda") % S).int()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    made = dict(d_x=torch.empty_like(x), dA=torch.empty(S, m, k, device="cuda"), dB=torch.empty(S, k, d, device="cuda"), d_x_low=torch.empty_like(x))

    def forward(status=status):
        out, kept = torch.empty(T, m, dtype=x.dtype, device="cuda"), torch.empty(T, k, device="cuda")
        B.mtpc_adapted_projection(x, W, A, Bf, None, which, out, out_low=kept, out_status=status)
        return out, kept

    def backward(*wanted, status=status):
        o = {key: torch.empty_like(t) if key in wanted else None for key, t in made.items()}
        B.mtpc_adapted_projection_backward(x, W, A, Bf, None, which, low, d_out, o["d_x"], o["dA"], o["dB"], d_x_low=o["d_x_low"], out_status=status)
        return tuple(t for t in o.values() if t is not None)

    calls = [forward] + [lambda w=w: backward(*w) for w in (("d_x",), ("d_x_low",), ("dA",), ("dB",), ("d_x", "dA", "dB"), ("d_x", "dA", "dB", "d_x_low"))]
    want = [call() for call in calls]
    torch.cuda.synchronize()
    assert status.item() == 0
    for call, right in zip(calls, want):
        limit(50)
        for _ in range(20):
            # a copy may have landed before its wait begins, since the waiting warp's instructions come from memory too the first time: no wait expires then
            got = call()
            torch.cuda.synchronize()                          # the kernels returned; the context is alive
            if status.item() != 0:
                break
            assert equal(got, right)
        assert status.item() == B.STATUS_TIMEOUT
        status.zero_()
        limit(0)
        assert equal(call(), right) and status.item() == 0
    limit(50)                                                 # nobody asks
    forward(status=None), backward("d_x", "dA", "dB", status=None)
    torch.cuda.synchronize()
    limit(0)
    assert equal(forward(), want[0]) and status.item() == 0


def test_captured_calls_keep_the_limit_that_they_were_captured_with(limit):
    T, d, m, k = 200, 256, 136, 16
    new = lambda *s: torch.randn(s, device="cuda").bfloat16()  # noqa: E731
    x, W, A, Bf, out, status = new(T, d), new(m, d), new(2, m, k), new(2, k, d), new(T, m), torch.zeros(1, dtype=torch.int32, device="cuda")

    def call():
        B.mtpc_adapted_projection(x, W, A, Bf, None, None, out, out_status=status)
    call()
    want = out.clone()
    graphs = []
    for ns in (50, 0):
        limit(ns)
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call()
    limit(0)
    for graph, bits in zip(graphs, (B.STATUS_TIMEOUT, 0)):
        status.zero_()
        for _ in range(20):
            graph.replay()
        torch.cuda.synchronize()
        assert status.item() == bits
    assert torch.equal(out, want)


def test_the_allocating_forms_say_so_too(limit):
    from paper_2511_11346_b200 import runner as R
    T, d, m, k = 200, 256, 136, 16
    new = lambda *s: torch.randn(s, device="cuda").bfloat16()  # noqa: E731
    x, W, A, Bf, d_out = new(T, d), new(m, d), new(2, m, k), new(2, k, d), new(T, m)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def forward():
        return R.adapted_projection(x, W, A, Bf, out_status=status)
    low = forward()[1]

    def backward():
        return R.adapted_projection_backward(x, W, A, Bf, low, d_out, x_low=x, out_status=status)
    backward()
    assert status.item() == 0
    for call in (forward, backward):
        limit(50)
        for _ in range(20):
            call()
        assert status.item() == B.STATUS_TIMEOUT
        status.zero_()
        limit(0)
        call()
        assert status.item() == 0
    none = torch.full((T,), 2, dtype=torch.int32, device="cuda")
    R.adapted_projection(x, W, A, Bf, row_adaptor=none, out_status=status)
    assert status.item() == B.STATUS_BAD_ADAPTOR
