"""The calls that fit a model to tasks, without a device: what they refuse, the workspaces they ask for."""
import ctypes

import pytest

from paper_2511_11346_b200 import binding as B

P, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(4098)           # never dereferenced: the argument checks come first
F32, BF16 = B.MTPC_F32, B.MTPC_BF16
NULL, SHAPE, UNSUPPORTED, WORKSPACE, CUDA = -1, -2, -3, -4, -5
BIG, NAN, INF = 1 << 40, float("nan"), float("inf")


def dropout(x=P, xs=64, xd=BF16, r=None, rs=64, T=4, d=64, p=0.1, rng=P, offset=0, out=P, os=64, od=BF16):
    return B.lib().mtpc_dropout(x, xs, xd, r, rs, T, d, p, rng, offset, out, os, od, None)


def policy(lp=P, old=P, ref=P, adv=P, per=0, mask=None, off=P, T=64, S=4, lo=0.2, hi=0.2, beta=0.1, seq=0, loss=P, stats=P, d=P, ws=P, wb=BIG, status=None):
    return B.lib().mtpc_policy_loss(lp, old, ref, adv, per, mask, off, T, S, lo, hi, beta, seq, loss, stats, d, ws, wb, status, None)


def preference(lp=P, ref=P, mask=None, off=P, T=64, S=4, beta=0.1, sm=0.0, loss=P, h=P, d=P, ws=P, wb=BIG, status=None):
    return B.lib().mtpc_preference_loss(lp, ref, mask, off, T, S, beta, sm, loss, h, d, ws, wb, status, None)


def project(x=P, xs=64, xl=None, xls=64, W=P, Ws=64, A=P, B_=P, sc=P, row=P, T=4, d=64, m=32, k=16, S=3, out=P, os=32, low=None, ws=P, wb=BIG, status=None):
    return B.lib().mtpc_adapted_projection(x, xs, xl, xls, W, Ws, A, B_, sc, row, T, d, m, k, S, out, os, low, ws, wb, status, None)


def project_back(xl=P, xls=64, W=P, Ws=64, A=P, B_=P, sc=P, row=P, low=P, T=4, d=64, m=32, k=16, S=3, g=P, gs=32, dx=P, dxs=64, dl=None, dls=64, dA=P, dB=P, ws=P, wb=BIG,
                 status=None):
    return B.lib().mtpc_adapted_projection_backward(xl, xls, W, Ws, A, B_, sc, row, low, T, d, m, k, S, g, gs, dx, dxs, dl, dls, dA, dB, ws, wb, status, None)


@pytest.mark.parametrize("call,kw,code", [
    (project, dict(x=None), NULL), (project, dict(W=None), NULL), (project, dict(A=None), NULL), (project, dict(B_=None), NULL), (project, dict(out=None), NULL),
    (project, dict(ws=None), NULL), (project, dict(wb=16), WORKSPACE), (project, dict(ws=ODD), WORKSPACE), (project, dict(T=-1), SHAPE), (project, dict(d=0), SHAPE),
    (project, dict(m=0), SHAPE), (project, dict(k=0), SHAPE), (project, dict(S=0), SHAPE), (project, dict(k=65), UNSUPPORTED), (project, dict(S=4097), UNSUPPORTED),
    (project, dict(T=(1 << 24) + 1), UNSUPPORTED), (project, dict(d=(1 << 17) + 1), UNSUPPORTED), (project, dict(m=(1 << 17) + 1, os=1 << 18), UNSUPPORTED),
    (project, dict(S=4096, k=64, d=1 << 17), UNSUPPORTED), (project, dict(xs=-64), SHAPE), (project, dict(Ws=-1), SHAPE), (project, dict(os=31), SHAPE), (project, dict(os=0), SHAPE),
    (project, dict(xl=P, xls=-1), SHAPE), (project, dict(x=ctypes.c_void_p(4097)), SHAPE), (project, dict(out=ctypes.c_void_p(4097)), SHAPE), (project, dict(sc=ODD), SHAPE),
    (project, dict(row=ODD), SHAPE), (project, dict(low=ODD), SHAPE), (project, dict(status=ODD), SHAPE),
    (project_back, dict(g=None), NULL), (project_back, dict(W=None), NULL), (project_back, dict(A=None), NULL), (project_back, dict(low=None), NULL),
    (project_back, dict(xl=None), NULL), (project_back, dict(ws=None), NULL), (project_back, dict(wb=16), WORKSPACE), (project_back, dict(dxs=63), SHAPE),
    (project_back, dict(dl=P, dls=0), SHAPE), (project_back, dict(gs=-1), SHAPE), (project_back, dict(dA=ODD), SHAPE), (project_back, dict(dB=ODD), SHAPE),
    (project_back, dict(k=65), UNSUPPORTED), (project_back, dict(T=-1), SHAPE),
    (dropout, dict(x=None), NULL), (dropout, dict(out=None), NULL), (dropout, dict(rng=None), NULL), (dropout, dict(T=-1), SHAPE), (dropout, dict(d=0), SHAPE),
    (dropout, dict(T=(1 << 30) + 1), SHAPE), (dropout, dict(d=(1 << 30) + 1), SHAPE), (dropout, dict(T=1 << 20, d=(1 << 20) + 1, os=1 << 21), UNSUPPORTED), (dropout, dict(p=1.0), SHAPE), (dropout, dict(p=-0.1), SHAPE),
    (dropout, dict(p=NAN), SHAPE), (dropout, dict(xd=2), SHAPE), (dropout, dict(od=-1), SHAPE), (dropout, dict(xs=-64), SHAPE), (dropout, dict(os=63), SHAPE),
    (dropout, dict(os=0), SHAPE), (dropout, dict(r=P, rs=-1), SHAPE), (dropout, dict(rng=ctypes.c_void_p(4100)), SHAPE), (dropout, dict(x=ODD, xd=F32), SHAPE),
    (dropout, dict(out=ODD, od=F32), SHAPE), (dropout, dict(r=ODD, od=F32), SHAPE),
    (policy, dict(lp=None), NULL), (policy, dict(old=None), NULL), (policy, dict(ref=None), NULL), (policy, dict(adv=None), NULL), (policy, dict(off=None), NULL),
    (policy, dict(loss=None), NULL), (policy, dict(d=None), NULL), (policy, dict(ws=None, T=1 << 20), NULL), (policy, dict(wb=16, T=1 << 20), WORKSPACE), (policy, dict(ws=ODD), WORKSPACE),
    (policy, dict(T=-1), SHAPE), (policy, dict(S=0), SHAPE), (policy, dict(S=(1 << 20) + 1), UNSUPPORTED), (policy, dict(T=(1 << 30) + 1), UNSUPPORTED),
    (policy, dict(lo=-0.1), SHAPE), (policy, dict(hi=NAN), SHAPE), (policy, dict(hi=INF), SHAPE), (policy, dict(beta=-1.0), SHAPE), (policy, dict(beta=NAN), SHAPE),
    (policy, dict(lp=ODD), SHAPE), (policy, dict(d=ODD), SHAPE), (policy, dict(off=ODD), SHAPE), (policy, dict(stats=ODD), SHAPE), (policy, dict(status=ODD), SHAPE),
    (preference, dict(lp=None), NULL), (preference, dict(ref=None), NULL), (preference, dict(off=None), NULL), (preference, dict(loss=None), NULL),
    (preference, dict(d=None), NULL), (preference, dict(ws=None, T=1 << 20), NULL), (preference, dict(wb=16, T=1 << 20), WORKSPACE), (preference, dict(ws=ODD), WORKSPACE), (preference, dict(S=3), SHAPE),
    (preference, dict(S=0), SHAPE), (preference, dict(beta=-0.1), SHAPE), (preference, dict(sm=1.5), SHAPE), (preference, dict(sm=NAN), SHAPE),
    (preference, dict(h=ODD), SHAPE), (preference, dict(ref=ODD), SHAPE),
])
def test_refusals(call, kw, code):
    assert call(**kw) == code


def test_what_is_allowed_reaches_the_check_for_a_device():
    import torch
    assert dropout(T=0, x=None, out=None, rng=None) == 0 and project(T=0, x=None, ws=None, wb=0) == 0
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    assert project() == project(T=1, xs=-1, os=0) == project(xl=P, sc=None, row=None, low=P) == project(x=ODD, k=5, d=33) == project(T=2, ws=None, wb=0) == CUDA
    assert project_back() == project_back(W=None, dx=None) == project_back(dA=None, low=None, dl=P) == project_back(dB=None, xl=None) == project_back(T=0) == CUDA
    assert dropout() == dropout(T=1, xs=-1, os=0) == dropout(x=ODD, out=ODD, p=0.0) == dropout(r=P, rs=0, od=F32) == CUDA
    assert policy() == policy(ws=None, wb=0) == policy(ref=None, beta=0.0, stats=None) == policy(lo=5.0, mask=ODD) == policy(T=0, lp=None, old=None, ref=None, d=None) == CUDA
    assert preference() == preference(ws=None, wb=0) == preference(h=None, sm=1.0) == preference(T=0, lp=None, ref=None, d=None) == CUDA


def test_workspaces():
    need, L = ctypes.c_size_t(0), B.lib()
    assert L.mtpc_objective_workspace_bytes(8, 8, None) == NULL and L.mtpc_objective_workspace_bytes(-1, 8, ctypes.byref(need)) == SHAPE
    for name in ("mtpc_adapted_projection_workspace_bytes", "mtpc_adapted_projection_backward_workspace_bytes"):
        f = getattr(L, name)
        assert f(8, 8, 8, 8, 8, 1, None) == NULL and f(8, 8, 8, 65, 8, 1, ctypes.byref(need)) == UNSUPPORTED and f(8, 8, 0, 8, 8, 1, ctypes.byref(need)) == SHAPE
        for T in (0, 1, 128, 129, 8192, 1 << 24):
            for d, m, k, S in ((1, 1, 1, 1), (4096, 4096, 16, 8), (1001, 2003, 12, 5), (1 << 17, 64, 64, 64)):
                sizes = []
                for rows in (1, 0):
                    assert f(T, d, m, k, S, rows, ctypes.byref(need)) == 0 and need.value % 256 == 0
                    sizes.append(need.value)
                assert sizes[0] <= sizes[1] and (T == 0 or sizes[1] >= 2 * m * d)
    assert L.mtpc_objective_workspace_bytes(8, 0, ctypes.byref(need)) == SHAPE and L.mtpc_objective_workspace_bytes(8, 1 << 21, ctypes.byref(need)) == UNSUPPORTED
    for T in (0, 1, 511, 65536, 65537, 1 << 20, 1 << 30):
        for S in (1, 2, 1000, 1 << 20):
            n = B.mtpc_objective_workspace_bytes(T, S)
            assert n % 256 == 0 and (n >= 18 * S or (n == 0 and S <= 1000 and T <= 65536))
    assert B.mtpc_objective_workspace_bytes(1 << 21, 256) < 1 << 20 and B.mtpc_objective_workspace_bytes(512, 8) == 0


def test_tensors_that_do_not_fit_are_refused():
    import torch
    x, i = torch.zeros(4, 8), torch.zeros(5, dtype=torch.int32)
    for call in (lambda: B.mtpc_dropout(x, x, 0.1, torch.zeros(2, dtype=torch.int64)), lambda: B.mtpc_policy_loss(x[0], x[0], x[0], x[1], i, 0.2, 0.2, 0.1, x[0], x[0]),
                 lambda: B.mtpc_preference_loss(x[0], x[0], i, 0.1, x[0], x[0])):
        with pytest.raises(B.MtpcError):
            call()                                        # no tensor of a device
