"""The calls beside the head, without a device: what they refuse, the workspaces they ask for, and that nothing is computed without a GPU."""
import ctypes

import pytest

from paper_2511_11346_b200 import binding as B

P = ctypes.c_void_p(4096)           # never dereferenced: the argument checks come first
ODD = ctypes.c_void_p(4098)
F32, BF16 = B.MTPC_F32, B.MTPC_BF16
NULL, SHAPE, UNSUPPORTED, WORKSPACE, CUDA = -1, -2, -3, -4, -5
BIG = 1 << 40


def embed(tokens=P, T=4, table=P, ts=64, td=BF16, v=320, d=64, out=P, os=64, od=BF16, status=None):
    return B.lib().mtpc_embed(tokens, T, table, ts, td, v, d, 1.0, out, os, od, status, None)


def embed_backward(tokens=P, T=4, do=P, ds=64, dd=F32, v=320, d=64, dt=P, dts=64, acc=0, ws=P, wb=BIG, status=None):
    return B.lib().mtpc_embed_backward(tokens, T, do, ds, dd, 1.0, v, d, dt, dts, acc, ws, wb, status, None)


def norm(x=P, xs=64, r=P, rs=64, w=P, wd=BF16, T=4, d=64, io=BF16, eps=1e-5, s=P, ss=64, out=P, os=64, q=None, qs=64, sc=None, group=0):
    return B.lib().mtpc_residual_rmsnorm(x, xs, r, rs, w, wd, T, d, io, eps, s, ss, out, os, q, qs, sc, group, None)


def norm_backward(s=P, ss=64, io=BF16, w=P, wd=BF16, T=4, d=64, eps=1e-5, do=P, dos=64, dod=F32, dm=None, dms=64, dx=P, dxs=64, dxd=BF16, dw=P,
                  ws=P, wb=BIG):
    return B.lib().mtpc_residual_rmsnorm_backward(s, ss, io, w, wd, T, d, eps, do, dos, dod, dm, dms, dx, dxs, dxd, dw, ws, wb, None)


@pytest.mark.parametrize("call,kw,code", [
    (embed, dict(tokens=None), NULL), (embed, dict(table=None), NULL), (embed, dict(out=None), NULL), (embed, dict(T=-1), SHAPE),
    (embed, dict(v=0), SHAPE), (embed, dict(d=0), SHAPE), (embed, dict(td=2), SHAPE), (embed, dict(od=-1), SHAPE), (embed, dict(ts=-64), SHAPE),
    (embed, dict(os=63), SHAPE), (embed, dict(os=0), SHAPE), (embed, dict(T=(1 << 26) + 1), UNSUPPORTED), (embed, dict(v=(1 << 20) + 1), UNSUPPORTED),
    (embed, dict(d=(1 << 20) + 1), UNSUPPORTED), (embed, dict(tokens=ODD), SHAPE), (embed, dict(table=ODD, td=F32), SHAPE), (embed, dict(status=ODD), SHAPE),
    (embed_backward, dict(tokens=None), NULL), (embed_backward, dict(do=None), NULL), (embed_backward, dict(dt=None), NULL),
    (embed_backward, dict(ws=None), NULL), (embed_backward, dict(wb=16), WORKSPACE), (embed_backward, dict(ws=ODD), WORKSPACE),
    (embed_backward, dict(dts=63), SHAPE), (embed_backward, dict(ds=-1), SHAPE), (embed_backward, dict(dd=2), SHAPE), (embed_backward, dict(T=-1), SHAPE),
    (embed_backward, dict(dt=ODD), SHAPE), (embed_backward, dict(v=(1 << 20) + 1), UNSUPPORTED),
    (norm, dict(x=None), NULL), (norm, dict(out=None), NULL), (norm, dict(q=P), NULL), (norm, dict(sc=P), NULL), (norm, dict(T=-1), SHAPE),
    (norm, dict(T=(1 << 30) + 1), SHAPE), (norm, dict(d=0), SHAPE), (norm, dict(io=2), SHAPE), (norm, dict(wd=2), SHAPE), (norm, dict(eps=0.0), SHAPE),
    (norm, dict(eps=-1.0), SHAPE), (norm, dict(eps=float("nan")), SHAPE), (norm, dict(eps=float("inf")), SHAPE), (norm, dict(xs=-64), SHAPE),
    (norm, dict(rs=-1), SHAPE), (norm, dict(ss=0), SHAPE), (norm, dict(os=63), SHAPE), (norm, dict(q=P, sc=P, qs=63), SHAPE),
    (norm, dict(d=32769, os=40000, ss=40000), UNSUPPORTED), (norm, dict(q=P, sc=P, group=16), UNSUPPORTED), (norm, dict(q=P, sc=P, group=-32), UNSUPPORTED),
    (norm, dict(q=P, sc=P, group=256), UNSUPPORTED), (norm, dict(x=ODD, io=F32), SHAPE), (norm, dict(w=ODD, wd=F32), SHAPE), (norm, dict(q=P, sc=ODD), SHAPE),
    (norm_backward, dict(s=None), NULL), (norm_backward, dict(do=None), NULL), (norm_backward, dict(dx=None), NULL), (norm_backward, dict(ws=None), NULL),
    (norm_backward, dict(wb=0), WORKSPACE), (norm_backward, dict(ws=ODD), WORKSPACE), (norm_backward, dict(eps=0.0), SHAPE), (norm_backward, dict(T=-1), SHAPE),
    (norm_backward, dict(dod=2), SHAPE), (norm_backward, dict(dxd=2), SHAPE), (norm_backward, dict(dxs=0), SHAPE), (norm_backward, dict(dm=P, dms=-1), SHAPE),
    (norm_backward, dict(do=ODD), SHAPE), (norm_backward, dict(d=32769, dxs=40000), UNSUPPORTED),
])
def test_refusals(call, kw, code):
    assert call(**kw) == code


def test_calls_without_work_need_no_device():
    assert embed(T=0, tokens=None, table=None, out=None) == 0
    assert embed_backward(T=0, tokens=None, do=None, ws=None, wb=0, acc=1) == 0
    assert norm(T=0, x=None, out=None) == 0
    assert norm_backward(T=0, s=None, do=None, dx=None, dw=None, ws=None) == 0


def test_one_row_needs_no_stride():
    """(the next check is the device's)"""
    import torch
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    assert embed(T=1, os=0) == CUDA and embed(v=1, ts=-5) == CUDA
    assert norm(T=1, xs=-3, rs=0, ss=0, os=0) == CUDA
    assert norm_backward(T=1, ss=-1, dos=-1, dxs=0) == CUDA and norm_backward(dw=None, ws=None, wb=0) == CUDA
    assert embed() == embed_backward() == norm() == norm(r=None, w=None, s=None) == norm_backward() == CUDA
    assert norm(out=None, q=P, sc=P, group=128) == CUDA


def test_workspaces():
    need = ctypes.c_size_t(0)
    L = B.lib()
    assert L.mtpc_embed_backward_workspace_bytes(8, 8, 8, None) == NULL and L.mtpc_residual_rmsnorm_backward_workspace_bytes(8, 8, None) == NULL
    assert L.mtpc_embed_backward_workspace_bytes(-1, 8, 8, ctypes.byref(need)) == SHAPE
    assert L.mtpc_embed_backward_workspace_bytes(8, 1 << 21, 8, ctypes.byref(need)) == UNSUPPORTED
    assert L.mtpc_residual_rmsnorm_backward_workspace_bytes(8, 0, ctypes.byref(need)) == SHAPE
    assert L.mtpc_residual_rmsnorm_backward_workspace_bytes(8, 40000, ctypes.byref(need)) == UNSUPPORTED
    for T in (0, 1, 16, 17, 8192, 16385, 1 << 26):
        for v in (1, 511, 512, 32768, 1 << 20):
            for d in (1, 33, 4096, 1 << 20):
                n = B.mtpc_embed_backward_workspace_bytes(T, v, d)
                assert n % 256 == 0 and n >= 8 * T + 8 * d            # keys, positions and a chunk's two parts at least
    assert B.mtpc_embed_backward_workspace_bytes(8192, 320, 4096) < 12 << 20
    assert B.mtpc_residual_rmsnorm_backward_workspace_bytes(8192, 4096) < 16 << 20


def entries(*rows):
    a = (B.MtpcGradient * max(1, len(rows)))()
    for e, (data, out, count, dtype, out_dtype) in zip(a, rows):
        e.data, e.out, e.count, e.dtype, e.out_dtype = data, out, count, dtype, out_dtype
    return a


def create(rows, ws=P, wb=BIG):
    handle = ctypes.c_void_p(0)
    code = B.lib().mtpc_create_gradient_list(entries(*rows), len(rows), ws, wb, None, ctypes.byref(handle))
    assert not handle.value or code == 0
    return code


@pytest.mark.parametrize("rows,code", [
    ([(None, None, 4, F32, F32)], NULL), ([(4096, 0, -1, F32, F32)], SHAPE), ([(4096, 0, 4, 2, F32)], SHAPE), ([(4096, 8192, 4, F32, 7)], SHAPE),
    ([(4098, 0, 4, F32, F32)], SHAPE), ([(4096, 8193, 4, F32, BF16)], SHAPE), ([(4096, 0, (1 << 40) + 1, F32, F32)], SHAPE),
    ([(4096, 4096, 4, F32, BF16)], SHAPE),                                                       # in place with another type
    ([(4096, 4100, 4, F32, F32)], SHAPE),                                                        # a result over its own data, moved
    ([(4096, 4096, 4, F32, F32), (4096, 4096, 4, F32, F32)], SHAPE),                             # twice in place
    ([(4096, 4096, 8, F32, F32), (4112, 0, 1, F32, F32)], SHAPE),                                # another entry's data within a result
    ([(4096, 8192, 4, F32, F32), (4112, 8204, 4, F32, F32)], SHAPE),                             # results that overlap
    ([(8192, 0, 4, F32, F32), (4096, 8184, 4, F32, F32)], SHAPE),
])
def test_gradient_lists_that_are_refused(rows, code):
    assert create(rows) == code


def test_gradient_lists():
    import torch
    L, need = B.lib(), ctypes.c_size_t(0)
    rows = [(4096, 4096, 4, F32, F32), (4112, 4112, 4, F32, F32), (4096, 0, 0, F32, F32), (9000, 9000, 7, BF16, BF16)]
    assert L.mtpc_gradient_list_workspace_bytes(entries(*rows), 4, ctypes.byref(need)) == 0 and need.value == 512
    assert L.mtpc_gradient_list_workspace_bytes(None, 0, ctypes.byref(need)) == 0 and L.mtpc_gradient_list_workspace_bytes(None, 1, ctypes.byref(need)) == NULL
    assert L.mtpc_gradient_list_workspace_bytes(None, -1, ctypes.byref(need)) == SHAPE and L.mtpc_gradient_list_workspace_bytes(entries(*rows), 4, None) == NULL
    assert create(rows, ws=None) == NULL and create(rows, wb=511) == WORKSPACE and create(rows, ws=ODD) == WORKSPACE
    assert L.mtpc_create_gradient_list(entries(*rows), 4, P, BIG, None, None) == NULL
    twice = [(4096, 8192, 4, F32, F32), (4096, 16384, 4, F32, F32), (4096, 0, 4, F32, F32)]       # read twice, written elsewhere: allowed
    if not torch.cuda.is_available():
        assert create(rows) == CUDA and create(twice) == CUDA
    assert L.mtpc_clip_gradients(None, 1.0, P, None) == NULL and L.mtpc_destroy_gradient_list(None) == NULL


def test_tensors_that_do_not_fit_are_refused():
    import torch
    x, w = torch.zeros(4, 8), torch.zeros(8)
    tokens = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: B.mtpc_embed(tokens, x, x), lambda: B.mtpc_embed_backward(tokens, x, x), lambda: B.mtpc_residual_rmsnorm(x, x, w, 1e-5, x),
                 lambda: B.mtpc_residual_rmsnorm_backward(x, w, 1e-5, x, None, x, w), lambda: B.GradientList([x]), lambda: B.GradientList([]),
                 lambda: B.mtpc_embed(tokens, w, x), lambda: B.mtpc_residual_rmsnorm(w, None, w, 1e-5, w)):
        with pytest.raises(B.MtpcError):
            call()                                        # no tensor of a device (or no matrix)
