"""Argument checks of layer norm, gradient norm and clipping, all made on the host before anything is launched: they need no
GPU, and the addresses below are never used."""
import ctypes

import numpy as np
import pytest

import paper_2301_08527_b200 as rk

EINVAL, EUNSUPPORTED = -1, -3
F32, F16, BF16 = 0, 1, 2
A, B, C, D, E, G = (0x7000000000 + (i << 32) for i in range(6))       # far apart


@pytest.fixture(scope="module")
def lib():
    from paper_2301_08527_b200.build import build
    build()
    return rk.load_library()


def _forward(lib, **kw):
    a = dict(x=A, xt=F32, xs=100, N=8, P=100, g=B, b=C, wt=F32, eps=1e-5, y=D, yt=F32, ys=100, mean=E, rstd=G, stream=None)
    a.update(kw)
    return lib.rocket_layer_norm(*a.values())


def _backward(lib, **kw):
    a = dict(dy=A, yt=F32, ds=100, x=B, xt=F32, xs=100, N=8, P=100, g=C, wt=F32, mean=D, rstd=D + 4096, dx=E, dxs=100, dg=G, db=G + 4096,
             ws=0x7f0000000000, bytes=1 << 40, stream=None)
    a.update(kw)
    return lib.rocket_layer_norm_backward(*a.values())


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(y=None), dict(N=-1), dict(P=0), dict(P=-5), dict(xt=3), dict(yt=-1), dict(wt=7), dict(eps=-1e-3),
    dict(eps=float("nan")), dict(eps=float("inf")), dict(xs=-100), dict(ys=99), dict(ys=0), dict(xs=1 << 62), dict(ys=1 << 62), dict(x=A + 2), dict(y=D + 1),
    dict(xt=F16, x=A + 1), dict(g=B + 2), dict(wt=BF16, b=C + 1), dict(mean=E + 2), dict(rstd=G + 1),
    dict(y=A), dict(y=A + 4), dict(y=A - 4), dict(y=A + 4 * 799), dict(y=B - 4 * 799), dict(y=C - 400), dict(mean=A + 400), dict(rstd=D + 32), dict(rstd=E + 28),
    # rows of one byte distance that reach into one another's gap
    dict(xs=300, ys=300, y=A + 4 * 99), dict(xs=300, ys=300, y=A + 4 * 201), dict(xs=300, ys=300, y=A - 4 * 99),
    # interleaved, but of different distances
    dict(xs=300, ys=250, y=A + 400),
])
def test_forward_refuses(lib, kw):
    assert _forward(lib, **kw) == EINVAL


@pytest.mark.parametrize("kw", [
    dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(dx=None, dg=None, db=None), dict(N=-1), dict(P=0), dict(xt=9), dict(yt=3),
    dict(wt=-1), dict(dxs=99), dict(xs=-1), dict(ds=-1), dict(dy=A + 2), dict(x=B + 1), dict(dx=E + 2), dict(dg=G + 1), dict(db=G + 4098), dict(mean=D + 2),
    dict(dx=A), dict(dx=B), dict(dg=C), dict(db=D), dict(dg=G, db=G), dict(dg=G, db=G + 396), dict(dg=E + 100), dict(bytes=-1),
    dict(ws=0x7f0000000008, N=100000, P=5000),
])
def test_backward_refuses(lib, kw):
    assert _backward(lib, **kw) == EINVAL


@pytest.mark.parametrize("N,P", [(0, 1), (0x7fffffff, 1), (0x7fffffff, 512), (1, 0x7fffffff), (0x7fffffff, 0x7fffffff), (3, 65536), (3, 65537), (3, 0x7fffffff - 4000)])
def test_workspace_sizes_at_the_ends(lib, N, P):
    assert 0 <= lib.rocket_layer_norm_backward_workspace(N, P) < 1 << 30


@pytest.mark.parametrize("N,P", [(1, 1), (32, 20000), (16384, 4096), (100003, 257), (5, 300000)])
def test_backward_refuses_a_workspace_that_is_too_small(lib, N, P):
    need = lib.rocket_layer_norm_backward_workspace(N, P)
    assert 0 <= need < 1 << 30
    if need > 0:
        kw = dict(N=N, P=P, ds=P, xs=P, dxs=P, dy=0x100000000000, x=0x200000000000, dx=0x300000000000, mean=0x400000000000, rstd=0x410000000000,
                  dg=0x420000000000, db=0x430000000000, g=0x440000000000)
        assert _backward(lib, bytes=need - 1, **kw) == EINVAL
        assert _backward(lib, ws=None, bytes=need, **kw) == EINVAL
        assert _backward(lib, ws=0x7f0000000004, bytes=need, **kw) == EINVAL
        assert _backward(lib, ws=0x200000000000, bytes=need, **kw) == EINVAL       # inside x


def test_workspace_sizes_out_of_range(lib):
    assert lib.rocket_layer_norm_backward_workspace(-1, 10) == EINVAL
    assert lib.rocket_layer_norm_backward_workspace(10, 0) == EINVAL
    sizes = (ctypes.c_int64 * 2)(1 << 30, 5)
    assert lib.rocket_grad_norm_workspace(-1, sizes) == EINVAL
    assert lib.rocket_grad_norm_workspace(1, None) == EINVAL
    assert lib.rocket_grad_norm_workspace(2, (ctypes.c_int64 * 2)(5, -1)) == EINVAL
    assert lib.rocket_grad_norm_workspace(1, (ctypes.c_int64 * 1)(1 << 60)) == EINVAL
    assert lib.rocket_grad_norm_workspace(0, None) == 0
    assert lib.rocket_grad_norm_workspace(2, (ctypes.c_int64 * 2)(100, 0)) == 0
    assert lib.rocket_grad_norm_workspace(2, sizes) > 0


def test_no_rows_are_a_no_op(lib):
    assert _forward(lib, N=0, x=None, y=None) == 0


def _grads(lib, tensors, out=None, max_norm=1.0, norm=E, ws=0x7f0000000000, nbytes=None, clip=True, count=None, null=()):
    """tensors, out: lists of (address, size, type)."""
    n = len(tensors) if count is None else count
    nbytes = 1 << 20 if nbytes is None else nbytes
    ptr = lambda ts: (ctypes.c_void_p * len(ts))(*[t[0] for t in ts])  # noqa: E731
    sizes = (ctypes.c_int64 * len(tensors))(*[t[1] for t in tensors])
    codes = lambda ts: (ctypes.c_int32 * len(ts))(*[t[2] for t in ts])  # noqa: E731
    a = [ptr(tensors), sizes, codes(tensors)]
    a = [None if i in null else v for i, v in enumerate(a)]
    if not clip:
        return lib.rocket_grad_norm(n, *a, norm, ws, nbytes, None)
    o = [ptr(out) if out is not None else None, codes(out) if out is not None and 3 not in null else None]
    return lib.rocket_clip_grad_norm(n, *a, *o, max_norm, norm, ws, nbytes, None)


ONE = [(A, 100, F32), (B, 7, F16)]
LARGE = [(A, 1 << 20, F32), (B, 7, F16)]


@pytest.mark.parametrize("clip", [False, True])
@pytest.mark.parametrize("kw", [
    dict(norm=None), dict(norm=E + 2), dict(tensors=LARGE, ws=None), dict(tensors=LARGE, ws=0x7f0000000008), dict(tensors=LARGE, nbytes=15), dict(nbytes=-1), dict(count=-1), dict(null=(0,)), dict(null=(1,)), dict(null=(2,)),
    dict(tensors=[(A, -1, F32)]), dict(tensors=[(A, 1, 3)]), dict(tensors=[(A, 1, -1)]), dict(tensors=[(None, 1, F32)]), dict(tensors=[(A + 2, 1, F32)]),
    dict(tensors=[(A + 1, 1, BF16)]), dict(tensors=[(A, 1 << 60, F32)]), dict(norm=A + 4), dict(tensors=LARGE, ws=A), dict(tensors=LARGE, ws=E - 64),
])
def test_norms_refuse(lib, clip, kw):
    kw = dict(kw)
    assert _grads(lib, kw.pop("tensors", ONE), clip=clip, **kw) == EINVAL


@pytest.mark.parametrize("kw", [
    dict(max_norm=-1.0), dict(max_norm=float("nan")),
    dict(tensors=[(A, 100, F32), (A, 100, F32)]), dict(tensors=[(A, 100, F32), (A + 396, 100, F32)]), dict(tensors=[(A, 100, F32), (A + 398, 1, F16)]),
    dict(out=[(C, 0, F32), (D, 0, BF16)]), dict(out=[(C, 0, F16), (D, 0, F16)]), dict(out=[(C, 0, 4), (D, 0, F16)]), dict(out=[(None, 0, F32), (D, 0, F16)]),
    dict(out=[(C, 0, F32), (D + 1, 0, F16)]), dict(out=[(C, 0, F32), (C + 398, 0, F16)]), dict(out=[(C, 0, F32), (D, 0, F16)], null=(3,)),
    dict(out=[(B, 0, F32), (A, 0, F16)]),             # one another's places
    dict(out=[(A + 4, 0, F32), (B, 0, F16)]),         # its own gradient, shifted
    dict(out=[(A, 0, F32), (B, 0, F32)]),             # its own gradient, wider
    dict(out=[(E, 0, F32), (B, 0, F16)]),             # the norm
])
def test_clipping_refuses(lib, kw):
    kw = dict(kw)
    assert _grads(lib, kw.pop("tensors", ONE), **kw) == EINVAL


def test_more_chunks_than_a_launch_can_number(lib):
    tensors = [(A + (i << 43), 1 << 40, F32) for i in range(1024)]
    assert _grads(lib, tensors, clip=False, ws=0x10, norm=0x1000000) in (EINVAL, EUNSUPPORTED)


@pytest.mark.parametrize("bad", ["array", "cpu", "none"])
def test_binding_takes_cuda_tensors_only(bad):
    import torch
    x = {"array": np.zeros((2, 3), np.float32), "cpu": torch.zeros(2, 3), "none": None}[bad]
    with pytest.raises(TypeError):
        rk.rocket_layer_norm(x)
    with pytest.raises(TypeError):
        rk.rocket_layer_norm_backward(x, x, x, x)
    with pytest.raises(TypeError):
        rk.rocket_grad_norm([x])
    with pytest.raises(TypeError):
        rk.rocket_clip_grad_norm([x], 1.0)
