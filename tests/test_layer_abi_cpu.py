"""Refusals of the layer operators through the C ABI, before anything touches a device."""
import ctypes
import os

import pytest

from paper_2609_40093_amd import _lib

D = ctypes.c_void_p(1 << 20)      # never dereferenced: the calls must fail first
ODD = ctypes.c_void_p((1 << 20) + 8)
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2609_40093_amd import build
        build.build()
    return _lib.load()


def refused(lib, status, name, what=b""):
    assert status == _lib.EP_ERR_INVALID_ARG
    text = lib.ep_last_error()
    assert name.encode() in text and what in text, text


def norm(lib, x=D, r=None, w=D, T=4, H=64, eps=1e-6, total=None, out=D, rows8=None):
    return lib.ep_rmsnorm(x, r, w, T, H, eps, total, out, rows8, None)


@pytest.mark.parametrize("bad", [dict(T=-1), dict(H=0), dict(H=12), dict(H=65544), dict(eps=-1.0), dict(eps=float("nan")),
                                 dict(x=None), dict(x=ODD), dict(r=ODD), dict(w=ODD), dict(out=ODD), dict(total=ODD),
                                 dict(rows8=ODD), dict(out=None), dict(H=72, rows8=D)])
def test_norm(lib, bad):
    refused(lib, norm(lib, **bad), "ep_rmsnorm")


def norm_grad(lib, s=D, w=D, d=D, t=None, T=4, H=64, eps=1e-6, dx=D, dw=D, ws=D, n=BIG):
    return lib.ep_rmsnorm_grad(s, w, d, t, T, H, eps, dx, dw, ws, n, None)


@pytest.mark.parametrize("bad", [dict(T=-1), dict(H=4), dict(H=20), dict(eps=-1e-9), dict(s=None), dict(d=None), dict(dx=None),
                                 dict(s=ODD), dict(t=ODD), dict(dx=ODD), dict(ws=None), dict(ws=ODD), dict(n=16)])
def test_norm_grad(lib, bad):
    refused(lib, norm_grad(lib, **bad), "ep_rmsnorm_grad")


def route(lib, z=D, bf16=0, mask=None, T=4, E=16, k=2, idx=D, w=D, counts=D, sums=D, loss=D, ws=D, n=BIG):
    return lib.ep_route(z, bf16, mask, T, E, k, 1, 0.1, idx, w, counts, sums, loss, ws, n, None)


@pytest.mark.parametrize("bad", [dict(T=-1), dict(E=0, k=0), dict(k=0), dict(k=17), dict(E=2049), dict(T=1 << 30), dict(z=None),
                                 dict(z=ODD), dict(idx=None), dict(w=None), dict(counts=None), dict(sums=None), dict(loss=None),
                                 dict(ws=None), dict(n=8)])
def test_route(lib, bad):
    refused(lib, route(lib, **bad), "ep_route")


def route_grad(lib, z=D, idx=D, counts=D, dw=D, dl=D, T=4, E=16, k=2, out=D):
    return lib.ep_route_grad(z, 0, None, idx, counts, dw, dl, T, E, k, 1, 0.1, out, None)


@pytest.mark.parametrize("bad", [dict(T=-1), dict(k=0), dict(E=4096), dict(z=None), dict(out=None), dict(out=ODD), dict(idx=None),
                                 dict(counts=None)])
def test_route_grad(lib, bad):
    refused(lib, route_grad(lib, **bad), "ep_route_grad")


def combine_grad(lib, d=D, y=D, rows=8, pos=D, w=D, T=4, H=64, k=2, dy=D, dw=D):
    return lib.ep_combine_grad(d, y, rows, pos, w, T, H, k, dy, dw, None)


@pytest.mark.parametrize("bad", [dict(T=-1), dict(rows=-1), dict(H=12), dict(k=0), dict(T=1 << 31), dict(d=None), dict(pos=None),
                                 dict(w=None), dict(y=None), dict(y=ODD), dict(dy=ODD), dict(dy=None, dw=None)])
def test_combine_grad(lib, bad):
    refused(lib, combine_grad(lib, **bad), "ep_combine_grad")


def product(lib, x=D, kind=0, rows=4, off=D, E=2, w=D, ws=None, K=64, N=32, bias=None, act=0, res=None, pre=None, y=D, dt=0,
            work=D, n=BIG):
    return lib.ep_expert_product(x, kind, rows, off, E, w, ws, K, N, bias, act, res, pre, y, dt, work, n, None)


@pytest.mark.parametrize("bad", [dict(kind=2), dict(act=5), dict(act=-1), dict(rows=-1), dict(rows=1 << 31), dict(E=0), dict(E=2049),
                                 dict(K=0), dict(K=12), dict(N=4), dict(N=20), dict(kind=1, ws=D, K=72), dict(kind=1), dict(ws=D),
                                 dict(K=262152), dict(N=262152), dict(N=131080, act=4), dict(K=262144, N=8192), dict(off=None),
                                 dict(x=None), dict(w=None), dict(y=None), dict(x=ODD), dict(w=ODD), dict(y=ODD), dict(bias=ODD),
                                 dict(res=ODD), dict(pre=ODD), dict(dt=2)])
def test_product(lib, bad):
    refused(lib, product(lib, **bad), "ep_expert_product")


def product_grad(lib, x=D, rows=4, off=D, E=2, w=D, K=64, N=32, act=2, pre=D, dy=D, dx=D, dw=D, db=D, work=D, n=BIG):
    return lib.ep_expert_product_grad(x, rows, off, E, w, K, N, act, pre, dy, dx, dw, db, work, n, None)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(E=0), dict(K=4), dict(N=12), dict(act=9), dict(off=None), dict(x=None), dict(w=None),
                                 dict(pre=None), dict(dy=None), dict(dx=ODD), dict(dw=ODD), dict(db=ODD), dict(pre=ODD),
                                 dict(dx=None, dw=None, db=None), dict(work=None), dict(n=64)])
def test_product_grad(lib, bad):
    refused(lib, product_grad(lib, **bad), "ep_expert_product_grad")


def test_workspace_queries(lib):
    n = ctypes.c_size_t()
    for call, args in ((lib.ep_rmsnorm_grad_workspace_bytes, (100, 64)), (lib.ep_route_workspace_bytes, (100, 64)),
                       (lib.ep_expert_product_workspace_bytes, (100, 2, 64, 32, 0, 0)),
                       (lib.ep_expert_product_grad_workspace_bytes, (100, 2, 64, 32, 2, 1))):
        assert call(*args, ctypes.byref(n)) == _lib.EP_OK
        assert call(*args, None) == _lib.EP_ERR_INVALID_ARG
        assert call(-1, *args[1:], ctypes.byref(n)) == _lib.EP_ERR_INVALID_ARG
    # dz of bf16 and the bias's partial sums
    lib.ep_expert_product_grad_workspace_bytes(1000, 2, 64, 32, 2, 0, ctypes.byref(n))
    assert n.value >= 1000 * 32 * 2
    lib.ep_expert_product_grad_workspace_bytes(1000, 2, 64, 32, 0, 0, ctypes.byref(n))
    assert n.value == 0


def test_nothing_to_do_is_no_error(lib):
    """No tokens, no rows: accepted without arrays, and nothing is launched."""
    assert norm(lib, T=0, x=None) == _lib.EP_OK
    assert norm_grad(lib, T=0, s=None, d=None, dx=None, dw=None, ws=None, n=0) == _lib.EP_OK
    assert route(lib, T=0, z=None, idx=None, w=None, counts=None, sums=None, loss=None, ws=None, n=0) == _lib.EP_OK
    assert route_grad(lib, T=0, z=None, out=None) == _lib.EP_OK
    assert combine_grad(lib, T=0, d=None, y=None, pos=None, w=None) == _lib.EP_OK
    assert product(lib, rows=0, x=None, w=None, y=None) == _lib.EP_OK
    assert product_grad(lib, rows=0, x=None, w=None, dy=None, pre=None, dw=None, db=None) == _lib.EP_OK


def test_gradient_workspace_goes_by_the_results(lib):
    """dx alone needs no parts of dw, the bias alone no dz; results that do not exist are refused."""
    n = ctypes.c_size_t()

    def need(results, rows=9000, E=2, K=520, N=264, act=3):
        assert lib.ep_expert_product_grad_workspace_bytes(rows, E, K, N, act, results, ctypes.byref(n)) == _lib.EP_OK
        return n.value

    dz = 9000 * 264 * 2
    everything, no_dx, no_dw = need(1), need(1 | _lib.EP_GRAD_WITHOUT_DX), need(1 | _lib.EP_GRAD_WITHOUT_DW)
    bias = need(1 | _lib.EP_GRAD_WITHOUT_DX | _lib.EP_GRAD_WITHOUT_DW)
    assert everything == no_dx and dz <= need(_lib.EP_GRAD_WITHOUT_DW) < dz + 256
    assert everything - no_dw >= 2 * 2 * 264 * 520 * 4      # dw's parts, two or more
    assert no_dw - bias == need(_lib.EP_GRAD_WITHOUT_DW) and 0 < bias < dz
    assert need(1, act=0) - need(1 | _lib.EP_GRAD_WITHOUT_DW, act=0) == everything - no_dw
    for bad in (-1, 8):
        refused(lib, lib.ep_expert_product_grad_workspace_bytes(9000, 2, 520, 264, 3, bad, ctypes.byref(n)),
                "ep_expert_product_grad_workspace_bytes", b"results")
