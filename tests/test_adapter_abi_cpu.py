"""Refusals of the adapters' and dropout's calls through the C ABI, before anything touches a device."""
import ctypes
import os

import pytest

from paper_2609_40093_amd import _lib

D = ctypes.c_void_p(1 << 20)      # never dereferenced: the calls must fail first
ODD = ctypes.c_void_p((1 << 20) + 8)
ODD4 = ctypes.c_void_p((1 << 20) + 2)
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2609_40093_amd import build
        build.build()
    return _lib.load()


def refused(lib, status, name):
    assert status == _lib.EP_ERR_INVALID_ARG
    text = lib.ep_last_error()
    assert name.encode() in text, text


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=1 << 31), dict(A=0), dict(A=2048), dict(ids=None), dict(order=None),
                                 dict(off=None), dict(ids=ODD4), dict(order=ODD4), dict(off=ODD4)])
def test_rows(lib, bad):
    a = {"ids": D, "rows": 4, "A": 3, "order": D, "off": D, **bad}
    refused(lib, lib.ep_adapter_rows(a["ids"], a["rows"], a["A"], a["order"], a["off"], None), "ep_adapter_rows")


SIZES = [dict(rows=-1), dict(rows=1 << 31), dict(A=0), dict(A=2048), dict(R=0), dict(R=12), dict(R=264), dict(K=0), dict(K=12),
         dict(N=4), dict(N=20), dict(K=262152), dict(N=262152), dict(N=131080, act=4), dict(act=-1), dict(act=5),
         dict(K=65536, N=65536), dict(A=2047, R=256, K=4096), dict(A=2047, R=256, N=4096)]


def product(lib, x=D, rows=4, order=None, off=D, A=2, R=16, a=D, b=D, scale=None, w=D, K=64, N=32, bias=None, act=0, res=None,
            pre=None, low=None, y=D, ws=D, n=BIG):
    return lib.ep_adapter_product(x, rows, order, off, A, R, a, b, scale, w, K, N, bias, act, res, pre, low, y, ws, n, None)


@pytest.mark.parametrize("bad", SIZES + [
    dict(off=None), dict(x=None), dict(a=None), dict(b=None), dict(y=None), dict(x=ODD), dict(a=ODD), dict(b=ODD), dict(w=ODD),
    dict(y=ODD), dict(bias=ODD), dict(res=ODD), dict(pre=ODD), dict(low=ODD), dict(order=ODD4), dict(off=ODD4), dict(scale=ODD4),
    dict(ws=None), dict(ws=ODD), dict(n=16), dict(order=D, rows=1 << 24, K=64),
    dict(order=D, w=None, rows=(1 << 25) + 1), dict(order=D, w=None, rows=1 << 24, R=40, K=72)])
def test_product(lib, bad):
    refused(lib, product(lib, **bad), "ep_adapter_product")


def test_product_workspace(lib):
    n = ctypes.c_size_t()

    def size(rows=64, A=8, R=16, K=7168, N=2048, w=1, act=0):
        assert lib.ep_adapter_product_workspace_bytes(rows, A, R, K, N, w, act, ctypes.byref(n)) == _lib.EP_OK
        return n.value

    assert size() > size(w=0) > 0
    assert size(rows=0) == 0 and size(rows=100000) >= 100000 * 32 * 2
    for bad in SIZES:
        a = {"rows": 4, "A": 2, "R": 16, "K": 64, "N": 32, "act": 0, **bad}
        refused(lib, lib.ep_adapter_product_workspace_bytes(a["rows"], a["A"], a["R"], a["K"], a["N"], 1, a["act"],
                                                            ctypes.byref(n)), "ep_adapter_product_workspace_bytes")
    refused(lib, lib.ep_adapter_product_workspace_bytes(4, 2, 16, 64, 32, 1, 0, None), "bytes is NULL")


def grad(lib, x=D, rows=4, order=None, off=D, A=2, R=16, a=D, b=D, scale=None, w=D, K=64, N=32, low=D, act=0, pre=None, d=D,
         dx=D, da=D, db=D, ws=D, n=BIG):
    return lib.ep_adapter_product_grad(x, rows, order, off, A, R, a, b, scale, w, K, N, low, act, pre, d, dx, da, db, ws, n,
                                       None)


@pytest.mark.parametrize("bad", SIZES + [
    dict(off=None), dict(x=None), dict(a=None), dict(b=None), dict(low=None), dict(d=None), dict(act=2), dict(x=ODD), dict(a=ODD),
    dict(b=ODD), dict(w=ODD), dict(low=ODD), dict(pre=ODD), dict(d=ODD), dict(dx=ODD), dict(da=ODD), dict(db=ODD),
    dict(order=ODD4), dict(off=ODD4), dict(scale=ODD4), dict(dx=None, da=None, db=None), dict(ws=None), dict(ws=ODD), dict(n=16)])
def test_grad(lib, bad):
    refused(lib, grad(lib, **bad), "ep_adapter_product_grad")


def test_grad_workspace(lib):
    n = ctypes.c_size_t()

    def size(results, act=0, order=0, rows=4096):
        assert lib.ep_adapter_product_grad_workspace_bytes(rows, 8, 16, 1024, 512, 1, act, order, results, ctypes.byref(n)) == 0
        return n.value

    every = _lib.EP_ADAPTER_DX | _lib.EP_ADAPTER_DA | _lib.EP_ADAPTER_DB
    assert size(0) == 0 and size(every) >= max(size(1), size(2), size(4))
    assert size(1, act=2) >= size(1) + 4096 * 512 * 2  # dz
    for bad in SIZES:
        a = {"rows": 4, "A": 2, "R": 16, "K": 64, "N": 32, "act": 0, **bad}
        refused(lib, lib.ep_adapter_product_grad_workspace_bytes(a["rows"], a["A"], a["R"], a["K"], a["N"], 1, a["act"],
                                                                 0, 7, ctypes.byref(n)), "ep_adapter_product_grad_workspace_bytes")
    for results in (-1, 8):
        refused(lib, lib.ep_adapter_product_grad_workspace_bytes(4, 2, 16, 64, 32, 1, 0, 0, results, ctypes.byref(n)), "results")
    refused(lib, lib.ep_adapter_product_grad_workspace_bytes(4, 2, 16, 64, 32, 1, 0, 0, 7, None), "bytes is NULL")


def dropout(lib, x=D, r=None, count=64, p=0.1, rng=D, out=D):
    return lib.ep_dropout(x, r, count, p, rng, 0, out, None)


@pytest.mark.parametrize("bad", [dict(count=-8), dict(count=12), dict(p=-0.1), dict(p=1.5), dict(p=float("nan")), dict(rng=None),
                                 dict(rng=ODD4), dict(x=None), dict(out=None), dict(x=ODD), dict(r=ODD), dict(out=ODD)])
def test_dropout(lib, bad):
    refused(lib, dropout(lib, **bad), "ep_dropout")


def norm(lib, x=D, r=None, w=D, T=4, H=64, eps=1e-6, p=0.1, rng=D, total=None, out=D, rows8=None):
    return lib.ep_dropout_rmsnorm(x, r, w, T, H, eps, p, rng, 0, total, out, rows8, None)


@pytest.mark.parametrize("bad", [dict(T=-1), dict(H=0), dict(H=12), dict(H=65544), dict(eps=-1.0), dict(p=2.0), dict(rng=None),
                                 dict(rng=ODD4), dict(x=None), dict(x=ODD), dict(r=ODD), dict(w=ODD), dict(out=ODD),
                                 dict(out=None), dict(H=72, rows8=D)])
def test_norm(lib, bad):
    refused(lib, norm(lib, **bad), "ep_dropout_rmsnorm")


def norm_grad(lib, s=D, w=D, d=D, t=None, T=4, H=64, eps=1e-6, p=0.1, rng=D, dx=D, dr=None, dw=D, ws=D, n=BIG):
    return lib.ep_dropout_rmsnorm_grad(s, w, d, t, T, H, eps, p, rng, 0, dx, dr, dw, ws, n, None)


@pytest.mark.parametrize("bad", [dict(T=-1), dict(H=20), dict(eps=-1e-9), dict(p=-1.0), dict(rng=None), dict(rng=ODD4),
                                 dict(s=None), dict(d=None), dict(dx=None), dict(dx=D, dr=D), dict(s=ODD), dict(t=ODD),
                                 dict(dx=ODD), dict(dr=ODD), dict(ws=None), dict(n=16)])
def test_norm_grad(lib, bad):
    refused(lib, norm_grad(lib, **bad), "ep_dropout_rmsnorm_grad")


def test_calls_without_rows_need_no_arrays(lib):
    assert lib.ep_dropout(None, None, 0, 0.5, None, 0, None, None) == _lib.EP_OK
    assert lib.ep_dropout_rmsnorm(None, None, None, 0, 64, 1e-6, 0.5, None, 0, None, None, None, None) == _lib.EP_OK
    assert product(lib, x=None, rows=0, a=None, b=None, w=None, y=None, ws=None, n=0) == _lib.EP_OK
