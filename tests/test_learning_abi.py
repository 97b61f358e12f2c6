"""The learning operators' host side without a GPU: refusals and the arithmetic of their workspaces."""
import ctypes
import math

import pytest

import paper_1102_3828_amd as pkg
from paper_1102_3828_amd import binding as b

F32, F16, BF16 = 0, 1, 2
P = 1 << 20   # an address that is never followed


def softmax(n=100, v=1000, d=64, kind=BF16, x=P, ldx=None, w=P, ldw=None, targets=P, offset=None, scale=1.0):
    return b.SoftmaxArgs(n, v, d, kind, x, d if ldx is None else ldx, w, d if ldw is None else ldw, targets, offset, scale, 0)


def need(args, grad=0):
    size = ctypes.c_int64(-1)
    return pkg.lib.ivfr_softmax_workspace(ctypes.byref(args), grad, ctypes.byref(size)), size.value


@pytest.mark.parametrize("change", [dict(n=-1), dict(n=1 << 31), dict(v=0), dict(v=1 << 31), dict(d=0), dict(d=65537), dict(kind=3), dict(kind=-1), dict(ldx=63),
                                    dict(ldw=63), dict(ldw=1 << 22), dict(scale=math.nan), dict(scale=math.inf)])
def test_softmax_refuses(change):
    args = softmax(**change)
    assert need(args)[0] == b.ERR_INVALID_ARG and b"softmax" in pkg.lib.ivfr_last_error()
    assert pkg.lib.ivfr_softmax_loss(ctypes.byref(args), P, P, P, 1 << 40, None) == b.ERR_INVALID_ARG
    assert pkg.lib.ivfr_softmax_loss_grad(ctypes.byref(args), P, None, P, P, P, P, 1 << 40, None) == b.ERR_INVALID_ARG


@pytest.mark.parametrize("change", [dict(x=None), dict(w=None), dict(targets=None), dict(x=P + 1), dict(w=P + 1), dict(targets=P + 4), dict(offset=P + 2)])
def test_softmax_refuses_pointers(change):
    args = softmax(**change)
    assert pkg.lib.ivfr_softmax_loss(ctypes.byref(args), P, P, P, 1 << 40, None) == b.ERR_INVALID_ARG
    assert pkg.lib.ivfr_softmax_loss_grad(ctypes.byref(args), P, None, P, P, P, P, 1 << 40, None) == b.ERR_INVALID_ARG


def test_softmax_refuses_workspaces():
    args = softmax()
    for grad in (0, 1):
        size = need(args, grad)[1]
        call = (lambda ws, size: pkg.lib.ivfr_softmax_loss_grad(ctypes.byref(args), P, None, P, P, P, ws, size, None)) if grad else \
            (lambda ws, size: pkg.lib.ivfr_softmax_loss(ctypes.byref(args), P, P, ws, size, None))
        assert size > 0
        assert call(P, size - 1) == b.ERR_INVALID_ARG and b"workspace" in pkg.lib.ivfr_last_error()
        assert call(P + 16, size) == b.ERR_INVALID_ARG
        assert call(None, size) == b.ERR_INVALID_ARG
    assert pkg.lib.ivfr_softmax_workspace(ctypes.byref(args), 0, None) == b.ERR_INVALID_ARG
    assert pkg.lib.ivfr_softmax_workspace(None, 0, None) == b.ERR_INVALID_ARG


def test_softmax_workspace_keeps_no_scores():
    """A loss of aligned 16-bit rows keeps statistics only; a gradient keeps at most pieces of 1 GiB of factors beside copies and partial sums."""
    n, v, d = 8192, 131072, 2048
    rc, size = need(softmax(n, v, d))
    assert rc == 0 and size < 0.05 * n * v
    rc, size = need(softmax(n, v, d), 1)
    copies, sums = 2 * n * d, 4 * n * d
    assert rc == 0 and size < (1 << 30) + copies + 8 * sums
    rc, size = need(softmax(0, v, d), 1)
    assert (rc, size) == (0, 0)


@pytest.mark.parametrize("n,v,d", [(1, 1, 1), (1, (1 << 31) - 257, 8), (100000, 1 << 20, 65536), (513, 33, 31)])
@pytest.mark.parametrize("kind", [F32, F16, BF16])
def test_softmax_workspace_of_any_sizes(n, v, d, kind):
    for grad in (0, 1):
        rc, size = need(softmax(n, v, d, kind), grad)
        assert rc == 0 and size % 256 == 0 and 0 < size < 1 << 45


def ortho(batch=1, rows=100, cols=50, kind=F32, steps=5, g=P, ld=None, stride=None, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7):
    flat = (ctypes.c_float * (3 * max(steps, 1)))(*(list(coefficients) * max(steps, 1)))
    a = b.OrthogonalizeArgs(batch, rows, cols, kind, steps, g, cols if ld is None else ld, rows * cols if stride is None else stride, ctypes.addressof(flat), 1.0, eps, 0)
    a.keep = flat
    return a


def ortho_need(a):
    size = ctypes.c_int64(-1)
    return pkg.lib.ivfr_orthogonalize_workspace(ctypes.byref(a), ctypes.byref(size)), size.value


@pytest.mark.parametrize("change", [dict(batch=-1), dict(batch=65536), dict(rows=0), dict(cols=0), dict(rows=(1 << 20) + 1), dict(kind=3), dict(steps=0), dict(steps=65),
                                    dict(ld=49), dict(coefficients=(math.nan, 0, 0)), dict(coefficients=(40.0, 0, 0)), dict(eps=-1.0)])
def test_orthogonalize_refuses(change):
    a = ortho(**change)
    assert ortho_need(a)[0] == b.ERR_INVALID_ARG and b"orthogonalize" in pkg.lib.ivfr_last_error()
    assert pkg.lib.ivfr_orthogonalize(ctypes.byref(a), P, P, 1 << 40, None) == b.ERR_INVALID_ARG


def test_orthogonalize_refuses_pointers_and_workspaces():
    a = ortho(rows=500, cols=600)
    rc, size = ortho_need(a)
    assert rc == 0 and size > 0
    assert pkg.lib.ivfr_orthogonalize(ctypes.byref(a), None, P, size, None) == b.ERR_INVALID_ARG
    assert pkg.lib.ivfr_orthogonalize(ctypes.byref(a), P, None, size, None) == b.ERR_INVALID_ARG
    assert pkg.lib.ivfr_orthogonalize(ctypes.byref(a), P, P, size - 1, None) == b.ERR_INVALID_ARG
    assert pkg.lib.ivfr_orthogonalize(ctypes.byref(ortho(g=None)), P, P, 1 << 40, None) == b.ERR_INVALID_ARG
    assert pkg.lib.ivfr_orthogonalize(ctypes.byref(ortho(g=P + 2)), P, P, 1 << 40, None) == b.ERR_INVALID_ARG


def test_orthogonalize_of_no_matrices_needs_nothing():
    assert ortho_need(ortho(batch=0)) == (0, 0)
    assert pkg.lib.ivfr_orthogonalize(ctypes.byref(ortho(batch=0)), None, None, 0, None) == 0
