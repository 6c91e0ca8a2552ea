"""Host-side argument checks of the 8-bit floating-point entry points: nothing is launched, no GPU is needed."""
import ctypes

import pytest

from paper_2405_18832_b200 import binding as B
from paper_2405_18832_b200 import build as build_mod

A = 1 << 20      # an aligned address that is never followed: the checks come first
UNSUPPORTED, INVALID, WORKSPACE = 2, 1, 3


@pytest.fixture(scope="module")
def L():
    build_mod.build()
    return B.lib()


def norm(L, **kw):
    a = dict(dtype=1, T=4, d=256, eps=1e-6, x=A, ld_x=256, residual=0, ld_residual=0, gamma=0, residual_out=0,
             ld_residual_out=0, y=A, ld_y=256, q=0, ld_q=0, scale=0, ld_scale=0)
    a.update(kw)
    return L.monde_rmsnorm_quant(*a.values(), None)


@pytest.mark.parametrize("bad,status", [(dict(T=-1), INVALID), (dict(d=0), INVALID), (dict(eps=-1.0), INVALID),
                                        (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
                                        (dict(dtype=2), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED),
                                        (dict(d=32769, ld_x=40000, ld_y=40000), UNSUPPORTED), (dict(y=0), INVALID),
                                        (dict(q=A, ld_q=256), INVALID), (dict(scale=A, ld_scale=2), INVALID),
                                        (dict(x=0), INVALID), (dict(ld_x=255), INVALID), (dict(ld_y=0), INVALID),
                                        (dict(residual=A, ld_residual=8), INVALID), (dict(x=A + 1), INVALID),
                                        (dict(q=A, ld_q=256, scale=A, ld_scale=1), INVALID),
                                        (dict(q=A, ld_q=256, scale=A + 2, ld_scale=2), INVALID)])
def test_norm_refusals(L, bad, status):
    assert norm(L, **bad) == status


def quant(L, **kw):
    a = dict(dtype=1, batch=1, rows=4, cols=256, block_rows=1, x=A, ld_x=256, q=A, ld_q=256, scale=A, ld_scale=2)
    a.update(kw)
    return L.monde_quantize_fp8(*a.values(), None)


@pytest.mark.parametrize("bad,status", [(dict(batch=-1), INVALID), (dict(rows=-1), INVALID), (dict(cols=0), INVALID),
                                        (dict(dtype=2), UNSUPPORTED), (dict(block_rows=64), UNSUPPORTED),
                                        (dict(block_rows=0), UNSUPPORTED), (dict(x=0), INVALID), (dict(q=0), INVALID),
                                        (dict(scale=0), INVALID), (dict(ld_x=100), INVALID), (dict(ld_scale=1), INVALID),
                                        (dict(x=A + 1), INVALID), (dict(scale=A + 1), INVALID)])
def test_quantisation_refusals(L, bad, status):
    assert quant(L, **bad) == status


def problem(**kw):
    a = dict(rows=4, N=256, K=128, E=1, src_rows=4, row_div=1, act=-1, out_dtype=1, ld_x=128, ld_x_scale=1, ld_out=256,
             ld_out_scale=2)
    a.update(kw)
    return B.monde_matmul_problem(*a.values())


BAD_SIZES = [(dict(rows=-1), INVALID), (dict(N=0), INVALID), (dict(K=0), INVALID), (dict(E=0), INVALID),
             (dict(src_rows=-1), INVALID), (dict(row_div=0), INVALID), (dict(K=120, ld_x=128), UNSUPPORTED),
             (dict(E=257), UNSUPPORTED), (dict(act=2), UNSUPPORTED), (dict(act=-2), UNSUPPORTED),
             (dict(out_dtype=3), UNSUPPORTED), (dict(ld_x=112), INVALID), (dict(ld_x=136), INVALID),
             (dict(ld_x_scale=0), INVALID), (dict(ld_out=255), INVALID), (dict(out_dtype=2, ld_out_scale=1), INVALID)]


@pytest.mark.parametrize("bad,status", BAD_SIZES)
def test_product_size_refusals(L, bad, status):
    p = problem(**bad)
    assert L.monde_matmul_workspace_bytes(ctypes.byref(p)) == 0
    assert L.monde_grouped_matmul_fp8(ctypes.byref(p), A, A, A, A, None, A, None, A, A, A, 1 << 30, None) == status


def test_product_pointer_refusals(L):
    def dense(p, x=A, xs=A, w=A, ws=A, bias=None, out=A, os=None, wk=A, n=1 << 30):
        return L.monde_matmul_fp8(ctypes.byref(p), x, xs, w, ws, bias, out, os, wk, n, None)

    def grouped(p, off=A, ids=None, wk=A):
        return L.monde_grouped_matmul_fp8(ctypes.byref(p), A, A, A, A, None, off, ids, A, None, wk, 1 << 30, None)

    p = problem()
    assert L.monde_matmul_fp8(None, A, A, A, A, None, A, None, A, 1 << 30, None) == INVALID
    assert L.monde_matmul_workspace_bytes(None) == 0
    for name in ("x", "xs", "w", "ws", "out", "wk"):
        assert dense(p, **{name: None}) == INVALID, name
    for name, addr in (("x", A + 8), ("w", A + 1), ("xs", A + 2), ("ws", A + 1), ("bias", A + 2), ("out", A + 1), ("wk", A + 8)):
        assert dense(p, **{name: addr}) == INVALID, name
    assert dense(problem(out_dtype=2)) == INVALID                    # no place for the scales
    assert dense(problem(out_dtype=0), out=A + 2) == INVALID
    assert dense(problem(E=2)) == INVALID                            # one matrix only
    assert dense(problem(src_rows=5)) == INVALID                     # without ids every row reads its own
    assert dense(p, n=1024) == WORKSPACE
    assert dense(problem(rows=0, src_rows=0), x=None, out=None) == 0
    assert grouped(p, off=None) == INVALID
    assert grouped(p, off=A + 2) == INVALID
    assert grouped(problem(src_rows=0), ids=A) == INVALID


def test_workspace_is_bounded(L):
    sizes = [(rows, N, K, E) for rows in (1, 7, 128, 5000, 1 << 20) for N in (1, 200, 8192, 300000) for K in (16, 8192)
             for E in (1, 64, 256)]
    for rows, N, K, E in sizes:
        n = B.monde_matmul_workspace_bytes(rows, N, K, E)
        assert 256 * 1024 <= n <= B.MATMUL_WS_MAX, (rows, N, K, E)
