"""Argument checks of the block-scaled 4-bit calls and the cache: what the host can see is refused with the documented status
before anything is launched (no GPU needed), and calls without rows are no-ops."""
import ctypes

import pytest

import paper_1901_09504_b200 as ocs
from paper_1901_09504_b200.binding import _CacheDesc

INVALID, SHAPE, WORKSPACE, UNSUPPORTED = 1, 2, 3, 4
P = 1 << 20            # a well-aligned address that is never dereferenced


def quantize(X=P, x_type=0, rows=4, C=32, ldx=32, S=0, idx=None, grid=2, codes=P, ld=16, scales=P, rs=P):
    return ocs.lib().ocs_quantize_mx4(X, x_type, rows, C, ldx, S, idx, grid, codes, ld, scales, rs, None, None)


def dequantize(codes=P, ld=16, scales=P, rs=P, rows=4, K=32, grid=2, Y=P, y_type=0, ldy=32):
    return ocs.lib().ocs_dequantize_mx4(codes, ld, scales, rs, rows, K, grid, Y, y_type, ldy, None)


def qlinear(A=P, a_s=P, a_r=P, M=4, K=32, lda=16, W=P, w_s=P, w_r=P, N=8, ldw=16, grid=2, bias=None, Y=P, y_type=0, ldy=8):
    return ocs.lib().ocs_qlinear_mx4(A, a_s, a_r, M, K, lda, W, w_s, w_r, N, ldw, grid, bias, Y, y_type, ldy, None, None)


def linear(X=P, x_type=0, M=4, C=32, ldx=32, S=0, idx=None, grid=2, W=P, w_s=P, w_r=P, N=8, ldw=16, bias=None, Y=P, y_type=0, ldy=8,
           ws=P, ws_bytes=1 << 20):
    return ocs.lib().ocs_linear_mx4(X, x_type, M, C, ldx, S, idx, grid, W, w_s, w_r, N, ldw, bias, Y, y_type, ldy, ws, ws_bytes, None, None)


def write(n_pages=4, page=8, heads=2, dim=32, grid=2, pages=P, X=P, ld=(64, 32), pages2=None, X2=None, x_type=0, tokens=3, slots=P):
    d = _CacheDesc(n_pages, page, heads, dim, grid)
    return ocs.lib().ocs_cache_write(ctypes.byref(d), pages, X, *ld, pages2, X2, *ld, x_type, tokens, slots, None, None)


def read(n_pages=4, page=8, heads=2, dim=32, grid=2, pages=P, pages2=None, table=P, ld_table=4, cols=4, starts=P, B=2, rows=9, Y=P, ld=(64, 32),
         Y2=None, y_type=0):
    d = _CacheDesc(n_pages, page, heads, dim, grid)
    return ocs.lib().ocs_cache_read(ctypes.byref(d), pages, pages2, table, ld_table, cols, starts, B, rows, Y, *ld, Y2, *ld, y_type, None, None)


@pytest.mark.parametrize("call,kw,status", [
    (quantize, dict(x_type=3), INVALID), (quantize, dict(grid=0), INVALID), (quantize, dict(grid=3), INVALID), (quantize, dict(S=-1), INVALID),
    (quantize, dict(X=None), INVALID), (quantize, dict(codes=None), INVALID), (quantize, dict(scales=None), INVALID),
    (quantize, dict(rs=None), INVALID), (quantize, dict(S=2, ld=17), INVALID), (quantize, dict(C=0), SHAPE), (quantize, dict(rows=-1), SHAPE),
    (quantize, dict(ldx=31), SHAPE), (quantize, dict(ld=15), SHAPE), (quantize, dict(S=1, idx=P), SHAPE), (quantize, dict(X=P + 2), SHAPE),
    (quantize, dict(scales=P + 8), SHAPE), (quantize, dict(rs=P + 2), SHAPE), (quantize, dict(S=2, ld=17, idx=P + 2), SHAPE),
    (quantize, dict(C=1 << 30, ldx=1 << 30, ld=1 << 29), UNSUPPORTED),
    (dequantize, dict(grid=0), INVALID), (dequantize, dict(y_type=3), INVALID), (dequantize, dict(codes=None), INVALID),
    (dequantize, dict(rs=None), INVALID), (dequantize, dict(Y=None), INVALID), (dequantize, dict(K=0), SHAPE), (dequantize, dict(rows=-1), SHAPE),
    (dequantize, dict(ld=15), SHAPE), (dequantize, dict(ldy=31), SHAPE), (dequantize, dict(Y=P + 2), SHAPE), (dequantize, dict(scales=P + 4), SHAPE),
    (dequantize, dict(K=1 << 30, ld=1 << 29, ldy=1 << 30), UNSUPPORTED),
    (qlinear, dict(y_type=-1), INVALID), (qlinear, dict(grid=0), INVALID), (qlinear, dict(A=None), INVALID), (qlinear, dict(a_s=None), INVALID),
    (qlinear, dict(a_r=None), INVALID), (qlinear, dict(W=None), INVALID), (qlinear, dict(w_s=None), INVALID), (qlinear, dict(w_r=None), INVALID),
    (qlinear, dict(Y=None), INVALID), (qlinear, dict(M=-1), SHAPE), (qlinear, dict(K=0), SHAPE), (qlinear, dict(N=0), SHAPE),
    (qlinear, dict(lda=24), SHAPE), (qlinear, dict(K=33), SHAPE), (qlinear, dict(ldw=8), SHAPE), (qlinear, dict(A=P + 8), SHAPE),
    (qlinear, dict(W=P + 8), SHAPE), (qlinear, dict(a_s=P + 8), SHAPE), (qlinear, dict(w_s=P + 8), SHAPE), (qlinear, dict(ldy=7), SHAPE),
    (qlinear, dict(Y=P + 2), SHAPE), (qlinear, dict(bias=P + 1), SHAPE), (qlinear, dict(w_r=P + 1), SHAPE),
    (qlinear, dict(M=1 << 30), UNSUPPORTED), (qlinear, dict(N=2 ** 31 - 511, ldy=2 ** 31 - 511), UNSUPPORTED),
    (qlinear, dict(K=1 << 30, lda=1 << 29, ldw=1 << 29), UNSUPPORTED),
    (linear, dict(M=40, ws=None), WORKSPACE), (linear, dict(M=40, ws_bytes=100), WORKSPACE), (linear, dict(M=40, ws=P + 16), WORKSPACE),
    (linear, dict(C=30000, ldx=30000, ldw=15008, ws=None), WORKSPACE),
    (linear, dict(x_type=7), INVALID), (linear, dict(grid=0), INVALID), (linear, dict(S=1), INVALID), (linear, dict(X=None), INVALID),
    (linear, dict(w_r=None), INVALID), (linear, dict(M=50, w_r=None), INVALID), (linear, dict(ldx=8), SHAPE), (linear, dict(S=8, idx=P), SHAPE), (linear, dict(M=-2), SHAPE),
    (linear, dict(N=2 ** 31 - 1, ldy=2 ** 31 - 1), UNSUPPORTED),
    (write, dict(grid=3), INVALID), (write, dict(grid=-1), INVALID), (write, dict(x_type=5), INVALID), (write, dict(pages=None), INVALID),
    (write, dict(X=None), INVALID), (write, dict(slots=None), INVALID), (write, dict(pages2=2 * P), INVALID), (write, dict(X2=P), INVALID),
    (write, dict(pages2=P, X2=P), INVALID), (write, dict(tokens=-1), SHAPE), (write, dict(page=0), SHAPE), (write, dict(heads=0), SHAPE),
    (write, dict(dim=0), SHAPE), (write, dict(n_pages=-1), SHAPE), (write, dict(pages=P + 8), SHAPE), (write, dict(X=P + 2), SHAPE),
    (write, dict(slots=P + 4), SHAPE), (write, dict(pages2=2 * P + 8, X2=P), SHAPE), (write, dict(dim=1025), UNSUPPORTED),
    (write, dict(page=1 << 20, heads=1 << 10), UNSUPPORTED), (write, dict(tokens=1 << 40), UNSUPPORTED),
    (read, dict(grid=7), INVALID), (read, dict(y_type=-2), INVALID), (read, dict(table=None), INVALID), (read, dict(starts=None), INVALID),
    (read, dict(Y=None), INVALID), (read, dict(pages=None), INVALID), (read, dict(Y2=P), INVALID), (read, dict(pages2=P), INVALID),
    (read, dict(rows=-1), SHAPE), (read, dict(B=-1), SHAPE), (read, dict(cols=-1), SHAPE), (read, dict(ld_table=3), SHAPE),
    (read, dict(ld=(64, 31)), SHAPE), (read, dict(ld=(31, 32)), SHAPE), (read, dict(starts=P + 2), SHAPE), (read, dict(Y=P + 2), SHAPE),
    (read, dict(dim=2000, ld=(4000, 2000)), UNSUPPORTED),
])
def test_refusals(call, kw, status):
    assert call(**kw) == status


def test_calls_without_rows_are_no_ops():
    assert quantize(rows=0, X=None) == 0 and dequantize(rows=0, codes=None) == 0
    assert qlinear(M=0, A=None) == 0 and linear(M=0, X=None, ws=None) == 0
    assert write(tokens=0, X=None) == 0 and read(rows=0, Y=None) == 0 and read(B=0, table=None) == 0


def test_sizes():
    L = ocs.lib()
    assert L.ocs_mx4_scale_bytes(0, 10, 1) == 0 and L.ocs_mx4_scale_bytes(1, 10, 0) == 0 and L.ocs_mx4_scale_bytes(1, 0, 1) == 0
    assert L.ocs_mx4_scale_bytes(1, 1, 1) == 512 and L.ocs_mx4_scale_bytes(129, 129, 1) == 4 * 512
    assert L.ocs_mx4_scale_bytes(128, 64, 2) == 512 and L.ocs_mx4_scale_bytes(128, 65, 2) == 1024
    assert L.ocs_mx4_scale_bytes(1 << 24, 1 << 16, 2) == 1 << 36

    def q(M, C, S, N, grid=2, y_type=0):
        return L.ocs_linear_mx4_workspace_bytes(M, C, S, grid, N, y_type)
    assert q(0, 10, 0, 10) == 0 and q(50, 10, 0, 10, grid=0) == 0 and q(50, 10, 0, 10, y_type=7) == 0 and q(50, 10, 0, 0) == 0
    assert q(5, 650, 13, 2600) == 0                               # few tokens: quantized inside the product
    assert q(50, 650, 13, 2600) >= 50 * (332 + 4) + 11 * 512
    assert q(1 << 20, 25088, 251, 4096) > (1 << 20) * 12669       # 32-bit products would wrap here

    def page(*a):
        return L.ocs_cache_page_bytes(ctypes.byref(_CacheDesc(0, *a)))
    assert page(16, 8, 128, 0) == 16 * 8 * (128 + 4)
    assert page(16, 8, 128, 1) == 16 * 8 * (64 + 4) and page(16, 8, 128, 2) == 16 * 8 * (64 + 8 + 4)
    assert page(1, 1, 1, 2) == 48 and page(1, 1, 17, 0) == 48
    assert page(0, 1, 1, 0) == 0 and page(1, 1, 1025, 0) == 0 and page(1, 1, 1, 3) == 0


def test_forced_plans():
    f = ocs.lib().ocs_selftest_force_mx4_plan
    assert f(48, 1, 1) == INVALID and f(64, 2, 1) == INVALID and f(256, 1, 1) == INVALID and f(64, 1, 3) == INVALID
    assert f(0, 1, 1) == 0
