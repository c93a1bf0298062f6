"""Argument checks of the row-wise calls: what the host can see is refused with the documented status before anything is
launched (no GPU needed), and calls without rows are no-ops."""
import pytest

import paper_1901_09504_b200 as ocs

INVALID, SHAPE, WORKSPACE, UNSUPPORTED = 1, 2, 3, 4
P = 1 << 20            # a well-aligned address that is never dereferenced


def quantize(X=P, x_type=0, rows=4, C=32, ldx=32, S=0, idx=None, bits=8, signed=1, codes=P, ld=32, scales=P):
    return ocs.lib().ocs_quantize_rows(X, x_type, rows, C, ldx, S, idx, bits, signed, codes, ld, scales, None, None)


def qlinear(A=P, signed=1, a_s=P, M=4, K=32, lda=32, W=P, w_s=P, N=8, ldw=32, bias=None, Y=P, y_type=0, ldy=8):
    return ocs.lib().ocs_qlinear_rows(A, signed, a_s, M, K, lda, W, w_s, N, ldw, bias, Y, y_type, ldy, None, None)


def linear(X=P, x_type=0, M=4, C=32, ldx=32, S=0, idx=None, bits=8, W=P, w_s=P, N=8, ldw=32, Y=P, y_type=0, ldy=8, ws=P,
           ws_bytes=1 << 20):
    return ocs.lib().ocs_linear_rows(X, x_type, M, C, ldx, S, idx, bits, 1, W, w_s, N, ldw, None, Y, y_type, ldy, ws, ws_bytes,
                                     None, None)


def logprobs(x=P, type=0, rows=4, V=100, ld=100, targets=P, beta=1.0, k=0, lp=P, H=P, ids=None, tlp=None, stats=P):
    return ocs.lib().ocs_token_logprobs(x, type, rows, V, ld, targets, beta, k, lp, H, ids, tlp, stats, None, None)


def backward(x=P, type=0, rows=4, V=100, ld=100, targets=P, beta=1.0, stats=P, g=P, gh=None, d=2 * P, ld_d=100):
    return ocs.lib().ocs_token_logprobs_backward(x, type, rows, V, ld, targets, beta, stats, g, gh, d, ld_d, None, None)


@pytest.mark.parametrize("call,kw,status", [
    (quantize, dict(x_type=3), INVALID), (quantize, dict(bits=1), INVALID), (quantize, dict(bits=9), INVALID),
    (quantize, dict(S=-1), INVALID), (quantize, dict(X=None), INVALID), (quantize, dict(scales=None), INVALID),
    (quantize, dict(S=2, ld=34), INVALID), (quantize, dict(C=0), SHAPE), (quantize, dict(rows=-1), SHAPE),
    (quantize, dict(ldx=31), SHAPE), (quantize, dict(S=1, idx=P, ld=32), SHAPE), (quantize, dict(X=P + 2), SHAPE),
    (quantize, dict(x_type=1, X=P + 1), SHAPE), (quantize, dict(C=1 << 30, ldx=1 << 30, ld=1 << 30), UNSUPPORTED),
    (qlinear, dict(y_type=-1), INVALID), (qlinear, dict(A=None), INVALID), (qlinear, dict(W=None), INVALID),
    (qlinear, dict(Y=None), INVALID), (qlinear, dict(w_s=None), INVALID), (qlinear, dict(a_s=None), INVALID),
    (qlinear, dict(M=-1), SHAPE), (qlinear, dict(K=0), SHAPE), (qlinear, dict(N=0), SHAPE),
    (qlinear, dict(lda=40), SHAPE), (qlinear, dict(lda=16), SHAPE), (qlinear, dict(ldw=16), SHAPE),
    (qlinear, dict(A=P + 4), SHAPE), (qlinear, dict(W=P + 8), SHAPE), (qlinear, dict(ldy=7), SHAPE),
    (qlinear, dict(Y=P + 2), SHAPE), (qlinear, dict(bias=P + 1), SHAPE),
    (qlinear, dict(K=140000, lda=140000, ldw=140000), UNSUPPORTED),
    (qlinear, dict(K=66000, lda=66000, ldw=66000, signed=0), UNSUPPORTED), (qlinear, dict(M=1 << 30), UNSUPPORTED),
    (linear, dict(M=900, N=5000, ldy=5000, ws=None), WORKSPACE), (linear, dict(M=900, N=5000, ldy=5000, ws_bytes=100), WORKSPACE),
    (linear, dict(M=900, N=5000, ldy=5000, ws=P + 16), WORKSPACE),
    (linear, dict(x_type=7), INVALID), (linear, dict(bits=0), INVALID), (linear, dict(S=1, ldw=48), INVALID),
    (linear, dict(X=None), INVALID), (linear, dict(ldx=8), SHAPE), (linear, dict(S=8, idx=P), SHAPE), (linear, dict(M=-2), SHAPE),
    (logprobs, dict(type=3), INVALID), (logprobs, dict(beta=0.0), INVALID), (logprobs, dict(beta=-1.0), INVALID),
    (logprobs, dict(beta=float("inf")), INVALID), (logprobs, dict(beta=float("nan")), INVALID), (logprobs, dict(k=-1), INVALID),
    (logprobs, dict(x=None), INVALID), (logprobs, dict(targets=None), INVALID), (logprobs, dict(V=0), SHAPE),
    (logprobs, dict(rows=-1), SHAPE), (logprobs, dict(ld=99), SHAPE), (logprobs, dict(k=101), SHAPE),
    (logprobs, dict(stats=P + 4), SHAPE), (logprobs, dict(x=P + 2), SHAPE), (logprobs, dict(k=65, ids=P), UNSUPPORTED),
    (logprobs, dict(V=1 << 30, ld=1 << 30), UNSUPPORTED),
    (backward, dict(type=5), INVALID), (backward, dict(beta=0.0), INVALID), (backward, dict(stats=None), INVALID),
    (backward, dict(d=None), INVALID), (backward, dict(targets=None), INVALID), (backward, dict(ld_d=99), SHAPE),
    (backward, dict(d=P, ld=128), SHAPE), (backward, dict(type=2, d=P + 1), SHAPE), (backward, dict(rows=-1), SHAPE),
])
def test_refusals(call, kw, status):
    assert call(**kw) == status


def test_calls_without_rows_are_no_ops():
    assert quantize(rows=0, X=None) == 0
    assert qlinear(M=0, A=None) == 0
    assert linear(M=0, X=None, ws=None) == 0
    assert logprobs(rows=0, x=None) == 0
    assert backward(rows=0, x=None) == 0


def test_workspace_query():
    def q(M, C, S, N, x_type=0, y_type=0, X=P, ldx=None):
        return ocs.lib().ocs_linear_rows_workspace_bytes(X, x_type, M, C, ldx or C, S, N, y_type)
    assert q(0, 10, 0, 10) == 0 and q(5, 10, 0, 10, x_type=7) == 0
    assert q(5, 650, 13, 2600) == 0                               # few tokens: quantized inside the product
    assert q(5, 650, 13, 2600, ldx=651) >= 5 * 672 + 20           # ... unless their rows start at any four bytes
    assert q(900, 650, 13, 2600) >= 900 * 672 + 900 * 4
    assert q(1 << 20, 25088, 251, 4096) > (1 << 20) * 25088       # 32-bit products would wrap here
