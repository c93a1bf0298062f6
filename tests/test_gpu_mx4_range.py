"""ocs_qlinear_mx4 on rows whose scales lie at the ends of fp32's range: outputs that fp32 holds come out right whatever a product
in between would do."""
import pytest
import torch

import paper_1901_09504_b200 as ocs

from test_gpu_mx4 import TYPES, _gen, check_product

pytestmark = pytest.mark.gpu


def _rows(seed, rows, K, exponent):
    x = torch.randn((rows, K), generator=_gen(seed), device="cuda")
    x[:, ::7] *= 9
    return x * 2.0 ** exponent


PLANS = [(0, 1, 1), (16, 1, 2), (64, 1, 1), (128, 1, 2), (256, 2, 1)]
# exponents of the tokens and of the channels.  Outputs are of the order of 2^(sum + 10)
FAR = [(115, -110), (-110, 115), (115, -115), (-115, 115), (110, -60), (-60, 110), (117, 0), (0, 117), (-125, 110), (110, -125)]


@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("a,w", FAR)
@pytest.mark.parametrize("M,K,N", [(9, 4100, 150), (150, 700, 270)])
def test_far_scales(M, K, N, a, w, plan):
    if (plan[0] == 16 and M > 16) or a + w + 20 > 127:
        return
    A, W = ocs.ocs_quantize_mx4(_rows(1, M, K, a)), ocs.ocs_quantize_mx4(_rows(2, N, K, w))
    bias = torch.randn(N, generator=_gen(3), device="cuda") * 2.0 ** min(a + w, 100)
    ocs.ocs_selftest_force_mx4_plan(*plan)
    try:
        y = ocs.ocs_qlinear_mx4(A, W, bias=bias)
    finally:
        ocs.ocs_selftest_force_mx4_plan(0)
    assert torch.isfinite(y).all()
    check_product(y, A, W, bias, torch.float32)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_far_scales_of_few_tokens(kind):
    """Quantized inside the product's kernel, every output type."""
    x, W = _rows(1, 3, 4100, 115), ocs.ocs_quantize_mx4(_rows(2, 150, 4100, -110))
    A = ocs.ocs_quantize_mx4(x)
    y = ocs.ocs_linear_mx4(x, W, out_dtype=TYPES[kind])
    exact = ocs.ocs_dequantize_mx4(A).double() @ ocs.ocs_dequantize_mx4(W).double().t()
    held = exact.abs() <= torch.finfo(TYPES[kind]).max      # (sums of 4100 products of the order of 2^8: some leave fp16's range)
    assert held.float().mean() > 0.5
    assert torch.equal(torch.isfinite(y), held)
    A64, W64 = (ocs.ocs_dequantize_mx4(q).double().abs() for q in (A, W))
    tol = (4100 / 16 + 12) * 2.0 ** -23 * (A64 @ W64.t()) + torch.finfo(TYPES[kind]).eps / 2 * exact.abs() * 1.01
    assert ((y.double() - exact).abs() <= tol)[held].all()


def test_outputs_outside_of_the_range():
    """Too large: infinite with the sum's sign; too small: zero; sums of zero stay zero."""
    W = torch.cat([_rows(2, 20, 64, 0).abs(), torch.zeros((4, 64), device="cuda")])
    x = _rows(1, 5, 64, 0).abs()
    x[3] *= -1
    up = ocs.ocs_qlinear_mx4(ocs.ocs_quantize_mx4(x * 2.0 ** 100), ocs.ocs_quantize_mx4(W * 2.0 ** 100))
    sign = torch.tensor([1, 1, 1, -1, 1.0], device="cuda")[:, None]
    assert (up[:, :20] == sign * float("inf")).all() and (up[:, 20:] == 0).all()
    down = ocs.ocs_qlinear_mx4(ocs.ocs_quantize_mx4(x * 2.0 ** -100), ocs.ocs_quantize_mx4(W * 2.0 ** -100))
    assert (down == 0).all()


@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("M,K,N", [(16, 300, 300), (200, 130, 300), (600, 300, 13000)])
def test_near_and_far_rows_side_by_side(M, K, N, plan):
    """Scales from one end of the range to the other among neighbouring tokens and channels, and more tiles than run at one time."""
    if plan[0] == 16 and M > 16:
        return
    x = _rows(1, M, K, 0) * (2.0 ** torch.tensor([110.0, -100, 0, 90, -117], device="cuda"))[torch.arange(M, device="cuda") % 5][:, None]
    w = _rows(2, N, K, 0) * (2.0 ** torch.tensor([-110.0, -60, 0, 10], device="cuda"))[torch.arange(N, device="cuda") % 4][:, None]
    A, W = ocs.ocs_quantize_mx4(x), ocs.ocs_quantize_mx4(w)
    ocs.ocs_selftest_force_mx4_plan(*plan)
    try:
        y = ocs.ocs_qlinear_mx4(A, W).double()
    finally:
        ocs.ocs_selftest_force_mx4_plan(0)
    a64, w64 = (ocs.ocs_dequantize_mx4(q).double() for q in (A, W))
    exact = a64 @ w64.t()
    # the sum's roundings, and one of the result (at most half of 2^-149 below the normal numbers)
    tol = (K / 16 + 12) * 2.0 ** -23 * (a64.abs() @ w64.abs().t()) + 2.0 ** -24 * exact.abs() * 1.01 + 2.0 ** -150
    top = torch.finfo(torch.float32).max
    inside, outside = exact.abs() + tol <= top, exact.abs() - tol > top
    assert inside.float().mean() > 0.9
    assert ((y - exact).abs() <= tol)[inside].all()
    assert (y == torch.sign(exact) * float("inf"))[outside].all()
