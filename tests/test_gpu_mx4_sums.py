"""The sums of the block-scaled product are fp32 and complete, also over the longest contractions.

check_product's bound holds for every order of summation and grows with the length; these hold for a length that is made of
n = K / 16 partial sums, each rounded to fp32 on its own: an addition is off by at most 2^-24 (cut off: 2^-23) of the partial sum,
whose mean square is at most that of the whole, s^2 = sum (a w)^2, for products of independent sign.  Independent errors add up
to at most sqrt(n) 2^-23 s; twice that is allowed, and the output's rounding, 2^-24 s.  Sums of 16 bits (2^-16 s a rounding), or a
product left out (s / sqrt(K)), are at least five times as far off at every K here."""
import pytest
import torch

import paper_1901_09504_b200 as ocs

from test_gpu_mx4 import GRIDS, _gen, _operand

pytestmark = pytest.mark.gpu

PLANS = [(0, 1, 1), (16, 1, 1), (32, 1, 8), (64, 1, 1), (64, 1, 8), (128, 1, 1), (128, 1, 4), (256, 2, 1)]


def _run(a, w, plan):
    ocs.ocs_selftest_force_mx4_plan(*plan)
    try:
        return ocs.ocs_qlinear_mx4(a, w)
    finally:
        ocs.ocs_selftest_force_mx4_plan(0)


def _tokens(plan):
    return plan[0] if 0 < plan[0] < 64 else 140


@pytest.mark.parametrize("grid", GRIDS)
@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("K", [2048, 25339, 65536])
def test_errors_are_those_of_32_bit_sums(K, plan, grid):
    M = _tokens(plan)
    a, w = _operand(K, M, K, grid), _operand(K + 1, 300, K, grid)
    y = _run(a, w, plan).double()
    A, W = (ocs.ocs_dequantize_mx4(q).double() for q in (a, w))
    exact, square = A @ W.t(), (A * A) @ (W * W).t()
    worst = (((y - exact) ** 2 / square).mean()).sqrt().item()
    allowed = (2 * (K / 16) ** 0.5 + 1) * 2.0 ** -23
    print(f"K {K} {plan} {worst:.2e} of {allowed:.2e}")
    assert worst <= allowed


@pytest.mark.parametrize("grid", GRIDS)
@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("K", [17, 300, 25339, 65535])
def test_the_last_block_is_whole(K, plan, grid):
    """Tokens that are zero but in their last block, which is not full: sums of its few products, all multiples of one unit and
    less than 2^24 of it, are exact."""
    M, n = _tokens(plan), {ocs.MX4_E8M0: 32, ocs.MX4_E4M3: 16}[grid]
    x = torch.zeros((M, K), device="cuda")
    first = (K - 1) // n * n
    x[:, first:] = torch.randn((M, K - first), generator=_gen(K), device="cuda")
    a, w = ocs.ocs_quantize_mx4(x, grid), _operand(K + 1, 300, K, grid)
    A, W = (ocs.ocs_dequantize_mx4(q).double() for q in (a, w))
    assert torch.equal(_run(a, w, plan).double(), A @ W.t())
    only = torch.zeros((M, K), device="cuda")                       # the very last channel
    only[:, -1] = x[:, -1]
    a = ocs.ocs_quantize_mx4(only, grid)
    got = _run(a, w, plan).double()
    assert torch.equal(got, ocs.ocs_dequantize_mx4(a).double() @ W.t()) and (got != 0).any()
