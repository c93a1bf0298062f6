"""ocs_linear_rows where few tokens are quantized inside the product's kernel: that this form is the one that runs, and that
it gives the bits of the two calls, for every number of tokens a tile, K split and several token tiles."""
import pytest
import torch

import paper_1901_09504_b200 as ocs

from test_gpu_rows import TYPES, _codes, _gen, _idx, _x, check_product

pytestmark = pytest.mark.gpu


def both_forms(M, C, S, N, x, y, signed, pad=0):
    """-> names of the kernels that ocs_linear_rows launched, after comparing it with its two halves."""
    X = _x(M, M, C, x, ld=C + pad)
    idx, W = _idx(M, C, S), _codes(N, N, C + S, True)
    w_s = torch.rand(N, generator=_gen(2), device="cuda") * 0.001
    bias = torch.randn(N, generator=_gen(3), device="cuda")
    st = ocs.new_status()
    query = ocs.lib().ocs_linear_rows_workspace_bytes(X.data_ptr(), ocs.binding.DTYPES[X.dtype], M, C, C + pad, S, N,
                                                      ocs.binding.DTYPES[TYPES[y]])
    torch.cuda.synchronize()
    ocs.ocs_trace_start()
    Y = ocs.ocs_linear_rows(X, W, w_s, idx_map=idx, S=S, is_signed=signed, bias=bias, out_dtype=TYPES[y], dev_status=st)
    torch.cuda.synchronize()
    kernels = set(ocs.ocs_trace_stop())
    codes, a_s = ocs.ocs_quantize_rows(X, 8, signed, idx_map=idx, S=S, dev_status=st)
    Y2 = ocs.ocs_qlinear_rows(codes, a_s, W, w_s, bias=bias, out_dtype=TYPES[y], dev_status=st)
    assert ocs.ocs_poll_status(st) == 0
    bits = torch.int32 if y == "f32" else torch.int16
    assert torch.equal(Y.view(bits), Y2.view(bits))
    check_product(codes, a_s, W, w_s, bias, Y)
    assert (query == 0) == (kernels == {"row_gemm_kernel(fused)"})
    return kernels


FUSED = {"row_gemm_kernel(fused)"}


@pytest.mark.parametrize("M,C,S,N,x,y,signed", [
    (1, 1, 0, 1, "f32", "f32", True), (1, 4096, 0, 512, "bf16", "bf16", True), (1, 8192, 0, 8192, "bf16", "bf16", True),
    (3, 127, 2, 300, "bf16", "bf16", False), (5, 1000, 24, 4000, "f16", "f16", True), (16, 1024, 0, 1000, "bf16", "f32", True),
    (20, 650, 13, 2600, "f32", "f32", True), (31, 96, 32, 64, "bf16", "f32", True), (2, 8192, 0, 2048, "bf16", "bf16", False),
])
def test_few_tokens_are_quantized_inside(M, C, S, N, x, y, signed):
    pad = -C % 4                                            # rows of whole 8 bytes
    assert both_forms(M, C, S, N, x, y, signed, pad) == FUSED


@pytest.mark.parametrize("M,C,S,N,x,pad", [(700, 650, 13, 2600, "f32", 0), (3, 127, 2, 300, "bf16", 0), (1, 16384, 0, 16384, "bf16", 0),
                                           (32, 4096, 0, 4096, "f32", 0)])
def test_many_long_or_unaligned_tokens_are_not(M, C, S, N, x, pad):
    assert "row_gemm_kernel" in both_forms(M, C, S, N, x, "bf16", True, pad)


@pytest.mark.parametrize("tn,slices,M,C,S,N,x,y", [
    (tn, s, M, C, S, 300, x, y)
    for tn, s, C, S in ((16, 1, 1400, 24), (16, 2, 1400, 500), (16, 4, 1400, 500), (32, 1, 760, 10), (32, 1, 760, 1140),
                        (32, 2, 760, 1140), (32, 4, 760, 1140), (32, 8, 760, 1140))
    for M, x, y in ((tn, "bf16", "f32"), (tn - 3, "f16", "bf16"), (2 * tn + 5, "bf16", "f16"), (3 * tn, "f16", "f32"), (1, "f32", "f32"))
])
def test_every_plan_of_the_fused_form(tn, slices, M, C, S, N, x, y):
    try:
        ocs.ocs_selftest_force_row_plan(tn, 1, slices)
        for signed in (True, False):
            assert both_forms(M, C, S, N, x, y, signed) == FUSED
    finally:
        ocs.ocs_selftest_force_row_plan(0)
