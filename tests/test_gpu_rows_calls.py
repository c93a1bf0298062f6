"""The row-wise calls put together as their signatures suggest, and what their binding refuses."""
import pytest
import torch

import paper_1901_09504_b200 as ocs

from test_gpu_rows import _codes, _gen, _idx, _x, check_product

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,C,S,N", [(5, 650, 13, 300), (1, 33, 0, 70), (200, 1001, 20, 513), (3, 64, 0, 64)])
@pytest.mark.parametrize("given", [False, True])
def test_codes_go_into_the_product_without_a_length(M, C, S, N, given):
    """Both halves of the layer quantized by ocs_quantize_rows and multiplied without a word about K: the bytes that pad the
    codes' rows to 16 are not part of them (and are not zero here)."""
    x, w, idx = _x(M, M, C, "f32"), _x(N, N, C + S, "f32"), _idx(C, C, S)
    K = C + S
    def room(rows):
        buf = torch.full((rows, ocs.round_up(K, 16)), 99, dtype=torch.int8, device="cuda")
        return (buf, torch.empty(rows, device="cuda")) if given else None
    if not given:                            # the allocator hands these bytes out again
        waste = [torch.full((n * ocs.round_up(K, 16),), 99, dtype=torch.int8, device="cuda") for n in (M, N) for _ in range(4)]
        del waste
    codes, a_s = ocs.ocs_quantize_rows(x, idx_map=idx, S=S, out=room(M))
    W, w_s = ocs.ocs_quantize_rows(w, out=room(N))
    assert codes.shape == (M, K) and W.shape == (N, K)
    Y = ocs.ocs_qlinear_rows(codes, a_s, W, w_s)
    check_product(codes, a_s, W, w_s, None, Y)
    assert torch.equal(Y, ocs.ocs_qlinear_rows(codes, a_s, W, w_s, K=K))
    assert torch.equal(Y, ocs.ocs_linear_rows(x, W, w_s, idx_map=idx, S=S))


@pytest.mark.parametrize("is_signed,kind", [(True, torch.uint8), (False, torch.int8), (True, torch.bool)])
def test_codes_of_the_other_sign_are_refused(is_signed, kind):
    """The product tells signed from unsigned codes by their type: -1 written as 255 would count as 255."""
    x = _x(1, 4, 32, "f32")
    with pytest.raises(AssertionError):
        ocs.ocs_quantize_rows(x, 8, is_signed, out=(torch.zeros((4, 32), dtype=kind, device="cuda"), torch.empty(4, device="cuda")))


def test_workspaces_and_status_words_on_the_host_are_refused():
    x, W, s = _x(1, 600, 32, "f32"), _codes(2, 5000, 32, True), torch.ones(5000, device="cuda")
    y, g = torch.zeros(600, dtype=torch.int32, device="cuda"), torch.ones(600, device="cuda")
    r = ocs.ocs_token_logprobs(x, y, want_stats=True)
    codes, a_s = ocs.ocs_quantize_rows(x)
    big = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    for ws in (big.cpu(), big.view(torch.int32), big[::2]):
        with pytest.raises(AssertionError):
            ocs.ocs_linear_rows(x, W, s, ws=ws)
    for st in (torch.zeros(1, dtype=torch.int32), torch.zeros(1, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")):
        for call in (lambda: ocs.ocs_quantize_rows(x, dev_status=st), lambda: ocs.ocs_qlinear_rows(codes, a_s, W, s, dev_status=st),
                     lambda: ocs.ocs_linear_rows(x, W, s, dev_status=st), lambda: ocs.ocs_token_logprobs(x, y, dev_status=st),
                     lambda: ocs.ocs_token_logprobs_backward(x, y, r.stats, g, dev_status=st)):
            with pytest.raises(AssertionError):
                call()
    with pytest.raises(AssertionError):
        ocs.ocs_quantize_rows(x, out=(codes, None))
