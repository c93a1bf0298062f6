"""The 4-bit layers as a model uses them: the layer in one call, and the recurrent language model on the 4-bit grids."""
import numpy as np
import pytest
import torch

import mx4_ref as ref
import paper_1901_09504_b200 as ocs
from ocs_inputs import configs
from paper_1901_09504_b200 import nets

from gpu_util import dev, host
from test_gpu_mx4 import GRIDS, TYPES, _idx, _x, check_product

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("grid", GRIDS)
@pytest.mark.parametrize("x_kind,y_kind", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f32", "f16")])
@pytest.mark.parametrize("M,C,S,N", [(1, 33, 0, 70), (5, 650, 13, 300), (16, 4096, 0, 129), (40, 1001, 20, 513), (129, 512, 5, 1024), (600, 2048, 40, 700)])
def test_the_layer_in_one_call_is_the_two_calls(M, C, S, N, x_kind, y_kind, grid):
    x, w, idx = _x(M, M, C, x_kind), _x(N, N, C + S, "f32", std=0.02), _idx(C, C, S)
    bias = torch.randn(N, device="cuda")
    st = ocs.new_status()
    W = ocs.ocs_quantize_mx4(w, grid, dev_status=st)
    a = ocs.ocs_quantize_mx4(x, grid, idx_map=idx, S=S, dev_status=st)
    y = ocs.ocs_linear_mx4(x, W, idx_map=idx, S=S, bias=bias, out_dtype=TYPES[y_kind], dev_status=st)
    two = ocs.ocs_qlinear_mx4(a, W, bias=bias, out_dtype=TYPES[y_kind], dev_status=st)
    assert ocs.ocs_poll_status(st) == 0
    assert torch.equal(y, two)
    check_product(y, a, W, bias, TYPES[y_kind])


@pytest.mark.parametrize("grid", GRIDS)
@pytest.mark.parametrize("plan", [(16, 1, 1), (16, 1, 2), (16, 1, 8), (32, 1, 1), (32, 1, 4), (64, 1, 1)])
@pytest.mark.parametrize("M,C,S,N,kind,ld,first", [(1, 8192, 0, 300, "bf16", 0, 0), (1, 700, 9, 129, "f16", 0, 1), (3, 5000, 50, 70, "bf16", 5001, 3),
                                                   (16, 650, 13, 257, "f32", 651, 1), (20, 577, 0, 130, "f16", 577, 5), (32, 333, 40, 500, "bf16", 0, 0),
                                                   (2, 31, 1, 16, "f32", 0, 0), (9, 1, 1, 5, "f32", 0, 0),
                                                   (32, 333, 200, 300, "f32", 0, 0), (32, 500, 500, 140, "bf16", 501, 1)])
def test_few_tokens_inside_the_product_give_the_two_calls_bits(M, C, S, N, kind, ld, first, plan, grid):
    x, w, idx = _x(M, M, C, kind, ld=ld or None, offset=first), _x(N, N, C + S, "f32", std=0.02), _idx(C, C, S)
    W = ocs.ocs_quantize_mx4(w, grid)
    st = ocs.new_status()
    a = ocs.ocs_quantize_mx4(x, grid, idx_map=idx, S=S, dev_status=st)
    ocs.ocs_selftest_force_mx4_plan(*plan)
    try:
        y = ocs.ocs_linear_mx4(x, W, idx_map=idx, S=S, dev_status=st, out_dtype=torch.float32)
        two = ocs.ocs_qlinear_mx4(a, W, dev_status=st)
    finally:
        ocs.ocs_selftest_force_mx4_plan(0)
    assert ocs.ocs_poll_status(st) == 0
    assert torch.equal(y, two)
    check_product(y, a, W, None, torch.float32)


@pytest.mark.parametrize("grid", GRIDS)
def test_bad_indices_of_few_tokens_are_flagged(grid):
    x, W, idx = _x(1, 3, 50, "bf16"), ocs.ocs_quantize_mx4(_x(2, 40, 53, "f32"), grid), _idx(1, 50, 3)
    for bad in (50, -1, 2 ** 30):
        idx[51] = bad
        st = ocs.new_status()
        ocs.ocs_linear_mx4(x, W, idx_map=idx, S=3, dev_status=st)
        assert ocs.ocs_poll_status(st) == ocs.DEV_BAD_INDEX


@pytest.mark.parametrize("grid", GRIDS)
def test_strided_inputs_and_outputs(grid):
    """Rows of a wider matrix in, columns of a wider matrix out; what lies between is left alone."""
    x = _x(1, 70, 300, "bf16", ld=333, offset=5)
    W = ocs.ocs_quantize_mx4(_x(2, 90, 300, "f32"), grid)
    buf = torch.full((70, 101), 7.0, device="cuda")
    ocs.ocs_linear_mx4(x, W, out=buf[:, 3:93])
    assert torch.equal(buf[:, 3:93], ocs.ocs_linear_mx4(x.contiguous(), W, out_dtype=torch.float32))
    assert (buf[:, :3] == 7).all() and (buf[:, 93:] == 7).all()


@pytest.mark.parametrize("grid", GRIDS)
def test_a_row_that_is_not_finite_stays_alone(grid):
    x = _x(1, 9, 200, "f32").clone()
    W = ocs.ocs_quantize_mx4(_x(2, 130, 200, "f32"), grid)
    want = ocs.ocs_linear_mx4(x, W)
    x[4, 7], x[6, 190] = float("nan"), float("inf")
    st = ocs.new_status()
    got = ocs.ocs_linear_mx4(x, W, dev_status=st)
    assert ocs.ocs_poll_status(st) == ocs.DEV_NONFINITE
    keep = [0, 1, 2, 3, 5, 7, 8]
    assert torch.equal(got[keep], want[keep])


@pytest.mark.parametrize("grid", GRIDS)
@pytest.mark.parametrize("M", [50, 7])
def test_calls_captured_with_their_own_workspaces(M, grid):
    """Two layers on two streams, captured together and replayed with new inputs (with workspaces, and without any)."""
    x = [_x(i, M, 512, "bf16").clone() for i in range(2)]
    W = [ocs.ocs_quantize_mx4(_x(5 + i, 400, 512, "f32"), grid) for i in range(2)]
    out = [torch.empty((M, 400), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    n = ocs.lib().ocs_linear_mx4_workspace_bytes(M, 512, 0, grid, 400, 2)
    assert (n == 0) == (M == 7)
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    side = torch.cuda.Stream()

    def run():
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        with torch.cuda.stream(side):
            ocs.ocs_linear_mx4(x[1], W[1], out=out[1], ws=ws[1])
        ocs.ocs_linear_mx4(x[0], W[0], out=out[0], ws=ws[0])
        main.wait_stream(side)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            run()
    torch.cuda.current_stream().wait_stream(s)
    for seed in (11, 12, 13):
        for i in range(2):
            x[i].copy_(_x(seed + i, M, 512, "bf16"))
        g.replay()
        for i in range(2):
            assert torch.equal(out[i], ocs.ocs_linear_mx4(x[i], W[i]))


def _layer64(L, x, grid):
    """The layer in 64 bits on its own weights and on activations quantized by the restatement."""
    z = host(x.double())[:, host(L.idx_map)]
    a = ref.values(*ref.quantize(z, grid, x.dtype == torch.float32), grid)
    w = host(ocs.ocs_dequantize_mx4(L.weights)).astype(np.float64)
    return a @ w.T + host(L.bias).astype(np.float64), np.abs(a) @ np.abs(w).T


@pytest.mark.parametrize("grid", GRIDS)
def test_a_layer_holds_the_split_weights(grid):
    W, A = configs.random_fc(5, 70, 130, 9)
    L = nets.prepare_mx4_layer(dev(W), dev(np.zeros(70, np.float32)), 0.05, grid)
    Wp, idx, _, _ = ocs.ocs_split(dev(W), L.S)
    w = host(Wp)[:, :130 + L.S].astype(np.float64)
    np.testing.assert_array_equal(host(L.idx_map), host(idx))
    np.testing.assert_array_equal(host(ocs.ocs_dequantize_mx4(L.weights)), ref.values(*ref.quantize(w, grid, True), grid))
    y = host(nets.mx4_linear_forward(L, dev(A)))
    want, size = _layer64(L, dev(A), grid)
    assert (np.abs(y - want) <= (137 / 16 + 12) * 2.0 ** -23 * size + 2.0 ** -24 * np.abs(want) * 1.01).all()


@pytest.mark.parametrize("grid", GRIDS)
def test_lstm_score_on_a_4_bit_grid(grid):
    cfg = configs.config5(vocab=3000, batch=4, seq=6)
    tokens = dev(cfg["tokens"])
    targets = torch.roll(tokens, -1, 0).contiguous()
    targets[-1] = -1
    st = ocs.new_status()
    layers = nets.prepare_lstm(cfg, torch.device("cuda"), dev_status=st, mx4=grid)
    r, logits = nets.lstm_score(cfg, layers, tokens, targets, top_k=5, dev_status=st, keep=True)
    again, t = nets.lstm_forward(cfg, layers, tokens, keep=True, dev_status=st)
    assert ocs.ocs_poll_status(st) == 0
    assert torch.equal(again, logits)
    want, size = _layer64(layers["W_dec"], t["tops"].view(24, -1), grid)
    assert (np.abs(host(logits) - want) <= (663 / 16 + 12) * 2.0 ** -23 * (size + 0.05) + 2.0 ** -24 * np.abs(want) * 1.01).all()
    z = logits.double()
    lp = torch.log_softmax(z, 1)
    given = targets.view(-1).long()
    ln = torch.where(given >= 0, lp.gather(1, given.clamp(min=0)[:, None])[:, 0], torch.zeros(24, dtype=torch.float64, device="cuda"))
    assert (r.logprob.double() - ln).abs().max() <= 170 * 2.0 ** -24       # (as in the test of the model with row scales)
    assert 0.5 * 3000 < float(torch.exp(-r.logprob[:20].mean())) < 2 * 3000
