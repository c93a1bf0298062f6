"""The language model with token and channel scales, and the scores of given tokens: the whole path against a restatement in
64 bits of what follows the quantized codes, and against the model with one scale per tensor."""
import numpy as np
import pytest
import torch

import paper_1901_09504_b200 as ocs
from ocs_inputs import configs
from paper_1901_09504_b200 import nets

from gpu_util import dev, host

pytestmark = pytest.mark.gpu


def _quantized64(L, x):
    """The layer in 64 bits on its own codes and the activation codes of an independent quantization (numpy, fp32 steps)."""
    z = host(x)
    alpha = np.abs(z).max(1)
    inv = np.where(alpha > 0, np.float32(127) / np.where(alpha > 0, alpha, 1), 0).astype(np.float32)
    q = np.rint(z * inv[:, None])[:, host(L.idx_map)].astype(np.float64)
    w = host(L.codes)[:, :L.C + L.S].astype(np.float64)
    y = (q @ w.T) * (alpha / np.float32(127)).astype(np.float64)[:, None] * host(L.w_scales).astype(np.float64)
    return y + host(L.bias).astype(np.float64)


def test_row_layer_has_the_split_weights_on_each_channels_own_grid():
    W, A = configs.random_fc(5, 70, 130, 9)
    L = nets.prepare_row_layer(dev(W), dev(np.zeros(70, np.float32)), 0.05, 6)
    Wp, idx, _, _ = ocs.ocs_split(dev(W), L.S)
    w = host(Wp)[:, :130 + L.S]
    step = np.abs(w).max(1) / 31
    np.testing.assert_array_equal(host(L.idx_map), host(idx))
    np.testing.assert_allclose(host(L.w_scales), step, rtol=2.0 ** -23)
    # half a step, and three roundings of a position of at most 31
    assert np.abs(host(L.codes)[:, :130 + L.S] - w / step[:, None]).max() <= 0.5 + 3 * 31 * 2.0 ** -24
    assert np.abs(host(L.codes)[:, :130 + L.S]).max() == 31
    y = nets.row_linear_forward(L, dev(A))
    ref = _quantized64(L, dev(A))
    assert np.abs(host(y) - ref).max() <= 4 * 2.0 ** -24 * np.abs(ref).max()
    # the layer tracks the float layer; a scale per channel and token does not lose against one for all
    exact = A.astype(np.float64) @ W.astype(np.float64).T
    Q = nets.prepare_layer(dev(W), dev(np.zeros(70, np.float32)), 0.05, 6)
    err_rows = np.abs(host(y) - exact).mean()
    err_tensor = np.abs(host(nets.linear_forward(Q, dev(A), False)) - exact).mean()
    assert err_rows <= err_tensor


@pytest.mark.parametrize("row_scales", [True, False])
def test_lstm_score(row_scales):
    cfg = configs.config5(vocab=3000, batch=4, seq=6)
    tokens = dev(cfg["tokens"])
    targets = torch.roll(tokens, -1, 0).contiguous()
    targets[-1] = -1                                       # nothing is given after the last tokens
    st = ocs.new_status()
    layers = nets.prepare_lstm(cfg, torch.device("cuda"), dev_status=st, row_scales=row_scales)
    r = nets.lstm_score(cfg, layers, tokens, targets, top_k=5, dev_status=st)
    logits, t = nets.lstm_forward(cfg, layers, tokens, keep=True, dev_status=st)
    assert ocs.ocs_poll_status(st) == 0
    if row_scales:
        ref = _quantized64(layers["W_dec"], t["tops"].view(24, -1))
        assert np.abs(host(logits) - ref).max() <= 4 * 2.0 ** -24 * np.abs(ref).max()
    z = logits.double()
    lp = torch.log_softmax(z, 1)
    given = targets.view(-1).long()
    want = torch.where(given >= 0, lp.gather(1, given.clamp(min=0)[:, None])[:, 0], torch.zeros(24, dtype=torch.float64, device="cuda"))
    # ln p around -8 and a sum of 3000 terms on chains of at most 158: 158 + 12 roundings
    assert (r.logprob.double() - want).abs().max() <= 170 * 2.0 ** -24
    assert (r.entropy.double() + (lp.exp() * lp).sum(1)).abs().max() <= 170 * 2.0 ** -24 * 9
    ids = torch.argsort(z, dim=1, descending=True, stable=True)[:, :5]
    assert torch.equal(r.top_ids.long(), ids)
    perplexity = float(torch.exp(-r.logprob[:20].mean()))
    assert 0.5 * 3000 < perplexity < 2 * 3000              # random weights: about as good as guessing


def test_row_scaled_model_stays_near_the_float_model():
    """The whole recurrent model with row scales against the float model in 64 bits: the hidden states' error is that of
    8-bit activations and 6-bit weights."""
    cfg = configs.config5(vocab=500, batch=3, seq=4)
    p, hidden = cfg["params"], cfg["hidden"]
    layers = nets.prepare_lstm(cfg, torch.device("cuda"), row_scales=True)
    _, t = nets.lstm_forward(cfg, layers, dev(cfg["tokens"]), keep=True)
    h = [np.zeros((3, hidden)) for _ in range(2)]
    c = [np.zeros((3, hidden)) for _ in range(2)]
    sig = lambda v: 1 / (1 + np.exp(-v))
    tops = []
    for s in range(4):
        x = p["emb"][cfg["tokens"][s]].astype(np.float64)
        for l in range(2):
            g = x @ p[f"W_ih{l}"].astype(np.float64).T + p[f"b_ih{l}"] + h[l] @ p[f"W_hh{l}"].astype(np.float64).T + p[f"b_hh{l}"]
            i, f, gg, o = np.split(g, 4, 1)
            c[l] = sig(f) * c[l] + sig(i) * np.tanh(gg)
            h[l] = sig(o) * np.tanh(c[l])
            x = h[l]
        tops.append(x)
    ref = np.stack(tops)
    # 6-bit weights: steps of max|w| / 31 = 0.29 / 31, error uniform in half a step; 650 of them against |x| <= 0.05 in the
    # gates -> 1e-3 a step, a few steps and layers of it
    assert np.abs(host(t["tops"]) - ref).max() < 0.02
