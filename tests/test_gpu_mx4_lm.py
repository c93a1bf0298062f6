"""The recurrent language model on the 4-bit grids against itself in floating point."""
import pytest
import torch

import paper_1901_09504_b200 as ocs
from ocs_inputs import configs
from paper_1901_09504_b200 import nets

from gpu_util import dev
from test_gpu_mx4 import GRIDS

pytestmark = pytest.mark.gpu


def float_logits(cfg, tokens):
    """The model in 64 bits, without any quantization."""
    p = {k: dev(v).double() for k, v in cfg["params"].items()}
    seq, batch = tokens.shape
    h, c = ([torch.zeros((batch, cfg["hidden"]), dtype=torch.float64, device="cuda") for _ in range(2)] for _ in range(2))
    tops = []
    for t in range(seq):
        x = p["emb"][tokens[t].long()]
        for l in range(2):
            g = x @ p[f"W_ih{l}"].t() + p[f"b_ih{l}"] + h[l] @ p[f"W_hh{l}"].t() + p[f"b_hh{l}"]
            i, f, n, o = g.chunk(4, 1)
            c[l] = torch.sigmoid(f) * c[l] + torch.sigmoid(i) * torch.tanh(n)
            x = h[l] = torch.sigmoid(o) * torch.tanh(c[l])
        tops.append(x)
    return torch.cat(tops) @ p["W_dec"].t() + p["b_dec"]


def rms(t):
    return float((t.double() ** 2).mean() ** 0.5)


@pytest.mark.parametrize("grid", GRIDS)
def test_logits_are_the_float_models_but_for_the_grid(grid):
    """A number on either grid is off by at most a quarter of itself or of half the smallest step, in the mean square by less
    than an eighth (steps of 1/4 to 1/2 of a code's size, errors spread evenly over them).  The decoder has two such operands, and the
    states it sees come from two cells with two each, whose gates flatten errors: together sqrt(6) / 8 = 0.31 of the products'
    size.  Logits that have nothing to do with the model would be off by 1.4."""
    cfg = configs.config5(vocab=3000, batch=4, seq=6)
    tokens = dev(cfg["tokens"])
    want = float_logits(cfg, tokens)
    bias = dev(cfg["params"]["b_dec"]).double()
    error = {}
    for name, kw in (("4 bits", dict(mx4=grid)), ("rows of 8 bits", dict(row_scales=True))):
        st = ocs.new_status()
        layers = nets.prepare_lstm({**cfg, "w_bits": 8}, torch.device("cuda"), dev_status=st, **kw)
        logits = nets.lstm_forward(cfg, layers, tokens, dev_status=st)
        assert ocs.ocs_poll_status(st) == 0
        error[name] = rms(logits - want) / rms(want - bias)
    print(f"grid {grid}: {error}")
    assert error["4 bits"] <= 0.31
    assert error["rows of 8 bits"] < error["4 bits"]
