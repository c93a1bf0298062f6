"""The gradient of a language model's scores, taken from what lstm_score hands out, against the definition in 64 bits."""
import pytest
import torch

import paper_1901_09504_b200 as ocs
from ocs_inputs import configs
from paper_1901_09504_b200 import nets

from gpu_util import dev

pytestmark = pytest.mark.gpu


def test_gradient_of_the_perplexity_of_a_model():
    cfg = configs.config5(vocab=3000, batch=4, seq=6)
    tokens = dev(cfg["tokens"])
    targets = torch.roll(tokens, -1, 0).contiguous()
    targets[-1] = -1                                       # nothing is given after the last tokens
    layers = nets.prepare_lstm(cfg, torch.device("cuda"), row_scales=True)
    r, logits = nets.lstm_score(cfg, layers, tokens, targets, want_stats=True, keep=True)
    assert torch.equal(r.logprob, nets.lstm_score(cfg, layers, tokens, targets).logprob)
    y = targets.view(-1)
    n = int((y >= 0).sum())
    g = torch.full((24,), -1.0 / n, device="cuda")         # of the mean of -ln p, the logarithm of the perplexity
    d = ocs.ocs_token_logprobs_backward(logits, y, r.stats, g)
    z = logits.double().requires_grad_()
    lp = torch.log_softmax(z, 1).gather(1, y.clamp(min=0).long()[:, None])[:, 0]
    (-lp[y >= 0].mean()).backward()
    # (p - 1[given]) / n: p around 1/3000 from an exponent around 8 and a sum of 3000 terms on chains of at most 158, that is
    # 158 + 2 * 8 + 10 roundings of p; one for the difference and one for the product at the given token
    p = torch.softmax(z.detach(), 1)
    tol = (184 * p + 4 * (torch.arange(3000, device="cuda") == y[:, None])) / n * 2.0 ** -24
    assert ((d.double() - z.grad).abs() <= tol).all()
    assert (d[y < 0] == 0).all()
