"""Token log probabilities where logits lie far from zero: stretches of the vocabulary that hold one finite mask value, rows
whose largest logit is huge, large inverse temperatures.  None of these rows holds NaN or infinity, so every result is a number,
within the tolerances of ordinary rows (they count roundings relative to distances from the row's maximum, not to its size)."""
import pytest
import torch

import paper_1901_09504_b200 as ocs

from test_gpu_logprobs import HALF_ULP, TYPES, U, _chain, _close, _gen, _logits, _ref_grad, _tol_sum, check

pytestmark = pytest.mark.gpu


def check_gradient(x, y, r, ref, beta):
    """Against the formula in 64 bits: p's relative error (its exponent's roundings and the sum's), the entropy's error, and the
    roundings of the formula itself."""
    T, V = x.shape
    g, gh = torch.randn(T, generator=_gen(8), device="cuda"), torch.randn(T, generator=_gen(9), device="cuda")
    d = ocs.ocs_token_logprobs_backward(x, y, r.stats, g, gh, inv_temperature=beta)
    want, one = _ref_grad(ref, y, beta, g, gh)
    limit = {torch.float16: 65520.0, torch.bfloat16: (2 - 2.0 ** -8) * 2.0 ** 127, torch.float32: (2 - 2.0 ** -24) * 2.0 ** 127}[x.dtype]
    want = torch.where(want.abs() >= limit, want.sign() * float("inf"), want)   # rounds beyond the type's largest value
    p, ts = ref["p"], (_tol_sum(ref, V) + U * 2 * ref["log_s"].abs())[:, None]
    tol_h = (_tol_sum(ref, V) + U * (2 * ref["E2"] + (6 + 2 * _chain(V)) * ref["E1"] + ref["H"].abs()))[:, None]
    live = lambda t: torch.where(p > 0, t.abs(), torch.zeros_like(t))
    eps_p = U * (2 * live(ref["d"]) + live(ref["logp"]) + 4) + ts
    G, GH = g.double().abs()[:, None], gh.double().abs()[:, None]
    lph = live(ref["logp"] + ref["H"][:, None])
    tol = beta * (p * (G + GH * lph) * (eps_p + 4 * U) + GH * p * (eps_p + tol_h) + 2 * U * G * one) + 2 * U * want.abs()
    tol = 1.01 * (tol + (HALF_ULP[x.dtype] * want.abs() if x.dtype != torch.float32 else 0))
    tol = tol + {torch.float16: 2.0 ** -25, torch.float32: 1e-44, torch.bfloat16: 1e-40}[x.dtype]
    tol = tol + beta * (G + GH * (lph + 1)) * 2.0 ** -125       # a p below fp32's normal range may be flushed to zero
    _close(d, want, torch.where(torch.isinf(want), torch.zeros_like(tol), tol), "gradient")


def masked_rows(V, kind, value):
    """Rows of ordinary logits in which a stretch holds `value`, and one that holds nothing else."""
    x = _logits(V, 12, V, kind).contiguous()
    n = min(V - 5, 6000)
    x[0, :n] = value
    x[1, V - n:] = value
    x[2, V // 3: V // 3 + n // 2] = value
    x[3, : V - 1] = value                    # one token left
    x[4, 1:] = value
    x[5] = value
    x[6, :256] = value                       # what the first warp's threads read first
    x[7, 256:768] = value
    x[8, ::2] = value
    x[9, : V // 2 + 1] = value
    x[10, n // 2:] = value
    x[11, : n // 2] = value
    x[11, V - n // 2:] = value
    return x


@pytest.mark.parametrize("kind,value", [(k, v) for k in ("f32", "bf16") for v in
                                        (-1e4, -1e7, -1e9, -1e10, -1e12, -1e18, -1e20, -1e25, -1e30, -3e38)] +
                         [("f16", -1e4), ("f16", -65504.0)])
@pytest.mark.parametrize("V", [700, 9001, 70001])
def test_finite_masks(kind, value, V):
    x = masked_rows(V, kind, value)
    y = torch.tensor([V - 1, 0, 1, V - 1, 0, 3, V - 1, 0, 1, V - 1, 0, V // 2], dtype=torch.int32, device="cuda")
    for beta in (1.0, 0.75):
        r, ref = check(x, y, 5, beta)
        for part in (r.logprob, r.entropy, r.top_logprob, r.stats):
            assert torch.isfinite(part).all()
        assert r.logprob[3] == 0 and r.entropy[3] == 0 and r.logprob[4] == 0 and r.entropy[4] == 0
        check_gradient(x, y, r, ref, beta)


@pytest.mark.parametrize("kind,value", [("f32", -1e10), ("bf16", -1e20), ("f16", -60000.0)])
@pytest.mark.parametrize("T,V,k", [(800, 3000, 0), (760, 20011, 5), (3, 200000, 64)])
def test_finite_masks_in_every_place(kind, value, T, V, k):
    """2048 masked neighbours that begin elsewhere in every row, for each way of sharing rows among CTAs and threads."""
    x = _logits(T, T, V, kind).contiguous()
    at = torch.randint(0, V - 2048, (T,), generator=_gen(5), device="cuda")
    at[0], at[1] = 0, V - 2048
    col = torch.arange(V, device="cuda")
    x[(col >= at[:, None]) & (col < at[:, None] + 2048)] = value
    y = torch.randint(0, V, (T,), generator=_gen(7), device="cuda", dtype=torch.int32)
    r, ref = check(x, y, k, 1.0)
    check_gradient(x, y, r, ref, 1.0)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("m", [1e6, 8e6, 2e7, 1e8, 1e9, 5e9, 1e10, 1e13, 1e20, 1e30, 1e38])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_rows_far_from_zero(kind, m, sign):
    """All logits within some 20 units in the last place of +-m, at an inverse temperature (a power of two: the reference's
    product is exact) that makes such a unit about one half; the first warp's share lower than the rest."""
    V = 5003
    bits = 23 if kind == "f32" else 7
    unit = 2.0 ** (torch.tensor(m, dtype=torch.float64).log2().floor().item() - bits)
    base = torch.tensor(sign * m, device="cuda").to(TYPES[kind]).double()
    steps = torch.randint(-20, 1, (6, V), generator=_gen(3), device="cuda").double()
    steps[:, :512] -= 12
    x = (base + unit * steps).to(TYPES[kind])
    y = torch.randint(0, V, (6,), generator=_gen(7), device="cuda", dtype=torch.int32)
    beta = 0.5 / unit
    r, ref = check(x, y, 3, beta)
    check_gradient(x, y, r, ref, beta)
    check(x, y, 3, 1.0)


@pytest.mark.parametrize("kind,value", [("f32", -1e9), ("bf16", -1e4), ("f16", -65504.0), ("f16", -3e4)])
@pytest.mark.parametrize("beta", [2.0 ** -12, 30.0, 1000.0, 4e4, 6e5, 1e7, 1e12])
def test_large_inverse_temperatures(kind, value, beta):
    x = masked_rows(9001, kind, value)
    x[10:, 100] += 200
    y = torch.zeros(12, dtype=torch.int32, device="cuda")
    r, ref = check(x, y, 5, beta)
    assert torch.isfinite(r.entropy).all()
    check_gradient(x, y, r, ref, beta)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 9001, 70001])
def test_inverse_temperature_whose_base_2_form_leaves_fp32(kind, V):
    """1.75 * 2^127 is finite, its product with log2 e is not: equal logits, one above the others, and logits so near to zero
    that their multiples of it are ordinary numbers."""
    beta = 1.75 * 2.0 ** 127
    x = torch.zeros((5, V), device="cuda").to(TYPES[kind])
    x[1] = 0.5
    x[2, V // 2] = 1.0
    x[3] = (torch.randint(-9, 10, (V,), generator=_gen(1), device="cuda").double() * 2.0 ** -126).to(TYPES[kind])
    x[4] = x[3]
    x[4, ::3] = -float("inf")
    y = torch.tensor([0, V - 1, V // 2, 1, 1], dtype=torch.int32, device="cuda")
    r, ref = check(x, y, 3, beta)
    check_gradient(x, y, r, ref, beta)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 9001, 70001])
def test_logits_whose_differences_leave_fp32(kind, V):
    """Logits up to the ends of fp32 with both signs, at an inverse temperature of 2^-126: their differences overflow, the
    differences' multiples are ordinary numbers."""
    beta = 2.0 ** -126
    x = (3.3e38 * (2 * torch.rand((4, V), generator=_gen(1), device="cuda") - 1)).to(TYPES[kind])
    x[1, :256] = torch.finfo(TYPES[kind]).min
    x[2, ::2] = -float("inf")
    x[3, V // 2:] = torch.finfo(TYPES[kind]).min
    y = torch.tensor([0, V - 1, 1, V // 2], dtype=torch.int32, device="cuda")
    r, ref = check(x, y, 3, beta)
    check_gradient(x, y, r, ref, beta)


def _device_us(f):
    """Shortest of several replays of ten calls, in us per call."""
    f()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(10):
            f()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    best = float("inf")
    for _ in range(8):
        begin.record()
        graph.replay()
        end.record()
        end.synchronize()
        best = min(best, begin.elapsed_time(end) * 100)
    del graph
    return best


@pytest.mark.parametrize("kind,T,V,k", [("bf16", 2000, 8000, 64), ("bf16", 800, 3000, 64), ("f16", 4096, 1116, 40), ("f32", 800, 3000, 64)])
def test_alternatives_of_equal_logits_take_no_pass_for_each(kind, T, V, k):
    """Rows of one value, and rows with fewer unmasked tokens than alternatives: the right ids, at a price near that of
    random rows (a pass over the row for each alternative would be ten to twenty times it)."""
    x = _logits(T, T, V, kind).contiguous()
    y = torch.zeros(T, dtype=torch.int32, device="cuda")
    out = ocs.ocs_token_logprobs(x, y, top_k=k)
    usual = _device_us(lambda: ocs.ocs_token_logprobs(x, y, top_k=k, out=out))
    for masked in (float("-inf"), -1e4, 1.0):
        z = torch.full_like(x, masked)
        z[:, 7::V // 10] = 1.0
        check(z, y, k, 1.0)
        took = _device_us(lambda: ocs.ocs_token_logprobs(z, y, top_k=k, out=out))
        assert took < 5 * usual + 5, (masked, took, usual)


@pytest.mark.parametrize("kind,V", [("bf16", 8000), ("f16", 8190), ("f32", 4090)])
def test_alternatives_that_few_threads_hold(kind, V):
    """The largest logits all in the vectors of 63 threads (of 128), far more of them than alternatives."""
    x = _logits(V, 5, V, kind).contiguous()
    ve = 8 if kind == "f32" else 16
    lucky = torch.arange(V, device="cuda") % (128 * ve) < 63 * ve
    x[:, lucky] += 40
    y = torch.zeros(5, dtype=torch.int32, device="cuda")
    for k in (5, 63, 64):
        check(x, y, k, 1.0)


@pytest.mark.parametrize("kind,T,V", [("bf16", 370, 128000), ("f32", 128, 128000)])
def test_masked_stretches_of_shared_rows_are_read_once(kind, T, V):
    """Nine tenths of rows that several CTAs share are masked: whatever the mask value, right and at one price."""
    x = _logits(T, T, V, kind).contiguous()
    y = torch.randint(0, V // 10, (T,), generator=_gen(7), device="cuda", dtype=torch.int32)
    took = {}
    for value in (-1e4, -1e9, -1e30):
        x[:, V // 10:] = value
        if T < 200:
            check(x, y, 0, 1.0)
        out = ocs.ocs_token_logprobs(x, y)
        took[value] = _device_us(lambda: ocs.ocs_token_logprobs(x, y, out=out))
    assert max(took.values()) < 1.25 * took[-1e4], took
