"""Log probabilities of given tokens, entropy, likeliest tokens and the gradient, against the definition in 64 bits.
Tolerances count roundings: u = 2^-24; d = (l - max) * beta carries two, exp two more, a sum of n positive terms one for
every addition on its longest chain."""
import numpy as np
import pytest
import torch

import paper_1901_09504_b200 as ocs

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = 2.0 ** -24
HALF_ULP = {torch.float32: U, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _logits(seed, T, V, kind, ld=None, offset=0):
    ld = ld or V
    z = 3.0 * torch.randn(T * ld + offset + 8, generator=_gen(seed), device="cuda")
    z[::131] += 9.0
    return z.to(TYPES[kind])[offset:offset + T * ld].view(T, ld)[:, :V]


def _chain(V):
    """Additions on the longest chain of a row's sum: at most V, and no more than V / 32 + 64 with a warp on the row."""
    return min(V, V // 32 + 64)


def _ref(logits, beta, targets, k):
    z = logits.double()
    live = ~torch.isneginf(z).all(1)
    zb = z * beta
    m = zb.max(1, keepdim=True).values
    d = torch.where(live[:, None], zb - m, torch.full_like(z, -float("inf")))
    p_un = d.exp()
    s = torch.where(live, p_un.sum(1), torch.ones_like(m[:, 0]))
    logp = d - s.log()[:, None]
    p = logp.exp()
    pd = torch.where(p > 0, p * d, torch.zeros_like(p))
    E1, E2 = -pd.sum(1), torch.where(p > 0, p * d * d, torch.zeros_like(p)).sum(1)   # E|d|, E d^2
    H = torch.where(live, s.log() + E1, torch.zeros_like(s))
    out = dict(logp=logp, p=p, H=H, E1=E1, E2=E2, d=d, live=live, log_s=s.log(), m=logits.double().max(1).values)
    if targets is not None:
        y = targets.long()
        ok = (y >= 0) & (y < z.shape[1])
        out["lp"] = torch.where(ok, logp.gather(1, y.clamp(0, z.shape[1] - 1)[:, None])[:, 0], torch.zeros_like(H))
        out["dy"] = torch.where(ok, d.gather(1, y.clamp(0, z.shape[1] - 1)[:, None])[:, 0], torch.zeros_like(H))
    if k:
        val = (logits.float() + 0.0).cpu().numpy()
        order = np.argsort(-val.astype(np.float64), axis=1, kind="stable")[:, :k]
        out["ids"] = order.astype(np.int32)
    return out


def _tol_sum(ref, V):
    """Error of ln s: each term's own (its d twice rounded, exp), then the additions."""
    return U * (2 * ref["E1"] + 4 + _chain(V) + ref["log_s"].abs())


def _close(got, want, tol, what):
    got, want = got.double(), want.double()
    same = torch.isinf(want) & (got == want)
    bad = ~same & ~((got - want).abs() <= tol)
    assert not bad.any(), (what, (got - want).abs()[bad].max().item(), bad.nonzero()[:4].tolist(), got[bad][:4], want[bad][:4])


def check(logits, targets, k, beta, status=0):
    T, V = logits.shape
    st = ocs.new_status()
    r = ocs.ocs_token_logprobs(logits, targets, top_k=k, inv_temperature=beta, want_stats=True, dev_status=st)
    assert ocs.ocs_poll_status(st) == status
    ref = _ref(logits, beta, targets, k)
    ts = _tol_sum(ref, V)
    if targets is not None:
        fin = lambda t: torch.where(torch.isinf(t), torch.zeros_like(t), t).abs()
        _close(r.logprob, ref["lp"], ts + U * (2 * fin(ref["dy"]) + fin(ref["lp"])), "logprob")
    tol_h = ts + U * (2 * ref["E2"] + (6 + 2 * _chain(V)) * ref["E1"] + ref["H"].abs())
    _close(r.entropy, ref["H"], tol_h, "entropy")
    _close(r.stats[:, 1], ref["log_s"], ts, "stats")
    assert torch.equal(r.stats[:, 0].double(), ref["m"]) and torch.equal(r.stats[:, 2], r.entropy)
    if k:
        np.testing.assert_array_equal(r.top_ids.cpu().numpy(), ref["ids"])
        ids = torch.from_numpy(ref["ids"]).cuda().long()
        want, dd = ref["logp"].gather(1, ids), ref["d"].gather(1, ids)
        zero = torch.zeros_like(want)
        tol = ts[:, None] + U * (2 * torch.where(torch.isinf(dd), zero, dd).abs() + torch.where(torch.isinf(want), zero, want).abs())
        _close(r.top_logprob, want, tol, "top_logprob")
    return r, ref


@pytest.mark.parametrize("T,V,kind,k,beta", [
    (1, 1, "f32", 1, 1.0), (3, 2, "bf16", 2, 1.0), (4, 5, "f16", 5, 0.7), (2, 64, "f32", 64, 1.0), (9, 63, "bf16", 20, 1.0),
    (5, 1000, "f32", 5, 1.0), (300, 1001, "bf16", 7, 1.25), (2, 4095, "f16", 64, 1.0), (33, 4096, "bf16", 0, 1.0),
    (20, 33278, "f32", 5, 1.0), (700, 3001, "f32", 1, 1.0), (1, 131072, "bf16", 20, 1.25), (8, 131072, "f32", 20, 0.5),
    (3, 262147, "bf16", 64, 1.0), (2, 50257, "f16", 3, 4.0), (1, 1000003, "bf16", 10, 1.0), (600, 8192, "f16", 20, 1.0),
    (1300, 517, "f32", 3, 1.0), (16, 200000, "f32", 64, 1.0),
])
@pytest.mark.parametrize("layout", ["dense", "strided"])
def test_logprobs(T, V, kind, k, beta, layout):
    x = _logits(T + V, T, V, kind) if layout == "dense" else _logits(T + V, T, V, kind, ld=V + 5, offset=3)
    y = torch.randint(0, V, (T,), generator=_gen(7), device="cuda", dtype=torch.int32)
    check(x, y, k, beta)


@pytest.mark.parametrize("T,V,kind,k,beta", [
    (800, 9001, "bf16", 20, 1.0), (760, 20011, "f32", 5, 0.8), (745, 16384, "f16", 64, 1.0), (741, 33278, "bf16", 9, 1.25),
    (400, 8191, "f32", 39, 1.0), (372, 16300, "f16", 1, 1.0),
])
@pytest.mark.parametrize("masked", [False, True])
def test_logprobs_many_rows(T, V, kind, k, beta, masked):
    """More rows than are resident at once and somewhat fewer, where a CTA has a row to itself."""
    x = _logits(T + V, T, V, kind, ld=V + 1, offset=1)
    if masked:
        x[:, 1::3] = float("-inf")
        x[5] = float("-inf")
        x[6, :V - 2] = float("-inf")
    y = torch.randint(0, V, (T,), generator=_gen(7), device="cuda", dtype=torch.int32)
    y[::11] = -1
    check(x, y, k, beta)


def test_parts_are_optional():
    x = _logits(1, 6, 999, "f32")
    y = torch.arange(6, dtype=torch.int32, device="cuda")
    full = ocs.ocs_token_logprobs(x, y, top_k=4)
    none = ocs.ocs_token_logprobs(x)
    assert none.logprob is None and none.top_ids is None and none.stats is None and torch.equal(none.entropy, full.entropy)
    only = ocs.TokenLogprobs(None, None, torch.empty((6, 4), dtype=torch.int32, device="cuda"), None, None)
    ocs.ocs_token_logprobs(x, None, top_k=4, out=only)
    assert torch.equal(only.top_ids, full.top_ids)
    assert ocs.ocs_token_logprobs(x[:0], y[:0], top_k=3).top_ids.shape == (0, 3)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [70, 3000, 70001])
def test_masks_and_ties(kind, V):
    """Rows that are masked in part or wholly (-infinity, the type's lowest value), rows of equal values, -0 beside 0."""
    t = TYPES[kind]
    x = _logits(V, 12, V, kind).contiguous()
    low = torch.finfo(t).min
    x[0, 1:] = -float("inf")                 # one token left
    x[1] = -float("inf")                     # nothing left
    x[2, ::2] = -float("inf")
    x[3] = low                               # nothing but the lowest value: uniform
    x[4, : V // 2] = low
    x[5] = 1.5                               # all equal
    x[6] = 0.0
    x[6, ::3] = -0.0
    x[7] = -float("inf")
    x[7, [V - 1, V // 2, 3]] = torch.tensor([1.0, 1.0, 2.0], dtype=t, device="cuda")   # three left, two of them equal
    x[8, V - 30:] = x[8].max() + 1           # the largest all in one place, equal
    x[9] = torch.finfo(t).max
    x[10] = (torch.arange(V, device="cuda") // 64).to(t)                                # ascending, with many equal ones
    x[11] = -torch.arange(V, device="cuda").to(t) / 8
    y = torch.tensor([0, 0, 0, 5, V - 1, 2, 6, 3, V - 1, 1, V - 1, 0], dtype=torch.int32, device="cuda")
    for k in (1, 20, 64):
        r, _ = check(x, y, k, 1.0)
    assert r.logprob[0] == 0 and r.entropy[0] == 0
    assert torch.isneginf(r.logprob[1]) and r.entropy[1] == 0 and torch.isneginf(r.top_logprob[1]).all()
    assert torch.isneginf(r.logprob[2])
    g = torch.ones(12, device="cuda")
    d = ocs.ocs_token_logprobs_backward(x, y, r.stats, g, g)
    assert torch.isfinite(d).all() and (d[1] == 0).all() and (d[0] == 0).all()


def test_targets_that_name_no_token():
    x = _logits(2, 5, 400, "bf16")
    y = torch.tensor([-1, 3, -100, 400, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    r, _ = check(x, y, 2, 1.0, status=ocs.DEV_BAD_INDEX)
    assert r.logprob[[0, 2, 3, 4]].eq(0).all() and r.logprob[1] < 0
    st = ocs.new_status()
    g = torch.ones(5, device="cuda")
    d = ocs.ocs_token_logprobs_backward(x, y, r.stats, g, dev_status=st)
    assert ocs.ocs_poll_status(st) == ocs.DEV_BAD_INDEX
    assert (d[[0, 2, 3, 4]] == 0).all() and (d[1] != 0).any()


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [50, 9000, 140001])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_rows_that_are_not_finite(kind, V, value):
    x = _logits(4, 6, V, kind).contiguous()
    x[1, 7] = value
    x[4, V - 1] = value
    x[5] = value
    y = torch.full((6,), 7, dtype=torch.int32, device="cuda")
    st = ocs.new_status()
    r = ocs.ocs_token_logprobs(x, y, top_k=5, dev_status=st)
    assert ocs.ocs_poll_status(st) == ocs.DEV_NONFINITE
    bad = [1, 4, 5]
    assert torch.isnan(r.logprob[bad]).all() and torch.isnan(r.entropy[bad]).all() and torch.isnan(r.top_logprob[bad]).all()
    assert (r.top_ids[bad] == -1).all()
    check(x[[0, 2, 3]], y[:3], 5, 1.0)
    for i in (0, 2, 3):                                    # the rows beside them are as ever
        assert torch.isfinite(r.logprob[i]) and torch.isfinite(r.entropy[i])


def _ref_grad(ref, targets, beta, g, gh):
    V = ref["p"].shape[1]
    y = targets.long()
    ok = (y >= 0) & (y < V)
    g = torch.where(ok, g.double(), torch.zeros_like(g.double()))[:, None]
    one = torch.zeros_like(ref["p"]).scatter_(1, y.clamp(0, V - 1)[:, None], ok.double()[:, None])
    lph = torch.where(ref["p"] > 0, ref["logp"] + ref["H"][:, None], torch.zeros_like(ref["p"]))
    return beta * (g * (one - ref["p"]) - gh.double()[:, None] * ref["p"] * lph) * ref["live"][:, None], one


@pytest.mark.parametrize("T,V,kind,beta", [
    (1, 1, "f32", 1.0), (3, 2, "bf16", 1.0), (5, 63, "f16", 0.7), (300, 1001, "bf16", 1.25), (20, 33278, "f32", 1.0),
    (4, 50257, "bf16", 1.0), (1, 131072, "f16", 2.0), (2, 262147, "f32", 1.0), (1300, 517, "f16", 1.0), (7, 4096, "bf16", 1.0),
])
@pytest.mark.parametrize("layout", ["dense", "strided", "in_place"])
def test_gradient(T, V, kind, beta, layout):
    x = _logits(T + V, T, V, kind) if layout != "strided" else _logits(T + V, T, V, kind, ld=V + 5, offset=3)
    y = torch.randint(0, V, (T,), generator=_gen(7), device="cuda", dtype=torch.int32)
    g, gh = torch.randn(T, generator=_gen(8), device="cuda"), torch.randn(T, generator=_gen(9), device="cuda")
    r, ref = check(x, y, 0, beta)
    out = None
    rest = None
    if layout == "strided":                                # rows at other alignments than the logits'
        buf = torch.full((T * (V + 2) + 9,), 3.0, dtype=x.dtype, device="cuda")
        out, rest = buf[1:1 + T * (V + 2)].view(T, V + 2)[:, :V], buf
    elif layout == "in_place":
        x = x.contiguous()
        out = x
    d = ocs.ocs_token_logprobs_backward(x, y, r.stats, g, gh, inv_temperature=beta, out=out)
    want, one = _ref_grad(ref, y, beta, g, gh)
    p, V_ = ref["p"], V
    ts = (_tol_sum(ref, V_) + U * 2 * ref["log_s"].abs())[:, None]
    tol_h = (_tol_sum(ref, V_) + U * (2 * ref["E2"] + (6 + 2 * _chain(V_)) * ref["E1"] + ref["H"].abs()))[:, None]
    dd = ref["d"].abs()
    eps_p = U * (2 * dd + ref["logp"].abs() + 4) + ts      # relative error of p
    G, GH = g.double().abs()[:, None], gh.double().abs()[:, None]
    lph = (ref["logp"] + ref["H"][:, None]).abs()
    tol = beta * (p * (G + GH * lph) * (eps_p + 4 * U) + GH * p * (eps_p + tol_h) + 2 * U * G * one) + 2 * U * want.abs()
    tol = tol * 1.01 + (HALF_ULP[x.dtype] * want.abs() * 1.01 if kind != "f32" else 0) + {"f16": 2.0 ** -25, "f32": 1e-44, "bf16": 1e-40}[kind]
    # a p below fp32's normal range may be flushed to zero
    tol = tol + beta * (G + GH * (lph + 1)) * 2.0 ** -125
    _close(d, want, tol, "gradient")
    if rest is not None:
        rest = rest.clone()
        rest[1:1 + T * (V + 2)].view(T, V + 2)[:, :V] = 3.0
        assert (rest == 3.0).all()


def test_gradient_against_differences():
    T, V, beta = 4, 37, 1.3
    x = _logits(11, T, V, "f32").contiguous()
    x[2, 5:9] = -float("inf")
    y = torch.tensor([3, 0, 36, -1], dtype=torch.int32, device="cuda")
    g, gh = torch.randn(T, generator=_gen(8), device="cuda"), torch.randn(T, generator=_gen(9), device="cuda")
    r = ocs.ocs_token_logprobs(x, y, inv_temperature=beta, want_stats=True)
    d = ocs.ocs_token_logprobs_backward(x, y, r.stats, g, gh, inv_temperature=beta).double()

    def value(z):
        f = _ref(z, beta, y, 0)
        return g.double() * f["lp"] + gh.double() * f["H"]
    h = 1e-4
    for v in range(V):
        e = torch.zeros((T, V), dtype=torch.float64, device="cuda")
        e[:, v] = h
        diff = (value(x.double() + e) - value(x.double() - e)) / (2 * h)
        # third derivatives of both terms stay below 50 here: h^2 / 6 * 50 < 1e-7, and differences of values ~10 carry 1e-12 / h
        torch.testing.assert_close(d[:, v], diff, rtol=1e-5, atol=2e-6)


def test_missing_gradients_count_as_zero():
    x = _logits(5, 3, 700, "f32")
    y = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    r = ocs.ocs_token_logprobs(x, y, want_stats=True)
    g, z = torch.randn(3, device="cuda"), torch.zeros(3, device="cuda")
    assert torch.equal(ocs.ocs_token_logprobs_backward(x, y, r.stats, g), ocs.ocs_token_logprobs_backward(x, y, r.stats, g, z))
    assert torch.equal(ocs.ocs_token_logprobs_backward(x, None, r.stats, None, g), ocs.ocs_token_logprobs_backward(x, y, r.stats, z, g))
    assert (ocs.ocs_token_logprobs_backward(x, y, r.stats) == 0).all()


def test_offsets_past_32_bits_and_another_stream():
    ld = (1 << 30) + 8
    buf = torch.zeros(2 * ld + 1000, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (3, 1000), (ld, 1))
    x.copy_(_logits(3, 3, 1000, "bf16"))
    y = torch.tensor([5, 6, 999], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r, ref = check(x, y, 5, 1.0)
        g = torch.ones(3, device="cuda")
        near = ocs.ocs_token_logprobs_backward(x.contiguous(), y, r.stats, g, g)
        ocs.ocs_token_logprobs_backward(x, y, r.stats, g, g, out=x)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(x, near)


def test_results_do_not_depend_on_the_rows_beside():
    """A row scored alone, in a small and in a large batch: the same whole numbers, and floats within the tolerance of one
    row's sum (how a row is split among CTAs may depend on how many rows there are)."""
    V = 33278
    x = _logits(6, 400, V, "bf16")
    y = torch.randint(0, V, (400,), generator=_gen(7), device="cuda", dtype=torch.int32)
    full = ocs.ocs_token_logprobs(x, y, top_k=20)
    for n in (1, 7, 64):
        part = ocs.ocs_token_logprobs(x[:n], y[:n], top_k=20)
        assert torch.equal(part.top_ids, full.top_ids[:n])
        torch.testing.assert_close(part.logprob, full.logprob[:n], rtol=0, atol=2 * U * (_chain(V) + 60))


def test_refusals_of_the_binding():
    x = torch.zeros((4, 32), device="cuda")
    y = torch.zeros(4, dtype=torch.int32, device="cuda")
    r = ocs.ocs_token_logprobs(x, y, want_stats=True)
    for bad in (lambda: ocs.ocs_token_logprobs(x.double(), y), lambda: ocs.ocs_token_logprobs(x, y.long()),
                lambda: ocs.ocs_token_logprobs(x, y[:3]), lambda: ocs.ocs_token_logprobs(x.t(), y),
                lambda: ocs.ocs_token_logprobs(x[0], y), lambda: ocs.ocs_token_logprobs(x[:1].expand(4, 32), y),
                lambda: ocs.ocs_token_logprobs_backward(x, y, r.stats[:2]),
                lambda: ocs.ocs_token_logprobs_backward(x, y, r.stats, out=torch.empty_like(x).half())):
        with pytest.raises(AssertionError):
            bad()
    for kw, status in ((dict(top_k=33), 2), (dict(top_k=-1), 1), (dict(inv_temperature=0.0), 1)):
        with pytest.raises(ocs.OcsError) as e:
            ocs.ocs_token_logprobs(x, y, **kw)
        assert e.value.status == status
    with pytest.raises(ocs.OcsError) as e:
        ocs.ocs_token_logprobs(torch.zeros((1, 100), device="cuda"), top_k=65)
    assert e.value.status == 4
