"""Cases for the library's language-model operators: integer layers with a scale per token and per output channel
(row quantization, the int8 product, both in one call) and log probabilities of given tokens with their gradient.

`own` False: the operators in elementary torch operations, in 32 bits; `own` True: this repository's calls.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    return [
        # One time step of the recurrent language model's gates (hidden 650, batch 20, 2 % duplicated channels): latency.
        dict(name="linear-gates", op="linear", M=20, C=650, N=2600, S=13, x="f32", y="f32", bias=True, signed=True),
        # One new token through a square projection: the weights are read once, nothing else weighs.
        dict(name="linear-token", op="linear", M=1, C=8192, N=8192, S=0, x="bf16", y="bf16", bias=False, signed=True),
        # A prompt of odd length with 2 % duplicated channels.
        dict(name="linear-prompt", op="linear", M=2047, C=4096, N=4096, S=82, x="bf16", y="bf16", bias=True, signed=True),
        # A full batch of tokens through a wide layer: bound by the tensor cores.
        dict(name="linear-batch", op="linear", M=8192, C=8192, N=8192, S=0, x="bf16", y="bf16", bias=False, signed=True),
        # The fc6-shaped layer of the sweep at r = 0.01: ReLU activations (unsigned codes), long contraction, few rows.
        dict(name="codes-fc6", op="codes", M=128, C=25088, N=4096, S=251, x="f32", y="f32", bias=True, signed=False),
        # The language model's vocabulary layer over a whole sequence batch (35 x 20 tokens): bound by its output.
        dict(name="codes-vocabulary", op="codes", M=700, C=650, N=33278, S=13, x="f32", y="f32", bias=True, signed=True),
        # A weight matrix quantized with one scale per output channel (fc6-shaped): a streaming pass.
        dict(name="rows-weights", op="rows", M=4096, C=25088, S=0, x="f32", signed=True),
        # Tokens of a short batch, odd width, duplicated channels: latency.
        dict(name="rows-tokens", op="rows", M=333, C=5000, S=50, x="bf16", signed=True),
        # Scoring a sequence batch of the language model: the given tokens and five alternatives.
        dict(name="logprobs-score", op="logprobs", T=700, V=33278, x="f32", top=5, beta=1.0),
        # A decoding step of eight sequences over a large vocabulary, with twenty alternatives and a temperature.
        dict(name="logprobs-step", op="logprobs", T=8, V=131072, x="bf16", top=20, beta=1.25),
        # The gradient for the same sequence batch.
        dict(name="gradient-score", op="gradient", T=700, V=33278, x="f32", beta=1.0),
        # The gradient for a long batch, odd vocabulary (rows that start at any two bytes).
        dict(name="gradient-long", op="gradient", T=2048, V=50257, x="bf16", beta=1.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("linear", "linear", "codes", "rows", "logprobs", "gradient"))
    x = rng.choice(("f32", "bf16", "f16"))
    if op in ("linear", "codes"):
        while True:
            M, C, N = _log_int(rng, 1, 8192), _log_int(rng, 64, 25088), _log_int(rng, 64, 33278)
            if M * C * N <= 8192 ** 3 and C * N <= 120_000_000 and M * C <= 70_000_000 and M * N <= 70_000_000:
                break
        S = rng.choice((0, max(1, C // 100), max(1, C // 50)))
        return dict(op=op, M=M, C=C, N=N, S=S, x=x, y=rng.choice(("f32", "bf16", "f16")), bias=rng.random() < 0.5,
                    signed=rng.random() < 0.7)
    if op == "rows":
        while True:
            M, C = _log_int(rng, 1, 16384), _log_int(rng, 32, 33278)
            if M * C <= 100_000_000:
                break
        return dict(op=op, M=M, C=C, S=rng.choice((0, max(1, C // 50))), x=x, signed=rng.random() < 0.7)
    while True:
        T, V = _log_int(rng, 1, 4096), _log_int(rng, 1000, 262144)
        if T * V <= 100_000_000:
            break
    beta = rng.choice((1.0, 1.0, 0.8, 1.25))
    if op == "logprobs":
        return dict(op=op, T=T, V=V, x=x, top=rng.choice((0, 1, 5, 20)), beta=beta)
    return dict(op=op, T=T, V=V, x=x, beta=beta)


# ---------------------------------------------------------------------------------------------------- inputs
def _laplace(g, *shape):
    e = torch.empty(shape, dtype=torch.float32, device="cuda").exponential_(generator=g)
    return torch.where(torch.rand(shape, generator=g, device="cuda") < 0.5, -e, e)


def _divided(a, b):
    """a / b, rounded once (a divisor that is a Python number would be turned into a multiplication)."""
    return torch.div(a, torch.full_like(a, b))


def _activations(g, M, C, signed, kind):
    """Normal activations of which one channel in a hundred is ten times as large; non-negative after a ReLU."""
    a = torch.randn((M, C), generator=g, device="cuda")
    a = a * torch.where(torch.rand(C, generator=g, device="cuda") < 0.01, 10.0, 1.0)
    return (a if signed else a.abs()).to(_TYPES[kind])


def _index_map(g, C, S):
    """The original channels, then the duplicated ones."""
    dup = torch.randint(0, C, (S,), generator=g, device="cuda", dtype=torch.int32)
    return torch.cat([torch.arange(C, dtype=torch.int32, device="cuda"), dup])


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op = case["op"]
    s = {"case": case}
    if op in ("linear", "codes", "rows"):
        M, C, S = case["M"], case["C"], case["S"]
        if op == "rows":
            x = 0.02 * _laplace(g, M, C)
            s["x"] = (x if case["signed"] else x.abs()).to(_TYPES[case["x"]])
        else:
            N = case["N"]
            w = 0.02 * _laplace(g, N, C + S)
            alpha = w.abs().amax(1)
            s["w_scale"] = _divided(alpha, 127.0)
            s["w"] = torch.zeros((N, (C + S + 15) // 16 * 16), dtype=torch.int8, device="cuda")
            s["w"][:, :C + S] = torch.round(w.mul_((127.0 / alpha)[:, None])).to(torch.int8)
            del w
            s["bias"] = torch.randn(N, generator=g, device="cuda") if case["bias"] else None
            if op == "linear":
                s["x"] = _activations(g, M, C, case["signed"], case["x"])
            else:  # the codes of an earlier step: rows of whole 16 bytes
                hi = 127 if case["signed"] else 255
                a = _activations(g, M, C + S, case["signed"], "f32")
                alpha = a.abs().amax(1)
                s["a_scale"] = _divided(alpha, float(hi))
                kind = torch.int8 if case["signed"] else torch.uint8
                s["a"] = torch.zeros((M, (C + S + 15) // 16 * 16), dtype=kind, device="cuda")
                s["a"][:, :C + S] = torch.round(a * (float(hi) / alpha)[:, None]).to(kind)
        s["idx"] = _index_map(g, C, S)
        return s
    T, V = case["T"], case["V"]
    z = 2.5 * torch.randn((T, V), generator=g, device="cuda")
    # a few likely tokens stand out in every row, as in a trained model's answers
    likely = torch.randint(0, V, (T, 8), generator=g, device="cuda")
    z.scatter_add_(1, likely, 12.0 * torch.rand((T, 8), generator=g, device="cuda"))
    s["logits"] = z.to(_TYPES[case["x"]])
    del z
    pick = torch.randint(0, 8, (T, 1), generator=g, device="cuda")
    s["targets"] = likely.gather(1, pick)[:, 0].to(torch.int32)
    if op == "gradient":
        l = s["logits"].float() * case["beta"]
        m = l.amax(1)
        e = (l - m[:, None]).exp_()
        total = e.sum(1)
        entropy = total.log() - (e * (l - m[:, None])).sum(1) / total
        # what the forward pass keeps for the gradient: the largest logit, the log of the sum relative to it, the entropy
        s["stats"] = torch.stack([s["logits"].amax(1).float(), total.log(), entropy, m + total.log()], 1).contiguous()
        s["g_logprob"] = torch.randn(T, generator=g, device="cuda") / T
        s["g_entropy"] = 0.01 * torch.randn(T, generator=g, device="cuda") / T
    return s


# ---------------------------------------------------------------------------------------------------- plain forms
def _levels(signed):
    return (127.0, -127.0) if signed else (255.0, 0.0)


def _plain_rows(x, idx, signed):
    hi, lo = _levels(signed)
    z = x.float()
    alpha = z.abs().amax(1)
    inv = torch.where(alpha > 0, torch.div(torch.full_like(alpha, hi), alpha), torch.zeros_like(alpha))
    q = torch.round(z * inv[:, None]).clamp_(lo, hi)
    if idx.numel() > x.shape[1]:
        q = q[:, idx.long()]
    return q, _divided(alpha, hi)


def _plain_product(q, a_scale, s):
    K = q.shape[1]
    acc = q @ s["w"][:, :K].float().t()
    y = acc * (a_scale[:, None] * s["w_scale"][None, :])
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(_TYPES[s["case"]["y"]])


def _plain_logprobs(s):
    case = s["case"]
    l = s["logits"].float()
    m = l.amax(1)
    d = (l - m[:, None]) * case["beta"]
    e = d.exp()
    total = e.sum(1)
    log_total = total.log()
    at = d.gather(1, s["targets"].long()[:, None])[:, 0]
    out = {"logprob": at - log_total, "entropy": log_total - (e * d).sum(1) / total}
    k = case["top"]
    if k:
        bits = (l + 0.0).view(torch.int32)
        order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long()   # whole numbers in the order of the logits
        V = l.shape[1]
        key = order * (1 << 32) + (V - 1 - torch.arange(V, device=l.device))   # of equal logits the lowest index first
        ids = V - 1 - (torch.topk(key, k, dim=1).values & 0xFFFFFFFF)
        out["top_ids"] = ids.to(torch.int32)
        out["top_logprob"] = d.gather(1, ids) - log_total[:, None]
    return out


def _plain_gradient(s):
    l = s["logits"].float()
    st, beta = s["stats"], s["case"]["beta"]
    logp = (l - st[:, 0:1]) * beta - st[:, 1:2]
    p = logp.exp()
    g = -(s["g_logprob"][:, None] + s["g_entropy"][:, None] * (logp + st[:, 2:3])) * p
    g.scatter_add_(1, s["targets"].long()[:, None], s["g_logprob"][:, None])
    return (g * beta).to(s["logits"].dtype)


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        import paper_1901_09504_b200 as ocs
        if op == "linear":
            return ocs.ocs_linear_rows(s["x"], s["w"], s["w_scale"], idx_map=s["idx"], S=case["S"], is_signed=case["signed"],
                                       bias=s["bias"], out_dtype=_TYPES[case["y"]])
        if op == "codes":
            return ocs.ocs_qlinear_rows(s["a"], s["a_scale"], s["w"], s["w_scale"], K=case["C"] + case["S"], bias=s["bias"],
                                        out_dtype=_TYPES[case["y"]])
        if op == "rows":
            codes, scale = ocs.ocs_quantize_rows(s["x"], idx_map=s["idx"], S=case["S"], is_signed=case["signed"])
            return {"values": codes[:, :case["C"] + case["S"]] * scale[:, None], "scale": scale}
        if op == "logprobs":
            r = ocs.ocs_token_logprobs(s["logits"], s["targets"], top_k=case["top"], inv_temperature=case["beta"])
            out = {"logprob": r.logprob, "entropy": r.entropy}
            if case["top"]:
                out["top_ids"], out["top_logprob"] = r.top_ids, r.top_logprob
            return out
        return ocs.ocs_token_logprobs_backward(s["logits"], s["targets"], s["stats"], g_logprob=s["g_logprob"],
                                               g_entropy=s["g_entropy"], inv_temperature=case["beta"])
    if op == "linear":
        q, scale = _plain_rows(s["x"], s["idx"], case["signed"])
        return _plain_product(q, scale, s)
    if op == "codes":
        return _plain_product(s["a"][:, :case["C"] + case["S"]].float(), s["a_scale"], s)
    if op == "rows":
        q, scale = _plain_rows(s["x"], s["idx"], case["signed"])
        return {"values": q * scale[:, None], "scale": scale}
    if op == "logprobs":
        return _plain_logprobs(s)
    return _plain_gradient(s)


# ---------------------------------------------------------------------------------------------------- what a pass needs
def work(case):
    op = case["op"]
    if op in ("linear", "codes"):
        M, C, N, S = case["M"], case["C"], case["N"], case["S"]
        K = C + S
        first = M * C * _BYTES[case["x"]] + 4 * S if op == "linear" else M * K + 4 * M
        return {"bytes": first + N * K + 4 * N + (4 * N if case["bias"] else 0) + M * N * _BYTES[case["y"]],
                "flops": 2.0 * M * N * K}
    if op == "rows":
        M, C, S = case["M"], case["C"], case["S"]
        return {"bytes": M * C * _BYTES[case["x"]] + 4 * S + M * (C + S) + 4 * M, "flops": 3.0 * M * C}
    T, V, b = case["T"], case["V"], _BYTES[case["x"]]
    if op == "logprobs":
        return {"bytes": T * V * b + T * (12 + 8 * case["top"]), "flops": 5.0 * T * V}
    return {"bytes": 2 * T * V * b + T * 28, "flops": 6.0 * T * V}


# ---------------------------------------------------------------------------------------------------- 64 bits
def _exact_codes(x, levels, lowest):
    """Grid codes of each row and the rows' steps, from the definition: step = largest magnitude / levels."""
    step = x.abs().max(dim=1, keepdim=True).values / levels
    ratio = torch.where(step > 0, x / torch.where(step > 0, step, torch.ones_like(step)), torch.zeros_like(x))
    return torch.clamp(torch.round(ratio), min=lowest, max=levels), step


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    f64 = torch.float64
    if op in ("linear", "codes", "rows"):
        K = case["C"] + case["S"]
        levels, lowest = (127, -127) if case["signed"] else (255, 0)
        if op == "codes":
            real = s["a"][:, :K].to(f64) * s["a_scale"].to(f64).unsqueeze(1)
        else:
            codes, step = _exact_codes(s["x"].to(f64), levels, lowest)
            real = torch.index_select(codes, 1, s["idx"].to(torch.int64)) * step
            if op == "rows":
                return {"values": real, "scale": step.squeeze(1)}
        weight = s["w"][:, :K].to(f64) * s["w_scale"].to(f64).unsqueeze(1)
        y = torch.matmul(real, weight.transpose(0, 1))
        return y if s["bias"] is None else y + s["bias"].to(f64).unsqueeze(0)
    T, V, beta = case["T"], case["V"], float(case["beta"])
    rows = []
    for t in range(0, T, 256):   # in slices: the matrices in 64 bits are large
        z = s["logits"][t:t + 256].to(f64) * beta
        y = s["targets"][t:t + 256].to(torch.int64)
        logp = z - torch.logsumexp(z, dim=1, keepdim=True)
        p = torch.exp(logp)
        h = -(p * logp).sum(dim=1)
        if op == "logprobs":
            part = {"logprob": logp[torch.arange(y.numel(), device=y.device), y], "entropy": h}
            if case["top"]:
                part["top_logprob"] = torch.sort(logp, dim=1, descending=True).values[:, :case["top"]]
        else:
            g1 = s["g_logprob"][t:t + 256].to(f64).unsqueeze(1)
            g2 = s["g_entropy"][t:t + 256].to(f64).unsqueeze(1)
            one = torch.zeros_like(p)
            one[torch.arange(y.numel(), device=y.device), y] = 1.0
            part = {"g": beta * (g1 * (one - p) - g2 * p * (logp + h.unsqueeze(1)))}
        rows.append(part)
    out = {k: torch.cat([r[k] for r in rows]) for k in rows[0]}
    if op == "gradient":
        return out["g"]
    if case["top"]:
        out["top_ids"] = None
    return out
