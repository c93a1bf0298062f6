"""Row quantization and the int8 layer with a scale per token and per output channel, against plain implementations in
64 bits.  Codes are equal bit for bit; the tolerance on Y counts the roundings of its definition."""
import numpy as np
import pytest
import torch

import paper_1901_09504_b200 as ocs

from gpu_util import host

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}   # half a unit in the last place


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _x(seed, M, C, kind, ld=None, offset=0, std=1.0):
    """Activations with a few outlier channels, as a view with row stride ld that starts `offset` elements in."""
    ld = ld or C
    buf = torch.randn(M * ld + offset + 8, generator=_gen(seed), device="cuda") * std
    buf[::97] *= 12
    return buf.to(TYPES[kind])[offset:offset + M * ld].view(M, ld)[:, :C]


def _idx(seed, C, S):
    dup = torch.randint(0, C, (S,), generator=_gen(seed + 1), device="cuda", dtype=torch.int32)
    return torch.cat([torch.arange(C, dtype=torch.int32, device="cuda"), dup])


def ref_rows(x, idx, bits, signed):
    """The definition step by step in IEEE fp32 (numpy), and the grid steps in 64 bits."""
    hi = np.float32(2 ** (bits - 1) - 1 if signed else 2 ** bits - 1)
    lo = -hi if signed else np.float32(0)
    z = x.float().cpu().numpy()
    alpha = np.abs(z).max(axis=1)
    with np.errstate(divide="ignore", over="ignore", invalid="ignore"):
        up = np.where(alpha < np.float32(2.0 ** -100), np.float32(2.0 ** 64), np.float32(1))
        inv = np.where(alpha > 0, hi / (alpha * up), np.float32(0)).astype(np.float32)
        q = np.clip(np.rint((z * up[:, None]) * inv[:, None]), lo, hi)
    q = q[:, idx.cpu().numpy()]
    return q.astype(np.int8 if signed else np.uint8), (alpha / hi).astype(np.float32)


@pytest.mark.parametrize("M,C,S,kind,bits,signed", [
    (1, 1, 0, "f32", 8, True), (1, 1, 1, "bf16", 8, True), (3, 7, 2, "f16", 8, False), (20, 650, 13, "f32", 8, True),
    (5, 33, 33, "bf16", 4, True), (17, 4096, 0, "bf16", 8, True), (17, 4096, 82, "f16", 8, False), (2, 5000, 50, "bf16", 6, True),
    (300, 129, 3, "f32", 2, True), (4, 25088, 251, "f32", 8, True), (3, 33278, 0, "f32", 8, True), (2, 70001, 7, "bf16", 8, True),
    (1500, 64, 0, "f16", 8, True), (1, 16384, 100, "f32", 8, False), (700, 1000, 10, "bf16", 5, False),
    # many long rows (staged through shared memory), rows shared by clusters
    (700, 25088, 251, "f32", 8, True), (301, 16400, 1500, "bf16", 8, False), (900, 9000, 0, "f32", 6, True), (450, 40000, 7, "f16", 8, True),
    (50, 25088, 251, "f32", 8, True), (300, 28928, 0, "f32", 4, True), (299, 28932, 1, "f32", 8, True),
])
@pytest.mark.parametrize("layout", ["dense", "strided"])
def test_quantize_rows(M, C, S, kind, bits, signed, layout):
    x = _x(M + C, M, C, kind) if layout == "dense" else _x(M + C, M, C, kind, ld=C + 3, offset=1)
    if not signed:
        x = x.abs() if layout == "dense" else x          # negative values clamp to 0 on the unsigned grid
    idx = _idx(C, C, S)
    st = ocs.new_status()
    ld = C + S + (0 if layout == "dense" else 5)
    codes = torch.full((M, ld), 77, dtype=torch.int8 if signed else torch.uint8, device="cuda")
    scales = torch.full((M,), -1.0, device="cuda")
    ocs.ocs_quantize_rows(x, bits, signed, idx_map=idx, S=S, out=(codes, scales), dev_status=st)
    q, sc = ref_rows(x, idx, bits, signed)
    assert ocs.ocs_poll_status(st) == 0
    np.testing.assert_array_equal(host(scales), sc)
    np.testing.assert_array_equal(host(codes)[:, :C + S], q)
    assert (host(codes)[:, C + S:] == 77).all()           # the padding is not ours to write
    # against 64 bits: a code is off its real-valued position by half a step plus three roundings of a number <= hi
    real = x.double().cpu().numpy()[:, idx.cpu().numpy()] / np.maximum(np.abs(x.double().cpu().numpy()).max(1, keepdims=True), 1e-300)
    hi = 2 ** (bits - 1) - 1 if signed else 2 ** bits - 1
    if signed:
        assert np.abs(host(codes)[:, :C + S] - real * hi).max() <= 0.5 + 3 * hi * 2.0 ** -24


@pytest.mark.parametrize("M,C,S", [(1, 1, 1), (9, 3, 2), (40, 31, 0), (200, 17, 5), (300, 513, 9), (160, 7279, 145), (20, 25001, 3),
                                   (310, 16389, 2), (3, 70003, 11), (2, 140009, 5)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("first", [0, 1, 6, 15])
@pytest.mark.parametrize("even", [True, False])
def test_quantize_rows_from_any_offset_to_any_offset(M, C, S, kind, first, even):
    """Rows that start anywhere relative to a 32-byte boundary, all of them alike (even) or each elsewhere, and codes that
    start at any byte; lengths of one piece up to more than a cluster's registers hold."""
    x = _x(M + C, M, C, kind, ld=-(-C // 32) * 32 if even else C + 1 + C % 2, offset=first)
    idx = _idx(C, C, S)
    ld = C + S + first % 4
    buf = torch.full((M * ld + first + 8,), 77, dtype=torch.int8, device="cuda")
    codes = buf[first:first + M * ld].view(M, ld)
    st = ocs.new_status()
    _, scales = ocs.ocs_quantize_rows(x, 8, True, idx_map=idx, S=S, out=(codes, torch.empty(M, device="cuda")), dev_status=st)
    q, sc = ref_rows(x, idx, 8, True)
    assert ocs.ocs_poll_status(st) == 0
    np.testing.assert_array_equal(host(scales), sc)
    np.testing.assert_array_equal(host(codes)[:, :C + S], q)
    assert (host(codes)[:, C + S:] == 77).all() and (host(buf)[:first] == 77).all() and (host(buf)[first + M * ld:] == 77).all()


def test_quantize_rows_zero_tiny_and_huge_rows():
    x = torch.zeros((6, 300), device="cuda")
    x[1, 5] = 1e-45                                       # the smallest subnormal
    x[2] = torch.linspace(-3e-38, 3e-38, 300, device="cuda")
    x[3, ::2] = 3.4028234e38
    x[4] = torch.linspace(-1e-31, 1e-30, 300, device="cuda")
    x[5, 7] = -2.0
    st = ocs.new_status()
    codes, scales = ocs.ocs_quantize_rows(x, dev_status=st)
    q, sc = ref_rows(x, torch.arange(300), 8, True)
    assert ocs.ocs_poll_status(st) == 0
    np.testing.assert_array_equal(host(codes)[:, :300], q)
    np.testing.assert_array_equal(host(scales), sc)
    assert (q[0] == 0).all() and sc[0] == 0 and q[1, 5] == 127 and q[5, 7] == -127


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("C", [40, 9000])
def test_quantize_rows_flags_what_is_not_finite(value, C):
    x = _x(3, 4, C, "f32").contiguous()
    x[2, C - 1] = value
    st = ocs.new_status()
    codes, scales = ocs.ocs_quantize_rows(x, dev_status=st)
    assert ocs.ocs_poll_status(st) == ocs.DEV_NONFINITE
    keep = [0, 1, 3]                                      # the other rows are as ever
    q, sc = ref_rows(x[keep], torch.arange(C), 8, True)
    np.testing.assert_array_equal(host(codes)[keep][:, :C], q)
    np.testing.assert_array_equal(host(scales)[keep], sc)


def test_quantize_rows_bad_index():
    x = _x(4, 3, 50, "bf16")
    idx = _idx(0, 50, 3)
    idx[51], idx[52] = 50, -1
    st = ocs.new_status()
    codes, _ = ocs.ocs_quantize_rows(x, idx_map=idx, S=3, dev_status=st)
    assert ocs.ocs_poll_status(st) == ocs.DEV_BAD_INDEX
    c = host(codes)
    np.testing.assert_array_equal(c[:, 51], c[:, 0])
    np.testing.assert_array_equal(c[:, 52], c[:, 0])


def _codes(seed, M, K, signed, pad=0):
    ld = ocs.round_up(K, 16) + pad
    t = torch.randint(-128 if signed else 0, 128 if signed else 256, (M, ld), generator=_gen(seed), device="cuda")
    return t.to(torch.int8 if signed else torch.uint8)[:, :K]


def check_product(A, a_s, W, w_s, bias, Y):
    """Y against 64 bits: float(acc), a*w and the sum each rounded once, then the output type."""
    acc = A.double() @ W.double().t()                      # whole numbers below 2^53: exact
    main = acc * a_s.double()[:, None] * w_s.double()[None, :]
    ref = main if bias is None else main + bias.double()[None, :]
    u = 2.0 ** -24
    tol = 1.01 * (2 * u * main.abs() + u * ref.abs() + (UNIT[Y.dtype] * ref.abs() if Y.dtype != torch.float32 else 0.0))
    tiny = {torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -134}[Y.dtype]
    bad = (Y.double() - ref).abs() > tol + tiny
    assert not bad.any(), (int(bad.sum()), (Y.double() - ref).abs().max().item(), bad.nonzero()[:4].tolist())


@pytest.mark.parametrize("M,K,N", [
    (1, 1, 1), (1, 128, 128), (1, 4096, 1000), (2, 129, 257), (7, 663, 2600), (8, 16, 5), (15, 4100, 129), (16, 127, 128),
    (17, 256, 300), (20, 663, 2600), (31, 1000, 33), (32, 2048, 640), (33, 64, 130), (63, 400, 127), (64, 4096, 4096),
    (65, 250, 2000), (100, 6339, 256), (127, 128, 384), (128, 25339, 256), (129, 777, 513), (200, 2250, 384), (255, 640, 255),
    (256, 512, 256), (257, 300, 511), (300, 25339, 64), (700, 663, 3000), (1000, 1000, 1000), (2047, 4178, 520), (520, 90, 40000),
    (3000, 2048, 2050), (2500, 130, 17),
])
@pytest.mark.parametrize("signed", [True, False])
def test_qlinear_rows(M, K, N, signed):
    A, W = _codes(M + K, M, K, signed, pad=16 if M % 3 == 0 else 0), _codes(N + K, N, K, True, pad=32 if N % 2 else 0)
    a_s = torch.rand(M, generator=_gen(1), device="cuda") * 0.02 + 1e-4
    w_s = torch.rand(N, generator=_gen(2), device="cuda") * 0.001 + 1e-6
    bias = torch.randn(N, generator=_gen(3), device="cuda") if (M + N) % 2 else None
    st = ocs.new_status()
    for y in (torch.float32, torch.bfloat16, torch.float16):
        # a row stride beyond N, and a first element that is aligned to nothing more than itself
        off, ldy = (0, N) if y == torch.float32 else ((1, N + 1) if M % 2 else (2, N + N % 2 + 2))
        buf = torch.full((off + M * ldy + 8,), 7.0, dtype=y, device="cuda")
        Y = buf[off:off + M * ldy].view(M, ldy)[:, :N]
        ocs.ocs_qlinear_rows(A, a_s, W, w_s, bias=bias, out=Y, dev_status=st)
        assert ocs.ocs_poll_status(st) == 0
        check_product(A, a_s, W, w_s, bias, Y)
        rest = buf.clone()
        rest[off:off + M * ldy].view(M, ldy)[:, :N] = 7.0
        assert (rest == 7.0).all()                         # nothing is written beside Y


@pytest.mark.parametrize("M,K,N", [(5, 4096, 300), (130, 2100, 520), (300, 1100, 777)])
def test_qlinear_rows_does_not_depend_on_the_plan(M, K, N):
    """Tokens per tile, pairs of CTAs and K splits: the same bits under every plan."""
    A, W = _codes(1, M, K, True), _codes(2, N, K, True)
    a_s, w_s = torch.rand(M, generator=_gen(1), device="cuda"), torch.rand(N, generator=_gen(2), device="cuda")
    bias = torch.randn(N, generator=_gen(3), device="cuda")
    st = ocs.new_status()
    first = ocs.ocs_qlinear_rows(A, a_s, W, w_s, bias=bias, dev_status=st)
    check_product(A, a_s, W, w_s, bias, first)
    try:
        for tn, cg, slices in [(16, 1, 1), (16, 1, 4), (32, 1, 1), (32, 1, 8), (64, 1, 1), (64, 1, 2), (64, 1, 8), (128, 1, 1),
                               (128, 1, 2), (128, 1, 4), (128, 1, 8), (256, 1, 1), (256, 2, 1)]:
            ocs.ocs_selftest_force_row_plan(tn, cg, slices)
            for _ in range(2):
                Y = ocs.ocs_qlinear_rows(A, a_s, W, w_s, bias=bias, dev_status=st)
                assert ocs.ocs_poll_status(st) == 0, (tn, cg, slices)
                assert torch.equal(Y, first), (tn, cg, slices)
    finally:
        ocs.ocs_selftest_force_row_plan(0)


def test_qlinear_rows_extreme_codes():
    """Accumulators at the ends of the documented range, and values that leave fp16."""
    for signed, K, a in ((True, 131071, -128), (False, 65793, 255)):
        A = torch.full((3, ocs.round_up(K, 16)), a, dtype=torch.int8 if signed else torch.uint8, device="cuda")[:, :K]
        W = torch.full((5, ocs.round_up(K, 16)), -128, dtype=torch.int8, device="cuda")[:, :K]
        one = torch.ones(5, device="cuda")
        Y = ocs.ocs_qlinear_rows(A, one[:3], W, one)
        assert (Y.double() == float(np.float32(a * -128 * K))).all()
        assert torch.isinf(ocs.ocs_qlinear_rows(A, one[:3], W, one, out_dtype=torch.float16)).all()


@pytest.mark.parametrize("M,C,S,N,x,y,signed", [
    (1, 4096, 0, 512, "bf16", "bf16", True), (1, 100, 3, 7, "f16", "f32", False), (20, 650, 13, 2600, "f32", "f32", True),
    (48, 5000, 100, 700, "bf16", "f16", True), (130, 650, 13, 33278, "f32", "f32", True), (333, 1000, 20, 1000, "f16", "bf16", False),
    (2047, 512, 10, 600, "bf16", "bf16", True), (8, 25088, 251, 128, "f32", "f32", False),
    # few tokens: quantized inside the product's kernel, by every row alignment, with K splits and many channel tiles
    (1, 1, 0, 1, "f32", "f32", True), (1, 1, 1, 5, "bf16", "f32", True), (3, 127, 2, 300, "bf16", "bf16", False),
    (5, 1000, 24, 40000, "f16", "f16", True), (16, 1024, 0, 4096, "f32", "bf16", True), (17, 640, 13, 3000, "f32", "f32", False),
    (20, 650, 0, 33278, "f32", "f32", True), (31, 96, 32, 64, "bf16", "f32", True), (32, 520, 5, 2000, "bf16", "bf16", True),
    (1, 16384, 300, 256, "f16", "f32", True), (2, 8192, 0, 8192, "bf16", "bf16", True), (40, 300, 3, 900, "f32", "f32", True),
])
@pytest.mark.parametrize("pad", [0, 1, 8])
def test_linear_rows_is_its_two_halves(M, C, S, N, x, y, signed, pad):
    X = _x(M, M, C, x, ld=(C + pad) if pad < 8 else ocs.round_up(C, 8) + 8)
    idx, W = _idx(M, C, S), _codes(N, N, C + S, True)
    w_s = torch.rand(N, generator=_gen(2), device="cuda") * 0.001
    bias = torch.randn(N, generator=_gen(3), device="cuda")
    st = ocs.new_status()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                          # on another stream than the tensors' own
        Y = ocs.ocs_linear_rows(X, W, w_s, idx_map=idx, S=S, is_signed=signed, bias=bias, out_dtype=TYPES[y], dev_status=st)
        codes, a_s = ocs.ocs_quantize_rows(X, 8, signed, idx_map=idx, S=S, dev_status=st)
        Y2 = ocs.ocs_qlinear_rows(codes, a_s, W, w_s, K=C + S, bias=bias, out_dtype=TYPES[y], dev_status=st)
    torch.cuda.current_stream().wait_stream(side)
    assert ocs.ocs_poll_status(st) == 0
    assert torch.equal(Y.view(torch.int32 if y == "f32" else torch.int16), Y2.view(torch.int32 if y == "f32" else torch.int16))
    check_product(codes[:, :C + S], a_s, W, w_s, bias, Y)


@pytest.mark.parametrize("M", [24, 300])
def test_linear_rows_back_to_back_and_in_a_graph(M):
    """Calls that follow one another reuse the same workspace, outputs and input buffers; then the same under graph replay."""
    C, N = 1024, 1152
    W, w_s = _codes(5, N, C, True), torch.rand(N, generator=_gen(2), device="cuda") * 0.001
    ws = torch.empty(max(256, ocs.lib().ocs_linear_rows_workspace_bytes(0, 2, M, C, C, 0, N, 0)), dtype=torch.uint8, device="cuda")
    xs = [_x(s, M, C, "bf16") for s in range(8)]
    refs = [ocs.ocs_linear_rows(x, W, w_s, out_dtype=torch.float32) for x in xs]
    torch.cuda.synchronize()
    x, out = torch.empty_like(xs[0]), torch.empty((M, N), device="cuda")
    got = []
    for _ in range(5):
        for s in xs:
            x.copy_(s)
            ocs.ocs_linear_rows(x, W, w_s, out=out, ws=ws)
            got.append(out.clone())
    assert all(torch.equal(g, refs[i % 8]) for i, g in enumerate(got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ocs.ocs_linear_rows(x, W, w_s, out=out, ws=ws)
    for i, s in enumerate(xs):
        x.copy_(s)
        graph.replay()
        assert torch.equal(out, refs[i])
    del graph


def test_linear_rows_zero_tiny_and_bad_rows():
    """Rows of zeros, rows below 2^-100, a row that is not finite and indices out of range, in both forms of the call."""
    for M in (12, 600):
        x = _x(9, M, 256, "f32").contiguous()
        x[1] = 0
        x[2] *= 1e-35
        x[3] = 0
        x[3, 255] = 1e-45
        idx = _idx(0, 256, 2)
        W, w_s = _codes(3, 130, 258, True), torch.rand(130, generator=_gen(2), device="cuda")
        st = ocs.new_status()
        Y = ocs.ocs_linear_rows(x, W, w_s, idx_map=idx, S=2, dev_status=st)
        q, sc = ref_rows(x, idx, 8, True)
        assert ocs.ocs_poll_status(st) == 0
        check_product(torch.from_numpy(q).cuda(), torch.from_numpy(sc).cuda(), W, w_s, None, Y)
        assert (Y[1] == 0).all()
        x[5, 77] = float("nan")
        Y2 = ocs.ocs_linear_rows(x, W, w_s, idx_map=idx, S=2, dev_status=st)
        assert ocs.ocs_poll_status(st) == ocs.DEV_NONFINITE
        keep = torch.arange(M, device="cuda") != 5
        assert torch.equal(Y2[keep], Y[keep])
        idx[257] = 256
        st = ocs.new_status()
        ocs.ocs_linear_rows(x[:5], W, w_s, idx_map=idx, S=2, dev_status=st)
        assert ocs.ocs_poll_status(st) == ocs.DEV_BAD_INDEX


def test_rows_beyond_32_bit_offsets():
    """Row strides that carry the last rows past 2^31 elements."""
    ld = (1 << 30) + 16
    buf = torch.zeros(2 * ld + 64, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (3, 64), (ld, 1))
    x.copy_(_x(1, 3, 64, "bf16"))
    codes, scales = ocs.ocs_quantize_rows(x)
    q, sc = ref_rows(x, torch.arange(64), 8, True)
    np.testing.assert_array_equal(host(codes)[:, :64], q)
    np.testing.assert_array_equal(host(scales), sc)
    W, w_s = _codes(2, 40, 64, True), torch.ones(40, device="cuda")
    Y = torch.as_strided(buf, (3, 40), (ld, 1))
    ocs.ocs_qlinear_rows(codes, scales, W, w_s, K=64, out=Y)
    check_product(codes[:, :64], scales, W, w_s, None, Y)
    del buf, x, Y
    cbuf = torch.zeros(2 * (1 << 31) + 64, dtype=torch.int8, device="cuda")
    A = torch.as_strided(cbuf, (3, 64), (1 << 31, 1))
    A.copy_(codes[:, :64])
    Y = ocs.ocs_qlinear_rows(A, scales, W, w_s, K=64)
    check_product(A, scales, W, w_s, None, Y)


def test_refusals_of_the_binding():
    x = torch.zeros((4, 32), device="cuda")
    W, s = torch.zeros((8, 32), dtype=torch.int8, device="cuda"), torch.ones(8, device="cuda")
    for bad in (lambda: ocs.ocs_quantize_rows(x.double()), lambda: ocs.ocs_quantize_rows(x.cpu()),
                lambda: ocs.ocs_quantize_rows(x[0]), lambda: ocs.ocs_quantize_rows(x.t()),
                lambda: ocs.ocs_quantize_rows(x[:1].expand(4, 32)), lambda: ocs.ocs_quantize_rows(x, S=2),
                lambda: ocs.ocs_qlinear_rows(x, s, W, s), lambda: ocs.ocs_qlinear_rows(W, s.double(), W, s),
                lambda: ocs.ocs_qlinear_rows(W, s, W, s[:4]), lambda: ocs.ocs_qlinear_rows(W, s, W, s, K=33),
                lambda: ocs.ocs_linear_rows(x, W[:, :16], s), lambda: ocs.ocs_linear_rows(x, W, s, out_dtype=torch.float64)):
        with pytest.raises((AssertionError, KeyError)):
            bad()
    with pytest.raises(ocs.OcsError) as e:
        ocs.ocs_quantize_rows(x, bits=9)
    assert e.value.status == 1
    with pytest.raises(ocs.OcsError) as e:
        ocs.ocs_qlinear_rows(W[:, :24].contiguous(), s, W, s)      # rows of 24 bytes
    assert e.value.status == 2
    with pytest.raises(ocs.OcsError) as e:
        big = torch.zeros((5000, 32), dtype=torch.int8, device="cuda")
        ocs.ocs_linear_rows(torch.zeros((900, 32), device="cuda"), big, torch.ones(5000, device="cuda"), ws=torch.empty(256, dtype=torch.uint8, device="cuda")[:128])
    assert e.value.status == 3
    empty = ocs.ocs_linear_rows(x[:0], W, s)
    assert empty.shape == (0, 8) and ocs.ocs_quantize_rows(x[:0])[0].shape == (0, 32)
