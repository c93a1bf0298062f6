"""Block-scaled 4-bit quantization and its product against plain implementations in 64 bits.  Codes and scales are equal bit
for bit; the tolerance on Y counts the roundings of its sums."""
import numpy as np
import pytest
import torch

import mx4_ref as ref
import paper_1901_09504_b200 as ocs

from gpu_util import host

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
GRIDS = [ocs.MX4_E8M0, ocs.MX4_E4M3]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _x(seed, M, C, kind, ld=None, offset=0, std=1.0):
    """Activations with a few outliers and a few tiny values, as a view with row stride ld that starts `offset` elements in."""
    ld = ld or C
    buf = torch.randn(M * ld + offset + 8, generator=_gen(seed), device="cuda") * std
    buf[::97] *= 12
    buf[::31] *= 1e-3
    return buf.to(TYPES[kind])[offset:offset + M * ld].view(M, ld)[:, :C]


def _idx(seed, C, S):
    dup = torch.randint(0, C, (S,), generator=_gen(seed + 1), device="cuda", dtype=torch.int32)
    return torch.cat([torch.arange(C, dtype=torch.int32, device="cuda"), dup])


def _outputs(rows, K, grid, ld=None):
    """An Mx4 whose memory is filled with a mark, and its buffers."""
    nb = (K + 1) // 2
    ld = ld or nb
    buf = torch.full((rows * ld + 16,), 0x5a, dtype=torch.uint8, device="cuda")
    n = ocs.lib().ocs_mx4_scale_bytes(rows, K, grid)
    scales = torch.full((n,), 0xa5, dtype=torch.uint8, device="cuda")
    return ocs.Mx4(buf[:rows * ld].view(rows, ld)[:, :nb], scales, torch.full((rows,), -1.0, device="cuda"), K, grid), buf, ld


def check_quantized(x, idx, S, grid, ld=None):
    M, C = x.shape
    K = C + S
    q, buf, ld = _outputs(M, K, grid, ld)
    st = ocs.new_status()
    ocs.ocs_quantize_mx4(x, grid, idx_map=idx, S=S, out=q, dev_status=st)
    assert ocs.ocs_poll_status(st) == 0
    z = host(x.double())[:, host(idx)] if S else host(x.double())
    codes, byte, r = ref.quantize(z, grid, x.dtype == torch.float32)
    got = host(buf)
    rows = got[:M * ld].reshape(M, ld)
    if grid == ocs.MX4_E4M3:
        np.testing.assert_array_equal(host(q.row_scales), r)
    blocks = byte.shape[1]
    at = ref.scale_index(M, ref.up(blocks, 4))
    sc = host(q.scales)
    np.testing.assert_array_equal(sc[at][:, :blocks], byte)
    assert (sc[at][:, blocks:] == 0).all()
    rest = np.ones(sc.size, bool)
    rest[at] = False
    assert (sc[rest] == 0xa5).all()                               # rows that do not exist
    np.testing.assert_array_equal(rows[:, :(K + 1) // 2], ref.pack(codes))
    assert (rows[:, (K + 1) // 2:] == 0x5a).all() and (got[M * ld:] == 0x5a).all()
    v = ref.values(codes, byte, r, grid)
    with np.errstate(over="ignore"):                              # (a block's 6 may lie above fp32's largest value)
        np.testing.assert_array_equal(host(ocs.ocs_dequantize_mx4(q)), v.astype(np.float32))
    return q, v


SHAPES = [(1, 1, 0), (1, 1, 1), (3, 7, 2), (2, 15, 0), (2, 16, 0), (5, 17, 3), (20, 650, 13), (5, 33, 33), (129, 31, 0), (17, 4096, 82),
          (2, 5000, 50), (300, 129, 3), (3, 25088, 251), (2, 33280, 0), (2, 70001, 7), (1500, 64, 0), (1, 16384, 100), (700, 1000, 10)]


@pytest.mark.parametrize("M,C,S", SHAPES)
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("grid", GRIDS)
def test_quantize(M, C, S, kind, grid):
    check_quantized(_x(M + C, M, C, kind), _idx(C, C, S), S, grid, ref.up((C + S + 1) // 2, 16))


@pytest.mark.parametrize("M,C,S,kind", [(200, 10000, 100, "f32"), (310, 25088, 251, "f32"), (300, 16641, 3, "f32"), (299, 28000, 0, "f32"),
                                        (297, 33280, 16, "bf16"), (150, 33281, 5, "f16"), (160, 20000, 0, "f16"), (299, 30000, 3000, "f32")])
@pytest.mark.parametrize("grid", GRIDS)
def test_quantize_many_long_rows(M, C, S, kind, grid):
    """Four pieces per thread, rows staged through shared memory, rows read twice, tails that shared memory does not hold."""
    check_quantized(_x(M + C, M, C, kind), _idx(C, C, S), S, grid, ref.up((C + S + 1) // 2, 16))


@pytest.mark.parametrize("M,C,S", [(1, 5, 1), (9, 3, 2), (40, 31, 0), (70, 513, 9), (3, 7279, 145), (2, 70003, 11)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("first,ld_codes", [(0, 0), (1, 1), (6, 4), (8, 3)])
@pytest.mark.parametrize("grid", GRIDS)
def test_quantize_from_any_offset_to_any_offset(M, C, S, kind, first, ld_codes, grid):
    x = _x(M + C, M, C, kind, ld=C + (first % 3 if first < 8 else -C % 8), offset=first)
    check_quantized(x, _idx(C, C, S), S, grid, (C + S + 1) // 2 + ld_codes)


@pytest.mark.parametrize("grid", GRIDS)
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_quantize_borders_and_ties(grid, kind):
    """Every border between codes times every scale, and its neighbours in x's type."""
    borders = np.array([.25, .75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.5, 3.0, 6.0])
    rows = []
    for s in ref.E4M3_POINTS[[8 * 7 + m for m in range(8)]]:                 # scales 1 .. 1.875
        v = torch.tensor(borders * s, device="cuda").to(TYPES[kind])
        inf = torch.full_like(v, float("inf"))
        n = ref.BLOCK[grid]
        for part in (v, torch.nextafter(v, inf) if kind == "f32" else v * (1 + 2 * HALF_STEP[v.dtype]), v * (1 - 2 * HALF_STEP[v.dtype])):
            row = torch.zeros(n, device="cuda", dtype=v.dtype)
            row[:10] = part
            row[10] = 6 * s                                                   # the block's largest: its scale is s
            row[11] = -float(part[3])
            rows.append(row)
    x = torch.stack(rows)
    x = torch.cat([x, torch.full_like(x, 2688.0)], 1)                         # the row's scale is 1
    check_quantized(x.contiguous(), _idx(0, x.shape[1], 0), 0, grid)


@pytest.mark.parametrize("grid", GRIDS)
def test_quantize_zero_tiny_and_huge_rows(grid):
    x = torch.zeros((9, 300), device="cuda")
    x[1, 5] = 1e-45
    x[2] = torch.linspace(-3e-38, 3e-38, 300, device="cuda")
    x[3, ::2] = 3.4028234e38
    x[4] = torch.linspace(-1e-31, 1e-30, 300, device="cuda")
    x[5, 7] = -2.0
    x[6, :40], x[6, 200:] = 1e30, 1e-5                                        # blocks far below their row's scale
    x[7, ::3] = -0.0
    x[8] = 2.0 ** -126
    check_quantized(x, _idx(0, 300, 0), 0, grid)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("C", [40, 9000, 40000])
@pytest.mark.parametrize("grid", GRIDS)
def test_quantize_flags_what_is_not_finite(value, C, grid):
    x = _x(1, 3, C, "f32").clone()
    x[1, C - 3] = value
    st = ocs.new_status()
    q = ocs.ocs_quantize_mx4(x, grid, dev_status=st)
    assert ocs.ocs_poll_status(st) == ocs.DEV_NONFINITE
    clean = ocs.ocs_quantize_mx4(x[::2].contiguous(), grid)
    assert torch.equal(ocs.ocs_dequantize_mx4(q)[::2], ocs.ocs_dequantize_mx4(clean))


def test_quantize_flags_bad_indices():
    x = _x(1, 4, 50, "bf16")
    for bad in (50, -1, 2 ** 30):
        idx = _idx(1, 50, 3)
        idx[51] = bad
        for grid in GRIDS:
            st = ocs.new_status()
            ocs.ocs_quantize_mx4(x, grid, idx_map=idx, S=3, dev_status=st)
            assert ocs.ocs_poll_status(st) == ocs.DEV_BAD_INDEX


@pytest.mark.parametrize("grid", GRIDS)
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,K,extra", [(1, 1, 0), (3, 7, 1), (5, 64, 0), (140, 333, 5), (33, 1024, 8)])
def test_dequantize_types_and_strides(M, K, extra, kind, grid):
    q = ocs.ocs_quantize_mx4(_x(7, M, K, "f32"), grid)
    want = ocs.ocs_dequantize_mx4(q).to(TYPES[kind])
    buf = torch.full((M, K + extra), 7.0, dtype=TYPES[kind], device="cuda")
    ocs.ocs_dequantize_mx4(q, out=buf[:, :K])
    assert torch.equal(buf[:, :K], want) and (buf[:, K:] == 7).all()


# ---------------------------------------------------------------------------------------------------- the product
def _operand(seed, rows, K, grid):
    return ocs.ocs_quantize_mx4(_x(seed, rows, K, "f32"), grid)


def check_product(y, a, w, bias, out_dtype):
    A, W = (ocs.ocs_dequantize_mx4(q).double() for q in (a, w))
    want = A @ W.t()
    size = A.abs() @ W.abs().t()
    if bias is not None:
        want = want + bias.double()
        size = size + bias.double().abs()
    # one rounding (at most a whole step, 2^-23, where it cuts off) for each 16 products, and a few at the end
    tol = (a.K / 16 + 12) * 2.0 ** -23 * size + HALF_STEP[out_dtype] * want.abs() * 1.01
    err = (y.double() - want).abs()
    worst = (err / tol.clamp_min(1e-300)).max().item()
    assert worst <= 1.0, worst
    return want


PLANS = [(16, 1, 1), (16, 1, 4), (32, 1, 1), (32, 1, 8), (64, 1, 1), (64, 1, 2), (128, 1, 1), (128, 1, 4), (256, 2, 1)]


@pytest.mark.parametrize("grid", GRIDS)
@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("M,K,N", [(1, 1, 1), (5, 64, 130), (16, 300, 128), (31, 1000, 257), (100, 257, 40), (300, 2048, 513), (515, 700, 700),
                                   (140, 1280, 30000), (9000, 100, 300), (1290, 513, 4100)])
def test_product_under_every_plan(M, K, N, plan, grid):
    a, w = _operand(M, M, K, grid), _operand(N + 1, N, K, grid)
    bias = torch.randn(N, generator=_gen(3), device="cuda")
    st = ocs.new_status()
    ocs.ocs_selftest_force_mx4_plan(*plan)
    try:
        y = ocs.ocs_qlinear_mx4(a, w, bias=bias, dev_status=st)
        again = ocs.ocs_qlinear_mx4(a, w, bias=bias, dev_status=st)
    finally:
        ocs.ocs_selftest_force_mx4_plan(0)
    assert ocs.ocs_poll_status(st) == 0
    check_product(y, a, w, bias, torch.float32)
    assert torch.equal(y, again)


@pytest.mark.parametrize("grid", GRIDS)
@pytest.mark.parametrize("M,K,N,bias,kind", [(1, 8192, 1000, False, "bf16"), (3, 25339, 70, True, "f32"), (130, 25088, 300, False, "f16"), (700, 663, 5001, True, "f32"),
                                             (2047, 4178, 517, True, "bf16"), (1025, 96, 33, False, "f32"), (64, 31, 20000, True, "f16"), (9000, 130, 257, False, "bf16")])
def test_product_as_planned(M, K, N, bias, kind, grid):
    a, w = _operand(M, M, K, grid), _operand(N + 1, N, K, grid)
    b = torch.randn(N, generator=_gen(3), device="cuda") if bias else None
    st = ocs.new_status()
    y = ocs.ocs_qlinear_mx4(a, w, bias=b, out_dtype=TYPES[kind], dev_status=st)
    assert ocs.ocs_poll_status(st) == 0
    check_product(y, a, w, b, TYPES[kind])
    assert torch.equal(y, ocs.ocs_qlinear_mx4(a, w, bias=b, out_dtype=TYPES[kind]))


@pytest.mark.parametrize("grid", GRIDS)
def test_scales_of_rows_that_do_not_exist_mean_nothing(grid):
    """The bytes of the last tile's missing rows are NaN in both formats here."""
    a, w = _operand(1, 70, 200, grid), _operand(2, 130, 200, grid)
    want = ocs.ocs_qlinear_mx4(a, w)
    for q in (a, w):
        rows = q.codes.shape[0]
        flat = q.scales.view(-1)
        at = torch.from_numpy(ref.scale_index(128 * q.scales.shape[0], 4 * q.scales.shape[1])).cuda()
        flat[at[rows:].reshape(-1)] = 255
    assert torch.equal(ocs.ocs_qlinear_mx4(a, w), want)


@pytest.mark.parametrize("grid", GRIDS)
def test_zero_rows_and_extreme_scales(grid):
    """Rows of zeros, and rows whose scales lie far apart (the sums' scale comes last)."""
    x, w = _x(1, 5, 300, "f32").clone(), _x(2, 140, 300, "f32").clone()
    x[1], w[7] = 0, 0
    x[2] *= 2.0 ** 60
    x[3] *= 2.0 ** -60
    w[9] *= 2.0 ** -70
    a, q = ocs.ocs_quantize_mx4(x, grid), ocs.ocs_quantize_mx4(w, grid)
    y = ocs.ocs_qlinear_mx4(a, q)
    check_product(y, a, q, None, torch.float32)
    assert (y[1] == 0).all() and (y[:, 7] == 0).all()


def test_grids_and_lengths_that_do_not_match_are_refused():
    a, b = _operand(1, 5, 64, ocs.MX4_E4M3), _operand(2, 7, 64, ocs.MX4_E8M0)
    c = _operand(3, 7, 65, ocs.MX4_E4M3)
    x = _x(1, 5, 64, "f32")
    for call in (lambda: ocs.ocs_qlinear_mx4(a, b), lambda: ocs.ocs_qlinear_mx4(a, c), lambda: ocs.ocs_linear_mx4(x, c),
                 lambda: ocs.ocs_quantize_mx4(x, ocs.GRID_I8), lambda: ocs.ocs_quantize_mx4(x, ocs.MX4_E4M3, out=c),
                 lambda: ocs.ocs_quantize_mx4(x, ocs.MX4_E4M3, idx_map=None, S=2), lambda: ocs.ocs_qlinear_mx4(a, a._replace(codes=a.codes.cpu())),
                 lambda: ocs.ocs_dequantize_mx4(a._replace(scales=a.scales[:, :0])), lambda: ocs.ocs_quantize_mx4(x.cpu()),
                 lambda: ocs.ocs_qlinear_mx4(a, a, dev_status=torch.zeros(1, dtype=torch.int32)),
                 lambda: ocs.ocs_linear_mx4(x, a, ws=torch.empty(1 << 20, dtype=torch.uint8))):
        with pytest.raises((AssertionError, AttributeError)):
            call()


def test_two_streams_at_once():
    """Products that run side by side, each with its own operands."""
    ops = [(_operand(i, 300, 2048, ocs.MX4_E4M3), _operand(i + 9, 1000, 2048, ocs.MX4_E4M3)) for i in range(4)]
    want = [ocs.ocs_qlinear_mx4(a, w) for a, w in ops]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ops]
    got = []
    for _ in range(5):
        for s, (a, w) in zip(streams, ops):
            with torch.cuda.stream(s):
                got.append(ocs.ocs_qlinear_mx4(a, w))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[i % 4]) for i, g in enumerate(got))
