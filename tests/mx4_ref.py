"""The block-scaled 4-bit grids and the cache's pages, restated in numpy from their definitions."""
import numpy as np

E8M0, E4M3, I8 = 1, 2, 0
BLOCK = {E8M0: 32, E4M3: 16}
E2M1 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
E4M3_POINTS = np.array([m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)][:-1])


def nearest(t, points):
    """Index of the point nearest to t >= 0, of two equally near ones the even index (point i has code i)."""
    hi = np.clip(np.searchsorted(points, t), 1, len(points) - 1)
    lo = hi - 1
    up, down = points[hi] - t, t - points[lo]
    return np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)


def up(v, m):
    return -(-v // m) * m


def quantize(z, grid, single):
    """z float64 [rows, K] (values of fp32 if `single`, else of a 16-bit type) -> (codes uint8 [rows, K], scale bytes
    uint8 [rows, blocks], row scales float64 [rows])."""
    n = BLOCK[grid]
    rows, K = z.shape
    b = np.zeros((rows, up(K, n)))
    b[:, :K] = z
    b = b.reshape(rows, -1, n)
    alpha = np.abs(b).max(2)
    r = np.ones(rows)
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        if grid == E8M0:
            e = np.where(alpha > 0, np.frexp(alpha)[1] - 1, -1000)
            byte = np.clip(e - 2 + 127, 0, 254)
            unit = np.ldexp(1.0, byte - 127)
        else:
            top = alpha.max(1)
            m, e = np.frexp(top / 2688)
            k = np.clip(np.where(top > 0, e - (m == 0.5), -117), -117, 117)
            r = np.ldexp(1.0, k)
            byte = nearest(((alpha / r[:, None]).astype(np.float32) / np.float32(6)).astype(np.float64), E4M3_POINTS)
            unit = E4M3_POINTS[byte] * r[:, None]
        t = np.where(unit[:, :, None] > 0, b / unit[:, :, None], 0.0)
        if single and grid == E4M3:
            t = t.astype(np.float32).astype(np.float64)
    code = nearest(np.abs(t), E2M1) | (np.signbit(b) * 8)
    return code.reshape(rows, -1)[:, :K].astype(np.uint8), byte.astype(np.uint8), r


def pack(codes):
    rows, K = codes.shape
    c = np.zeros((rows, up(K, 2)), np.uint8)
    c[:, :K] = codes
    return c[:, 0::2] | (c[:, 1::2] << 4)


def unpack(b, K):
    c = np.zeros((b.shape[0], 2 * b.shape[1]), np.uint8)
    c[:, 0::2], c[:, 1::2] = b & 15, b >> 4
    return c[:, :K]


def values(codes, byte, r, grid):
    """float64 values of codes [rows, K] with scale bytes [rows, blocks] and row scales [rows]."""
    v = np.where(codes & 8, -1.0, 1.0) * E2M1[codes & 7]
    s = np.ldexp(1.0, byte.astype(int) - 127) if grid == E8M0 else E4M3_POINTS[byte]
    return v * np.repeat(s, BLOCK[grid], axis=1)[:, :codes.shape[1]] * r[:, None]


def scale_index(rows, blocks):
    """Byte offsets of the scales of `rows` rows and `blocks` blocks in their tiles."""
    m, b = np.arange(rows)[:, None], np.arange(blocks)[None, :]
    P = -(-blocks // 4)
    return ((m // 128 * P + b // 4) * 32 + m % 32) * 16 + m // 32 % 4 * 4 + b % 4


def cache_sections(page_size, heads, dim, grid):
    n = page_size * heads
    cb = up(dim if grid == I8 else (dim + 1) // 2, 16)
    sb = 0 if grid == I8 else up(-(-dim // BLOCK[grid]), 4)
    at_s = n * cb
    at_r = up(at_s + n * sb, 16)
    return cb, sb, at_s, at_r, up(at_r + (0 if grid == E8M0 else 4 * n), 16)


def i8(z):
    """z float32 [rows, dim] -> (codes int8, steps float32): ocs_quantize_rows' signed 8-bit grid."""
    alpha = np.abs(z).max(1)
    with np.errstate(divide="ignore", over="ignore", invalid="ignore"):
        upf = np.where(alpha < np.float32(2.0 ** -100), np.float32(2.0 ** 64), np.float32(1))
        inv = np.where(alpha > 0, np.float32(127) / (alpha * upf), np.float32(0)).astype(np.float32)
        q = np.rint((z * upf[:, None]) * inv[:, None])
    return q.astype(np.int8), (alpha / np.float32(127)).astype(np.float32)
