"""Every byte of two codes at every place of a row, read back in every form: whole words, rows that start anywhere, pages of the
cache.  Every scale byte of both formats that a quantization can write."""
import numpy as np
import pytest
import torch

import mx4_ref as ref
import paper_1901_09504_b200 as ocs

from gpu_util import host

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
GRIDS = [ocs.MX4_E8M0, ocs.MX4_E4M3]
R, K = 256, 512
CODES = ((np.arange(R)[:, None] + np.arange(K // 2)[None, :]) % 256).astype(np.uint8)


def _scale_bytes(rows, blocks, grid):
    """E8M0: 0 .. 252 (E4M3: 0 .. 126) in turn."""
    return ((np.arange(rows)[:, None] * 5 + np.arange(blocks)[None, :]) % (253 if grid == ocs.MX4_E8M0 else 127)).astype(np.uint8)


def _want(codes, byte, r, grid, dtype):
    v = ref.values(ref.unpack(codes, 2 * codes.shape[1]), byte, r, grid)
    with np.errstate(over="ignore"):
        return torch.from_numpy(v.astype(np.float32)).to(dtype)       # (exact in fp32 but for infinities)


@pytest.mark.parametrize("grid", GRIDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("ld,first", [(K, 0), (K + 16, 16), (K + 8, 0), (K + 1, 0), (K + 3, 1), (K + 5, 7)])
@pytest.mark.parametrize("ld_codes,at", [(256, 0), (264, 8), (260, 4), (257, 3)])
def test_dequantize(ld_codes, at, ld, first, dtype, grid):
    blocks = K // ref.BLOCK[grid]
    byte, r = _scale_bytes(R, blocks, grid), 2.0 ** (np.arange(R) % 20 - 10)
    scales = np.zeros(ocs.lib().ocs_mx4_scale_bytes(R, K, grid), np.uint8)
    scales[ref.scale_index(R, blocks)] = byte
    buf = torch.zeros(R * ld_codes + 16, dtype=torch.uint8, device="cuda")
    codes = buf[at:at + R * ld_codes].view(R, ld_codes)[:, :K // 2]
    codes.copy_(torch.from_numpy(CODES))
    q = ocs.Mx4(codes, torch.from_numpy(scales).cuda(), torch.from_numpy(r).float().cuda(), K, grid)
    out = torch.full((R * ld + 16,), 7.0, dtype=dtype, device="cuda")
    y = out[first:first + R * ld].view(R, ld)[:, :K]
    ocs.ocs_dequantize_mx4(q, out=y)
    if grid == ocs.MX4_E8M0:
        r = np.ones(R)
    np.testing.assert_array_equal(host(y.float()), host(_want(CODES, byte, r, grid, dtype).float()))
    assert (out.view(-1)[:first] == 7).all() and (out.view(-1)[first + R * ld:] == 7).all()


@pytest.mark.parametrize("grid", [ocs.GRID_I8] + GRIDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad", [0, 1, 8])
def test_cache_read(pad, dtype, grid):
    """One head of 512 numbers (int8: 256), four tokens a page."""
    P, D = 4, 256 if grid == ocs.GRID_I8 else K
    cache = ocs.ocs_cache_new(R // P, P, 1, D, grid)
    cb, sb, at_s, at_r, size = ref.cache_sections(P, 1, D, grid)
    pages, r = np.zeros((R // P, size), np.uint8), 2.0 ** (np.arange(R) % 20 - 10)
    pages[:, :at_s] = CODES.reshape(R // P, at_s)
    if grid != ocs.GRID_I8:
        byte = _scale_bytes(R, D // ref.BLOCK[grid], grid)
        pages[:, at_s:at_s + P * sb].reshape(R // P, P, sb)[:, :, :byte.shape[1]] = byte.reshape(R // P, P, -1)
    if grid != ocs.MX4_E8M0:
        pages[:, at_r:at_r + 4 * P] = r.astype(np.float32).view(np.uint8).reshape(R // P, 4 * P)
    cache.pages.copy_(torch.from_numpy(pages))
    out = torch.full((R, 1, D + pad), 7.0, dtype=dtype, device="cuda")
    table = torch.arange(R // P, dtype=torch.int32, device="cuda")[None]
    ocs.ocs_cache_read(cache, table, torch.tensor([0, R], dtype=torch.int32, device="cuda"), R, out=out[:, :, :D])
    if grid == ocs.GRID_I8:
        want = torch.from_numpy((CODES.view(np.int8) * r[:, None]).astype(np.float32)).to(dtype)
    else:
        want = _want(CODES, byte, r if grid == ocs.MX4_E4M3 else np.ones(R), grid, dtype)
    np.testing.assert_array_equal(host(out[:, 0, :D].float()), host(want.float()))
    assert (out[:, :, D:] == 7).all()
