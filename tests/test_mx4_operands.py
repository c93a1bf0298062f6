"""What the 4-bit and cache calls' Python side refuses before anything reaches the library (no GPU needed: tensors that only
claim to be on one)."""
import pytest
import torch

import paper_1901_09504_b200 as ocs
from paper_1901_09504_b200 import binding


class OnDevice(torch.Tensor):
    """A host tensor that passes for a device tensor."""
    is_cuda = True


def u8(*shape):
    return torch.zeros(shape, dtype=torch.uint8).as_subclass(OnDevice)


def f32(*shape):
    return torch.zeros(shape).as_subclass(OnDevice)


def rows_of_codes(codes, grid=ocs.MX4_E4M3, K=128):
    return ocs.Mx4(codes, u8(4096), f32(max(codes.shape[0], 1)), K, grid)


# one row of a matrix that is kept column by column: 64 codes, 8 bytes apart; every other byte of one row; one byte for all
SCATTERED = [lambda: u8(64, 8)[:, 3:4].t(), lambda: u8(1, 128)[:, ::2], lambda: u8(1, 1).expand(1, 64)]


@pytest.mark.parametrize("grid", [ocs.MX4_E8M0, ocs.MX4_E4M3])
@pytest.mark.parametrize("codes", SCATTERED)
def test_a_single_row_of_codes_has_to_be_dense(codes, grid):
    q, x = rows_of_codes(codes(), grid), f32(1, 128)
    w = rows_of_codes(u8(8, 64), grid)
    for call in (lambda: ocs.ocs_dequantize_mx4(q), lambda: ocs.ocs_qlinear_mx4(q, w), lambda: ocs.ocs_qlinear_mx4(w, q),
                 lambda: ocs.ocs_linear_mx4(x, q), lambda: ocs.ocs_quantize_mx4(x, grid, out=q)):
        with pytest.raises(AssertionError):
            call()


def test_rows_that_are_dense_are_taken():
    check = binding._check_mx4
    assert check(rows_of_codes(u8(1, 64))) == (1, 64)
    assert check(rows_of_codes(u8(5, 64)[3:4])) == (1, 64)                  # a row of a matrix
    assert check(rows_of_codes(u8(5, 200)[2:3, 16:80])) == (1, 64)
    assert check(rows_of_codes(u8(1, 64).as_strided((1, 64), (1, 1)))) == (1, 64)   # (a single row has no stride of its own)
    assert check(rows_of_codes(u8(5, 80)[:, :64])) == (5, 80)
    assert check(rows_of_codes(u8(1, 1), K=2)) == (1, 16)
    assert check(rows_of_codes(u8(8, 1).t()[:, :1], K=2)) == (1, 16)        # one byte: its stride says nothing
    assert check(rows_of_codes(u8(0, 64)))[0] == 0


class Elsewhere(OnDevice):
    def get_device(self):
        return 1


def test_tensors_of_a_device_that_is_not_the_current_one(monkeypatch):
    """Their stream would be another device's: refused before the library is called."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0)

    class Library:
        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return getattr(real, name)

            def called(*_):
                raise RuntimeError(f"{name} was called")
            return called
    real = ocs.lib()
    monkeypatch.setattr(binding, "_lib", Library())
    there = lambda *shape: torch.zeros(shape).as_subclass(Elsewhere)  # noqa: E731
    bytes_there = lambda *shape: torch.zeros(shape, dtype=torch.uint8).as_subclass(Elsewhere)  # noqa: E731
    q = ocs.Mx4(bytes_there(4, 64), bytes_there(4096), there(4), 128, ocs.MX4_E4M3)
    cache = ocs.QuantCache(bytes_there(2, real.ocs_cache_page_bytes(binding.C.byref(binding._CacheDesc(0, 4, 2, 32, 0)))), 4, 2, 32, 0)
    ints = lambda dtype, *shape: torch.zeros(shape, dtype=dtype).as_subclass(Elsewhere)  # noqa: E731
    for call in (lambda: ocs.ocs_dequantize_mx4(q, out=there(4, 128)), lambda: ocs.ocs_qlinear_mx4(q, q, out=there(4, 4)),
                 lambda: ocs.ocs_linear_mx4(there(4, 128), q, out=there(4, 4)), lambda: ocs.ocs_quantize_mx4(there(4, 128), out=q),
                 lambda: ocs.ocs_cache_write(cache, there(3, 2, 32), ints(torch.int64, 3)),
                 lambda: ocs.ocs_cache_read(cache, ints(torch.int32, 1, 2), ints(torch.int32, 2), 3, out=there(3, 2, 32))):
        with pytest.raises(AssertionError):
            call()
