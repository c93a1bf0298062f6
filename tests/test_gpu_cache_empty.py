"""Reading a cache where nothing is in it yet."""
import pytest
import torch

import paper_1901_09504_b200 as ocs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("grid", [ocs.GRID_I8, ocs.MX4_E8M0, ocs.MX4_E4M3])
def test_a_table_without_columns(grid):
    cache = ocs.ocs_cache_new(2, 4, 3, 64, grid)
    ocs.ocs_cache_write(cache, torch.ones((8, 3, 64), device="cuda"), torch.arange(8, device="cuda"))
    table = torch.zeros((5, 0), dtype=torch.int32, device="cuda")
    out, st = torch.full((7, 3, 64), 9.0, device="cuda"), ocs.new_status()
    starts = torch.full((6,), 2, dtype=torch.int32, device="cuda")
    ocs.ocs_cache_read(cache, table, starts, 7, out=out, dev_status=st)          # five sequences without tokens
    assert (out == 9).all() and ocs.ocs_poll_status(st) == 0
    starts[3:] = 4
    ocs.ocs_cache_read(cache, table, starts, 7, out=out, dev_status=st)          # one with two that no column holds
    assert (out[2:4] == 0).all() and (out[:2] == 9).all() and (out[4:] == 9).all()
    assert ocs.ocs_poll_status(st) == ocs.DEV_BAD_INDEX
