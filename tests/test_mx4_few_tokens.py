"""Which ocs_linear_mx4 calls quantize their tokens inside the product: up to 1024 blocks of 16 (E4M3) or 2048 of 32 channels
(E8M0) in all, the duplicated ones among them.  Those calls ask for no workspace."""
import pytest
import torch

import mx4_ref as ref
import paper_1901_09504_b200 as ocs

LIMIT = {ocs.MX4_E4M3: 1024, ocs.MX4_E8M0: 2048}


def workspace(M, C, S, grid, N=2600, y_type=0):
    return ocs.lib().ocs_linear_mx4_workspace_bytes(M, C, S, grid, N, y_type)


@pytest.mark.parametrize("grid", LIMIT)
@pytest.mark.parametrize("M", [4, 16, 20, 32])
def test_blocks_of_duplicated_channels_count(M, grid):
    K = LIMIT[grid] // M * ref.BLOCK[grid]                       # the longest row that is within the limit
    for S in (0, 1, K // 100, K // 2, K - 8):
        assert workspace(M, K - S, S, grid) == 0
        assert workspace(M, K - S, S + 1, grid) >= M * (K + 1) // 2
        assert workspace(M, K + 1 - S, S, grid) >= M * (K + 1) // 2


@pytest.mark.gpu
@pytest.mark.parametrize("grid,M,C,S", [(ocs.MX4_E4M3, 32, 200, 300), (ocs.MX4_E4M3, 32, 200, 312), (ocs.MX4_E4M3, 32, 200, 313),
                                        (ocs.MX4_E4M3, 5, 1000, 2264), (ocs.MX4_E4M3, 5, 1000, 2265), (ocs.MX4_E4M3, 1, 64, 16000),
                                        (ocs.MX4_E8M0, 32, 1000, 1048), (ocs.MX4_E8M0, 32, 1000, 1049), (ocs.MX4_E8M0, 16, 70, 4000)])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_many_duplicated_channels_on_both_sides_of_the_limit(grid, M, C, S, kind):
    """Tails that shared memory does not hold, inside the product and before it: the bits of the two calls."""
    g = torch.Generator(device="cuda").manual_seed(M + S)
    x = torch.randn((M, C), generator=g, device="cuda").to(kind)
    dup = torch.randint(0, C, (S,), generator=g, device="cuda", dtype=torch.int32)
    idx = torch.cat([torch.arange(C, dtype=torch.int32, device="cuda"), dup])
    w = ocs.ocs_quantize_mx4(torch.randn((300, C + S), generator=g, device="cuda"), grid)
    st = ocs.new_status()
    y = ocs.ocs_linear_mx4(x, w, idx_map=idx, S=S, out_dtype=torch.float32, dev_status=st)
    two = ocs.ocs_qlinear_mx4(ocs.ocs_quantize_mx4(x, grid, idx_map=idx, S=S, dev_status=st), w, dev_status=st)
    assert ocs.ocs_poll_status(st) == 0
    assert torch.equal(y, two)
