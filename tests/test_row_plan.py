"""The forced plan of the row product is one value: a call in another thread sees the plan before or after a change, never
parts of both (the workspace query makes the same choice as the product)."""
import threading
import time

import pytest
import torch

import paper_1901_09504_b200 as ocs

P = 1 << 20            # a well-aligned address that is never dereferenced


def test_a_forced_plan_changes_as_a_whole():
    def query():
        return ocs.lib().ocs_linear_rows_workspace_bytes(P, 1, 1, 16384, 16384, 0, 256, 0)
    try:
        # 16 tokens a tile and no split: the codes of 16384 channels do not fit beside the weights.  64 tokens: never
        # quantized inside.  16 tokens of the one with eight slices of the other would be (no workspace).
        ocs.ocs_selftest_force_row_plan(16, 1, 1)
        assert query() > 0
        ocs.ocs_selftest_force_row_plan(64, 1, 8)
        assert query() > 0
        ocs.ocs_selftest_force_row_plan(16, 1, 8)
        assert query() == 0
        ocs.ocs_selftest_force_row_plan(16, 1, 1)
        stop = threading.Event()

        def flip():
            L = ocs.lib()
            while not stop.is_set():
                for _ in range(100):
                    L.ocs_selftest_force_row_plan(64, 1, 8)
                    L.ocs_selftest_force_row_plan(16, 1, 1)
        t = threading.Thread(target=flip)
        t.start()
        try:
            end = time.monotonic() + 2.0
            seen = set()
            while time.monotonic() < end:
                seen.update(query() > 0 for _ in range(100))
        finally:
            stop.set()
            t.join()
        assert seen == {True}
    finally:
        ocs.ocs_selftest_force_row_plan(0)


@pytest.mark.gpu
def test_calls_under_a_changing_plan():
    """Each call takes one plan from its check of the workspace to its launches: the same bits whatever another thread forces
    meanwhile."""
    x = torch.randn((3, 16384), device="cuda").half()
    W = torch.randint(-127, 128, (256, 16384), device="cuda", dtype=torch.int8)
    w_s = torch.rand(256, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    want = ocs.ocs_linear_rows(x, W, w_s, ws=ws)
    st = ocs.new_status()
    stop = threading.Event()

    def flip():
        while not stop.is_set():
            for plan in ((16, 1, 8), (64, 1, 8), (16, 1, 1), (32, 1, 8), (256, 2, 1), (128, 1, 4)):
                ocs.ocs_selftest_force_row_plan(*plan)
    t = threading.Thread(target=flip)
    t.start()
    try:
        end = time.monotonic() + 2.0
        while time.monotonic() < end:
            got = [ocs.ocs_linear_rows(x, W, w_s, ws=ws, dev_status=st) for _ in range(50)]
            assert all(torch.equal(g, want) for g in got)
    finally:
        stop.set()
        t.join()
        ocs.ocs_selftest_force_row_plan(0)
    assert ocs.ocs_poll_status(st) == 0
