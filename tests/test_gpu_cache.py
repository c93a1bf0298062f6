"""The quantized key/value cache against a plain restatement: every byte of a page, and the values read back."""
import numpy as np
import pytest
import torch

import mx4_ref as ref
import paper_1901_09504_b200 as ocs

from gpu_util import host

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
GRIDS = [ocs.GRID_I8, ocs.MX4_E8M0, ocs.MX4_E4M3]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _vectors(seed, n, H, D, kind, layout="dense"):
    if layout == "dense":
        x = torch.randn((n, H, D), generator=_gen(seed), device="cuda")
    elif layout == "heads first":        # [H][n][D] in memory, rows of any alignment
        x = torch.randn((H, n, D + 1), generator=_gen(seed), device="cuda")
    else:                                # part of a wider projection
        x = torch.randn((n, 3 * H * D + 5), generator=_gen(seed), device="cuda")
    x.view(-1)[::37] *= 15
    x = x.to(TYPES[kind])
    if layout == "dense":
        return x
    if layout == "heads first":
        return x[:, :, :D].transpose(0, 1)
    return x[:, H * D:2 * H * D].view(n, H, D)


def _expect(pages, x, slots, cache):
    """pages (numpy, changed in place) after a write."""
    P, H, D, grid = cache.page_size, cache.heads, cache.dim, cache.grid
    cb, sb, at_s, at_r, size = ref.cache_sections(P, H, D, grid)
    assert pages.shape[1] == size
    z = host(x.double())
    for t, s in enumerate(host(slots)):
        if s < 0:
            continue
        page = pages[s // P]
        for h in range(H):
            v = s % P * H + h
            if grid == ocs.GRID_I8:
                q, step = ref.i8(z[t, h:h + 1].astype(np.float32))
                row = np.zeros(ref.up(D, 16), np.uint8)
                row[:D] = q[0].view(np.uint8)
                page[v * cb:v * cb + row.size] = row
                page[at_r + 4 * v:at_r + 4 * v + 4] = step.view(np.uint8)
                continue
            codes, byte, r = ref.quantize(z[t, h:h + 1], grid, x.dtype == torch.float32)
            n = byte.shape[1]
            row = np.zeros(ref.up(D, 16) // 2, np.uint8)
            packed = ref.pack(codes)[0]
            row[:packed.size] = packed
            page[v * cb:v * cb + row.size] = row
            page[at_s + v * sb:at_s + v * sb + n] = byte[0]
            if grid == ocs.MX4_E4M3:
                page[at_r + 4 * v:at_r + 4 * v + 4] = r.astype(np.float32).view(np.uint8)


def _values(pages, slots, cache):
    """float64 [n, H, D]: what the slots hold."""
    P, H, D, grid = cache.page_size, cache.heads, cache.dim, cache.grid
    cb, sb, at_s, at_r, _ = ref.cache_sections(P, H, D, grid)
    out = np.zeros((len(slots), H, D))
    for t, s in enumerate(slots):
        page = pages[s // P]
        for h in range(H):
            v = s % P * H + h
            r = page[at_r + 4 * v:at_r + 4 * v + 4].copy().view(np.float32).astype(float) if grid != ocs.MX4_E8M0 else np.ones(1)
            row = page[v * cb:(v + 1) * cb]
            if grid == ocs.GRID_I8:
                out[t, h] = row[:D].view(np.int8).astype(float) * r
            else:
                n = -(-D // ref.BLOCK[grid])
                out[t, h] = ref.values(ref.unpack(row[None], D), page[None, at_s + v * sb:at_s + v * sb + n], r, grid)[0]
    return out


@pytest.mark.parametrize("grid", GRIDS)
@pytest.mark.parametrize("kind,layout", [("f32", "dense"), ("f16", "heads first"), ("bf16", "part"), ("bf16", "dense"), ("f32", "part")])
@pytest.mark.parametrize("n,H,D,P", [(1, 1, 1, 1), (5, 3, 20, 4), (33, 2, 64, 16), (9, 5, 80, 16), (7, 2, 96, 8), (4, 1, 128, 32), (3, 2, 257, 2),
                                     (2, 3, 576, 3), (2, 1, 1024, 1)])
def test_write_then_read(n, H, D, P, kind, layout, grid):
    x = _vectors(n + D, n, H, D, kind, layout)
    pages = -(-n // P) + 3
    cache = ocs.ocs_cache_new(pages, P, H, D, grid)
    cache.pages.fill_(0x33)
    other = cache._replace(pages=cache.pages.clone())
    x2 = _vectors(n + D + 1, n, H, D, kind, "dense")
    order = torch.randperm(pages * P, generator=_gen(n), device="cuda")[:n]
    slots = order.clone()
    if n > 4:
        slots[2], slots[4] = -1, -(2 ** 40)
    want, want2 = host(cache.pages).copy(), host(other.pages).copy()
    st = ocs.new_status()
    ocs.ocs_cache_write(cache, x, slots, cache2=other, x2=x2, dev_status=st)
    assert ocs.ocs_poll_status(st) == 0
    _expect(want, x, slots, cache)
    _expect(want2, x2, slots, other)
    cb, sb, at_s, at_r, _ = ref.cache_sections(P, H, D, grid)
    np.testing.assert_array_equal(host(cache.pages), want)
    np.testing.assert_array_equal(host(other.pages), want2)

    # read one sequence whose pages are the cache's in another order
    pg = torch.randperm(pages, generator=_gen(D), device="cuda").to(torch.int32)
    length = pages * P - (1 if pages * P > 2 else 0)
    starts = torch.tensor([2, 2 + length], dtype=torch.int32, device="cuda")
    out = torch.full((length + 5, H, D + (layout == "part")), 9.0, device="cuda", dtype=TYPES[kind])
    out2 = torch.full((length + 5, H, D), 9.0, device="cuda", dtype=TYPES[kind])
    got, got2 = ocs.ocs_cache_read(cache, pg[None], starts, length + 5, cache2=other, out=out[:, :, :D], out2=out2, dev_status=st)
    assert ocs.ocs_poll_status(st) == 0
    at = [int(p) * P + o for p in host(pg) for o in range(P)][:length]
    written = [i for i, s in enumerate(at) if s in host(slots)]   # (the mark is no vector: its row scale is no power of two)
    for g, w in ((got, want), (got2, want2)):
        v = torch.from_numpy(_values(w, [at[i] for i in written], cache)).float().to(TYPES[kind])
        assert torch.equal(g[2:2 + length].cpu()[written], v)
        assert (g[:2] == 9).all() and (g[2 + length:] == 9).all()
    assert (out[:, :, D:] == 9).all()


@pytest.mark.parametrize("grid", GRIDS)
@pytest.mark.parametrize("lengths", [[1], [0, 5, 0, 0, 40, 1, 0], [17, 16, 15, 33], [0, 0], [3] * 70])
def test_ragged_sequences(lengths, grid):
    """Sequences without tokens, lengths around a page's end, shared pages (a common prefix)."""
    P, H, D = 16, 2, 48
    cols = max(1, max(-(-n // P) for n in lengths))
    cache = ocs.ocs_cache_new(50, P, H, D, grid)
    slots = torch.arange(50 * P, device="cuda")
    x = _vectors(5, 50 * P, H, D, "bf16")
    ocs.ocs_cache_write(cache, x, slots)
    table = torch.randint(0, 50, (len(lengths), cols + 2), generator=_gen(1), device="cuda", dtype=torch.int32)[:, :cols]
    starts = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device="cuda")
    total = sum(lengths)
    out = torch.full((total + 3, H, D), 9.0, device="cuda")
    st = ocs.new_status()
    ocs.ocs_cache_read(cache, table, starts, total + 3, out=out, dev_status=st)
    assert ocs.ocs_poll_status(st) == 0
    at = [int(host(table)[b, i // P]) * P + i % P for b, n in enumerate(lengths) for i in range(n)]
    assert torch.equal(out[:total].cpu().double(), torch.from_numpy(_values(host(cache.pages), at, cache)).float().double())
    assert (out[total:] == 9).all()


def test_bad_slots_and_pages_are_flagged():
    cache = ocs.ocs_cache_new(4, 8, 2, 32, ocs.MX4_E4M3)
    x = _vectors(1, 5, 2, 32, "f32")
    for bad in (32, 2 ** 40):
        st = ocs.new_status()
        ocs.ocs_cache_write(cache, x, torch.tensor([3, bad, -1, 31, 0], device="cuda"), dev_status=st)
        assert ocs.ocs_poll_status(st) == ocs.DEV_BAD_INDEX
    good = host(cache.pages).copy()
    starts = torch.tensor([0, 20], dtype=torch.int32, device="cuda")
    for row in ([0, 4, 3], [0, -1, 3], [0, 2 ** 31 - 1, 3]):
        st = ocs.new_status()
        out = ocs.ocs_cache_read(cache, torch.tensor([row], dtype=torch.int32, device="cuda"), starts, 20, torch.float32, dev_status=st)
        assert ocs.ocs_poll_status(st) == ocs.DEV_BAD_INDEX
        assert (out[8:16] == 0).all()
        assert torch.equal(out[:8].cpu().double(), torch.from_numpy(_values(good, list(range(8)), cache)))
    st = ocs.new_status()   # a sequence that is longer than its table's row
    out = ocs.ocs_cache_read(cache, torch.tensor([[0, 3]], dtype=torch.int32, device="cuda"), starts, 20, torch.float32, dev_status=st)
    assert ocs.ocs_poll_status(st) == ocs.DEV_BAD_INDEX and (out[16:] == 0).all()


@pytest.mark.parametrize("P", [1, 4])
def test_starts_before_the_first_row(P):
    """A negative first start leaves out a sequence's first tokens; one so low that no table has the column reads zeros."""
    cache = ocs.ocs_cache_new(12, P, 2, 24, ocs.GRID_I8)
    x = _vectors(11, 9, 2, 24, "f32")
    ocs.ocs_cache_write(cache, x, torch.arange(9, device="cuda"))
    table = torch.arange(12, dtype=torch.int32, device="cuda").view(1, 12)
    whole = ocs.ocs_cache_read(cache, table, torch.tensor([0, 9], dtype=torch.int32, device="cuda"), 9, torch.float32)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    rest = ocs.ocs_cache_read(cache, table, torch.tensor([-4, 5], dtype=torch.int32, device="cuda"), 5, torch.float32, dev_status=st)
    assert torch.equal(rest, whole[4:]) and ocs.ocs_poll_status(st) == 0
    for first in (-2 ** 31, -2 ** 31 + 3, -10 ** 9):
        low = ocs.ocs_cache_read(cache, table, torch.tensor([first, 5], dtype=torch.int32, device="cuda"), 5, torch.float32, dev_status=st)
        assert (low == 0).all() and ocs.ocs_poll_status(st) == ocs.DEV_BAD_INDEX


@pytest.mark.parametrize("grid", GRIDS)
def test_not_finite_is_flagged_and_stays_in_its_vector(grid):
    x = _vectors(1, 4, 3, 64, "f32")
    bad = x.clone()
    bad[2, 1, 5] = float("nan")
    a, b = ocs.ocs_cache_new(2, 4, 3, 64, grid), ocs.ocs_cache_new(2, 4, 3, 64, grid)
    slots = torch.arange(4, device="cuda")
    st = ocs.new_status()
    ocs.ocs_cache_write(a, x, slots), ocs.ocs_cache_write(b, bad, slots, dev_status=st)
    assert ocs.ocs_poll_status(st) == ocs.DEV_NONFINITE
    table, starts = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    va, vb = (ocs.ocs_cache_read(c, table, starts, 4, torch.float32) for c in (a, b))
    va[2, 1] = vb[2, 1] = 0
    assert torch.equal(va, vb)


def test_empty_calls_are_no_ops():
    cache = ocs.ocs_cache_new(2, 4, 3, 64)
    ocs.ocs_cache_write(cache, torch.empty((0, 3, 64), device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"))
    out = ocs.ocs_cache_read(cache, torch.zeros((0, 1), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), 0)
    assert out.shape == (0, 3, 64)


def test_pages_behind_four_gigabytes():
    """Byte offsets past 32 bits."""
    P, H, D = 64, 16, 256
    size = ocs.ocs_cache_new(0, P, H, D).pages.shape[1]
    n = 2 ** 32 // size + 20
    cache = ocs.ocs_cache_new(n, P, H, D)
    x = _vectors(1, 3, H, D, "bf16")
    last = (n - 1) * P
    ocs.ocs_cache_write(cache, x, torch.tensor([last, last + 63, last + 1], device="cuda"))
    starts = torch.tensor([0, P], dtype=torch.int32, device="cuda")
    out = ocs.ocs_cache_read(cache, torch.tensor([[n - 1]], dtype=torch.int32, device="cuda"), starts, P, torch.float32)
    want = torch.from_numpy(_values(host(cache.pages[n - 1:]), [0, 1, 63], cache)).float()
    assert torch.equal(out[[0, 1, 63]].cpu(), want) and (out[2:63] == 0).all()
    assert (want - x[[0, 2, 1]].float().cpu()).abs().max() <= 0.5 / 127 * x.float().abs().max().item() * 1.02 and not cache.pages[0].any()


def test_a_decoding_loop_captured_and_replayed():
    """Write one token per sequence, read all: captured once, replayed with new tokens, slots and lengths in the same buffers."""
    B, P, H, D, n = 3, 4, 2, 64, 10
    k, v = ocs.ocs_cache_new(B * 4, P, H, D, ocs.MX4_E4M3), ocs.ocs_cache_new(B * 4, P, H, D, ocs.MX4_E4M3)
    table = torch.arange(B * 4, device="cuda", dtype=torch.int32).view(B, 4)
    xk, xv = _vectors(1, B * n, H, D, "bf16").view(n, B, H, D), _vectors(2, B * n, H, D, "bf16").view(n, B, H, D)
    bk, bv, slots = xk[0].clone(), xv[0].clone(), torch.zeros(B, dtype=torch.int64, device="cuda")
    starts = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    ok, ov = torch.zeros((B * n, H, D), device="cuda", dtype=torch.bfloat16), torch.zeros((B * n, H, D), device="cuda", dtype=torch.bfloat16)

    def step():
        ocs.ocs_cache_write(k, bk, slots, cache2=v, x2=bv)
        ocs.ocs_cache_read(k, table, starts, B * n, cache2=v, out=ok, out2=ov)
    slots.fill_(-1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for t in range(n):
        bk.copy_(xk[t]), bv.copy_(xv[t])
        slots.copy_(table[:, t // P].long() * P + t % P)
        starts.copy_(torch.arange(B + 1, device="cuda") * (t + 1))
        g.replay()
    a, b = ocs.ocs_cache_new(B * 4, P, H, D, ocs.MX4_E4M3), None
    ocs.ocs_cache_write(a, xk.transpose(0, 1).reshape(B * n, H, D).contiguous(),
                        torch.cat([table[i].long().repeat_interleave(P)[:n] * P + torch.arange(n, device="cuda") % P for i in range(B)]))
    assert torch.equal(a.pages, k.pages)
    assert torch.equal(ocs.ocs_cache_read(a, table, starts, B * n), ok)
    assert torch.equal(ocs.ocs_cache_read(v, table, starts, B * n), ov)


def test_what_does_not_fit_the_cache_is_refused():
    c = ocs.ocs_cache_new(4, 8, 2, 32, ocs.MX4_E4M3)
    x, slots = _vectors(1, 3, 2, 32, "f32"), torch.arange(3, device="cuda")
    table, starts = torch.zeros((1, 2), dtype=torch.int32, device="cuda"), torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    for call in (lambda: ocs.ocs_cache_write(c, x[:, :1], slots), lambda: ocs.ocs_cache_write(c, x, slots[:2]),
                 lambda: ocs.ocs_cache_write(c, x, slots.int()), lambda: ocs.ocs_cache_write(c._replace(dim=48), x, slots),
                 lambda: ocs.ocs_cache_write(c, x.double(), slots), lambda: ocs.ocs_cache_write(c, x, slots, cache2=c._replace(grid=ocs.MX4_E8M0), x2=x),
                 lambda: ocs.ocs_cache_write(c, x, slots, x2=x), lambda: ocs.ocs_cache_write(c, x.transpose(1, 2), slots),
                 lambda: ocs.ocs_cache_read(c, table.long(), starts, 3), lambda: ocs.ocs_cache_read(c, table, starts[:1], 3),
                 lambda: ocs.ocs_cache_read(c, table, starts, 3, out=x[:2]), lambda: ocs.ocs_cache_read(c, table, starts, 3, out2=x),
                 lambda: ocs.ocs_cache_read(c, table, starts, 3, cache2=c, out2=x.half()), lambda: ocs.ocs_cache_read(c, table, starts.cpu(), 3)):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(ocs.OcsError):
        ocs.ocs_cache_new(1, 8, 2, 2000)
    with pytest.raises(ocs.OcsError):
        ocs.ocs_cache_write(c, x, slots, cache2=c, x2=x)          # the same cache twice
