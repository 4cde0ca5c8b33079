"""Block tables and slot maps built on the GPU (kv_tables_grow, include/kvr_tables.h)
against a plain loop over the requests: integer results, equal in every element,
including the ones a call must leave alone."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_14635_amd import kvr  # noqa: E402

KEPT = -77  # what table entries hold that a call must not write


def loop(held, lens, B, free, tables, max_rows):
    """The definition, request by request."""
    tables, wide = tables.copy(), tables.shape[1]
    slots, positions, offsets, used, unplaced = [], [], [0], 0, 0
    for r, (h, n) in enumerate(zip(held, lens)):
        h = max(int(h), 0)
        for j in range(-(-h // B), min(-(-int(n) // B), wide)):
            tables[r, j] = free[used] if used < len(free) else -1
            used += 1
        for p in range(h, int(n)):
            b = tables[r, p // B] if p // B < wide else -1
            slots.append(int(b) * B + p % B if b >= 0 else -1)
            positions.append(p)
            unplaced += b < 0
        offsets.append(len(slots))
    total = len(slots)
    pad = [-1] * max(0, max_rows - total)
    counts = [min(used, len(free)), max(used - len(free), 0), total, unplaced]
    return (tables, np.array(offsets), np.array(slots + pad, np.int64)[:max_rows],
            np.array(positions + pad)[:max_rows], np.array(counts))


class Call:
    """The device arrays of one request set, with guard entries behind each output."""

    def __init__(self, held, lens, B, free, tables, max_rows):
        dev = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
        self.R, self.B, self.max_rows, self.nfree = len(lens), B, max_rows, len(free)
        self.held = None if held is None else dev(held)
        self.lens, self.free, self.tables = dev(lens), dev(free), dev(tables)
        self.offsets = torch.full((self.R + 1 + 4,), KEPT, dtype=torch.int32, device="cuda")
        self.slots = torch.full((max_rows + 4,), KEPT, dtype=torch.int64, device="cuda")
        self.positions = torch.full((max_rows + 4,), KEPT, dtype=torch.int32, device="cuda")
        self.counts = torch.full((8,), KEPT, dtype=torch.int32, device="cuda")

    def run(self, with_positions=True):
        kvr.kv_tables_grow(self.held.data_ptr() if self.held is not None else 0, self.lens.data_ptr(), self.R,
                           self.B, self.free.data_ptr(), self.nfree, self.tables.data_ptr(), self.tables.shape[1],
                           self.max_rows, self.offsets.data_ptr(), self.slots.data_ptr(),
                           self.positions.data_ptr() if with_positions else 0, self.counts.data_ptr(),
                           stream=torch.cuda.current_stream().cuda_stream)

    def check(self, want, with_positions=True):
        tables, offsets, slots, positions, counts = want
        n = self.max_rows
        assert np.array_equal(self.counts.cpu().numpy()[:4], counts)
        assert np.array_equal(self.offsets.cpu().numpy()[:self.R + 1], offsets)
        assert np.array_equal(self.tables.cpu().numpy(), tables)
        assert np.array_equal(self.slots.cpu().numpy()[:n], slots)
        got = self.positions.cpu().numpy()
        assert np.array_equal(got[:n], positions) if with_positions else (got == KEPT).all()
        for t, end in ((self.offsets, self.R + 1), (self.slots, n), (self.positions, n), (self.counts, 4)):
            assert (t[end:] == KEPT).all()


def request_set(R, low, high, grow, B, seed, wide_extra=1):
    rng = np.random.default_rng(seed)
    lens = rng.integers(low, high + 1, size=R).astype(np.int32)
    held = np.maximum(0, lens - rng.integers(0, grow + 1, size=R)).astype(np.int32) if grow else np.zeros(R, np.int32)
    wide = max(1, -(-int(lens.max(initial=0)) // B)) + wide_extra
    ids = rng.permutation(R * wide + 7).astype(np.int32)
    tables = np.full((R, wide), KEPT, np.int32)
    o = 0
    for r in range(R):
        k = -(-int(held[r]) // B)
        tables[r, :k] = ids[o:o + k]
        o += k
    return held, lens, ids[o:], tables


# one request of one position; the scan's step of 512 requests and the window of
# 2048 rows from both sides; requests without new positions; blocks of one slot
# and of odd sizes; more requests than one window's rows
CASES = {
    "one": (1, 1, 1, 0, 16), "one_long": (1, 5000, 5000, 0, 16), "step_64": (64, 200, 900, 1, 16),
    "ragged_511": (511, 0, 40, 0, 16), "ragged_512": (512, 0, 40, 9, 8), "ragged_513": (513, 0, 40, 9, 24),
    "rows_2048": (128, 16, 16, 0, 16), "odd_block": (37, 0, 333, 50, 7), "block_one": (9, 0, 30, 4, 1),
    "wide_block": (50, 0, 300, 20, 1000), "none_new": (20, 5, 5, 0, 16), "many_requests": (5000, 0, 3, 2, 16),
    "many_long": (700, 0, 500, 0, 32),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(CASES))
def test_tables_grow(name):
    R, low, high, grow, B = CASES[name]
    held, lens, free, tables = request_set(R, low, high, grow, B, seed=len(name))
    if name == "none_new":
        held = lens.copy()
        tables[:, 0] = np.arange(R)
    total = int((lens - held).sum())
    # exactly the rows, some behind them, fewer than there are
    for max_rows, free_n in ((total, len(free)), (total + 2500, len(free)), (max(0, total // 2 - 3), len(free)),
                             (total, total // B // 3), (total + 1, 0)):
        c = Call(held, lens, B, free[:free_n], tables, max_rows)
        want = loop(held, lens, B, free[:free_n], tables, max_rows)
        c.run()
        c.run()  # the same call again
        c.check(want)


@pytest.mark.gpu
def test_tables_grow_of_full_and_broken_tables():
    """Tables narrower than the lengths, an old last block that is none, requests
    that shrink, a negative held, no held array, no positions array."""
    B = 16
    held = np.array([0, 20, 33, 50, -5, 40, 16], np.int32)
    lens = np.array([100, 45, 90, 40, 10, 41, 17], np.int32)
    free = np.arange(100, 140, dtype=np.int32)
    tables = np.full((7, 4), KEPT, np.int32)
    tables[1, :2], tables[2, :3], tables[3, :4], tables[5, :3], tables[6, :1] = [3, 4], [5, 6, -1], 7, [8, 9, 10], 11
    c = Call(held, lens, B, free, tables, 200)
    c.run()
    c.check(loop(held, lens, B, free, tables, 200))
    narrow = np.full((7, 2), KEPT, np.int32)
    c = Call(None, lens, B, free, narrow, 300)
    c.run(with_positions=False)
    c.check(loop(np.zeros(7, np.int32), lens, B, free, narrow, 300), with_positions=False)
    # held beyond the table's width: rows there have no slot, nothing is taken
    held = np.array([70, 64], np.int32)
    lens = np.array([75, 66], np.int32)
    c = Call(held, lens, B, free, tables[:2], 9)
    c.run()
    c.check(loop(held, lens, B, free, tables[:2], 9))


@pytest.mark.gpu
def test_tables_grow_of_no_requests_and_no_rows():
    c = Call([], [], 16, np.zeros(0, np.int32), np.zeros((0, 3), np.int32), 10)
    c.run()
    c.check(loop([], [], 16, [], np.zeros((0, 3), np.int32), 10))
    held, lens, free, tables = request_set(3, 5, 50, 0, 16, 1)
    c = Call(held, lens, 16, free, tables, 0)
    c.run()
    c.check(loop(held, lens, 16, free, tables, 0))


@pytest.mark.gpu
def test_tables_grow_in_a_graph_follows_the_lengths():
    """A captured call replayed over changing lengths, on a stream of its own."""
    B, R = 16, 40
    held, lens, free, tables = request_set(R, 3, 200, 5, B, 21, wide_extra=4)
    c = Call(held, lens, B, free, tables, 300)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c.run()
    rng = np.random.default_rng(3)
    for _ in range(4):
        tables = c.tables.cpu().numpy()
        lens = (held + rng.integers(0, 7, size=R)).astype(np.int32)
        c.lens.copy_(torch.tensor(lens))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        c.check(loop(held, lens, B, free, tables, 300))


def call_with(**kw):
    a = dict(held=0x1000, lens=0x2000, num_requests=4, block_size=16, free_blocks=0x3000, num_free=9, tables=0x4000,
             max_blocks=5, max_rows=64, row_offsets=0x5000, slots=0x6000, positions=0x7000, counts=0x8000)
    a.update(kw)
    kvr.kv_tables_grow(**a)


@pytest.mark.parametrize("bad", [
    dict(num_requests=-1), dict(num_requests=(1 << 30) + 1), dict(num_free=-1), dict(max_blocks=-1), dict(max_rows=-1), dict(max_rows=1 << 31),
    dict(block_size=0), dict(lens=0), dict(tables=0), dict(free_blocks=0), dict(slots=0), dict(row_offsets=0),
    dict(counts=0), dict(lens=0x2002), dict(slots=0x6004), dict(tables=0x4001)])
def test_tables_grow_refusals(bad):
    with pytest.raises(kvr.KvError) as e:
        call_with(**bad)
    assert e.value.status == kvr.KV_EINVAL and e.value.message


def test_tables_grow_on_a_device_that_is_not_there():
    with pytest.raises(kvr.KvError) as e:
        call_with(device=4096)
    assert e.value.status == kvr.KV_EDEVICE and e.value.message
