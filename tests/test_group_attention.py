"""Attention over the arena with shared prefixes (kv_group_attention,
include/kvr_attention.h) against softmax(q k^T / sqrt(d)) v in 64 bits.  Slots outside the
contexts hold NaN.

Tolerance, per output element, with u = 2^-24 and A the largest sum_e |q_e k_je| /
sqrt(d) of the row's positions:
  a score is a fp32 sum of d products and a scaling, |ds| <= (d + 8) u A;
  weights then differ by 2 |ds| relative, the exponential and its argument's
  rounding (the argument is at most 1.5 * 2 A) add (8 + 4 A) u;
  sums over n positions add 2 (n + 16) u;
  in bf16 models weights enter the product with V as two bf16 numbers (2^-17 relative), and
  their exponents lie 32 to 72 below zero, where half a step is 2^-18 at most (2^-18
  relative, in the product and in the sum of weights): 2^-16 in all;
all times max |v|, plus half a step of the output type and its least number."""
import dataclasses

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_14635_amd import harness as Hn  # noqa: E402
from paper_2608_14635_amd import kvr  # noqa: E402
from paper_2608_14635_amd import workloads as W  # noqa: E402

U = 2.0 ** -24
KEPT = 7.0


def heads(name, g=4, nkv=2):
    if name == "bf16":
        return dataclasses.replace(W.TINY_BF16, num_layers=2, num_q_heads=g * nkv, num_kv_heads=nkv)
    d = int(name[4:])
    nkv = max(nkv, 128 // d)
    return dataclasses.replace(W.TINY_F32, num_layers=2, num_q_heads=g * nkv, num_kv_heads=nkv, head_dim=d)


def torch_dtype(shape):
    return torch.bfloat16 if shape.dtype == W.BF16 else torch.float32


def to64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Batch:
    """Requests of lens[r] positions and counts[r] query rows over an arena of NaN; sizes[g] of
    them in group g (what is left over in none), prefix[g] positions shared."""

    def __init__(self, shape, lens, counts=None, sizes=(), prefix=(), before=0, B=16, seed=0, layer=1, extra_rows=0,
                 std=1.3, copies=True):
        self.shape, self.lens, self.B, self.layer = shape, np.array(lens, np.int64), B, layer
        self.counts = np.ones(len(lens), int) if counts is None else np.array(counts)
        self.plain = counts is None and not extra_rows  # one row a request: no offsets
        self.group_off = before + np.concatenate([[0], np.cumsum(sizes)]).astype(int)
        self.prefix = np.array(prefix, int)
        rng = np.random.default_rng(seed)
        need = -(-np.maximum(self.lens, 0) // B)
        self.blocks = int(need.sum()) + 3
        ids = list(rng.permutation(self.blocks))
        self.tables = np.full((len(lens), int(need.max(initial=0)) + 1), -1, np.int32)
        same = []
        group = {r: g for g in range(len(sizes)) for r in range(self.group_off[g], self.group_off[g + 1])}
        for r, k in enumerate(need):
            first = self.group_off[group[r]] if r in group else r
            shared = min(self.prefix[group[r]], self.lens[r], self.lens[first]) if first != r else 0
            whole = shared // B
            self.tables[r, :whole] = self.tables[first, :whole]
            for b in range(whole, k):
                self.tables[r, b] = ids.pop()
            # the prefix's last block: a copy of its own
            same += [(self.slot(first, j), self.slot(r, j)) for j in range(whole * B, shared)]
        self.slots = [np.array([self.slot(r, j) for j in range(n)], np.int64) for r, n in enumerate(self.lens)]
        dt = torch_dtype(shape)
        nkv, d = shape.num_kv_heads, shape.head_dim
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        lead = 4 // (2 if dt == torch.bfloat16 else 4)
        n = 2 * 2 * self.blocks * B * nkv * d
        self.raw = torch.full((n + lead,), float("nan"), dtype=dt, device="cuda")
        self.arena = self.raw[lead:].view(2, 2, self.blocks * B, nkv, d)
        flat = np.unique(np.concatenate(self.slots)) if len(lens) else np.zeros(0, np.int64)
        if len(flat):
            self.arena[layer][:, torch.tensor(flat)] = torch.randn(2, len(flat), nkv, d, generator=g,
                                                                   device="cuda").mul_(std).to(dt)
        if copies and same:
            src, dst = torch.tensor(same, device="cuda").unbind(1)
            self.arena[layer][:, dst] = self.arena[layer][:, src]
        self.handle = kvr.kv_arena_bind(self.arena.data_ptr(), n * self.arena.element_size(), shape, B, self.blocks)
        self.rows = int(self.counts.sum()) + extra_rows
        self.off = np.concatenate([[0], np.cumsum(self.counts)])
        # query rows wider than their heads, 4 bytes past a 16-byte boundary
        w = shape.num_q_heads * d
        flat_q = torch.randn(self.rows * (w + 2 * lead) + lead, generator=g, device="cuda").mul_(std).to(dt)
        self.q = flat_q[lead:].view(self.rows, w + 2 * lead)[:, :w]
        self.out = torch.full((self.rows, w + 4), KEPT, dtype=dt, device="cuda")
        self.bind()

    def slot(self, r, j):
        return int(self.tables[r, j // self.B]) * self.B + j % self.B

    def bind(self, max_query=None, max_len=None):
        dev = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
        self.d_lens, self.d_tables, self.d_off = dev(self.lens), dev(self.tables), dev(self.off)
        self.d_groups, self.d_prefix = dev(self.group_off), dev(self.prefix)
        self.max_query = max_query or max(1, int(self.counts.max(initial=1)))
        self.max_len = max_len or max(1, int(self.lens.max(initial=1)))
        self.ws_bytes = kvr.kv_group_attention_workspace_bytes(self.shape, max(1, len(self.lens)), max(1, self.rows),
                                                               len(self.prefix), self.max_query, self.max_len)
        assert self.ws_bytes > 0
        # every byte 255: whatever is read without having been written is NaN
        self.ws = torch.full((self.ws_bytes + 64,), 255, dtype=torch.uint8, device="cuda")

    def run(self, ws=None, stream=None, groups=True):
        kvr.kv_group_attention(self.handle, self.layer, self.q.data_ptr(), self.q.stride(0),
                               0 if self.plain else self.d_off.data_ptr(), self.rows, self.d_lens.data_ptr(),
                               self.d_tables.data_ptr(), len(self.lens), self.tables.shape[1], self.d_groups.data_ptr(),
                               self.d_prefix.data_ptr(), len(self.prefix) if groups else 0, self.max_query, self.max_len,
                               self.out.data_ptr(), self.out.stride(0), (self.ws if ws is None else ws).data_ptr(),
                               self.ws_bytes, Hn.stream_ptr() if stream is None else stream)

    def reference(self):
        """out and its tolerance, [rows, nq, d], 64 bits; a prefix through its first request's table."""
        s, B = self.shape, self.B
        nq, nkv, d = s.num_q_heads, s.num_kv_heads, s.head_dim
        plane = to64(self.arena[self.layer])
        q = to64(self.q).reshape(self.rows, nq, d)
        out, tol = np.zeros((self.rows, nq, d)), np.zeros((self.rows, nq, d))
        split = 2.0 ** -16 if s.dtype == W.BF16 else 0.0
        half = torch.finfo(torch_dtype(s)).eps / 2
        for r, n in enumerate(self.lens):
            m = self.counts[r]
            tables = np.repeat(self.tables[r:r + 1], 1, 0)[0]
            j = np.arange(max(0, min(n, self.tables.shape[1] * B, self.max_len)))
            blk = tables[j // B].astype(np.int64)
            for g in range(len(self.prefix)):
                if self.group_off[g] <= r < self.group_off[g + 1]:
                    first = self.tables[self.group_off[g]][j // B].astype(np.int64)
                    blk = np.where(j < self.prefix[g], first, blk)
            there = (blk >= 0) & (blk < self.blocks)
            slots = (blk * B + j % B)[there]
            k, v = plane[0, slots], plane[1, slots]
            for i in range(min(m, self.max_query)):
                row = self.off[r] + i
                seen = j[there] <= n - m + i
                if not seen.any():
                    continue
                for h in range(nq):
                    kk, vv = k[seen, h // (nq // nkv)], v[seen, h // (nq // nkv)]
                    with np.errstate(all="ignore"):
                        x = kk @ q[row, h] / np.sqrt(d)
                        p = np.exp(x - x.max())
                        # p 0 times NaN is NaN: every position that is seen counts
                        out[row, h] = (p[:, None] * vv).sum(0) / p.sum()
                        a = (np.abs(kk) @ np.abs(q[row, h])).max() / np.sqrt(d)
                        rel = (2 * (d + 8) * a + 8 + 4 * a + 2 * (len(x) + 16)) * U + split
                        tol[row, h] = rel * np.abs(vv).max() + half * np.abs(out[row, h]) + 1e-37
        return out, tol

    def check(self):
        want, tol = self.reference()
        w = want.shape[1] * want.shape[2]
        got = to64(self.out)
        assert (got[:, w:] == KEPT).all()
        used = int(self.counts.sum())
        assert (got[used:] == KEPT).all()
        assert bool((self.ws[self.ws_bytes:] == 255).all())
        got, want, tol = got[:used, :w], want.reshape(len(want), w)[:used], tol.reshape(len(tol), w)[:used]
        nan = ~np.isfinite(want)
        assert np.array_equal(~np.isfinite(got), nan)
        with np.errstate(invalid="ignore"):
            bad = np.abs(got - want)[~nan] > tol[~nan]
        assert not bad.any(), (int(bad.sum()), float(np.abs(got - want)[~nan].max()), float(tol[~nan].min()))

    def release(self):
        kvr.kv_arena_release(self.handle)


def run_and_check(b, once=False):
    """As it is and, unless `once`, with bounds that no short call has."""
    b.run()
    torch.cuda.synchronize()
    b.check()
    if not once:
        wider = max(0, -(-1200 // b.B) - b.tables.shape[1])
        b.tables = np.pad(b.tables, ((0, 0), (0, wider)), constant_values=-1)
        b.bind(b.max_query, max(b.max_len, 1100))
        b.out.fill_(KEPT)
        b.run()
        torch.cuda.synchronize()
        b.check()
    b.release()


RAGGED = [1, 15, 16, 17, 31, 32, 33, 0, 64, 100, 257]
TYPES = [("bf16", 1), ("bf16", 4), ("bf16", 5), ("bf16", 16), ("f32_32", 3), ("f32_64", 1), ("f32_64", 8),
         ("f32_128", 4), ("f32_128", 16)]


@pytest.mark.gpu
@pytest.mark.parametrize("name,g", TYPES)
@pytest.mark.parametrize("B", [16, 24, 1])
def test_without_groups(name, g, B):
    run_and_check(Batch(heads(name, g), RAGGED, B=B, seed=g))


@pytest.mark.gpu
@pytest.mark.parametrize("name,g", TYPES)
@pytest.mark.parametrize("B", [16, 8, 48])
def test_groups(name, g, B):
    """Prefixes that end in and between blocks and tiles; groups of one request, of none; requests
    that end in the prefix, before it and with it; requests in no group."""
    lens = [50, 70, 41, 300, 33, 64, 40, 20, 65, 90, 1, 129, 7, 200]
    run_and_check(Batch(heads(name, g), lens, sizes=[3, 1, 0, 4, 3], prefix=[37, 30, 9, 40, 64], before=1, B=B, seed=g))


@pytest.mark.gpu
@pytest.mark.parametrize("name,g", [("bf16", 1), ("bf16", 5), ("bf16", 16), ("f32_32", 8), ("f32_64", 3), ("f32_128", 4)])
def test_several_rows_a_request(name, g):
    """Row counts that fill a matrix tile's columns, cross it, and take several; a
    request without rows, one with more rows than positions, rows behind the last; rows
    that begin before the prefix's end."""
    lens = [1, 40, 17, 300, 0, 64, 5, 33, 150, 151]
    counts = [1, 4, 0, 2, 9, 64, 8, 3, 5, 1]
    b = Batch(heads(name, g), lens, counts, sizes=[2, 5, 2], prefix=[20, 30, 148], before=1, B=32, seed=g, extra_rows=3)
    run_and_check(b)


@pytest.mark.gpu
@pytest.mark.parametrize("name,g,size,prefix", [("bf16", 4, 4, 500), ("bf16", 4, 8, 777), ("bf16", 4, 33, 1030), ("bf16", 8, 40, 4000),
                                                ("f32_64", 4, 17, 600), ("f32_128", 2, 20, 333)])
def test_long_prefixes(name, g, size, prefix):
    """One, two, four and more column tiles; a tail of one position in every third request."""
    lens = [prefix + (1 if i % 3 == 0 else 5 + 41 * i % 150) for i in range(size)]
    run_and_check(Batch(heads(name, g), lens, sizes=[size], prefix=[prefix], seed=size))


@pytest.mark.gpu
@pytest.mark.parametrize("name,lens,sizes,prefix", [
    ("bf16", [70001], [], []), ("bf16", [9000, 1, 4097, 20000, 21000], [2], [1]),
    ("f32_64", [5000, 3], [], []), ("bf16", [1 + (37 * i) % 90 for i in range(1100)], [2] * 550, [1] * 550),
    ("f32_32", [30 + (5 * i) % 40 for i in range(300)], [30] * 10, [11 * i for i in range(10)]),
    ("bf16", [40 + (7 * i) % 60 for i in range(600)], [600], [39])])
def test_long_and_many(name, lens, sizes, prefix):
    run_and_check(Batch(heads(name, 4), lens, sizes=sizes, prefix=prefix, seed=len(lens)))


@pytest.mark.gpu
@pytest.mark.parametrize("name,g", [("bf16", 4), ("bf16", 3), ("f32_32", 4), ("f32_64", 2), ("f32_128", 4)])
def test_a_prompts_piece(name, g):
    """Many query rows of several requests: several column tiles each, causal inside."""
    run_and_check(Batch(heads(name, g), [500, 222, 260], [150, 222, 60], sizes=[3], prefix=[200], seed=2))


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["bf16", "f32_64"])
def test_a_whole_prompt(name):
    """A thousand query rows over as many positions and more, and one row beside them."""
    run_and_check(Batch(heads(name, 1), [1300, 900], [1000, 1], sizes=[2], prefix=[250], seed=3))


@pytest.mark.gpu
@pytest.mark.parametrize("long", [False, True])
@pytest.mark.parametrize("name", ["bf16", "f32_64"])
def test_blocks_that_are_not_there(name, long):
    """Table entries outside the arena, tables narrower than the lengths, a request
    of which nothing is left, lengths above max_len and below zero, prefixes of any number."""
    b = Batch(heads(name, 4), [100, 64, 33, 1400 if long else 200, 50, 10, 90, 80], [1, 3, 2, 1, 1, 2, 1, 2], sizes=[2, 3, 1, 2],
              prefix=[30, 33, 5, 60], B=16, seed=5)
    b.tables[0, [0, 3]] = -1
    b.tables[1, 2] = b.blocks
    b.tables[2, :3] = [-5, 1 << 30, -(1 << 31)]
    b.tables = np.ascontiguousarray(b.tables[:, :80 if long else 9])  # request 3 has 88 or 13 blocks
    b.lens[5] = -3
    b.prefix[2], b.prefix[3] = -7, 2 ** 31 - 1
    b.bind(max_len=1200 if long else 64)
    run_and_check(b, once=True)


@pytest.mark.gpu
@pytest.mark.parametrize("name,counts", [("bf16", None), ("bf16", [3, 5, 2]), ("f32_64", [3, 5, 2]), ("f32_128", None)])
def test_values_that_are_not_finite(name, counts):
    """A NaN or infinity in K or V reaches exactly the rows that see its position, and in V its
    dim alone; infinite queries give NaN rows."""
    b = Batch(heads(name, 4), [50, 70, 40], counts, seed=6)
    a = b.arena[b.layer]
    # the last two of request 1 and one of 2: masked for earlier query rows
    for r, j, which, x in ((0, 20, 1, float("nan")), (1, 69, 1, float("inf")), (1, 67, 0, float("nan")),
                           (2, 39, 1, float("-inf")), (2, 38, 1, float("nan"))):
        a[which, int(b.slots[r][j]), :, 5 + j % 2] = x
    b.q[0, 3] = float("inf")
    run_and_check(b)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["bf16", "f32_64"])
def test_what_a_row_does_not_see_in_a_prefix(name):
    """Rows before the prefix's end, values behind them that are not finite."""
    b = Batch(heads(name, 4), [30, 36, 60, 33], [2, 3, 1, 4], sizes=[4], prefix=[40], seed=7)
    for j in (34, 35, 39):
        b.arena[b.layer][1, int(b.slots[2][j]), :, j] = float("nan")
        b.arena[b.layer][0, int(b.slots[2][j]), :, 3] = float("inf")
    b.tables[0] = b.tables[2]  # the group's first table
    b.bind()
    run_and_check(b)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["bf16", "f32_64"])
def test_scores_of_any_size(name):
    """Scores in the thousands, equal scores, and queries of zero."""
    b = Batch(heads(name, 4), [300, 129, 64, 200], sizes=[4], prefix=[60], seed=7, std=30.0)
    b.q[1] = 0
    run_and_check(b)


@pytest.mark.gpu
@pytest.mark.parametrize("name,counts", [("bf16", None), ("bf16", [9, 5, 1, 12]), ("f32_32", None), ("f32_64", [9, 5, 1, 12]),
                                         ("f32_128", None)])
@pytest.mark.parametrize("high,value", [(20, 0), (28, 0), (33, 0), (34, 0), (34, 127), (34, -60), (35, 0), (36, 0), (60, 0),
                                        (120, 0)])
def test_large_scores(name, counts, high, value):
    """Scores of about 2^high and values of about 2^value.  Queries and keys have two dims that are
    not zero, whose products and sum are fp32 numbers: a score is exact.  Many positions of each
    sixth share their large product, and differ by what the other adds, few by 2^(high - 20).
    An exponent's argument, at most 150 where its weight does not vanish, has the roundings of
    the scale and of two products."""
    b = Batch(heads(name, 5), [500, 300, 250, 30], counts, sizes=[3], prefix=[200], seed=high)
    dt, shape = torch_dtype(b.shape), b.shape
    g = torch.Generator(device="cuda")
    g.manual_seed(high)
    of = lambda n, *size: torch.randint(0, n, size, generator=g, device="cuda")  # noqa: E731
    q = torch.zeros(b.rows, shape.num_q_heads, shape.head_dim, device="cuda")
    q[..., 7] = (1 + of(128, b.rows, shape.num_q_heads) / 128.0) * 2.0 ** (high // 2)
    q[1::2, :, 7] *= -1
    q[..., 9] = 1
    b.q.copy_(q.flatten(1))
    keys, values = b.arena[b.layer]
    new = torch.zeros_like(keys, dtype=torch.float32)
    steps = torch.tensor([-1.0, -0.75, -127 / 128, 127 / 128, 0.25, 1.0], device="cuda")
    new[..., 7] = steps[of(6, len(keys), 1)] * 2.0 ** (high - high // 2)
    new[..., 9] = of(4, len(keys), 1) * 2.0 ** (high - 20)
    keys.copy_(torch.where(keys.isnan(), torch.nan, new.to(dt)))
    values.mul_(2.0 ** (value - 4 if value > 0 else value))  # of std 1.3, none above 2^4
    for copy in (1, 2):  # the prefix's last block is each request's own copy
        for plane in (keys, values):
            plane[torch.tensor(b.slots[copy][192:200])] = plane[torch.tensor(b.slots[0][192:200])]
    q, keys, values = to64(b.q).reshape(q.shape), to64(keys), to64(values)
    each, half = shape.num_q_heads // shape.num_kv_heads, torch.finfo(dt).eps / 2
    for wide in (0, 100):  # in a short call, and by its bounds in another
        b.tables = np.pad(b.tables, ((0, 0), (0, wide)), constant_values=-1)
        b.bind(b.max_query, max(b.max_len, 12 * wide))
        b.out.fill_(KEPT)
        b.run()
        torch.cuda.synchronize()
        got = to64(b.out[:, :b.q.shape[1]]).reshape(q.shape)
        for r, n in enumerate(b.lens):
            for i in range(b.counts[r]):
                seen, row = b.slots[r][:n - b.counts[r] + i + 1], b.off[r] + i
                for h in range(shape.num_q_heads):
                    x, v = keys[seen, h // each] @ q[row, h], values[seen, h // each]
                    p = np.exp((x - x.max()) / np.sqrt(shape.head_dim))
                    want = (p[:, None] * v).sum(0) / p.sum()
                    rel = (8 + 4 * 150 + 2 * (len(x) + 16)) * U + (2.0 ** -16 if dt == torch.bfloat16 else 0.0)
                    off = rel * np.abs(v).max() + half * np.abs(want) + 1e-37
                    assert (np.abs(got[row, h] - want) <= off).all(), (wide, r, i, h, got[row, h, :3], want[:3])
    b.release()


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["bf16", "f32_64"])
def test_values_next_to_the_largest(name):
    """Sums of values next to the largest number stay finite, in a prefix and behind it."""
    b = Batch(heads(name, 4), [1000, 700, 650], sizes=[3], prefix=[600], seed=8)
    top = torch.finfo(torch_dtype(b.shape)).max
    b.arena[b.layer][1] = torch.where(b.arena[b.layer][1] > 0, top, top / 2)
    b.q.mul_(0.01)
    run_and_check(b)


@pytest.mark.gpu
@pytest.mark.parametrize("name,g", [("bf16", 2), ("bf16", 5), ("f32_64", 16)])
@pytest.mark.parametrize("wide", [0, 100])
def test_more_rows_than_max_query(name, g, wide):
    """Rows past max_query are left out; those before them keep their positions."""
    counts = [5, 9, 2, 7]
    b = Batch(heads(name, g), [40, 9, 70, 44], counts, sizes=[4], prefix=[8], seed=12)
    b.tables = np.pad(b.tables, ((0, 0), (0, wide)), constant_values=-1)
    b.bind(max_query=4, max_len=1100 if wide else None)
    b.run()
    torch.cuda.synchronize()
    want, tol = b.reference()
    got = to64(b.out[:, :b.q.shape[1]]).reshape(want.shape)
    for r, m in enumerate(counts):
        rows = slice(b.off[r], b.off[r] + min(m, 4))
        assert (np.abs(got[rows] - want[rows]) <= tol[rows]).all(), r
        assert (got[rows.stop:b.off[r] + m] == KEPT).all(), r
    b.release()


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["bf16", "f32_64"])
@pytest.mark.parametrize("wide", [0, 100])
def test_the_prefix_is_the_first_requests(name, wide):
    """What other requests' tables say of shared positions is not read, in a short call and, by its
    bounds (`wide` entries more in the tables), another."""
    b = Batch(heads(name, 4), [100, 90, 80], sizes=[3], prefix=[64], seed=13)
    b.tables = np.pad(b.tables, ((0, 0), (0, wide)), constant_values=-1)
    b.bind(max_len=1100 if wide else None)
    b.run()
    want = b.out.clone()
    b.tables[1:, :4] = -1
    b.bind(max_len=1100 if wide else None)
    b.out.fill_(KEPT)
    b.run()
    torch.cuda.synchronize()
    assert torch.equal(b.out, want)
    b.release()


@pytest.mark.gpu
def test_groups_that_share_nothing_change_nothing():
    """The same call with and without groups, by its tolerance; without groups by the bits of
    groups of one request."""
    lens = [100, 500, 33, 64]
    a = Batch(heads("bf16", 4), lens, sizes=[4], prefix=[0], seed=14)
    a.run(groups=False)
    torch.cuda.synchronize()
    a.check()
    a.out.fill_(KEPT)
    run_and_check(a)


@pytest.mark.gpu
@pytest.mark.parametrize("name,g,counts,same", [("bf16", 4, None, True), ("bf16", 16, None, True), ("f32_64", 3, None, True),
                                                ("f32_128", 8, None, True), ("bf16", 5, [4, 4, 4, 4], True),
                                                ("bf16", 5, [9, 1, 1, 1], False), ("f32_64", 5, [9, 1, 1, 1], False)])
@pytest.mark.parametrize("long", [False, True])
def test_groups_of_one_request_share_nothing(name, g, counts, same, long):
    """Whatever their prefixes: by the bits of the call without groups where an item has as many
    columns in both, by its tolerance elsewhere."""
    lens = [100, 2500 if long else 500, 33, 64]
    b = Batch(heads(name, g), lens, counts, sizes=[1] * 4, prefix=[50, 300, 33, 1000], seed=15)
    b.run(groups=False)
    torch.cuda.synchronize()
    b.check()
    want = b.out.clone()
    b.out.fill_(KEPT)
    b.run()
    torch.cuda.synchronize()
    b.check()
    assert not same or torch.equal(b.out, want)
    b.release()


@pytest.mark.gpu
@pytest.mark.parametrize("each,B", [(9, 16), (40, 24)])
def test_a_long_prefix_of_many_heads(each, B):
    """Heads so many that a workgroup's stretch of the prefix is longer than the positions it looks
    up at once (2048), column tiles of 18 and 80 columns; in 64 bits on the device."""
    g, nkv, d, P = 2, 64, 128, 19001
    shape = dataclasses.replace(W.TINY_BF16, num_layers=1, num_q_heads=g * nkv, num_kv_heads=nkv)
    lens = [P + 1 + 3 * r for r in range(each)]
    blocks = -(-P // B) + each * (-(-lens[-1] // B) - P // B) + 1
    gen = torch.Generator(device="cuda")
    gen.manual_seed(each)
    arena = torch.randn(2, blocks * B, nkv, d, generator=gen, device="cuda", dtype=torch.bfloat16)
    h = kvr.kv_arena_bind(arena.data_ptr(), arena.numel() * 2, shape, B, blocks)
    tables = np.full((each, -(-lens[-1] // B)), -1, np.int32)
    ids = iter(np.random.default_rng(each).permutation(blocks))
    tables[:, :P // B] = [next(ids) for _ in range(P // B)]
    for r, n in enumerate(lens):
        for b in range(P // B, -(-n // B)):
            tables[r, b] = next(ids)
    dev = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
    q = torch.randn(each, g * nkv * d, generator=gen, device="cuda", dtype=torch.bfloat16)
    out = torch.full_like(q, KEPT)
    n = kvr.kv_group_attention_workspace_bytes(shape, each, each, 1, 1, lens[-1])
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    args = dev(lens), dev(tables), dev([0, each]), dev([P])
    kvr.kv_group_attention(h, 0, q.data_ptr(), q.stride(0), 0, each, args[0].data_ptr(), args[1].data_ptr(), each,
                           tables.shape[1], args[2].data_ptr(), args[3].data_ptr(), 1, 1, lens[-1], out.data_ptr(),
                           out.stride(0), ws.data_ptr(), n, Hn.stream_ptr())
    torch.cuda.synchronize()
    for r in (0, 7, each - 1):
        j = np.arange(lens[r])
        at = np.where(j < P, tables[0, j // B], tables[r, j // B]).astype(np.int64) * B + j % B
        at = torch.tensor(at, device="cuda")
        for head in range(0, nkv, 9):
            k, v = (arena[c, at, head].double() for c in (0, 1))
            x = q[r].view(g * nkv, d)[head * g:(head + 1) * g].double()
            score = x @ k.t().contiguous() / d ** 0.5
            want = torch.softmax(score, 1) @ v
            A = float((x.abs() @ k.abs().t().contiguous()).max()) / d ** 0.5
            off = ((2 * (d + 8) * A + 8 + 6 * A + 2 * (lens[r] + 16)) * U + 2.0 ** -16) * float(v.abs().max())
            got = out[r].view(g * nkv, d)[head * g:(head + 1) * g].double()
            assert ((got - want).abs() <= off + 2.0 ** -8 * want.abs() + 1e-37).all(), (r, head)
    kvr.kv_arena_release(h)


@pytest.mark.gpu
@pytest.mark.parametrize("name,g", [("bf16", 4), ("bf16", 1), ("f32_32", 4), ("f32_64", 3), ("f32_128", 2)])
@pytest.mark.parametrize("most", [255, 256, 257, 511, 512, 513, 1023, 1024, 1025])
def test_lengths_about_a_short_calls(name, g, most):
    """Lengths up to, at and past those that a workgroup takes at once, of prefixes and behind them."""
    lens = [most, most - 1, 1, most // 2, most, 64]
    run_and_check(Batch(heads(name, g), lens, [2, 1, 1, 3, 1, 5], sizes=[2, 3], prefix=[most - 3, 40], before=0, B=24, seed=g), once=True)


@pytest.mark.gpu
def test_slots_past_four_gib():
    shape = dataclasses.replace(heads("bf16", 4), num_layers=1)
    blocks = (5 << 30) // (2 * 2 * 128 * 16)  # a plane of 5 GiB
    raw = torch.empty(2, blocks, 16, 2, 128, dtype=torch.bfloat16, device="cuda")
    h = kvr.kv_arena_bind(raw.data_ptr(), raw.numel() * 2, shape, 16, blocks)
    small = Batch(shape, [90, 80], sizes=[2], prefix=[50], seed=8, layer=0)
    small.run()
    want = small.out.clone()
    near = np.unique(small.tables[small.tables >= 0])
    far = {int(b): blocks - 1 - i * (blocks // 16) for i, b in enumerate(near)}
    for b, f in far.items():
        raw[:, f] = small.arena[0].view(2, small.blocks, 16, 2, 128)[:, b]
    small.tables = np.vectorize(lambda b: far.get(int(b), -1))(small.tables)
    small.bind()
    handle, small.handle = small.handle, h
    small.out.fill_(KEPT)
    small.run()
    torch.cuda.synchronize()
    assert torch.equal(small.out, want)
    small.handle = handle
    small.release()
    kvr.kv_arena_release(h)


@pytest.mark.gpu
def test_graphs_follow_the_lengths_and_share_a_workspace():
    """Two captured calls over one workspace, replayed in turn with eager calls
    between them, while lengths, queries and prefixes change; every replay equals eager."""
    a = Batch(heads("bf16", 4), [600, 433, 900, 405], sizes=[4], prefix=[300], seed=9)
    b = Batch(heads("bf16", 4), [40, 300], [3, 2], sizes=[2], prefix=[30], seed=10)
    ws = torch.full((max(a.ws_bytes, b.ws_bytes),), 255, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = []
    for x in (a, b):
        with torch.cuda.stream(s):
            x.run(ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            x.run(ws)
        graphs.append(g)
    rng = np.random.default_rng(1)
    for step in range(4):
        for x, g in zip((a, b), graphs):
            x.lens = np.array([int(rng.integers(0, len(t) + 1)) for t in x.slots])
            x.prefix = np.array([int(rng.integers(0, 300 if x is a else 30))])
            x.d_lens.copy_(torch.tensor(x.lens, dtype=torch.int32))
            x.d_prefix.copy_(torch.tensor(x.prefix, dtype=torch.int32))
            x.q.copy_(torch.randn(x.q.shape, device="cuda"))
            x.out.fill_(KEPT)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            x.check()
            replayed = x.out.clone()
            x.out.fill_(KEPT)
            x.run()
            torch.cuda.synchronize()
            assert torch.equal(x.out, replayed)
    a.release()
    b.release()


@pytest.mark.gpu
def test_two_streams_at_once():
    """Calls in flight together over one arena, a workspace each."""
    b = Batch(heads("bf16", 4), [3000, 2001, 2700, 2257], sizes=[4], prefix=[2000], seed=14)
    b.run()
    torch.cuda.synchronize()
    b.check()
    want, outs = b.out.clone(), []
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [torch.full_like(b.ws, 255) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(8):
        for s, w in zip(streams, ws):
            with torch.cuda.stream(s):
                b.out = torch.full_like(want, KEPT)
                b.run(w, s.cuda_stream)
                outs.append(b.out)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    b.release()


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["bf16", "f32_64"])
@pytest.mark.parametrize("sizes", [[], [3]])
@pytest.mark.parametrize("wide", [0, 100])
def test_output_over_the_queries(name, sizes, wide):
    """out may be q itself."""
    b = Batch(heads(name, 5), [70, 500, 63, 90], [4, 2, 1, 30], sizes=sizes, prefix=[60] * len(sizes), seed=11)
    b.tables = np.pad(b.tables, ((0, 0), (0, wide)), constant_values=-1)
    b.bind(max_len=1100 if wide else None)
    b.run()
    want = b.out[:, :b.q.shape[1]].clone()
    b.out = b.q
    b.run()
    torch.cuda.synchronize()
    assert torch.equal(b.q, want)
    b.release()


@pytest.mark.gpu
@pytest.mark.parametrize("wide", [0, 100])
def test_output_over_the_queries_takes_their_stride(wide):
    """Rows at another stride would lie over other requests' queries."""
    b = Batch(heads("bf16", 5), [70, 500, 63, 90], seed=11)
    b.tables = np.pad(b.tables, ((0, 0), (0, wide)), constant_values=-1)
    b.bind(max_len=1100 if wide else None)
    before, q = b.q.clone(), b.q
    w = q.shape[1]
    for out_stride in (w, q.stride(0) - 2):
        b.out = torch.as_strided(q, q.shape, (out_stride, 1))
        with pytest.raises(kvr.KvError) as e:
            b.run()
        assert e.value.status == kvr.KV_EINVAL
    torch.cuda.synchronize()
    assert torch.equal(b.q, before)
    b.release()


# ---- sizes and refusals -----------------------------------------------------
def test_workspace_bytes():
    s, f = W.LLAMA8B, kvr.kv_group_attention_workspace_bytes
    assert f(s, 4, 4, 1, 1, 1000) > 0 and f(s, 4, 4, 0, 1, 1000) > 0
    for bad in ((0, 4, 1, 1, 10), (4, 0, 1, 1, 10), (4, 4, -1, 1, 10), (4, 4, 1, 0, 10), (4, 4, 1, 1, 0),
                ((1 << 24) + 1, 4, 1, 1, 10), (4, (1 << 24) + 1, 1, 1, 10), (4, 4, (1 << 24) + 1, 1, 10),
                (4, 4, 1, 1, 1 << 31)):
        assert f(s, *bad) == 0, bad
    assert f(dataclasses.replace(s, num_q_heads=8 * 17), 4, 4, 1, 1, 1000) == 0
    assert f(dataclasses.replace(W.TINY_F32, head_dim=16, num_kv_heads=8, num_q_heads=8), 4, 4, 1, 1, 1000) == 0


@pytest.mark.parametrize("name,g", [("bf16", 1), ("bf16", 4), ("bf16", 16), ("f32_32", 3), ("f32_128", 4)])
def test_workspaces_take_every_smaller_call(name, g):
    s, rng, f = heads(name, g), np.random.default_rng(5), kvr.kv_group_attention_workspace_bytes
    for _ in range(3000):
        big = [int(2 ** rng.uniform(0, e)) for e in (9, 12, 8, 7, 16)]
        small = [int(rng.integers(1, n + 1)) if rng.random() < 0.7 else n for n in big]
        small[2] = 0 if rng.random() < 0.3 else small[2]
        assert 0 < f(s, *small) <= f(s, *big), (small, big)


def test_attention_of_an_unknown_arena_is_refused():
    with pytest.raises(kvr.KvError) as e:
        kvr.kv_group_attention(0x1234, 0, 0x1000, 4096, 0, 1, 0x2000, 0x3000, 1, 1, 0, 0, 0, 1, 16, 0x4000, 4096, 0x10000,
                               1 << 20)
    assert e.value.status == kvr.KV_ESTATE


@pytest.mark.gpu
def test_refusals():
    b = Batch(heads("bf16", 4), [20, 30], sizes=[2], prefix=[10], seed=1)
    w = b.shape.num_q_heads * 128
    ok = dict(arena=b.handle, layer=0, q=0x1000, q_stride=w, q_offsets=0x2000, rows=2, lens=0x3000, tables=0x4000,
              num_requests=2, max_blocks=4, group_offsets=0x6000, prefix_lens=0x7000, num_groups=1, max_query=1, max_len=64,
              out=0x5000, out_stride=w, workspace=0x10000, workspace_bytes=b.ws_bytes * 4)
    for bad in (dict(layer=-1), dict(layer=2), dict(q=0), dict(out=0), dict(lens=0), dict(tables=0), dict(rows=-1),
                dict(rows=1 << 31), dict(num_requests=-1), dict(num_requests=(1 << 24) + 1), dict(max_blocks=-1),
                dict(max_query=0), dict(max_len=0), dict(q_stride=w - 2), dict(out_stride=w - 2), dict(q_stride=w + 1),
                dict(q=0x1002), dict(lens=0x3001), dict(q_offsets=0, rows=3), dict(max_len=1 << 31), dict(q_stride=1 << 62),
                dict(rows=1 << 24, max_len=1 << 26), dict(workspace=0), dict(workspace=0x10008), dict(num_groups=-1),
                dict(num_groups=(1 << 24) + 1), dict(group_offsets=0), dict(prefix_lens=0), dict(group_offsets=0x6002)):
        with pytest.raises(kvr.KvError) as e:
            kvr.kv_group_attention(**{**ok, **bad})
        assert e.value.status == kvr.KV_EINVAL, bad
    need = kvr.kv_group_attention_workspace_bytes(b.shape, 2, 2, 1, 1, 64)
    with pytest.raises(kvr.KvError) as e:
        kvr.kv_group_attention(**{**ok, "workspace_bytes": need - 1})
    assert e.value.status == kvr.KV_ENOMEM
    kvr.kv_group_attention(**{**ok, "rows": 0})  # nothing to do
    kvr.kv_group_attention(**{**ok, "num_requests": 0})
    b.release()
