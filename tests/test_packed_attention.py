"""Attention over a packed arena (kv_packed_attention, include/kvr_packed.h)
against softmax(q k^T / sqrt(d)) v in 64 bits over the values the arena's bytes
stand for.  Slots outside the contexts hold arbitrary bytes, NaN scales among them.

Tolerance, per output element, with u = 2^-24 and A the largest sum_e |q_e k_je| /
sqrt(d) of the row's positions:
  a score is a fp32 sum of d products and a scaling, |ds| <= (d + 8) u A;
  weights then differ by 2 |ds| relative, the exponential and its argument's
  rounding (the argument is at most 1.5 * 2 A) add (8 + 4 A) u;
  sums over n positions add 2 (n + 16) u;
  weights enter the product with V as sums of two bf16 numbers in bf16 models
  (2^-17 relative), of three in fp32 ones (u);
all times max |v|, plus half a step of the output type and its least number."""
import dataclasses

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_14635_amd import harness as Hn  # noqa: E402
from paper_2608_14635_amd import kvr  # noqa: E402
from paper_2608_14635_amd import workloads as W  # noqa: E402

import packed_util as P  # noqa: E402

U = 2.0 ** -24
KEPT = 7.0


def heads(name, g=None):
    s = dataclasses.replace(P.SHAPES[name], num_layers=2)
    return s if g is None else dataclasses.replace(s, num_q_heads=g * s.num_kv_heads)


class Batch:
    """Requests over a packed arena: lens[r] positions, counts[r] query rows."""

    def __init__(self, shape, lens, counts=None, B=16, seed=0, layer=1, extra_rows=0, blocks=None, std=1.3,
                 wide_extra=1):
        self.shape, self.lens, self.B, self.layer = shape, np.array(lens), B, layer
        self.counts = np.ones(len(lens), int) if counts is None else np.array(counts)
        self.plain = counts is None and not extra_rows  # one row a request: no offsets
        rng = np.random.default_rng(seed)
        need = -(-self.lens // B)
        self.blocks = blocks or int(need.sum()) + 3
        self.arena = P.PackedArena(shape, B, self.blocks, seed=seed)
        ids = rng.permutation(self.blocks)
        self.tables = np.full((len(lens), int(need.max(initial=0)) + wide_extra), -1, np.int32)
        o = 0
        for r, k in enumerate(need):
            self.tables[r, :k] = ids[o:o + k]
            o += k
        self.slots = [self.tables[r, np.arange(n) // B].astype(np.int64) * B + np.arange(n) % B
                      for r, n in enumerate(self.lens)]
        dt = P.torch_dtype(shape)
        nkv, d = shape.num_kv_heads, shape.head_dim
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        flat = np.concatenate(self.slots) if len(lens) else np.zeros(0, np.int64)
        n = len(flat)
        if n:
            k, v = (torch.randn(n, nkv * d, generator=g, device="cuda").mul_(std).to(dt) for _ in range(2))
            self.store(k, v, flat)
        self.rows = int(self.counts.sum()) + extra_rows
        self.off = np.concatenate([[0], np.cumsum(self.counts)])
        # query rows wider than their heads, 4 bytes past a 16-byte boundary
        w, lead = shape.num_q_heads * d, 4 // (2 if dt == torch.bfloat16 else 4)
        flat_q = torch.randn(self.rows * (w + 2 * lead) + lead, generator=g, device="cuda").mul_(std).to(dt)
        self.q = flat_q[lead:].view(self.rows, w + 2 * lead)[:, :w]
        self.out = torch.full((self.rows, w + 4), KEPT, dtype=dt, device="cuda")
        self.bind()

    def store(self, k, v, slots):
        w = k.shape[1]
        sl = torch.tensor(slots, device="cuda")
        kvr.kv_packed_store(self.arena.handle, self.layer, k.data_ptr(), w, v.data_ptr(), w, sl.data_ptr(), len(slots),
                            Hn.stream_ptr())
        torch.cuda.synchronize()

    def bind(self, max_query=None, max_len=None):
        dev = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
        self.d_lens, self.d_tables, self.d_off = dev(self.lens), dev(self.tables), dev(self.off)
        self.max_query = max_query or max(1, int(self.counts.max(initial=1)))
        self.max_len = max_len or max(1, int(self.lens.max(initial=1)))
        self.ws_bytes = kvr.kv_packed_attention_workspace_bytes(self.shape, max(1, len(self.lens)), max(1, self.rows),
                                                                self.max_query, self.max_len)
        # every byte 255: whatever is read without having been written is NaN
        self.ws = torch.full((self.ws_bytes,), 255, dtype=torch.uint8, device="cuda")

    def run(self, ws=None, stream=None):
        kvr.kv_packed_attention(self.arena.handle, self.layer, self.q.data_ptr(), self.q.stride(0),
                                0 if self.plain else self.d_off.data_ptr(), self.rows, self.d_lens.data_ptr(),
                                self.d_tables.data_ptr(), len(self.lens), self.tables.shape[1], self.max_query,
                                self.max_len, self.out.data_ptr(), self.out.stride(0),
                                (self.ws if ws is None else ws).data_ptr(), self.ws_bytes,
                                Hn.stream_ptr() if stream is None else stream)

    def reference(self):
        """out and its tolerance, [rows, nq, d], 64 bits."""
        s, B = self.shape, self.B
        nq, nkv, d = s.num_q_heads, s.num_kv_heads, s.head_dim
        kc, vc, ks, vs = (a[self.layer] for a in self.arena.parts())
        q = self.q.float().cpu().numpy().astype(np.float64).reshape(self.rows, nq, d)
        out, tol = np.zeros((self.rows, nq, d)), np.zeros((self.rows, nq, d))
        split = 2.0 ** -17 if s.dtype == W.BF16 else U
        half = torch.finfo(P.torch_dtype(s)).eps / 2
        for r, n in enumerate(self.lens):
            m = self.counts[r]
            j = np.arange(max(0, min(n, self.tables.shape[1] * B, self.max_len)))
            blk = self.tables[r, j // B].astype(np.int64)
            there = (blk >= 0) & (blk < self.blocks)
            slots = (blk * B + j % B)[there]
            k, v = P.values(kc[slots], ks[slots]), P.values(vc[slots], vs[slots])
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
        got = self.out.float().cpu().numpy().astype(np.float64)
        assert (got[:, w:] == KEPT).all()
        used = int(self.counts.sum())
        assert (got[used:] == KEPT).all()
        got, want, tol = got[:used, :w], want.reshape(len(want), w)[:used], tol.reshape(len(tol), w)[:used]
        nan = np.isnan(want)
        assert np.array_equal(np.isnan(got), nan)
        bad = np.abs(got - want)[~nan] > tol[~nan]
        assert not bad.any(), (int(bad.sum()), float(np.abs(got - want)[~nan].max()), float(tol[~nan].min()))

    def release(self):
        self.arena.release()


RAGGED = [1, 15, 16, 17, 31, 32, 33, 0, 64, 100, 257]


@pytest.mark.gpu
@pytest.mark.parametrize("name,g", [("bf16", 1), ("bf16", 4), ("bf16", 5), ("bf16", 16), ("f32_32", 3), ("f32_64", 1),
                                    ("f32_64", 8), ("f32_128", 4), ("f32_128", 16)])
@pytest.mark.parametrize("B", [16, 48])
def test_one_row_a_request(name, g, B):
    b = Batch(heads(name, g), RAGGED, B=B, seed=g)
    b.run()
    torch.cuda.synchronize()
    b.check()
    b.release()


@pytest.mark.gpu
@pytest.mark.parametrize("name,g", [("bf16", 1), ("bf16", 5), ("bf16", 16), ("f32_32", 8), ("f32_64", 3), ("f32_128", 4)])
def test_several_rows_a_request(name, g):
    """Row counts that fill a matrix tile's columns, cross it, and take several; a
    request without rows, one with more rows than positions, rows behind the last."""
    lens = [1, 40, 17, 0, 300, 64, 5, 33]
    counts = [1, 4, 0, 2, 9, 64, 8, 3]
    b = Batch(heads(name, g), lens, counts, B=32, seed=g, extra_rows=3)
    b.run()
    torch.cuda.synchronize()
    b.check()
    b.release()


@pytest.mark.gpu
@pytest.mark.parametrize("name,lens", [("bf16", [70001]), ("bf16", [9000, 1, 4097, 20000]), ("f32_64", [5000, 3]),
                                       ("bf16", [1 + (37 * i) % 90 for i in range(1100)]),
                                       ("f32_32", [1 + (5 * i) % 40 for i in range(300)])])
def test_long_and_many(name, lens):
    b = Batch(heads(name, 4), lens, seed=len(lens))
    b.run()
    torch.cuda.synchronize()
    b.check()
    b.release()


@pytest.mark.gpu
@pytest.mark.parametrize("name,g", [("bf16", 4), ("bf16", 3), ("f32_32", 4), ("f32_64", 2), ("f32_128", 4)])
def test_a_prompts_piece(name, g):
    """Many query rows of two requests: several column tiles each, causal inside."""
    b = Batch(heads(name, g), [500, 222], [150, 222], seed=2)
    b.run()
    torch.cuda.synchronize()
    b.check()
    b.release()


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["bf16", "f32_64"])
def test_blocks_that_are_not_there(name):
    """Table entries outside the arena, tables narrower than the lengths, a request
    of which nothing is left, and lengths above max_len and below zero."""
    b = Batch(heads(name, 4), [100, 64, 33, 200, 50, 10], [1, 3, 2, 1, 1, 2], B=16, seed=5)
    b.tables[0, [0, 3]] = -1
    b.tables[1, 2] = b.blocks
    b.tables[2, :3] = [-5, 1 << 30, -(1 << 31)]
    b.tables = np.ascontiguousarray(b.tables[:, :9])  # request 3 has 13 blocks
    b.lens[5] = -3
    b.bind(max_len=64)
    b.run()
    torch.cuda.synchronize()
    b.check()
    b.release()


@pytest.mark.gpu
@pytest.mark.parametrize("name,counts", [("bf16", None), ("bf16", [3, 5, 2]), ("f32_64", [3, 5, 2]), ("f32_128", None)])
def test_values_that_are_not_finite(name, counts):
    """A NaN in K or V reaches exactly the rows that see its position, and in V the
    group's dims alone; infinite queries give NaN rows."""
    b = Batch(heads(name, 4), [50, 70, 40], counts, seed=6)
    dt, w = P.torch_dtype(b.shape), b.shape.num_kv_heads * b.shape.head_dim
    bad = {(0, 20): "v", (1, 69): "v", (1, 67): "k", (2, 39): "k"}  # the last two of request 1 and one of 2: masked
    for (r, j), which in bad.items():                                # for earlier query rows
        k, v = (torch.randn(1, w, device="cuda").to(dt) for _ in range(2))
        (k if which == "k" else v)[0, 5] = float("nan")
        b.store(k, v, b.slots[r][j:j + 1])
    b.q[0, 3] = float("inf")
    b.run()
    torch.cuda.synchronize()
    b.check()
    b.release()


@pytest.mark.gpu
def test_scores_of_any_size():
    """Scores in the thousands, equal scores, and queries of zero."""
    b = Batch(heads("bf16", 4), [300, 129, 64], seed=7, std=30.0)
    b.q[1] = 0
    b.run()
    torch.cuda.synchronize()
    b.check()
    b.release()


@pytest.mark.gpu
def test_records_past_four_gib():
    shape = dataclasses.replace(heads("bf16", 4), num_layers=1)
    blocks = (6 << 30) // (17 * 128 * shape.num_kv_heads)
    n = kvr.kv_packed_bytes(shape, 16, blocks)
    raw = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    h = kvr.kv_packed_bind(raw.data_ptr(), n, shape, 16, blocks)
    small = Batch(shape, [90], seed=8, layer=0, blocks=9)
    # the same bytes, blocks far apart
    far = np.array([blocks - 1 - i * (blocks // 8) for i in range(6)])
    rec = shape.num_kv_heads * 17 * 128
    for i, f in enumerate(far):
        src = int(small.tables[0, i]) * rec
        raw[int(f) * rec:int(f) * rec + rec] = small.arena.raw[src:src + rec]
    small.run()
    want = small.out.clone()
    small.tables[0, :6] = far
    small.bind()
    handle, small.arena.handle = small.arena.handle, h
    small.out.fill_(KEPT)
    small.run()
    torch.cuda.synchronize()
    assert torch.equal(small.out, want)
    small.arena.handle = handle
    small.release()
    kvr.kv_packed_release(h)


@pytest.mark.gpu
def test_graphs_follow_the_lengths_and_share_a_workspace():
    """Two captured calls over one workspace, replayed in turn with eager calls
    between them, while lengths and queries change; every replay equals eager."""
    a = Batch(heads("bf16", 4), [600, 33, 900, 5], seed=9)
    b = Batch(heads("bf16", 4), [40, 300], [3, 2], seed=10)
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
            x.lens = np.array([int(rng.integers(0, n + 1)) for n in [len(t) for t in x.slots]])
            x.d_lens.copy_(torch.tensor(x.lens, dtype=torch.int32))
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
@pytest.mark.parametrize("name,g", [("bf16", 2), ("bf16", 5), ("f32_64", 16)])
def test_more_rows_than_max_query(name, g):
    """Rows past max_query are left out; those before them keep their positions."""
    counts = [5, 9, 2, 7]
    b = Batch(heads(name, g), [40, 9, 70, 4], counts, seed=12)
    b.bind(max_query=4)
    b.run()
    torch.cuda.synchronize()
    want, tol = b.reference()
    got = b.out[:, :b.q.shape[1]].float().cpu().numpy().astype(np.float64).reshape(want.shape)
    for r, m in enumerate(counts):
        rows = slice(b.off[r], b.off[r] + min(m, 4))
        assert (np.abs(got[rows] - want[rows]) <= tol[rows]).all(), r
        assert (got[rows.stop:b.off[r] + m] == KEPT).all(), r
    b.release()


@pytest.mark.gpu
def test_requests_that_share_blocks():
    """A common prefix: two requests' tables name the same blocks, one block twice in a
    third's."""
    b = Batch(heads("bf16", 4), [100, 90, 64], [2, 3, 1], seed=13)
    b.tables[1, :5] = b.tables[0, :5]
    b.tables[2, 3] = b.tables[2, 0]
    b.bind()
    b.run()
    torch.cuda.synchronize()
    b.check()
    b.release()


@pytest.mark.gpu
def test_attention_on_two_streams_at_once():
    """Calls in flight together over one arena, a workspace each."""
    b = Batch(heads("bf16", 4), [3000, 1, 700, 257], seed=14)
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
def test_output_over_the_queries():
    """out may be q itself."""
    b = Batch(heads("bf16", 5), [70, 500, 3], [4, 2, 1], seed=11)
    b.run()
    c = b.q.clone()
    b.q.copy_(c)
    want = b.out[:, :c.shape[1]].clone()
    kvr.kv_packed_attention(b.arena.handle, b.layer, b.q.data_ptr(), b.q.stride(0), b.d_off.data_ptr(), b.rows,
                            b.d_lens.data_ptr(), b.d_tables.data_ptr(), 3, b.tables.shape[1], b.max_query, b.max_len,
                            b.q.data_ptr(), b.q.stride(0), b.ws.data_ptr(), b.ws_bytes, Hn.stream_ptr())
    torch.cuda.synchronize()
    assert torch.equal(b.q, want)
    b.release()


# ---- sizes and refusals -----------------------------------------------------
def test_workspace_bytes():
    s = W.LLAMA8B
    assert kvr.kv_packed_attention_workspace_bytes(s, 4, 4, 1, 1000) > 0
    for bad in ((0, 4, 1, 10), (4, 0, 1, 10), (4, 4, 0, 10), (4, 4, 1, 0), ((1 << 24) + 1, 4, 1, 10),
                (4, (1 << 24) + 1, 1, 10), (4, 1 << 62, 1 << 30, 10), (4, 4, 1, 1 << 31), (4, 4, 1, 1 << 62)):
        assert kvr.kv_packed_attention_workspace_bytes(s, *bad) == 0
    wide = dataclasses.replace(s, num_q_heads=8 * 17)
    assert kvr.kv_packed_attention_workspace_bytes(wide, 4, 4, 1, 1000) == 0


@pytest.mark.parametrize("name,g", [("bf16", 1), ("bf16", 4), ("bf16", 16), ("f32_32", 3), ("f32_128", 4)])
def test_workspaces_take_every_smaller_call(name, g):
    s, rng = heads(name, g), np.random.default_rng(5)
    sizes = lambda: [int(2 ** rng.uniform(0, e)) for e in (9, 12, 7, 16)]  # noqa: E731
    for _ in range(3000):
        big = sizes()
        small = [int(rng.integers(1, n + 1)) if rng.random() < 0.7 else n for n in big]
        a, b = (kvr.kv_packed_attention_workspace_bytes(s, *x) for x in (small, big))
        assert 0 < a <= b, (small, big)


def test_attention_of_an_unknown_arena_is_refused():
    with pytest.raises(kvr.KvError) as e:
        kvr.kv_packed_attention(0x1234, 0, 0x1000, 4096, 0, 1, 0x2000, 0x3000, 1, 1, 1, 16, 0x4000, 4096, 0x10000, 1 << 20)
    assert e.value.status == kvr.KV_ESTATE


@pytest.mark.gpu
def test_attention_refusals():
    b = Batch(heads("bf16", 4), [20, 30], seed=1)
    w = b.shape.num_q_heads * 128
    ok = dict(packed=b.arena.handle, layer=0, q=0x1000, q_stride=w, q_offsets=0x2000, rows=2, lens=0x3000,
              tables=0x4000, num_requests=2, max_blocks=4, max_query=1, max_len=64, out=0x5000, out_stride=w,
              workspace=0x10000, workspace_bytes=b.ws_bytes)
    for bad in (dict(layer=-1), dict(layer=2), dict(q=0), dict(out=0), dict(lens=0), dict(tables=0), dict(rows=-1),
                dict(rows=1 << 31), dict(num_requests=-1), dict(num_requests=(1 << 24) + 1), dict(max_blocks=-1), dict(max_query=0), dict(max_len=0),
                dict(q_stride=w - 2), dict(out_stride=w - 2), dict(q_stride=w + 1), dict(q=0x1002), dict(lens=0x3001),
                dict(q_offsets=0, rows=3), dict(max_len=1 << 31), dict(rows=1 << 24, max_len=1 << 26), dict(workspace=0), dict(workspace=0x10008)):
        with pytest.raises(kvr.KvError) as e:
            kvr.kv_packed_attention(**{**ok, **bad})
        assert e.value.status == kvr.KV_EINVAL, bad
    with pytest.raises(kvr.KvError) as e:
        kvr.kv_packed_attention(**{**ok, "workspace_bytes": b.ws_bytes - 1})
    assert e.value.status == kvr.KV_ENOMEM
    kvr.kv_packed_attention(**{**ok, "rows": 0})  # nothing to do
    kvr.kv_packed_attention(**{**ok, "num_requests": 0})
    b.release()
