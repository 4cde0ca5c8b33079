"""Attention over a packed arena (kv_packed_attention, include/kvr_packed.h) at the ends
of its range: blocks and lengths past 32-bit offsets, values and queries next to the
largest numbers, and sums in which every position counts by itself."""
import dataclasses

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_14635_amd import harness as Hn  # noqa: E402
from paper_2608_14635_amd import kvr  # noqa: E402
from paper_2608_14635_amd import workloads as W  # noqa: E402

import packed_util as P  # noqa: E402
import test_packed_attention as TA  # noqa: E402

U = 2.0 ** -24
ONE_HEAD = dataclasses.replace(P.F32[128], num_layers=1, num_q_heads=4, num_kv_heads=1)


def dev(a, dtype=torch.int32):
    return torch.tensor(np.asarray(a), dtype=dtype, device="cuda")


class Zeros:
    """A packed arena of zeros (K and V 0 in every slot), with chosen rows stored."""

    def __init__(self, shape, B, blocks):
        self.shape, self.B, self.blocks = shape, B, blocks
        n = kvr.kv_packed_bytes(shape, B, blocks)
        self.raw = torch.zeros(n, dtype=torch.uint8, device="cuda")
        self.handle = kvr.kv_packed_bind(self.raw.data_ptr(), n, shape, B, blocks)

    def store(self, slots, k, v):
        """k, v [n, nkv, d], values that the arena holds exactly."""
        dt, w = P.torch_dtype(self.shape), self.shape.num_kv_heads * self.shape.head_dim
        kd, vd = (torch.tensor(np.asarray(x).reshape(-1, w), dtype=torch.float32).to(dt).cuda() for x in (k, v))
        sl = dev(slots, torch.int64)
        kvr.kv_packed_store(self.handle, 0, kd.data_ptr(), w, vd.data_ptr(), w, sl.data_ptr(), len(sl), Hn.stream_ptr())
        torch.cuda.synchronize()

    def attend(self, q, lens, tables, counts=None, max_len=None):
        """q [rows, nq, d] -> out [rows, nq, d] in 64 bits; counts: query rows of each request."""
        s, lens, tables = self.shape, np.asarray(lens), np.asarray(tables, np.int32)
        counts = np.ones(len(lens), int) if counts is None else np.asarray(counts)
        w = s.num_q_heads * s.head_dim
        qd = torch.tensor(np.asarray(q).reshape(-1, w), dtype=torch.float32).to(P.torch_dtype(s)).cuda()
        out = torch.full_like(qd, 7.0)
        off, ln, tab = dev(np.concatenate([[0], np.cumsum(counts)])), dev(lens), dev(tables)
        m, n = int(counts.max()), int(max_len or lens.max())
        size = kvr.kv_packed_attention_workspace_bytes(s, len(lens), len(qd), m, n)
        ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        kvr.kv_packed_attention(self.handle, 0, qd.data_ptr(), w, off.data_ptr(), len(qd), ln.data_ptr(), tab.data_ptr(),
                                len(lens), tables.shape[1], m, n, out.data_ptr(), w, ws.data_ptr(), size, Hn.stream_ptr())
        torch.cuda.synchronize()
        return out.double().cpu().numpy().reshape(-1, s.num_q_heads, s.head_dim)

    def release(self):
        kvr.kv_packed_release(self.handle)


def marks(n, d, seed=0):
    """Values [n, 1, d] that the arena holds exactly, different in every row."""
    rng = np.random.default_rng(seed)
    v = rng.choice(P.VALUES, size=(n, 1, d))
    v[..., ::32] = 6.0  # each group's scale is 1
    return v


@pytest.mark.gpu
def test_records_past_two_gib_of_one_block():
    """A block of 15.8 million slots: its last records lie more than 2^31 bytes behind its
    first.  K is 0 but for a few positions, each of which outweighs all before it
    by e^60 and more: what a request sees is the V of the last of them."""
    d, B = 128, 15_800_000
    border = 16 * ((1 << 31) // (17 * d) + 1)  # the first slot of a record that starts past 2^31
    at = [100, border - 1, border, border + 13, B - 1]
    a = Zeros(ONE_HEAD, B, 1)
    k = np.zeros((len(at), 1, d))
    for i in range(len(at)):
        k[i, 0, :i + 1] = 6.0
    v = marks(len(at), d)
    a.store(at, k, v)
    q = np.zeros((1, 4, d))
    q[..., :len(at)] = 128.0  # scores 128 * 6 * (i + 1) / sqrt(128): 68 apart
    lens = [p + 1 for p in at]
    out = a.attend(np.repeat(q, len(at), 0), lens, np.zeros((len(at), 1)))
    # the rest weighs at most 1.6e7 e^-67 of V's 6; the quotient and the weight's parts round by a few u
    assert np.abs(out - v).max() <= 6 * 8 * U
    a.release()


@pytest.mark.gpu
def test_lengths_up_to_the_largest_number():
    """Contexts whose last positions are next to 2^31, over one block listed many times;
    the last of several query rows see them, as do requests some positions shorter."""
    d, B = 128, 1 << 16
    top, wide = (1 << 31) - 1, (1 << 31) // B
    a = Zeros(ONE_HEAD, B, 2)
    last = [B - 71, B - 41, B - 4, B - 3, B - 2]  # of block 1: positions 2^31 - 71 .. 2^31 - 2
    k = np.zeros((len(last), 1, d))
    for i in range(len(last)):
        k[i, 0, :i + 1] = 6.0
    v = marks(len(last), d, seed=1)
    a.store([B + x for x in last], k, v)
    q = np.zeros((5, 4, d))
    q[..., :len(last)] = 128.0
    table = np.zeros((3, wide))
    table[:, -1] = 1
    # rows at positions 2^31 - 71, 2^31 - 41, and the last three
    out = a.attend(q, [top - 69, top - 39, top], table, counts=[1, 1, 3])
    # 2^31 positions of weight e^-67 at most, V 0 there: 1.7e-20
    assert np.abs(out - v).max() <= 6 * 8 * U
    # a length beyond them, and a max_len below: its positions are left out
    out = a.attend(q[:1], [top], table[:1], max_len=top - 39)
    assert np.abs(out - v[1]).max() <= 6 * 8 * U
    out = a.attend(q[:2], [-5, -(1 << 31)], table[:2], max_len=40)
    assert (out == 0).all()
    a.release()


class ByDim(TA.Batch):
    """A batch whose K and V the test chooses, and whose tolerance goes by each dim's own
    values: an output element is sum p_j v_j of its dim, so the errors of the weights
    (test_packed_attention.py lists them) count times the largest |v_j| there.  Where V comes
    near the largest number an exponential's argument may be some 40 more and rounded to 2^-19, in
    the weights and where sums meet: 4 ln 2 2^-19 relative."""

    def put(self, k, v):
        dt, w = P.torch_dtype(self.shape), self.shape.num_kv_heads * self.shape.head_dim
        k, v = (torch.tensor(x, dtype=torch.float64).to(dt).cuda().view(-1, w) for x in (k, v))
        self.store(k, v, np.concatenate(self.slots))

    def reference(self):
        s, g = self.shape, self.shape.num_q_heads // self.shape.num_kv_heads
        d = s.head_dim
        kc, vc, ks, vs = (a[self.layer] for a in self.arena.parts())
        q = self.q.float().cpu().numpy().astype(np.float64).reshape(self.rows, -1, g, d)
        out, tol = np.zeros(q.shape), np.zeros(q.shape)
        split = 2.0 ** -17 if s.dtype == W.BF16 else U
        half = torch.finfo(P.torch_dtype(s)).eps / 2
        for r, n in enumerate(self.lens):
            sl = self.slots[r]
            k, v = (P.values(c[sl], x[sl]).swapaxes(0, 1) for c, x in ((kc, ks), (vc, vs)))  # [nkv, n, d]
            for i in range(self.counts[r]):
                row, seen = self.off[r] + i, n - self.counts[r] + i + 1
                if seen < 1:
                    continue
                x = q[row] @ k[:, :seen].swapaxes(1, 2) / np.sqrt(d)                        # [nkv, g, seen]
                a = (np.abs(q[row]) @ np.abs(k[:, :seen]).swapaxes(1, 2)).max(-1) / np.sqrt(d)
                p = np.exp(x - x.max(-1, keepdims=True))
                p /= p.sum(-1, keepdims=True)
                out[row] = p @ v[:, :seen]
                rel = (2 * (d + 8) * a + 8 + 4 * a + 2 * (seen + 16)) * U + split
                rel += 2.8 * 2.0 ** -19 * (np.abs(v).max() >= 2.0 ** 65)
                tol[row] = rel[..., None] * np.abs(v[:, :seen]).max(1)[:, None] + half * np.abs(out[row])
        return out.reshape(self.rows, -1, d), tol.reshape(self.rows, -1, d) + 2.0 ** -120


HUGE = 6 * 2.0 ** 125  # the largest value a packed arena holds


def large_values(kind, b, rng):
    """V [n, nkv, d] over all requests' positions: all of them large; the first half of each
    request's ordinary and the second large; one position's in one group; and all tiny."""
    n, nkv, d = int(b.lens.sum()), b.shape.num_kv_heads, b.shape.head_dim
    v = rng.choice(P.VALUES, size=(n, nkv, d))
    o = np.concatenate([[0], np.cumsum(b.lens)])
    if kind == "all":
        return v * 2.0 ** 125
    if kind == "tiny":
        return v * 2.0 ** -100
    for r, m in enumerate(b.lens):
        if kind == "late":
            v[o[r] + m // 2:o[r + 1]] *= 2.0 ** 125
        elif m:
            v[o[r] + m // 3, :, 32 * (r % (d // 32)):][..., :32] = HUGE * rng.choice([-1, 1])
    return v


# one request whose sums come together from a few workgroups up to (two kv heads alone) more
# than the second kernel loads at a time
TOGETHER = {"bf16": ([1 + 32 * 4 * n for n in (3, 7, 15, 31)], 8), "bf16_2": ([32 * 4 * 90], 2),
            "f32_32": ([1 + 32 * 4 * n for n in (3, 7, 15, 31)], 8), "f32_64": ([32 * 4 * n + 9 for n in (4, 13, 30)], 4),
            "f32_128": ([32 * 4 * n + 9 for n in (4, 13, 30)], 2), "f32_128_1": ([32 * 4 * 70 + 5], 1)}


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["all", "late"])
@pytest.mark.parametrize("case", list(TOGETHER))
def test_large_values_from_many_workgroups(case, kind):
    lens, nkv = TOGETHER[case]
    name = case if case in P.SHAPES else case.rsplit("_", 1)[0]
    shape = dataclasses.replace(TA.heads(name), num_kv_heads=nkv, num_q_heads=3 * nkv if nkv > 1 else 4)
    for n in lens:
        b = ByDim(shape, [n], [2], seed=n)
        rng = np.random.default_rng(n)
        b.put(rng.normal(size=(n, nkv, shape.head_dim)), large_values(kind, b, rng))
        b.run()
        torch.cuda.synchronize()
        b.check()
        b.release()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["all", "late", "one", "tiny"])
@pytest.mark.parametrize("name,g", [("bf16", 4), ("f32_32", 3), ("f32_64", 8), ("f32_128", 4)])
@pytest.mark.parametrize("lens,counts", [([3000, 1, 700, 257, 33, 0], None), ([90, 40, 300], [1, 9, 70])])
def test_values_next_to_the_largest(name, g, kind, lens, counts):
    """V up to 1.5 * 2^127: outputs lie between the values, whatever their sums are."""
    b = ByDim(TA.heads(name, g), lens, counts, seed=len(lens))
    rng = np.random.default_rng(len(kind))
    k = rng.normal(size=(int(b.lens.sum()), b.shape.num_kv_heads, b.shape.head_dim))
    b.put(k * np.linspace(0.3, 1.5, len(k))[:, None, None], large_values(kind, b, rng))
    b.run()
    torch.cuda.synchronize()
    b.check()
    b.release()


@pytest.mark.gpu
@pytest.mark.parametrize("name,g", [("f32_32", 3), ("f32_64", 8), ("f32_128", 4), ("bf16", 4)])
def test_queries_next_to_the_largest(name, g):
    """Queries up to the largest number of their type, above the largest bf16 one in fp32,
    against K whose products with them are ordinary; infinite and NaN ones beside them."""
    b = ByDim(TA.heads(name, g), [300, 70, 33, 40, 50], [2, 5, 1, 1, 1], seed=3)
    n, nkv, d = int(b.lens.sum()), b.shape.num_kv_heads, b.shape.head_dim
    rng = np.random.default_rng(4)
    k = np.zeros((n, nkv, d))
    k[..., :32] = rng.choice(P.VALUES, size=(n, nkv, 32)) * 2.0 ** -120
    b.put(k, rng.choice(P.VALUES, size=(n, nkv, d)))
    most = torch.finfo(b.q.dtype).max
    q = torch.tensor(rng.choice([-1, -0.999, -0.99609375, 0.998, 1, 0.5], size=(b.rows, b.q.shape[1])))
    q = torch.where(torch.arange(b.q.shape[1]) % d % 32 < 5, q * most, q * 2.0 ** 100).to(b.q.dtype)
    q[8, 0] = float("inf")
    q[9, 2] = float("nan")
    b.q.copy_(q)
    b.run()
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        want, tol = b.reference()
    got = b.out[:, :b.q.shape[1]].double().cpu().numpy().reshape(want.shape)
    assert (np.abs(got[:8] - want[:8]) <= tol[:8]).all()
    assert np.isnan(got[8:, 0]).all() and np.isfinite(got[8:, 1:]).all()
    b.release()


def equal_weights(b, codes):
    """Queries of 0 weigh all positions alike: with V = 1 in one dim a position (codes: of each
    request, [nkv, n] dims, -1 for none) an output is the share of positions of that
    dim.  Counts and sums are whole numbers, exact in fp32; the quotient takes two roundings and
    the output's own."""
    nkv, d = b.shape.num_kv_heads, b.shape.head_dim
    g, dt = b.shape.num_q_heads // nkv, P.torch_dtype(b.shape)
    tol = torch.finfo(dt).eps / 2 + 4 * U
    for r, code in enumerate(codes):
        n = code.shape[1]
        if n == 0:
            continue
        v = torch.zeros(n, nkv, d + 1, dtype=dt, device="cuda").scatter_(2, torch.where(code < 0, d, code).t()[..., None], 1.0)[..., :d]
        k = torch.randn(n, nkv * d, device="cuda").to(dt)
        b.store(k, v.reshape(n, -1).contiguous(), b.slots[r])
    b.q.zero_()
    b.out.fill_(TA.KEPT)
    b.run()
    torch.cuda.synchronize()
    out = b.out[:, :b.q.shape[1]].double().view(b.rows, nkv, g, d)
    for r, code in enumerate(codes):
        for i in range(b.counts[r]):
            seen = code.shape[1] - b.counts[r] + i + 1
            if seen < 1:
                assert (out[b.off[r] + i] == 0).all()
                continue
            count = torch.stack([torch.bincount(c[c >= 0], minlength=d) for c in code[:, :seen]]).double()
            want = (count / seen)[:, None].expand(nkv, g, d)
            assert ((out[b.off[r] + i] - want).abs() <= tol * want).all(), (r, i)
    return tol


EVERY = {"bf16": (8, 4, [70001], [1]), "bf16_2": (2, 4, [70001, 5], [3, 1]), "bf16_ragged": (8, 4, [9000, 1, 4097, 20000, 0], [1, 1, 4, 1, 1]),
         "f32_32": (8, 2, [20011], [1]), "f32_64": (4, 1, [5000, 3], [2, 1]), "f32_128": (1, 4, [40000, 333], [1, 70]),
         "bf16_many": (8, 4, [1 + (37 * i) % 90 for i in range(520)], [1] * 520)}


@pytest.mark.gpu
@pytest.mark.parametrize("case", list(EVERY))
def test_every_position_counts_once(case):
    """In every kv head, first by units of 32 positions, each in one dim of its own choice, then
    position by position, a window of each request in each kv head, in turn."""
    nkv, g, lens, counts = EVERY[case]
    name = case if case in P.SHAPES else "bf16"
    b = TA.Batch(dataclasses.replace(TA.heads(name), num_kv_heads=nkv, num_q_heads=g * nkv), lens, counts, seed=nkv)
    d = b.shape.head_dim
    pos = [torch.arange(n, device="cuda").expand(nkv, n) for n in lens]
    head = torch.arange(nkv, device="cuda")[:, None]
    tol = equal_weights(b, [(p // 32 * (2 * head + 3) + 7 * head) % d for p in pos])
    # a unit that were left out, the shortest and the fullest dim's: beyond the tolerance
    for n in lens:
        most = 32 * -(-n // (32 * d))
        assert n < 64 or 32 / most - 32 / n > 4 * tol
    parts = max(nkv, -(-max(lens) // (d * 64)))  # windows in which a position shows beside its dim's others
    for turn in range(parts):
        # window (turn + head) mod parts of each request
        equal_weights(b, [torch.where(p * parts // max(n, 1) == (turn + head) % parts, p % d, -1) for p, n in zip(pos, lens)])
    assert 1 / 65 > 2 * tol
    b.release()
