"""The packed arena's entry points (include/kvr_packed.h) at sizes that only large calls
reach: steps that the decode over it does not take, and rows in such numbers that a wave moves
two steps of them at a time, or that the workgroups of the largest grid walk on.  What one large
call does is compared, bit for bit, with many small ones (which the other tests compare with the
format's definition), and rows picked from it with the definition itself."""
import dataclasses

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_14635_amd import harness as Hn  # noqa: E402
from paper_2608_14635_amd import kvr  # noqa: E402
from paper_2608_14635_amd import workloads as W  # noqa: E402

import packed_util as P  # noqa: E402
import test_packed as TP  # noqa: E402


def bound(shape, B, blocks):
    n = kvr.kv_packed_bytes(shape, B, blocks)
    raw = torch.empty(n, dtype=torch.uint8, device="cuda")
    return raw, kvr.kv_packed_bind(raw.data_ptr(), n, shape, B, blocks)


def step_status(shape, handle, positions, tables, size):
    """What a step with a workspace of `size` bytes that is never touched answers."""
    w = kvr.Weights(kvr.make_desc(shape), 0x1000, [{k: 0x1000 for k in kvr.LAYER_FIELDS}] * shape.num_layers)
    with pytest.raises(kvr.KvError) as e:
        kvr.kv_packed_decode_step(w, 0x1000, 0x1000, np.zeros(len(positions), np.int32), positions, tables, handle,
                                  0x10000, size, 0x2000)
    assert e.value.message
    return e.value.status


@pytest.mark.gpu
def test_decode_steps_of_positions_that_the_attention_does_not_take():
    """Requests whose tables name one block over and over, but for the block that they write."""
    shape, B = dataclasses.replace(W.TINY_BF16, num_layers=1), 1 << 14
    raw, h = bound(shape, B, 41)
    top = (1 << 31) - 1

    def tables(n):
        t = np.zeros((n, (1 << 31) // B), np.int32)
        t[:, -1] = np.arange(1, n + 1)
        return t
    assert step_status(shape, h, [top], tables(1), 1 << 62) == kvr.KV_EINVAL
    assert step_status(shape, h, [5, top], np.vstack([np.full(1 << 17, 7, np.int32), tables(1)[0]]), 1 << 62) == kvr.KV_EINVAL
    assert step_status(shape, h, [top - 1] * 40, tables(40), 1 << 62) == kvr.KV_EINVAL
    # one position less, and fewer requests: the workspace is what is missing
    assert step_status(shape, h, [top - 1], tables(1), 16) == kvr.KV_ENOMEM
    assert step_status(shape, h, [top - 1] * 8, tables(8), 16) == kvr.KV_ENOMEM
    kvr.kv_packed_release(h)


@pytest.mark.gpu
def test_decode_steps_of_more_requests_than_the_attention_takes():
    shape, n = dataclasses.replace(P.F32[32], num_layers=1, num_q_heads=4, num_kv_heads=4), (1 << 24) + 1
    raw, h = bound(shape, 16, n)
    assert step_status(shape, h, np.zeros(n, np.int32), np.arange(n, dtype=np.int32)[:, None], 1 << 62) == kvr.KV_EINVAL
    kvr.kv_packed_release(h)


def wave_items(shape, rows, layers, steps):
    """Wave items of a call whose waves take `steps` times as many rows as fill their lanes."""
    each = steps * 64 // (shape.head_dim // 8)
    return -(-rows // each) * shape.num_kv_heads * layers


def pick(n, seed):
    """Places [n] of a permutation over n + n/8, some of them outside."""
    rng = np.random.default_rng(seed)
    s = rng.permutation(n + n // 8)[:n].astype(np.int64)
    s[rng.integers(0, n, size=7)] = [-1, -(1 << 40), 1 << 40, -2, n * 3, 1 << 31, -1]
    return s


class Rows:
    """A retained arena of ordinary values and a packed one of arbitrary bytes, pairs of slots."""

    def __init__(self, shape, n):
        self.shape, self.n, dt = shape, n, P.torch_dtype(shape)
        L, nkv, d, B = shape.num_layers, shape.num_kv_heads, shape.head_dim, 32
        self.blocks = -(-(n + n // 8) // B)
        g = torch.Generator(device="cuda")
        g.manual_seed(n)
        self.plain = torch.empty(L, 2, self.blocks * B, nkv, d, dtype=dt, device="cuda")
        for layer in self.plain:
            layer.normal_(generator=g)
            layer *= torch.exp2(torch.randint(-8, 9, (2, self.blocks * B, 1, 1), generator=g, device="cuda")).to(dt)
        self.arena = self.bind(self.plain)
        self.bytes = kvr.kv_packed_bytes(shape, B, self.blocks)
        self.before = torch.randint(0, 256, (self.bytes,), generator=g, device="cuda", dtype=torch.uint8)
        self.host = (pick(n, 1), pick(n, 2))
        self.slots = [torch.tensor(s, device="cuda") for s in self.host]
        self.B = B

    def bind(self, t):
        return kvr.kv_arena_bind(t.data_ptr(), t.numel() * t.element_size(), self.shape, 32, self.blocks)

    def calls(self, call, each):
        for i in range(0, self.n, each):
            a, b = (s[i:i + each] for s in self.slots)
            call(a.data_ptr(), b.data_ptr(), len(a))
        torch.cuda.synchronize()

    def park(self, each):
        """The packed bytes after a park of `each` pairs a call."""
        raw = self.before.clone()
        h = kvr.kv_packed_bind(raw.data_ptr(), self.bytes, self.shape, self.B, self.blocks)
        self.calls(lambda a, p, n: kvr.kv_packed_park(self.arena, a, h, p, n, Hn.stream_ptr()), each)
        kvr.kv_packed_release(h)
        return raw

    def restore(self, raw, each):
        """A retained arena after a restore from those bytes."""
        out = self.plain.flip(0).contiguous()
        h, a = kvr.kv_packed_bind(raw.data_ptr(), self.bytes, self.shape, self.B, self.blocks), self.bind(out)
        self.calls(lambda s, p, n: kvr.kv_packed_restore(h, p, a, s, n, Hn.stream_ptr()), each)
        kvr.kv_packed_release(h)
        kvr.kv_arena_release(a)
        return out


TWICE, WALK = 2 * 8192, 4 << 16  # wave items above which a wave takes two steps of rows, a workgroup more items
PARKS = {"bf16": (32, 301, 8205), "f32_32": (64, 519, 16411), "f32_64": (64, 519, 16411), "f32_128": (64, 519, 16411)}


@pytest.mark.gpu
@pytest.mark.parametrize("size", ["twice", "walk"])
@pytest.mark.parametrize("name", list(PARKS))
def test_large_parks_and_restores(name, size):
    layers, some, many = PARKS[name]
    shape = dataclasses.replace(P.SHAPES[name], num_layers=layers)
    n, each = some if size == "twice" else many, 101
    assert wave_items(shape, n, layers, 1) > TWICE >= wave_items(shape, each, layers, 1)
    assert (wave_items(shape, n, layers, 2) > WALK) == (size == "walk")
    r = Rows(shape, n)
    raw = r.park(n)
    assert torch.equal(raw, r.park(each))
    out = r.restore(raw, n)
    assert torch.equal(out.view(torch.int16), r.restore(raw, each).view(torch.int16))
    # rows at the ends and between them, of the first and the last layer, against the definition
    a, p = r.host
    good = (a >= 0) & (a < r.blocks * r.B) & (p >= 0) & (p < r.blocks * r.B)
    rows = np.flatnonzero(good)
    rows = np.unique(np.concatenate([rows[:9], rows[-9:], rows[::len(rows) // 20 + 1]]))
    for l in (0, layers - 1):
        got = out[l][:, torch.tensor(a[rows], device="cuda")].double().cpu().numpy()
        x = r.plain[l][:, torch.tensor(a[rows], device="cuda")].double().cpu().numpy()
        assert np.array_equal(got, P.values(*P.quantise(x)))
    # and every slot that is not listed as it was
    kept = torch.ones(r.blocks * r.B, dtype=torch.bool, device="cuda")
    kept[torch.tensor(a[good], device="cuda")] = False
    assert torch.equal(out[:, :, kept], r.plain.flip(0)[:, :, kept])
    kvr.kv_arena_release(r.arena)


@pytest.mark.gpu
@pytest.mark.parametrize("name,n", [("bf16", 8235), ("f32_32", 32801), ("f32_64", 32801), ("f32_128", 32801)])
def test_large_stores_and_loads(name, n):
    """Rows of one layer, on strides of their own."""
    shape, each, B = P.SHAPES[name], 1001, 48
    assert wave_items(shape, n, 1, 1) > TWICE >= wave_items(shape, each, 1, 1)
    dt, w = P.torch_dtype(shape), shape.num_kv_heads * shape.head_dim
    blocks = -(-(n + n // 8) // B)
    size = kvr.kv_packed_bytes(shape, B, blocks)
    some = TP.rows_of(shape, 300, 3).view(300, w).cuda()  # zeros, ties, tiny, huge and non-finite ones among them
    k = some[torch.arange(n, device="cuda") * 7 % 300].clone()
    v = torch.zeros(n, w + 6, dtype=dt, device="cuda")
    v[:, :w] = some[torch.arange(n, device="cuda") * 11 % 300]
    slots = torch.tensor(pick(n, 5), device="cuda")
    before = torch.randint(0, 256, (size,), device="cuda", dtype=torch.uint8)
    raws, outs = [], []
    for part in (n, each):
        raw, out = before.clone(), torch.full((2, n, w + 2), 7.0, dtype=dt, device="cuda")
        h = kvr.kv_packed_bind(raw.data_ptr(), size, shape, B, blocks)
        for i in range(0, n, part):
            m = min(part, n - i)
            kvr.kv_packed_store(h, 1, k[i:].data_ptr(), w, v[i:].data_ptr(), w + 6, slots[i:].data_ptr(), m, Hn.stream_ptr())
            kvr.kv_packed_load(h, 1, out[0, i:].data_ptr(), w + 2, out[1, i:].data_ptr(), w + 2, slots[i:].data_ptr(), m,
                               Hn.stream_ptr())
        torch.cuda.synchronize()
        kvr.kv_packed_release(h)
        raws.append(raw)
        outs.append(out)
    assert torch.equal(*raws) and torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))
    good = (slots >= 0) & (slots < B * blocks)
    want = P.values(*P.quantise(some.view(300, -1, shape.head_dim).double().cpu().numpy())).reshape(300, w)
    want = torch.tensor(want, device="cuda")
    for out, mul in zip(outs[0], (7, 11)):
        got = out[good, :w].double()
        exp = want[torch.arange(n, device="cuda")[good] * mul % 300]
        assert torch.equal(got.isnan(), exp.isnan()) and torch.equal(got.nan_to_num(), exp.nan_to_num())
        assert (out[~good] == 7.0).all() and (out[:, w:] == 7.0).all()
