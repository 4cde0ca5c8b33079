"""The packed arena (include/kvr_packed.h): rows stored, loaded, parked and
restored, against the format written out in numpy.  Codes, scales and the values
they stand for are exact, so everything is compared bit for bit, the bytes that a
call must leave alone included."""
import dataclasses

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_14635_amd import harness as Hn  # noqa: E402
from paper_2608_14635_amd import kvr  # noqa: E402
from paper_2608_14635_amd import workloads as W  # noqa: E402

import packed_util as P  # noqa: E402


def rows_of(shape, n, seed, special=True):
    """Plain rows [n, nkv, d] in the model dtype: values over many magnitudes, ties
    between codes, groups of zeros, of tiny and of huge values, and some that are
    not finite."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(n, shape.num_kv_heads, shape.head_dim)) * np.exp2(rng.integers(-8, 9, size=(n, 1, 1)))
    if special:
        g = x.reshape(n, -1, 32)
        ties = np.array([6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -5, 0, -0.0, 4.999, 5.001, 3, -6])
        for i in range(0, n, 3):
            g[i, i % g.shape[1], :16] = ties * 2.0 ** (i % 40 - 20)
        g[0, 0] = 0
        g[n // 2, 0] = 1e-39 if shape.dtype == W.F32 else 2.0 ** -130
        g[n // 3, -1] = 3.0e38
        g[n - 1, 0] = 2.0 ** -118
        if n > 4:
            g[1, 0, 5], g[2, -1, 31], g[3, 0, 0] = np.nan, np.inf, -np.inf
            g[4, 0, 3] = 1.5 * 2.0 ** 20   # the border between two scales, met from both sides
            g[4, -1, 3] = 1.5078125 * 2.0 ** 20
    return torch.tensor(x, dtype=torch.float32).to(P.torch_dtype(shape))


def check_slots(got, before, layer, slots, k, v):
    """The layer's listed slots hold k, v [n, nkv, d]; every other byte is as before."""
    want = P.quantise(k.float().numpy().astype(np.float64)) + P.quantise(v.float().numpy().astype(np.float64))
    for part, was, new in zip(got, before, (want[0], want[2], want[1], want[3])):
        exp = was.copy()
        nan = None
        if new.shape[-1] == k.shape[-1]:  # codes of a NaN group stand for nothing
            nan = np.repeat((want[1] if new is want[0] else want[3]) == 255, 32, axis=-1)
            new = np.where(nan, part[layer][slots], new)
        exp[layer, slots] = new
        assert np.array_equal(part, exp)


SIZES = {"one": (1, 16, 3), "fifteen": (15, 32, 3), "seventeen": (17, 16, 5), "many": (300, 48, 9)}


@pytest.mark.gpu
@pytest.mark.parametrize("size", list(SIZES))
@pytest.mark.parametrize("name", list(P.SHAPES))
def test_store_and_load(name, size):
    shape, (n, B, blocks) = P.SHAPES[name], SIZES[size]
    rng = np.random.default_rng(n)
    a = P.PackedArena(shape, B, blocks, seed=n)
    slots = rng.permutation(B * blocks)[:n]
    nkv, d, dt = shape.num_kv_heads, shape.head_dim, P.torch_dtype(shape)
    k, v = rows_of(shape, n, 1), rows_of(shape, n, 2)
    # K: rows apart and 4 bytes past a 16-byte boundary; V: dense rows
    off = 2 if dt == torch.bfloat16 else 1
    wide = torch.zeros(n * (nkv * d + 6) + off, dtype=dt, device="cuda")
    ks = wide[off:].view(n, nkv * d + 6)[:, :nkv * d]
    ks.copy_(k.view(n, -1))
    vs, sl = v.cuda(), torch.tensor(slots, device="cuda")
    kvr.kv_packed_store(a.handle, 1, ks.data_ptr(), ks.stride(0), vs.data_ptr(), nkv * d, sl.data_ptr(), n,
                        Hn.stream_ptr())
    torch.cuda.synchronize()
    check_slots(a.parts(), a.parts(before=True), 1, slots, k, v)
    # and back, into rows of other strides with guards between them
    out = torch.full((2, n, nkv * d + 2), 7.0, dtype=dt, device="cuda")
    kvr.kv_packed_load(a.handle, 1, out[0].data_ptr(), nkv * d + 2, out[1].data_ptr(), nkv * d + 2, sl.data_ptr(),
                       n, Hn.stream_ptr())
    torch.cuda.synchronize()
    for got, x in zip(out, (k, v)):
        want = P.values(*P.quantise(x.float().numpy().astype(np.float64))).reshape(n, -1)
        assert np.array_equal(got[:, :nkv * d].float().cpu().numpy().astype(np.float64), want, equal_nan=True)
        assert (got[:, nkv * d:] == 7.0).all()
    a.release()


@pytest.mark.gpu
def test_rows_without_a_slot_are_passed_over():
    shape, B, blocks, n = P.BF16, 16, 4, 9
    a = P.PackedArena(shape, B, blocks, seed=3)
    k, v = rows_of(shape, n, 4, special=False), rows_of(shape, n, 5, special=False)
    slots = np.array([-1, 5, B * blocks, 6, -(1 << 40), 1 << 40, 63, 0, B * blocks + 1])
    good = (slots >= 0) & (slots < B * blocks)
    kd, vd, sl = k.cuda(), v.cuda(), torch.tensor(slots, device="cuda")
    w = shape.num_kv_heads * shape.head_dim
    kvr.kv_packed_store(a.handle, 0, kd.data_ptr(), w, vd.data_ptr(), w, sl.data_ptr(), n, Hn.stream_ptr())
    torch.cuda.synchronize()
    check_slots(a.parts(), a.parts(before=True), 0, slots[good], k[good], v[good])
    out = torch.full((2, n, w), 7.0, dtype=torch.bfloat16, device="cuda")
    kvr.kv_packed_load(a.handle, 0, out[0].data_ptr(), w, out[1].data_ptr(), w, sl.data_ptr(), n, Hn.stream_ptr())
    torch.cuda.synchronize()
    keep = torch.tensor(~good, device="cuda")
    assert (out[:, keep] == 7.0).all() and not (out[:, ~keep] == 7.0).all(-1).any()
    kvr.kv_packed_store(a.handle, 0, 0, w, 0, w, 0, 0)  # no rows
    a.release()


def bound_arena(shape, wl):
    arena = Hn.DeviceArena(wl)
    arena.bind()
    return arena


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(P.SHAPES))
def test_park_and_restore(name):
    """Every layer of a request set into a packed arena of other block size and
    tables, then back into other slots of a second arena."""
    shape = dataclasses.replace(P.SHAPES[name], num_layers=3)
    lens = [1, 40, 0, 17, 130]
    wl = W.small_workload(shape, lens, block_size=8, seed=3, other_live_frac=0.2)
    arena, back = bound_arena(shape, wl), bound_arena(shape, wl)
    n = sum(lens)
    rows = rows_of(shape, n * 6, 6).view(3, 2, n, shape.num_kv_heads, shape.head_dim)
    src = np.concatenate([wl.block_tables[r, np.arange(m) // 8] * 8 + np.arange(m) % 8
                          for r, m in enumerate(lens)]).astype(np.int64)
    flat = arena.bits.view(3, 2, -1, shape.num_kv_heads, shape.head_dim)
    flat[:, :, torch.tensor(src, device="cuda")] = rows.cuda().view(flat.dtype)
    rng = np.random.default_rng(8)
    a = P.PackedArena(shape, 48, 6, seed=4)
    mid = rng.permutation(48 * 6)[:n]
    total = wl.num_blocks * 8
    dst = rng.permutation(total)[:n]
    mid2, dst2 = mid.copy(), dst.copy()
    mid2[7], dst2[9] = -1, total  # passed over on one way and on the other
    up = lambda x: torch.tensor(np.asarray(x, np.int64), device="cuda")  # noqa: E731
    s1, m1, m2, d2 = up(src), up(mid), up(mid2), up(dst2)
    before = back.bits.clone()
    kvr.kv_packed_park(arena.handle, s1.data_ptr(), a.handle, m1.data_ptr(), n, Hn.stream_ptr())
    kvr.kv_packed_restore(a.handle, m2.data_ptr(), back.handle, d2.data_ptr(), n, Hn.stream_ptr())
    torch.cuda.synchronize()
    for l in range(3):
        check_slots([p[l:l + 1] for p in a.parts()], [p[l:l + 1] for p in a.parts(before=True)], 0, mid,
                    rows[l, 0], rows[l, 1])
    dt = P.torch_dtype(shape)
    got = back.bits.view(dt).view(3, 2, total, shape.num_kv_heads, shape.head_dim).float().cpu().numpy()
    want = before.view(dt).view(*got.shape).float().cpu().numpy()
    kept = np.setdiff1d(np.arange(n), [7, 9])
    want[:, :, dst[kept]] = P.values(*P.quantise(rows.float().numpy().astype(np.float64)))[:, :, kept]
    assert np.array_equal(got, want, equal_nan=True)
    untouched = np.setdiff1d(np.arange(total), dst[kept])
    bits = lambda t: t.view(3, 2, total, -1)[:, :, torch.tensor(untouched, device="cuda")]  # noqa: E731
    assert torch.equal(bits(back.bits), bits(before))
    for x in (arena, back, a):
        x.release()


@pytest.mark.gpu
def test_slots_past_four_gib_of_records():
    """A packed arena whose records lie past 32-bit offsets."""
    shape = dataclasses.replace(P.BF16, num_layers=1)
    blocks = (1 << 33) // (17 * 128 * shape.num_kv_heads)  # 8 GiB
    n = kvr.kv_packed_bytes(shape, 16, blocks)
    raw = torch.zeros(n, dtype=torch.uint8, device="cuda")
    h = kvr.kv_packed_bind(raw.data_ptr(), n, shape, 16, blocks)
    slots = np.array([0, blocks * 16 - 1, blocks * 4 + 3, blocks * 8 + 5])
    k, v = rows_of(shape, 4, 7, special=False), rows_of(shape, 4, 8, special=False)
    kd, vd, sl = k.cuda(), v.cuda(), torch.tensor(slots, device="cuda")
    w = shape.num_kv_heads * 128
    out = torch.zeros(2, 4, w, dtype=torch.bfloat16, device="cuda")
    kvr.kv_packed_store(h, 0, kd.data_ptr(), w, vd.data_ptr(), w, sl.data_ptr(), 4, Hn.stream_ptr())
    kvr.kv_packed_load(h, 0, out[0].data_ptr(), w, out[1].data_ptr(), w, sl.data_ptr(), 4, Hn.stream_ptr())
    torch.cuda.synchronize()
    for got, x in zip(out, (k, v)):
        want = P.values(*P.quantise(x.float().numpy().astype(np.float64))).reshape(4, -1)
        assert np.array_equal(got.float().cpu().numpy(), want)
    # the four slots' records alone were written
    assert int((raw.view(-1, 17 * 128) != 0).any(1).sum()) == 4 * shape.num_kv_heads
    kvr.kv_packed_release(h)


# ---- refusals (no device access) ------------------------------------------
def status(call, *a, **kw):
    with pytest.raises(kvr.KvError) as e:
        call(*a, **kw)
    assert e.value.message
    return e.value.status


def test_packed_bytes():
    s = W.LLAMA8B
    assert kvr.kv_packed_bytes(s, 16, 10) == 32 * 10 * 8 * 17 * 128
    assert kvr.kv_packed_bytes(s, 48, 10) == 3 * kvr.kv_packed_bytes(s, 16, 10)
    for bad in ((s, 0, 10), (s, -16, 10), (s, 8, 10), (s, 24, 10), (s, 16, 0), (s, 16, -3), (s, 16, 1 << 62),
                (dataclasses.replace(s, head_dim=64), 16, 10),
                (dataclasses.replace(W.TINY_F32, head_dim=16, num_kv_heads=8, num_q_heads=8), 16, 10)):
        assert kvr.kv_packed_bytes(*bad) == 0


def test_packed_bind_refusals(monkeypatch):
    s = W.TINY_BF16
    n = kvr.kv_packed_bytes(s, 16, 10)
    assert status(kvr.kv_packed_bind, 0, n, s, 16, 10) == kvr.KV_EINVAL
    assert status(kvr.kv_packed_bind, 0x10000, n - 1, s, 16, 10) == kvr.KV_EINVAL
    assert status(kvr.kv_packed_bind, 0x10008, n, s, 16, 10) == kvr.KV_EINVAL
    assert status(kvr.kv_packed_bind, 0x10000, n, s, 24, 10) == kvr.KV_EINVAL
    assert status(kvr.kv_packed_bind, 0x10000, n, dataclasses.replace(s, dtype=7), 16, 10) == kvr.KV_EINVAL
    monkeypatch.setenv("KVR_DEBUG_FAIL_PROBE", "1")
    assert status(kvr.kv_packed_bind, 0x10000, n, s, 16, 10) == kvr.KV_EDEVICE


def test_unknown_packed_handles_are_refused():
    assert status(kvr.kv_packed_release, 0x1234) == kvr.KV_ESTATE
    assert status(kvr.kv_packed_store, 0x1234, 0, 0x1000, 256, 0x2000, 256, 0x3000, 1) == kvr.KV_ESTATE
    assert status(kvr.kv_packed_load, 0x1234, 0, 0x1000, 256, 0x2000, 256, 0x3000, 1) == kvr.KV_ESTATE
    assert status(kvr.kv_packed_park, 0x1234, 0x1000, 0x1234, 0x2000, 1) == kvr.KV_ESTATE
    assert status(kvr.kv_packed_restore, 0x1234, 0x1000, 0x1234, 0x2000, 1) == kvr.KV_ESTATE


@pytest.mark.gpu
def test_packed_refusals_on_live_handles():
    shape = P.BF16
    a = P.PackedArena(shape, 16, 4)
    w = shape.num_kv_heads * 128
    ok = dict(packed=a.handle, layer=0, k=0x1000, k_stride=w, v=0x2000, v_stride=w, slots=0x3000, rows=2)
    for bad in (dict(layer=-1), dict(layer=2), dict(rows=-1), dict(rows=1 << 31), dict(k=0), dict(v=0), dict(slots=0),
                dict(k_stride=w - 2), dict(v_stride=w - 2), dict(k_stride=w + 1), dict(k=0x1002), dict(slots=0x3004)):
        for call in (kvr.kv_packed_store, kvr.kv_packed_load):
            assert status(call, **{**ok, **bad}) == kvr.KV_EINVAL
    wl = W.small_workload(shape, [5], seed=1)
    arena = bound_arena(shape, wl)
    other = bound_arena(W.TINY_BF16, W.small_workload(W.TINY_BF16, [5], seed=1))
    assert status(kvr.kv_packed_park, other.handle, 0x1000, a.handle, 0x2000, 1) == kvr.KV_ESTATE
    for args in ((0, 0x2000, 1), (0x1000, 0, 1), (0x1000, 0x2000, -1), (0x1000, 0x2000, 1 << 31), (0x1004, 0x2000, 1)):
        s, p, n = args
        assert status(kvr.kv_packed_park, arena.handle, s, a.handle, p, n) == kvr.KV_EINVAL
        assert status(kvr.kv_packed_restore, a.handle, p, arena.handle, s, n) == kvr.KV_EINVAL
    for x in (arena, other, a):
        x.release()
    assert status(kvr.kv_packed_store, **ok) == kvr.KV_ESTATE
