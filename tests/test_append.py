"""Rows of q, k and v into the arena (kv_append, include/kvr_append.h) against the
formula in 64 bits.

Tolerance, with u = 2^-24, a and b a pair of the head with its bias:
  the bias adds u of |x| + |bias|; the norm is a sum of d squares (d u), halved by the
  root, its division and root (3 u) and two products (2 u);
  a turned value is two products and a sum with a cosine and a sine rounded once (u) of an
  angle that is off by 2^-48 of itself (the reference's own rounding among it), so at most
  (4 u + 2^-48 angle + 2^-46) (|a| + |b|);
then half a step of the output type and its least number."""
import dataclasses

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_14635_amd import harness as Hn  # noqa: E402
from paper_2608_14635_amd import kvr  # noqa: E402
from paper_2608_14635_amd import workloads as W  # noqa: E402

U = 2.0 ** -24
KEPT = 7.0
NAMES = ("q_norm", "k_norm", "bq", "bk", "bv")


def shape_of(name, qk_norm=False, qkv_bias=False, g=4):
    if name == "bf16":
        s = dataclasses.replace(W.TINY_BF16, num_layers=2, num_q_heads=2 * g, num_kv_heads=2)
    else:
        d = int(name[4:])
        s = dataclasses.replace(W.TINY_F32, num_layers=2, num_q_heads=g * 256 // d, num_kv_heads=256 // d, head_dim=d)
    return dataclasses.replace(s, qk_norm=qk_norm, qkv_bias=qkv_bias, rope_theta=5e5)


def torch_dtype(shape):
    return torch.bfloat16 if shape.dtype == W.BF16 else torch.float32


def to64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Rows:
    """Rows of one product, q, k and v side by side, and an arena of arbitrary bits."""

    def __init__(self, shape, rows, B=16, seed=0, layer=1, far=5000, blocks=None, lead=2, pad=2):
        self.shape, self.rows, self.B, self.layer = shape, rows, B, layer
        nq, nkv, d = shape.num_q_heads, shape.num_kv_heads, shape.head_dim
        dt = torch_dtype(shape)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        rand = lambda *n: torch.randn(*n, generator=g, device="cuda").mul_(1.3).to(dt)  # noqa: E731
        self.blocks = blocks or rows // B + 3
        slots = self.blocks * B
        n = 2 * shape.num_layers * slots * nkv * d
        lead //= 1 if dt == torch.bfloat16 else 2  # 4 bytes
        self.raw = rand(n + 2 * lead)  # the arena starts on a boundary of 4 bytes, a guard behind it
        self.arena = self.raw[lead:lead + n]
        self.handle = kvr.kv_arena_bind(self.arena.data_ptr(), n * self.arena.element_size(), shape, B, self.blocks)
        width = (nq + 2 * nkv) * d
        self.width = width + pad
        self.flat = rand(rows * self.width + lead)
        self.x = self.flat[lead:].view(rows, self.width)
        self.slots = torch.randperm(slots, generator=g, device="cuda")[:rows]
        self.positions = torch.randint(0, far, (rows,), generator=g, device="cuda", dtype=torch.int32)
        self.q_out = torch.full((rows, nq * d + pad), KEPT, dtype=dt, device="cuda")
        self.weights = {}
        if shape.qk_norm:
            self.weights.update({k: 1 + 0.1 * rand(d) for k in NAMES[:2]})
        if shape.qkv_bias:
            self.weights.update({k: rand((nq if k == "bq" else nkv) * d) for k in NAMES[2:]})

    def run(self, with_q=True, in_place=False, stream=None):
        s = self.shape
        nq, nkv, d = s.num_q_heads, s.num_kv_heads, s.head_dim
        at, e, w = self.x.data_ptr(), self.x.element_size(), self.x.stride(0)
        out, out_w = (at, w) if in_place else (self.q_out.data_ptr(), self.q_out.stride(0))
        kvr.kv_append(self.handle, self.layer, {k: t.data_ptr() for k, t in self.weights.items()}, at if with_q else 0,
                      w, at + nq * d * e, w, at + (nq + nkv) * d * e, w, self.positions.data_ptr(),
                      self.slots.data_ptr(), self.rows, out if with_q else 0, out_w,
                      Hn.stream_ptr() if stream is None else stream)

    def reference(self):
        """Heads [rows, nq + 2 nkv, d] and their tolerance, 64 bits."""
        s = self.shape
        nq, nkv, d = s.num_q_heads, s.num_kv_heads, s.head_dim
        n = nq + 2 * nkv
        x = to64(self.x)[:, :n * d].reshape(self.rows, n, d)
        err = np.zeros_like(x)
        w = {k: to64(t) for k, t in self.weights.items()}
        if s.qkv_bias:
            bias = np.concatenate([w["bq"], w["bk"], w["bv"]]).reshape(n, d)
            err += U * (np.abs(x) + np.abs(bias))
            x = x + bias
        qk = slice(0, nq + nkv)
        if s.qk_norm:
            gain = np.concatenate([np.tile(w["q_norm"], (nq, 1)), np.tile(w["k_norm"], (nkv, 1))])
            inv = 1 / np.sqrt((x[:, qk] ** 2).mean(-1, keepdims=True) + s.rms_eps)
            # a bias's rounding moves the norm by its largest share
            moved = np.sqrt((err[:, qk] ** 2).sum(-1, keepdims=True) / np.maximum((x[:, qk] ** 2).sum(-1, keepdims=True), 1e-300))
            new = x[:, qk] * inv * gain
            err[:, qk] = err[:, qk] * inv * np.abs(gain) + np.abs(new) * ((d / 2 + 6) * U + moved)
            x[:, qk] = new
        pos = self.positions.cpu().numpy().astype(np.float64)
        angle = pos[:, None, None] * s.rope_theta ** (-2.0 * np.arange(d // 2) / d)
        cos, sin = np.cos(angle), np.sin(angle)
        a, b = x[:, qk, :d // 2].copy(), x[:, qk, d // 2:].copy()
        ea, eb = err[:, qk, :d // 2].copy(), err[:, qk, d // 2:].copy()
        off = (4 * U + 2.0 ** -48 * angle + 2.0 ** -46) * (np.abs(a) + np.abs(b)) + ea + eb
        x[:, qk, :d // 2], x[:, qk, d // 2:] = a * cos - b * sin, b * cos + a * sin
        err[:, qk, :d // 2], err[:, qk, d // 2:] = off, off
        return x, err + torch.finfo(torch_dtype(s)).eps / 2 * np.abs(x) + 1e-37

    def planes(self, raw=None):
        s = self.shape
        a = self.arena if raw is None else raw
        return a.view(s.num_layers, 2, self.blocks * self.B, s.num_kv_heads, s.head_dim)

    def check(self, before, stored, turned, want=None):
        """`before`: the whole memory; stored, turned: rows whose K/V, whose q is written."""
        s = self.shape
        nq, nkv, d = s.num_q_heads, s.num_kv_heads, s.head_dim
        x, tol = self.reference() if want is None else want
        lead = (len(self.raw) - len(self.arena)) // 2
        bits = torch.int16 if self.raw.dtype == torch.bfloat16 else torch.int32
        kept = torch.ones(self.raw.shape, dtype=torch.bool, device="cuda")
        self.planes(kept[lead:lead + len(self.arena)])[self.layer, :, self.slots[stored]] = False
        assert torch.equal(self.raw.view(bits)[kept], before.view(bits)[kept])
        got = to64(self.planes()[self.layer][:, self.slots[stored]])
        st = stored.cpu().numpy()
        for i, part in enumerate((slice(nq, nq + nkv), slice(nq + nkv, None))):
            assert_close(got[i], x[st, part], tol[st, part])
        tu = turned.cpu().numpy()
        out = to64(self.q_out)
        assert_close(out[tu, :nq * d].reshape(-1, nq, d), x[tu, :nq], tol[tu, :nq])
        assert (out[~tu] == KEPT).all() and (out[:, nq * d:] == KEPT).all()

    def release(self):
        kvr.kv_arena_release(self.handle)


def assert_close(got, want, tol):
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan)
    with np.errstate(invalid="ignore"):
        bad = ~nan & ~(np.abs(got - want) <= tol) & ~(got == want)
    assert not bad.any(), (int(bad.sum()), float(np.abs(got - want)[bad].max()), float(tol[bad].min()))


def all_rows(r):
    return torch.ones(r.rows, dtype=torch.bool, device="cuda")


def run_and_check(r, **kw):
    before = r.raw.clone()
    r.run(**kw)
    torch.cuda.synchronize()
    r.check(before, all_rows(r), all_rows(r) if kw.get("with_q", True) else ~all_rows(r))
    r.release()


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["bf16", "f32_16", "f32_32", "f32_64", "f32_128"])
@pytest.mark.parametrize("variant", ["", "norm", "bias", "both"])
@pytest.mark.parametrize("rows", [1, 5, 67])
def test_rows(name, variant, rows):
    if "f32_16" == name and variant in ("norm", "both"):
        return  # such a model is refused
    s = shape_of(name, variant in ("norm", "both"), variant in ("bias", "both"), g=3 if rows == 5 else 4)
    run_and_check(Rows(s, rows, B=16 if rows > 1 else 24, seed=rows))


@pytest.mark.gpu
@pytest.mark.parametrize("name,rows", [("bf16", 1025), ("bf16", 2048), ("bf16", 4097), ("f32_64", 2051), ("f32_16", 2500),
                                       ("f32_32", 2049), ("f32_128", 2050)])
def test_many_rows(name, rows):
    run_and_check(Rows(shape_of(name, name != "f32_16", True), rows, seed=rows))


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["bf16", "f32_64"])
@pytest.mark.parametrize("far", [1, 200000, 2 ** 31 - 1])
def test_positions(name, far):
    r = Rows(shape_of(name), 130, seed=far % 97, far=far)
    r.positions[0], r.positions[-1] = 0, far if far < 2 ** 31 else 2 ** 31 - 1
    run_and_check(r)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["bf16", "f32_32"])
@pytest.mark.parametrize("rows", [40, 1100, 2101])
def test_rows_that_are_passed_over(name, rows):
    """Negative positions; slots of -1, behind the arena, of 2^62 and of the least number."""
    r = Rows(shape_of(name, qk_norm=True, qkv_bias=True), rows, seed=3)
    r.positions[torch.tensor([0, 7, rows - 1])] = torch.tensor([-1, -2 ** 31, -5], dtype=torch.int32, device="cuda")
    r.slots[torch.tensor([2, 7, 9, 11, 12])] = torch.tensor([-1, 3, r.blocks * r.B, 1 << 62, -2 ** 63], device="cuda")
    before = r.raw.clone()
    r.run()
    torch.cuda.synchronize()
    turned = r.positions >= 0
    stored = turned & (r.slots >= 0) & (r.slots < r.blocks * r.B)
    assert int(turned.sum()) == rows - 3 and int(stored.sum()) == rows - 7
    r.check(before, stored, turned)
    r.release()


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["bf16", "f32_64"])
def test_k_and_v_alone(name):
    run_and_check(Rows(shape_of(name, True, True), 33, seed=4), with_q=False)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [9, 1200, 2050])
def test_over_the_queries(rows):
    r = Rows(shape_of("bf16", True), rows, seed=5)
    r.run()
    torch.cuda.synchronize()
    want, x = r.q_out.clone(), r.x.clone()
    w = r.shape.num_q_heads * 128
    r.run(in_place=True)
    torch.cuda.synchronize()
    assert torch.equal(r.x[:, :w], want[:, :w]) and torch.equal(r.x[:, w:], x[:, w:])
    r.release()


@pytest.mark.gpu
def test_values_that_are_not_finite():
    """They stay in their pair, or in their head where it is normed."""
    for norm in (False, True):
        r = Rows(shape_of("bf16", norm), 6, seed=6)
        d, nq = 128, r.shape.num_q_heads
        clean = r.reference()
        bad = [(1, 3, float("nan")), (2, nq, float("inf")), (3, nq + 3, float("-inf"))]  # a q, a k and a v head
        for row, h, x in bad:
            r.x[row, h * d + 5] = x
        before = r.raw.clone()
        r.run()
        torch.cuda.synchronize()
        heads = np.concatenate([to64(r.q_out)[:, :nq * d].reshape(6, nq, d),
                                np.moveaxis(to64(r.planes()[1][:, r.slots]), 0, 1).reshape(6, -1, d)], 1)
        kept = np.ones(heads.shape, bool)
        for row, h, x in bad:
            touched = [5] if h == nq + 3 else range(d) if norm else [5, 69]
            kept[row, h, touched] = False
            assert not np.isfinite(heads[row, h, [5] if norm else touched]).any()
        assert (np.abs(heads - clean[0]) <= clean[1])[kept].all()
        assert not torch.equal(before, r.raw)
        r.release()


@pytest.mark.gpu
def test_slots_past_four_gib():
    s = dataclasses.replace(shape_of("bf16"), num_layers=1)
    blocks = (5 << 30) // (2 * 2 * 128 * 16)  # a plane of 5 GiB
    arena = torch.empty(2 * blocks * 16 * 2 * 128, dtype=torch.bfloat16, device="cuda")
    h = kvr.kv_arena_bind(arena.data_ptr(), arena.numel() * 2, s, 16, blocks)
    r = Rows(s, 20, seed=8, layer=0)
    r.run()
    want = r.planes()[0][:, r.slots].clone()
    far = blocks * 16 - 1 - torch.arange(20, device="cuda") * (blocks * 16 // 21)
    near, r.slots, handle, r.handle = r.slots, far, r.handle, h
    r.run()
    torch.cuda.synchronize()
    assert torch.equal(arena.view(2, -1, 2, 128)[:, far], want)
    r.handle = handle
    r.release()
    kvr.kv_arena_release(h)


@pytest.mark.gpu
def test_captured_calls_follow_their_arrays():
    r = Rows(shape_of("bf16", True, True), 70, seed=9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        r.run()
    for step in range(3):
        r.positions.copy_(torch.randint(-3, 90000, (70,), device="cuda"))
        r.slots.copy_(torch.randperm(r.blocks * r.B, device="cuda")[:70])
        r.x.copy_(torch.randn(r.x.shape, device="cuda"))
        r.q_out.fill_(KEPT)
        before = r.raw.clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        r.check(before, r.positions >= 0, r.positions >= 0)
    r.release()


@pytest.mark.gpu
def test_two_streams_at_once():
    """Calls on two layers of one arena, and on the same rows."""
    rs = Rows(shape_of("bf16"), 300, seed=10)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    torch.cuda.synchronize()
    for layer, s in enumerate(streams):
        with torch.cuda.stream(s):
            rs.layer, rs.q_out = layer, torch.full_like(rs.q_out, KEPT)
            rs.run(stream=s.cuda_stream)
            outs.append(rs.q_out)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
    p = rs.planes()
    assert torch.equal(p[0][:, rs.slots], p[1][:, rs.slots])
    rs.release()


# ---- refusals ---------------------------------------------------------------
def test_append_to_an_unknown_arena_is_refused():
    with pytest.raises(kvr.KvError) as e:
        kvr.kv_append(0x1234, 0, None, 0x1000, 1024, 0x2000, 256, 0x3000, 256, 0x4000, 0x5000, 1, 0x6000, 1024)
    assert e.value.status == kvr.KV_ESTATE


@pytest.mark.gpu
def test_refusals():
    w = {k: 0x100 * (i + 1) for i, k in enumerate(NAMES)}
    r = Rows(shape_of("bf16", True, True), 2, seed=1)
    ok = dict(arena=r.handle, layer=0, layer_weights=w, q=0x1000, q_stride=1024, k=0x2000, k_stride=256, v=0x3000,
              v_stride=256, positions=0x4000, slots=0x5000, rows=2, q_out=0x6000, q_out_stride=1024)
    bads = [dict(layer=-1), dict(layer=2), dict(rows=-1), dict(rows=1 << 31), dict(k=0), dict(v=0), dict(positions=0),
            dict(slots=0), dict(q=0), dict(q_out=0), dict(q_stride=1022), dict(k_stride=254), dict(v_stride=254),
            dict(q_out_stride=1022), dict(q_stride=1025), dict(k_stride=257), dict(q=0x1002), dict(k=0x2002),
            dict(q_out=0x6002), dict(positions=0x4002), dict(slots=0x5004), dict(layer_weights=None),
            dict(k_stride=1 << 61), dict(q=0x6000, q_stride=1026)]
    bads += [dict(layer_weights={**w, k: 0}) for k in NAMES] + [dict(layer_weights={**w, "bk": 0x102})]
    for bad in bads:
        with pytest.raises(kvr.KvError) as e:
            kvr.kv_append(**{**ok, **bad})
        assert e.value.status == kvr.KV_EINVAL, bad
    kvr.kv_append(**{**ok, "rows": 0})  # nothing to do
    r.release()
    with pytest.raises(kvr.KvError) as e:
        kvr.kv_append(**ok)
    assert e.value.status == kvr.KV_ESTATE
