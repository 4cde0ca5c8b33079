"""The resumed decode step over a packed arena (kv_packed_decode_step), and the
serving operators in one run: tables grown on the GPU, rebuilt K/V parked, steps
taken over the packed arena, their tokens' log probabilities read off the logits.

The step is compared with the same decoder in 64 bits (roundings at the library's
declared sites), which takes the K/V of every position, the new one's included, as
the packed arena holds them; the new rows' codes are compared with those of the
reference's own K and V.  Tolerances are the decode step's: 1e-4 (fp32) and 2e-2
(bf16) of the largest logit.  A code differs where a K or V one rounding away falls
on the other side of a border: a bf16 step is 2^-8 of a value, a code's at least a
sixth of it, so no code is further than one off, and less than 2^-8 * 6 = 2.4 % of
them at the most, were every value a step off; in fp32 a 1e-4th of that."""
import dataclasses

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_14635_amd import harness as Hn  # noqa: E402
from paper_2608_14635_amd import kvr  # noqa: E402
from paper_2608_14635_amd import workloads as W  # noqa: E402

import packed_util as P  # noqa: E402
import parity_util as PU  # noqa: E402
import test_gpu_decode as TD  # noqa: E402

CASES = {
    "tiny_f32": (W.TINY_F32, [1, 6, 23, 100], 16),
    "tiny_bf16": (W.TINY_BF16, [1, 6, 23, 300], 16),
    "tiny_bf16_b48_40req": (W.TINY_BF16.with_layers(2), [1 + (7 * i) % 90 for i in range(40)], 48),
    "tiny_bf16_70req": (dataclasses.replace(W.TINY_BF16, num_layers=2, vocab=1024), [1 + (5 * i) % 60 for i in range(70)], 16),
    "qwen3_8b_2l": (TD.SHAPES["qwen3_8b_2l"], [1, 6, 23, 300], 32),
    "qwen25_1_5b_2l": (TD.SHAPES["qwen25_1_5b_2l"], [2, 40, 150], 16),
    "g16_bf16": (TD.SHAPES["g16_bf16"], [1, 33, 90], 16),
}
STEPS = 2


def dev(a, dtype=torch.int32):
    return torch.tensor(np.asarray(a), dtype=dtype, device="cuda")


class Tables:
    """Block tables kept on the device, grown with kv_tables_grow."""

    def __init__(self, R, B, wide, blocks, seed):
        self.B, self.R = B, R
        self.tables = torch.full((R, wide), -1, dtype=torch.int32, device="cuda")
        self.free = dev(np.random.default_rng(seed).permutation(blocks))
        self.taken = 0
        self.held = torch.zeros(R, dtype=torch.int32, device="cuda")

    def grow(self, lens, max_rows):
        lens = dev(lens)
        off = torch.empty(self.R + 1, dtype=torch.int32, device="cuda")
        slots = torch.empty(max_rows, dtype=torch.int64, device="cuda")
        counts = torch.empty(4, dtype=torch.int32, device="cuda")
        free = self.free[self.taken:]
        kvr.kv_tables_grow(self.held.data_ptr(), lens.data_ptr(), self.R, self.B, free.data_ptr(), len(free),
                           self.tables.data_ptr(), self.tables.shape[1], max_rows, off.data_ptr(), slots.data_ptr(),
                           0, counts.data_ptr(), stream=Hn.stream_ptr())
        taken, lacked, rows, unplaced = counts.tolist()
        assert lacked == 0 and unplaced == 0 and rows == max_rows
        self.taken += taken
        self.held = lens
        return slots


def reference_step(shape, w, head, tokens, positions, tables, B, parts):
    """Logits [R, vocab] and the new K, V [L, R, nkv, d], 64 bits; parts: the packed
    arena's codes and scales after the step."""
    H, d, nq, nkv = shape.hidden, shape.head_dim, shape.num_q_heads, shape.num_kv_heads
    kc, vc, ks, vs = parts
    wide = lambda x: x.astype(np.float32).astype(np.float64)  # noqa: E731
    if shape.dtype == W.BF16:
        rnd = lambda x: W.bf16_bits_to_f32(W.f32_to_bf16_bits(x.astype(np.float32))).astype(np.float64)  # noqa: E731
    else:
        rnd = wide
    norm = lambda x, gain: x / np.sqrt((x * x).mean(-1, keepdims=True) + shape.rms_eps) * gain  # noqa: E731
    pos = np.asarray(positions, np.float64)
    ang = pos[:, None] * float(shape.rope_theta) ** (-np.arange(0, d, 2) / d)
    c, s = wide(np.cos(ang))[:, None], wide(np.sin(ang))[:, None]

    def rope(x):
        a, b = x[..., :d // 2], x[..., d // 2:]
        return np.concatenate([a * c - b * s, b * c + a * s], -1)
    x = w["embed"][tokens].astype(np.float64)
    R, new = len(tokens), ([], [])
    for l, lw in enumerate(w["layers"]):
        lw = {k: np.asarray(v, np.float64) for k, v in lw.items()}
        a = rnd(norm(x, lw["attn_norm"]))
        q, k, v = (a @ lw[n].T + (lw[b] if shape.qkv_bias else 0) for n, b in (("wq", "bq"), ("wk", "bk"), ("wv", "bv")))
        q, k, v = q.reshape(R, nq, d), k.reshape(R, nkv, d), v.reshape(R, nkv, d)
        if shape.qk_norm:
            q, k = norm(q, lw["q_norm"]), norm(k, lw["k_norm"])
        q, k, v = rnd(rope(q)), rnd(rope(k)), rnd(v)
        new[0].append(k)
        new[1].append(v)
        o = np.zeros((R, nq, d))
        for r in range(R):
            j = np.arange(positions[r] + 1)
            slots = tables[r, j // B].astype(np.int64) * B + j % B
            K, V = P.values(kc[l, slots], ks[l, slots]), P.values(vc[l, slots], vs[l, slots])
            for h in range(nq):
                z = K[:, h // (nq // nkv)] @ q[r, h] / np.sqrt(d)
                p = np.exp(z - z.max())
                o[r, h] = p @ V[:, h // (nq // nkv)] / p.sum()
        x = x + rnd(o).reshape(R, nq * d) @ lw["wo"].T
        b = rnd(norm(x, lw["ffn_norm"]))
        gate = b @ lw["w_gate"].T
        x = x + rnd(gate / (1 + np.exp(-gate)) * (b @ lw["w_up"].T)) @ lw["w_down"].T
    logits = rnd(norm(x, np.asarray(head["final_norm"], np.float64))) @ np.asarray(head["lm_head"], np.float64).T
    return logits, np.stack(new[0]), np.stack(new[1])


def check_codes(shape, parts, slots, k, v):
    share = 0.024 if shape.dtype == W.BF16 else 2.4e-6 * 100
    for codes, scales, x in ((parts[0], parts[2], k), (parts[1], parts[3], v)):
        got = P.values(codes[:, slots], scales[:, slots])
        want_codes, want_scales = P.quantise(x)
        want = P.values(want_codes, want_scales)
        # a code's step is at most 2 scales of the group; a scale may itself be one off
        step = np.repeat(2 * 2.0 ** (np.maximum(scales[:, slots], want_scales) - 127.0), 32, axis=-1)
        assert (np.abs(got - want) <= 2 * step).all()
        same_scale = np.repeat(scales[:, slots] == want_scales, 32, axis=-1)
        assert (got != want)[same_scale].mean() <= share
        assert (~same_scale).mean() <= 0.05


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(CASES))
def test_rebuild_park_decode_and_logprobs(name):
    shape, prefix, B = CASES[name]
    R, tol = len(prefix), PU.TOL[shape.dtype]
    wl = TD.resume_workload(shape, prefix, steps=STEPS, seed=901)
    pre, last = TD.split_last(wl)
    host_w, head = W.host_weights(shape, seed=902), W.host_head_weights(shape, seed=903)
    f = W.weights_as_f32(host_w, shape.dtype)
    fh = {k: W.bf16_bits_to_f32(a) if shape.dtype == W.BF16 else a for k, a in head.items()}
    model, hd = Hn.device_model_from_host(shape, host_w), Hn.device_head_from_host(shape, head)
    # the prefixes rebuilt in the retained arena, then parked
    arena = Hn.DeviceArena(wl)
    arena.bind()
    n = int(pre.lens.sum())
    ws, nbytes = Hn.alloc_workspace(shape, R, n, n)
    kvr.kv_rebuild(model.weights, pre.tokens, pre.lens, wl.block_tables, arena.handle, ws.data_ptr(), nbytes,
                   Hn.stream_ptr())
    lens = np.array(pre.lens, np.int64)
    blocks = int((-(-(lens + STEPS) // B)).sum()) + 2
    packed = P.PackedArena(shape, B, blocks, seed=5)
    tabs = Tables(R, B, int((-(-(lens + STEPS) // B)).max()), blocks, 6)
    to = tabs.grow(lens, n)
    src = dev(np.concatenate([wl.block_tables[r, np.arange(m) // 16].astype(np.int64) * 16 + np.arange(m) % 16
                              for r, m in enumerate(lens)]), torch.int64)
    kvr.kv_packed_park(arena.handle, src.data_ptr(), packed.handle, to.data_ptr(), n, Hn.stream_ptr())
    # greedy steps over the packed arena
    size = kvr.kv_packed_decode_workspace_bytes(shape, R, int(lens.max()) + STEPS)
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    nxt = torch.zeros(R, dtype=torch.int32, device="cuda")
    logits = torch.zeros(R, shape.vocab, device="cuda")
    lp, ent = torch.zeros(R, device="cuda"), torch.zeros(R, device="cuda")
    lp_ws = torch.empty(kvr.kv_logprobs_workspace_bytes(R, shape.vocab, 3), dtype=torch.uint8, device="cuda")
    top_lp = torch.zeros(R, 3, device="cuda")
    top = torch.zeros(R, 3, dtype=torch.int32, device="cuda")
    tokens = last
    for step in range(STEPS):
        before = packed.raw.clone()
        slots = tabs.grow(lens + 1, R).cpu().numpy()
        tables = tabs.tables.cpu().numpy()
        kvr.kv_packed_decode_step(model.weights, hd["final_norm"].data_ptr(), hd["lm_head"].data_ptr(), tokens, lens,
                                  tables, packed.handle, ws.data_ptr(), size, nxt.data_ptr(), logits.data_ptr(),
                                  Hn.stream_ptr())
        kvr.kv_logprobs(logits.data_ptr(), kvr.KV_F32, R, shape.vocab, shape.vocab, 1.0, nxt.data_ptr(), 3, lp.data_ptr(),
                        ent.data_ptr(), top_lp.data_ptr(), top.data_ptr(), lp_ws.data_ptr(), lp_ws.numel(),
                        stream=Hn.stream_ptr())
        torch.cuda.synchronize()
        parts = packed.parts()
        # nothing but the new slots changed
        was = P.unpack(before.cpu().numpy()[:packed.n], shape, blocks, B)
        others = np.setdiff1d(np.arange(blocks * B), slots)
        for a, b in zip(parts, was):
            assert np.array_equal(a[:, others], b[:, others])
        want, k, v = reference_step(shape, f, fh, tokens, lens, tables, B, parts)
        check_codes(shape, parts, slots, k, v)
        got = logits.cpu().numpy()
        worst = max(TD.rel(got[r], want[r]) for r in range(R))
        TD.say(f"{name} step {step}: logits off by {worst:.1e}")
        assert worst <= tol
        TD.assert_valid_argmax(nxt.cpu().numpy(), want, tol)
        # the tokens taken are the likeliest, and their log probabilities the logits'
        assert torch.equal(top[:, 0], nxt) and torch.equal(top_lp[:, 0], lp)
        ref = torch.log_softmax(logits.double(), -1)
        near = (lp.double() - ref.gather(1, nxt.long()[:, None])[:, 0]).abs()
        assert (near <= 1e-5).all() and (ent.double() + (ref * ref.exp()).sum(-1)).abs().max() <= 1e-4
        tokens, lens = nxt.cpu().numpy(), lens + 1
    arena.release()
    packed.release()


@pytest.mark.gpu
def test_a_captured_serving_step():
    """Tables grown, rows stored, attended over and scored inside one graph, replayed
    as the lengths grow; every replay equals the same calls made eagerly over a
    second arena."""
    shape = dataclasses.replace(P.BF16, num_layers=1)
    R, B, V, wide, blocks = 6, 16, 5000, 8, 60
    rng = np.random.default_rng(1)
    nkv, nq, d = shape.num_kv_heads, shape.num_q_heads, 128
    start = rng.integers(0, 40, size=R)

    class Side:
        def __init__(self):
            self.arena = P.PackedArena(shape, B, blocks, seed=2)
            self.held, self.lens = dev(np.zeros(R)), dev(start)
            self.tables = torch.full((R, wide), -1, dtype=torch.int32, device="cuda")
            self.free = dev(np.random.default_rng(3).permutation(blocks))
            self.n = int(start.sum()) + 20
            self.off, self.counts = dev(np.zeros(R + 1)), dev(np.zeros(4))
            self.slots = torch.zeros(self.n, dtype=torch.int64, device="cuda")
            self.k, self.v = (torch.zeros(self.n, nkv * d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            self.q = torch.zeros(R, nq * d, dtype=torch.bfloat16, device="cuda")
            self.out = torch.zeros_like(self.q)
            self.bytes = kvr.kv_packed_attention_workspace_bytes(shape, R, R, 1, wide * B)
            self.ws = torch.full((self.bytes,), 255, dtype=torch.uint8, device="cuda")
            self.logits, self.tok = torch.zeros(R, V, device="cuda"), dev(np.arange(R))
            self.lp = torch.zeros(R, device="cuda")
            self.lws = torch.zeros(kvr.kv_logprobs_workspace_bytes(R, V, 0), dtype=torch.uint8, device="cuda")

        def calls(self):
            s = Hn.stream_ptr()
            kvr.kv_tables_grow(self.held.data_ptr(), self.lens.data_ptr(), R, B, self.free.data_ptr(), blocks,
                               self.tables.data_ptr(), wide, self.n, self.off.data_ptr(), self.slots.data_ptr(), 0,
                               self.counts.data_ptr(), stream=s)
            kvr.kv_packed_store(self.arena.handle, 0, self.k.data_ptr(), nkv * d, self.v.data_ptr(), nkv * d,
                                self.slots.data_ptr(), self.n, s)
            kvr.kv_packed_attention(self.arena.handle, 0, self.q.data_ptr(), nq * d, 0, R, self.lens.data_ptr(),
                                    self.tables.data_ptr(), R, wide, 1, wide * B, self.out.data_ptr(), nq * d,
                                    self.ws.data_ptr(), self.bytes, s)
            kvr.kv_logprobs(self.logits.data_ptr(), kvr.KV_F32, R, V, V, 1.0, self.tok.data_ptr(), 0, self.lp.data_ptr(), 0,
                            0, 0, self.lws.data_ptr(), self.lws.numel(), stream=s)

        def feed(self, step):
            g = torch.Generator(device="cuda")
            g.manual_seed(step)
            for t in (self.k, self.v, self.q, self.logits):
                t.copy_(torch.randn(t.shape, generator=g, device="cuda"))

    a, b = Side(), Side()
    s = torch.cuda.Stream()
    a.feed(0)
    b.feed(0)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a.calls()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        a.calls()
    for step in range(5):
        for x in (a, b):
            x.feed(step)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        b.calls()
        torch.cuda.synchronize()
        for n in ("tables", "slots", "counts", "out", "lp"):
            assert torch.equal(getattr(a, n), getattr(b, n)), (step, n)
        assert torch.equal(a.arena.raw, b.arena.raw) and a.counts[1] == 0
        taken = int(a.counts[0])
        for x in (a, b):  # the step's blocks are gone from the list, its positions held
            x.free.copy_(torch.roll(x.free, -taken))
            x.held.copy_(x.lens)
            x.lens += dev([1, 0, 2, 1, 1, 3])
        torch.cuda.synchronize()
    a.arena.release()
    b.arena.release()


@pytest.mark.parametrize("name", ["tiny_f32", "qwen3_8b_2l", "g16_bf16"])
def test_packed_decode_workspaces_take_every_smaller_step(name):
    shape, rng = CASES[name][0], np.random.default_rng(6)
    for _ in range(1000):
        R, n = (int(2 ** rng.uniform(0, e)) for e in (8, 17))
        r, m = int(rng.integers(1, R + 1)), int(rng.integers(1, n + 1))
        for size in (kvr.kv_packed_decode_workspace_bytes, kvr.kv_decode_workspace_bytes):
            assert 0 < size(shape, r, m) <= size(shape, R, n)


def test_packed_decode_sizes_and_refusals():
    s = W.LLAMA8B
    a = kvr.kv_packed_decode_workspace_bytes(s, 4, 1000)
    assert 0 < a < kvr.kv_packed_decode_workspace_bytes(s, 16, 65536)
    for bad in ((s, 0, 10), (s, 4, 0), (dataclasses.replace(s, head_dim=64), 4, 10),
                (dataclasses.replace(W.TINY_F32, head_dim=16, num_q_heads=8, num_kv_heads=8), 4, 10)):
        assert kvr.kv_packed_decode_workspace_bytes(*bad) == 0
    w = kvr.Weights(kvr.make_desc(s), 0x1000, [{k: 0x1000 for k in kvr.LAYER_FIELDS}] * s.num_layers)
    with pytest.raises(kvr.KvError) as e:
        kvr.kv_packed_decode_step(w, 0x1000, 0x1000, [1], [0], [[0]], 0x1234, 0x10000, 1 << 30, 0x2000)
    assert e.value.status == kvr.KV_ESTATE


@pytest.mark.gpu
def test_packed_decode_refusals_on_a_live_arena():
    s = W.TINY_BF16
    a = P.PackedArena(s, 16, 4)
    before = a.raw.clone()
    w = kvr.Weights(kvr.make_desc(s), 0x1000, [{k: 0x1000 for k in kvr.LAYER_FIELDS}] * s.num_layers)
    ok = dict(weights=w, final_norm=0x1000, lm_head=0x1000, tokens=[1, 2], positions=[3, 20], tables=[[0, -1], [1, 2]],
              packed=a.handle, workspace=0x10000, workspace_bytes=1 << 34, next_tokens=0x2000)
    other = kvr.Weights(kvr.make_desc(W.TINY_F32), 0x1000, [{k: 0x1000 for k in kvr.LAYER_FIELDS}] * 2)
    for bad, st in ((dict(tokens=[1, s.vocab]), kvr.KV_ERANGE), (dict(positions=[3, -1]), kvr.KV_EINVAL),
                    (dict(positions=[3, 40]), kvr.KV_ECAPACITY), (dict(tables=[[0, -1], [1, 4]]), kvr.KV_ERANGE),
                    (dict(tables=[[2, -1], [1, 2]]), kvr.KV_EALIAS), (dict(next_tokens=0), kvr.KV_EINVAL),
                    (dict(final_norm=0), kvr.KV_EINVAL), (dict(workspace=0), kvr.KV_EINVAL),
                    (dict(workspace=0x10008), kvr.KV_EINVAL), (dict(workspace_bytes=1000), kvr.KV_ENOMEM),
                    (dict(weights=other), kvr.KV_ESTATE)):
        with pytest.raises(kvr.KvError) as e:
            kvr.kv_packed_decode_step(**{**ok, **bad})
        assert e.value.status == st, bad
    kvr.kv_packed_decode_step(**{**ok, "tokens": [], "positions": [], "tables": np.zeros((0, 0), np.int32)})
    torch.cuda.synchronize()
    assert torch.equal(a.raw, before)
    a.release()
