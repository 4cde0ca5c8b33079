"""The performance cases of the serving operators beside the KV rebuild: what a
rollout worker calls around a decode step.

A case names one call:

  tables    kv_tables_grow: block tables and slot maps from the requests' lengths
  park      kv_packed_park, kv_packed_restore: interrupted requests' K/V put from
            the arena into a packed one (4-bit values, one power of two for 32) and
            brought back
  attend    kv_packed_attention: queries over a packed arena, through block tables
  logprob   kv_logprobs: log probabilities of given tokens, entropy, alternatives

Heads and vocabularies are those of the package's decoder shapes.  Lengths follow
the case's own `mix` number, everything else the seed.  Where `own` is false, the
same results are computed in their plain form, elementary torch operations.
"""
import math
import random

import torch

own = False

# heads, head dim and dtype of the decoder shapes
HEADS = {"tiny_f32": (4, 4, 64, "f32"), "tiny_bf16": (8, 2, 128, "bf16"), "qwen25_1_5b": (12, 2, 128, "bf16"),
         "llama8b": (32, 8, 128, "bf16"), "qwen14b": (40, 8, 128, "bf16"), "qwen3_32b": (64, 8, 128, "bf16")}
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
KV_STD = 1.3
TILE = 16     # slots of a packed tile
GROUP = 32    # values that share a scale
LOW_SCALE, HIGH_SCALE, NAN_SCALE = 7, 252, 255


def listed():
    return [
        # the tables of a whole batch before one decode step: a position each
        dict(name="tables_step", kind="tables", requests=64, low=200, high=16000, grow=1, block=16, mix=1),
        # the tables of a recovering worker's whole queue, every position new
        dict(name="tables_fill", kind="tables", requests=333, low=1, high=16384, grow=0, block=32, mix=2),
        # one interrupted request of a small model parked and brought back, every layer
        dict(name="park_one", kind="park", shape="qwen25_1_5b", layers=28, requests=1, low=171, high=171,
             block=16, mix=3),
        # a batch of the 8B shape parked, a few layers of it
        dict(name="park_batch", kind="park", shape="llama8b", layers=4, requests=16, low=1024, high=8192,
             block=16, mix=4),
        # the tiny fp32 decoder's heads, short ragged requests
        dict(name="attend_f32", kind="attend", shape="tiny_f32", requests=33, low=1, high=300, query=1,
             block=16, mix=5),
        # one request of about two thousand positions: latency
        dict(name="attend_one", kind="attend", shape="llama8b", requests=1, low=2001, high=2001, query=1,
             block=16, mix=6),
        # the whole batch over long contexts
        dict(name="attend_batch", kind="attend", shape="llama8b", requests=16, low=2048, high=16384, query=1,
             block=16, mix=7),
        # one to five drafted tokens of each request checked in one pass, 14B heads, 32-slot blocks
        dict(name="attend_draft", kind="attend", shape="qwen14b", requests=40, low=300, high=4000, query=5,
             block=32, mix=8),
        # two agentic requests of very long context
        dict(name="attend_long", kind="attend", shape="qwen14b", requests=2, low=150000, high=200000, query=1,
             block=16, mix=9),
        # a single request's step: its token's log probability and the five likeliest
        dict(name="logprob_one", kind="logprob", rows=1, vocab=151936, dtype="f32", pad=0, top=5, banned=0.0,
             scale=1.0, mix=10),
        # a batch's step, some tokens banned, the 20 likeliest
        dict(name="logprob_step", kind="logprob", rows=64, vocab=128256, dtype="f32", pad=0, top=20, banned=0.02,
             scale=1.25, mix=11),
        # a prompt's tokens scored from bf16 logits, rows on an odd stride
        dict(name="logprob_prompt", kind="logprob", rows=1024, vocab=151936, dtype="bf16", pad=3, top=0,
             banned=0.0, scale=1.0, mix=12),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    """One more case of the same ranges."""
    while True:
        kind = rng.choice(["tables", "park", "attend", "attend", "attend", "logprob", "logprob"])
        c = dict(kind=kind, mix=rng.randrange(1 << 20))
        if kind == "logprob":
            c.update(rows=_log_int(rng, 1, 1024), vocab=_log_int(rng, 1000, 152064),
                     dtype=rng.choice(["f32", "bf16"]), pad=rng.choice([0, 0, 1, 3, 8]),
                     top=rng.choice([0, 1, 5, 20, 64]), banned=rng.choice([0.0, 0.0, 0.02, 0.9]),
                     scale=rng.choice([1.0, 1.25, 0.7]))
            if c["rows"] * c["vocab"] <= (1 << 26 if c["top"] else 1 << 27):
                return c
            continue
        c.update(requests=_log_int(rng, 1, 256), block=rng.choice([16, 16, 32, 64]))
        c["high"] = _log_int(rng, 1, 32768)
        c["low"] = max(1, int(c["high"] * rng.uniform(0.02, 1.0)))
        if kind == "tables":
            c["requests"] = _log_int(rng, 1, 2048)
            c["block"] = rng.choice([8, 16, 16, 24, 32, 64])
            c["grow"] = rng.choice([0, 1, 1, 7, 300])
            c["scarce"] = rng.random() < 0.25  # the free list ends before the last request
        else:
            c["shape"] = rng.choice(list(HEADS))
        if kind == "park":
            c["layers"] = rng.randint(1, 8)
        if kind == "attend":
            c["query"] = rng.choice([1, 1, 1, 2, 4, 8])
        w, most = work(c), {"tables": 5.0e7, "park": 1.4e9, "attend": 3.5e8}[kind]
        # what the plain form spreads out: every context as long as the longest
        spread = c["requests"] * c["high"] * 1024 if kind == "attend" else 0
        if w["bytes"] <= most and spread <= 5.0e8:
            return c


# --------------------------------------------------------------------------
# Sizes of a case
# --------------------------------------------------------------------------
def _lens(case):
    rng = random.Random(case["mix"])
    return [rng.randint(case["low"], case["high"]) for _ in range(case["requests"])]


def _held(case, lens):
    """Positions placed before the call: all but `grow` of each request's (0: none)."""
    return [max(0, n - case["grow"]) if case["grow"] else 0 for n in lens]


def _queries(case, lens):
    """Query rows of each request."""
    rng = random.Random(case["mix"] + 1)
    return [min(n, rng.randint(1, case["query"])) for n in lens]


def _blocks(n, B):
    return (n + B - 1) // B


def work(case):
    kind = case["kind"]
    if kind == "logprob":
        e = 4 if case["dtype"] == "f32" else 2
        n = case["rows"] * case["vocab"]
        return {"bytes": float(n * e + case["rows"] * (12 + 8 * case["top"])), "flops": 6.0 * n}
    lens, B = _lens(case), case["block"]
    R = len(lens)
    if kind == "tables":
        held = _held(case, lens)
        rows = sum(lens) - sum(held)
        taken = sum(_blocks(n, B) - _blocks(h, B) for n, h in zip(lens, held))
        return {"bytes": float(12 * R + 8 * taken + 12 * rows), "flops": float(rows)}
    nq, nkv, d, dt = HEADS[case["shape"]]
    e = 4 if dt == "f32" else 2
    packed = 2 * nkv * (d // 2 + d // GROUP)  # bytes of a position
    if kind == "park":
        each = case["layers"] * (2 * 2 * nkv * d * e + 2 * packed) + 4 * 8
        return {"bytes": float(sum(lens) * each), "flops": float(sum(lens) * case["layers"] * 2 * nkv * d * 4)}
    qn = _queries(case, lens)
    pairs = sum(q * n - q * (q - 1) // 2 for q, n in zip(qn, lens))
    return {"bytes": float(sum(lens) * packed + 2 * sum(qn) * nq * d * e + 4 * sum(_blocks(n, B) for n in lens)),
            "flops": 4.0 * nq * d * pairs}


# --------------------------------------------------------------------------
# The packed layout, in torch.  Per layer, block, kv head and tile of 16 slots,
# 17 d bytes: K values [16][d/2], V values [4][16][4][d/32] (slots four by four, a
# sixteenth of the dims, slot), K scales [16][d/32], V scales [4][d/32][4].
# A byte holds two values, the even dim low: a sign and one of 0 .5 1 1.5 2 3 4 6.
# A scale byte s stands for 2^(s - 127), 255 for NaN.
# --------------------------------------------------------------------------
def _parts(packed, d):
    w = d // GROUP
    return (packed[..., :8 * d].unflatten(-1, (16, d // 2)),
            packed[..., 8 * d:16 * d].unflatten(-1, (4, 16, 4, w)),
            packed[..., 16 * d:16 * d + 16 * w].unflatten(-1, (16, w)),
            packed[..., 16 * d + 16 * w:].unflatten(-1, (4, w, 4)))


def _quantise(x):
    """x [n, nkv, d] fp32 -> bytes of two values [n, nkv, d/2], scale bytes [n, nkv, d/32].
    The scale is the least power of two that takes the group's largest magnitude to
    at most 6; values round to the nearest, ties to the even code."""
    g = x.unflatten(-1, (-1, GROUP))
    most = g.abs().amax(-1)
    frac, ex = torch.frexp(most)
    byte = (ex - torch.where(frac <= 0.75, 3, 2) + 127).clamp(LOW_SCALE, HIGH_SCALE)
    byte = torch.where(most > 0, byte, LOW_SCALE)
    a = (g * _two_to(254 - byte)[..., None]).abs()
    code = (a > 0.25).to(torch.uint8)
    for edge, up in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= edge) if up else (a > edge)
    code += 8 * (torch.signbit(g)).to(torch.uint8)
    byte = torch.where(torch.isfinite(most), byte, NAN_SCALE)
    code = code.flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), byte.to(torch.uint8)


def _two_to(byte):
    return (byte.to(torch.int32) << 23).view(torch.float32)


def _values(codes, scales, dtype=torch.float32):
    """The values that bytes [..., d/2] and scale bytes [..., d/32] stand for."""
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=dtype,
                         device=codes.device)
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).to(torch.int32)
    v = table[code].unflatten(-1, (-1, GROUP))
    s = torch.where(scales == NAN_SCALE, math.nan, _two_to(scales.clamp(max=254)).to(dtype))
    return (v * s[..., None]).flatten(-2)


def _slot_parts(slots, B):
    return slots // B, slots % B // TILE, slots % TILE


def _write_packed(packed, layer, k, v, slots, B):
    """Rows k, v [n, nkv, d] into their slots of packed [layers, blocks, nkv, tiles, 17 d]."""
    kc, vc, ks, vs = _parts(packed[layer], k.shape[-1])
    b, t, c = _slot_parts(slots, B)
    codes, scales = _quantise(k.float())
    kc[b, :, t, c], ks[b, :, t, c] = codes, scales
    codes, scales = _quantise(v.float())
    vc[b, :, t, c // 4, :, c % 4] = codes.unflatten(-1, (16, -1))
    vs[b, :, t, c // 4, :, c % 4] = scales


def _read_packed(packed, layer, slots, B, d):
    kc, vc, ks, vs = _parts(packed[layer], d)
    b, t, c = _slot_parts(slots, B)
    k = _values(kc[b, :, t, c], ks[b, :, t, c])
    return k, _values(vc[b, :, t, c // 4, :, c % 4].flatten(-2), vs[b, :, t, c // 4, :, c % 4])


# --------------------------------------------------------------------------
# Inputs, from the seed alone
# --------------------------------------------------------------------------
class _State(dict):
    """A worker's handles; the bindings are given back with it."""

    def __del__(self):
        for give_back, handle in self.pop("handles", ()):
            give_back(handle)


def _tables(lens, B, seed):
    """Block tables over a random order of an arena a quarter larger, and the number of its blocks."""
    need = [_blocks(n, B) for n in lens]
    total = sum(need) + max(2, sum(need) // 4)
    g = torch.Generator().manual_seed(seed)
    perm = torch.randperm(total, generator=g, dtype=torch.int64)
    tables = torch.full((len(lens), max(need)), -1, dtype=torch.int32)
    o = 0
    for r, k in enumerate(need):
        tables[r, :k] = perm[o:o + k]
        o += k
    return tables, total


def _all_slots(tables, lens, B):
    """Slots of every position of every request, request by request."""
    out = []
    for r, n in enumerate(lens):
        p = torch.arange(n)
        out.append(tables[r].long()[p // B] * B + p % B)
    return torch.cat(out)


def _randn(g, *shape, std=1.0, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).to(dtype)


def _inputs(case, seed):
    kind = case["kind"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if kind == "logprob":
        R, V, dt = case["rows"], case["vocab"], DTYPE[case["dtype"]]
        logits = _randn(g, R, V + case["pad"], std=3.0, dtype=dt)[:, :V]
        tokens = torch.randint(0, V, (R,), generator=g, device="cuda", dtype=torch.int32)
        if case["banned"]:
            kept = torch.rand(R, V, generator=g, device="cuda") >= case["banned"]
            kept[torch.arange(R, device="cuda"), tokens.long()] = True
            logits.masked_fill_(~kept, -math.inf)
        return dict(case=case, logits=logits, tokens=tokens)
    lens, B = _lens(case), case["block"]
    if kind == "tables":
        held = _held(case, lens)
        R, wide = len(lens), _blocks(case["high"], B)
        tables, total = _tables(lens, B, seed)
        free = []
        grown = torch.full((R, wide), -1, dtype=torch.int32)
        for r, (n, h) in enumerate(zip(lens, held)):
            k = _blocks(h, B)
            grown[r, :k] = tables[r, :k]
            free += tables[r, k:_blocks(n, B)].tolist()
        free = free[:len(free) * 2 // 3] if case.get("scarce") else free
        rows = sum(lens) - sum(held)
        return dict(case=case, held=torch.tensor(held, dtype=torch.int32, device="cuda"),
                    lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), tables=grown.cuda(),
                    free=torch.tensor(free or [0], dtype=torch.int32, device="cuda"), num_free=len(free),
                    max_rows=rows + 5)
    nq, nkv, d, dt = HEADS[case["shape"]]
    dt = DTYPE[dt]
    tables, total = _tables(lens, B, seed)
    slots = _all_slots(tables, lens, B).cuda()
    if kind == "park":
        L = case["layers"]
        arena = torch.empty(L, 2, total * B, nkv, d, dtype=dt, device="cuda")
        for l in range(L):
            arena[l].normal_(0.0, KV_STD, generator=g)
        to, packed_blocks = _tables(lens, 2 * B, seed + 1)  # the packed arena's blocks are its own
        return dict(case=case, arena=arena, back=torch.zeros_like(arena), slots=slots, blocks=total,
                    packed=torch.zeros(L, packed_blocks, nkv, 2 * B // TILE, 17 * d, dtype=torch.uint8,
                                       device="cuda"),
                    packed_slots=_all_slots(to, lens, 2 * B).cuda(), packed_blocks=packed_blocks)
    # attend: every slot outside the contexts holds arbitrary bytes
    packed = torch.randint(0, 256, (1, total, nkv, B // TILE, 17 * d), generator=g, device="cuda",
                           dtype=torch.uint8)
    for i in range(0, len(slots), 1 << 16):
        part = slots[i:i + (1 << 16)]
        k, v = (_randn(g, len(part), nkv, d, std=KV_STD) for _ in range(2))
        _write_packed(packed, 0, k, v, part, B)
    qn = _queries(case, lens)
    off = torch.cat([torch.zeros(1, dtype=torch.int64), torch.tensor(qn).cumsum(0)])
    return dict(case=case, packed=packed, blocks=total, q=_randn(g, sum(qn), nq, d, std=KV_STD, dtype=dt),
                offsets=off.to(torch.int32).cuda(), lens=torch.tensor(lens, dtype=torch.int32, device="cuda"),
                tables=tables.clamp(min=0).cuda(), rows=sum(qn), max_query=max(qn), max_len=max(lens))


def prepare(case, seed):
    st = _State(_inputs(case, seed))
    if not own:
        return st
    import dataclasses

    from paper_2608_14635_amd import kvr
    from paper_2608_14635_amd import workloads as W

    st["kvr"], st["stream"], kind = kvr, torch.cuda.current_stream().cuda_stream, case["kind"]
    cuda = dict(device="cuda")
    if kind == "tables":
        n = st["max_rows"]
        st["row_offsets"] = torch.empty(len(st["lens"]) + 1, dtype=torch.int32, **cuda)
        st["slots"] = torch.empty(n, dtype=torch.int64, **cuda)
        st["positions"] = torch.empty(n, dtype=torch.int32, **cuda)
        st["counts"] = torch.empty(4, dtype=torch.int32, **cuda)
        return st
    if kind == "logprob":
        R, n = case["rows"], case["top"]
        st["ws_bytes"] = kvr.kv_logprobs_workspace_bytes(R, case["vocab"], n)
        st["ws"] = torch.empty(max(1, st["ws_bytes"]), dtype=torch.uint8, **cuda)
        st["logprobs"], st["entropy"] = torch.empty(R, **cuda), torch.empty(R, **cuda)
        st["top_logprobs"] = torch.empty(R, n, **cuda)
        st["top_tokens"] = torch.empty(R, n, dtype=torch.int32, **cuda)
        return st
    B = case["block"]
    shape = dataclasses.replace(W.SHAPES[case["shape"]], num_layers=case.get("layers", 1))
    st["handles"] = []

    def bound(bind, give_back, t, block, blocks):
        h = bind(t.data_ptr(), t.numel() * t.element_size(), shape, block, blocks)
        st["handles"].append((give_back, h))
        return h

    if kind == "park":
        for name in ("arena", "back"):
            st[name + "_handle"] = bound(kvr.kv_arena_bind, kvr.kv_arena_release, st[name], B, st["blocks"])
        st["packed_handle"] = bound(kvr.kv_packed_bind, kvr.kv_packed_release, st["packed"], 2 * B,
                                    st["packed_blocks"])
        return st
    st["packed_handle"] = bound(kvr.kv_packed_bind, kvr.kv_packed_release, st["packed"], B, st["blocks"])
    st["out"] = torch.empty_like(st["q"])
    st["ws_bytes"] = kvr.kv_packed_attention_workspace_bytes(shape, len(st["lens"]), st["rows"], st["max_query"],
                                                             st["max_len"])
    st["ws"] = torch.empty(st["ws_bytes"], dtype=torch.uint8, **cuda)
    return st


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------
def run(st):
    return (_run_own if own else _run_plain)[st["case"]["kind"]](st)


def _own_tables(st):
    st["kvr"].kv_tables_grow(st["held"].data_ptr(), st["lens"].data_ptr(), len(st["lens"]), st["case"]["block"],
                             st["free"].data_ptr(), st["num_free"], st["tables"].data_ptr(), st["tables"].shape[1],
                             st["max_rows"], st["row_offsets"].data_ptr(), st["slots"].data_ptr(),
                             st["positions"].data_ptr(), st["counts"].data_ptr(), stream=st["stream"])
    return {k: st[k] for k in ("tables", "row_offsets", "slots", "positions", "counts")}


def _own_park(st):
    kvr, n = st["kvr"], len(st["slots"])
    kvr.kv_packed_park(st["arena_handle"], st["slots"].data_ptr(), st["packed_handle"],
                       st["packed_slots"].data_ptr(), n, st["stream"])
    kvr.kv_packed_restore(st["packed_handle"], st["packed_slots"].data_ptr(), st["back_handle"],
                          st["slots"].data_ptr(), n, st["stream"])
    return {"arena": st["back"]}


def _own_attend(st):
    q, out = st["q"], st["out"]
    st["kvr"].kv_packed_attention(st["packed_handle"], 0, q.data_ptr(), q.stride(0), st["offsets"].data_ptr(),
                                  st["rows"], st["lens"].data_ptr(), st["tables"].data_ptr(), len(st["lens"]),
                                  st["tables"].shape[1], st["max_query"], st["max_len"], out.data_ptr(),
                                  out.stride(0), st["ws"].data_ptr(), st["ws_bytes"], st["stream"])
    return {"out": out}


def _own_logprob(st):
    c, z = st["case"], st["logits"]
    kvr = st["kvr"]
    kvr.kv_logprobs(z.data_ptr(), kvr.KV_F32 if c["dtype"] == "f32" else kvr.KV_BF16, c["rows"], c["vocab"],
                    z.stride(0), c["scale"], st["tokens"].data_ptr(), c["top"], st["logprobs"].data_ptr(),
                    st["entropy"].data_ptr(), st["top_logprobs"].data_ptr(), st["top_tokens"].data_ptr(),
                    st["ws"].data_ptr(), st["ws_bytes"], stream=st["stream"])
    return {k: st[k] for k in ("logprobs", "entropy", "top_logprobs", "top_tokens")}


def _plain_tables(st):
    B, held, lens, tables, free = st["case"]["block"], st["held"].long(), st["lens"].long(), st["tables"], st["free"]
    dev, (R, wide) = tables.device, tables.shape
    first, last = _blocks(held, B), _blocks(lens, B).clamp(max=wide)
    need = (last - first).clamp(min=0)
    at = need.cumsum(0) - need
    col = torch.arange(wide, device=dev)
    i = at[:, None] + col - first[:, None]
    new = torch.where(i < st["num_free"], free[i.clamp(0, len(free) - 1)], -1)
    tables = torch.where((col >= first[:, None]) & (col < last[:, None]), new, tables)
    n = (lens - held).clamp(min=0)
    off = torch.cat([torch.zeros(1, dtype=torch.int64, device=dev), n.cumsum(0)])
    row = torch.arange(st["max_rows"], device=dev)
    r = torch.searchsorted(off[1:], row, right=True).clamp(max=R - 1)
    pos = held[r] + row - off[r]
    entry = torch.where(pos // B < wide, tables[r, (pos // B).clamp(0, wide - 1)].long(), -1)
    there = row < off[R]
    slots = torch.where(there & (entry >= 0), entry * B + pos % B, -1)
    total = need.sum()
    taken = total.clamp(max=st["num_free"])
    counts = torch.stack([taken, total - taken, off[R], (there & (slots < 0)).sum()])
    return {"tables": tables, "row_offsets": off.to(torch.int32), "slots": slots,
            "positions": torch.where(there, pos, -1).to(torch.int32), "counts": counts.to(torch.int32)}


def _plain_park(st):
    B, slots, to = st["case"]["block"], st["slots"], st["packed_slots"]
    for l in range(st["case"]["layers"]):
        _write_packed(st["packed"], l, st["arena"][l, 0, slots], st["arena"][l, 1, slots], to, 2 * B)
        k, v = _read_packed(st["packed"], l, to, 2 * B, st["arena"].shape[-1])
        st["back"][l, 0, slots], st["back"][l, 1, slots] = k.to(st["back"].dtype), v.to(st["back"].dtype)
    return {"arena": st["back"]}


def _plain_attend(st):
    q, lens, B = st["q"], st["lens"].long(), st["case"]["block"]
    nq, nkv, d, _ = HEADS[st["case"]["shape"]]
    R, n, dev = len(lens), st["max_len"], q.device
    key = torch.arange(n, device=dev)
    inside = key < lens[:, None]
    slots = torch.where(inside, st["tables"].long()[:, key // B] * B + key % B, 0)
    k, v = _read_packed(st["packed"], 0, slots.flatten(), B, d)
    k = k.unflatten(0, (R, n)).transpose(1, 2).contiguous()
    v = v.unflatten(0, (R, n)).masked_fill(~inside[:, :, None, None], 0.0).transpose(1, 2).contiguous()
    # queries padded to the largest count; query i of a request is at position len - count + i
    off = st["offsets"].long()
    count, i = off[1:] - off[:-1], torch.arange(st["max_query"], device=dev)
    there = i < count[:, None]
    row = torch.where(there, off[:-1, None] + i, 0)
    x = q.float()[row].unflatten(2, (nkv, nq // nkv)).permute(0, 2, 3, 1, 4).flatten(2, 3)
    s = (x.contiguous() @ k.transpose(2, 3)).mul_(1.0 / math.sqrt(d))
    pos = lens[:, None] - count[:, None] + i
    seen = (key <= pos[:, :, None]) & inside[:, None]                          # [R, query, key]
    s = s.unflatten(2, (nq // nkv, -1)).masked_fill_(~seen[:, None, None], -math.inf).flatten(2, 3)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    o = (p @ v) / p.sum(-1, keepdim=True)
    o = o.unflatten(2, (nq // nkv, -1)).permute(0, 3, 1, 2, 4).flatten(2, 3)   # [R, query, nq, d]
    return {"out": o[there].to(q.dtype)}


def _plain_logprob(st):
    c = st["case"]
    z = st["logits"].float() + 0.0
    most = z.amax(-1, keepdim=True)
    x = (z - most) * c["scale"]
    e = torch.exp(x)
    total = e.sum(-1)
    lse = torch.log(total)
    mean = (torch.where(e > 0, x, 0.0) * e).sum(-1) / total
    out = {"logprobs": x.gather(1, st["tokens"].long()[:, None])[:, 0] - lse, "entropy": lse - mean}
    # the likeliest, ties to the lowest index: one key orders value and index
    top, R, V = c["top"], c["rows"], c["vocab"]
    vals, idx = [z.new_empty(R, 0)], [torch.empty(R, 0, dtype=torch.int32, device=z.device)]
    for i in range(0, R if top else 0, 64):
        bits = z[i:i + 64].contiguous().view(torch.int32)
        bits = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long()
        key = (bits << 32) + (0x7FFFFFFF - torch.arange(V, device=z.device))
        best = 0x7FFFFFFF - (torch.topk(key, top, dim=1).values & 0xFFFFFFFF)
        vals.append(x[i:i + 64].gather(1, best) - lse[i:i + 64, None])
        idx.append(best.to(torch.int32))
    out["top_logprobs"] = torch.cat(vals[1:] or vals)
    out["top_tokens"] = torch.cat(idx[1:] or idx)
    return out


_run_own = dict(tables=_own_tables, park=_own_park, attend=_own_attend, logprob=_own_logprob)
_run_plain = dict(tables=_plain_tables, park=_plain_park, attend=_plain_attend, logprob=_plain_logprob)


# --------------------------------------------------------------------------
# The same results in 64 bits, from the definitions
# --------------------------------------------------------------------------
def _exact_tables(st):
    case, B = st["case"], st["case"]["block"]
    held, lens, free = (st[k].tolist() for k in ("held", "lens", "free"))
    tables, slots, positions, offsets, used, unplaced = st["tables"].tolist(), [], [], [0], 0, 0
    for r, (h, n) in enumerate(zip(held, lens)):
        for j in range(-(-h // B), -(-n // B)):
            tables[r][j] = free[used] if used < st["num_free"] else -1
            used += 1
        for p in range(h, n):
            b = tables[r][p // B]
            slots.append(b * B + p % B if b >= 0 else -1)
            unplaced += b < 0
            positions.append(p)
        offsets.append(len(slots))
    rest = [-1] * (st["max_rows"] - len(slots))
    taken = min(used, st["num_free"])
    back = dict(device="cuda")
    return {"tables": torch.tensor(tables, **back), "row_offsets": torch.tensor(offsets, **back),
            "slots": torch.tensor(slots + rest, **back), "positions": torch.tensor(positions + rest, **back),
            "counts": torch.tensor([taken, used - taken, len(slots), unplaced], **back)}


def _nearest(x):
    """x [..., d] in 64 bits -> the values a packed arena holds for it, found by
    trying all of a group's values at its scale."""
    grid = [0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0]  # those of even codes first
    g = x.unflatten(-1, (-1, GROUP))
    most = g.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(most.clamp(min=2.0 ** -140) / 6)) - 1
    for _ in range(3):
        e += most > 6 * torch.exp2(e)
    e = e.clamp(LOW_SCALE - 127, HIGH_SCALE - 127)
    s = torch.exp2(e)
    best = torch.zeros_like(g)
    err = torch.full_like(g, math.inf)
    for val in grid:  # a tie keeps the even code, which came first
        diff = (g.abs() - val * s).abs()
        best, err = torch.where(diff < err, val * s, best), torch.minimum(diff, err)
    return (best * torch.where(g < 0, -1.0, 1.0)).flatten(-2)


def _exact_park(st):
    slots = st["slots"]
    out = torch.zeros(st["arena"].shape, dtype=torch.float64, device="cuda")
    for l in range(st["case"]["layers"]):
        for kv in range(2):
            for i in range(0, len(slots), 1 << 14):
                s = slots[i:i + (1 << 14)]
                out[l, kv, s] = _nearest(st["arena"][l, kv, s].double())
    return {"arena": out}


def _exact_attend(st):
    case, q, B = st["case"], st["q"].double(), st["case"]["block"]
    nq, nkv, d, _ = HEADS[case["shape"]]
    off, out = st["offsets"].tolist(), torch.empty_like(q)
    kc, vc, ks, vs = _parts(st["packed"][0], d)
    for r, n in enumerate(st["lens"].tolist()):
        blocks = st["tables"][r, :_blocks(n, B)].long()

        def flat(t):  # [blocks, nkv, tiles, 16 slots, x] -> [nkv, positions, x]
            return t.transpose(0, 1).flatten(1, 3)[:, :n]
        for h in range(nkv):
            pick = lambda t: t[blocks, h:h + 1]  # noqa: E731
            k = _values(flat(pick(kc)), flat(pick(ks)), torch.float64)[0]
            v = _values(flat(pick(vc).transpose(4, 5).flatten(3, 4).flatten(4, 5)),
                        flat(pick(vs).transpose(4, 5).flatten(3, 4)), torch.float64)[0]
            rows = slice(off[r], off[r + 1])
            m = off[r + 1] - off[r]
            for j in range(h * (nq // nkv), (h + 1) * (nq // nkv)):
                s = (q[rows, j] @ k.t()) / math.sqrt(d)
                pos = torch.arange(n - m, n, device="cuda")
                s = s.masked_fill(torch.arange(n, device="cuda") > pos[:, None], -math.inf)
                out[rows, j] = torch.softmax(s, -1) @ v
    return {"out": out}


def _exact_logprob(st):
    c = st["case"]
    out = {"logprobs": [], "entropy": [], "top_logprobs": [], "top_tokens": []}
    for i in range(0, c["rows"], 64):
        z = st["logits"][i:i + 64].double()
        lp = torch.log_softmax(z * c["scale"], -1)
        out["logprobs"].append(lp.gather(1, st["tokens"][i:i + 64].long()[:, None])[:, 0])
        out["entropy"].append(torch.special.entr(lp.exp()).sum(-1))
        order = torch.sort(z, dim=-1, descending=True, stable=True).indices[:, :c["top"]]
        out["top_logprobs"].append(lp.gather(1, order))
        out["top_tokens"].append(order.to(torch.int32))
    return {k: torch.cat(v) for k, v in out.items()}


@torch.no_grad()
def exact(case, seed):
    w = work(case)
    if (case["kind"] == "tables" and w["flops"] > 4e6) or (case["kind"] == "park" and w["bytes"] > 4e9):
        return None
    st = _inputs(case, seed)
    return dict(tables=_exact_tables, park=_exact_park, attend=_exact_attend, logprob=_exact_logprob)[
        case["kind"]](st)
