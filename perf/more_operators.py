"""The performance cases of the operators around a group of rollouts: several answers
sampled from one prompt, and the loss of their tokens.

A case names one call:

  append    kv_append: rows of a layer's q, k, v products with bias, per-head norm and
            rotation applied, K and V put into the arena's slots
  group     kv_group_attention: queries over the arena through block tables, a prefix
            that a group of requests shares read once for the group
  policy    kv_policy_loss: the clipped policy loss of given tokens with its KL term,
            and the gradient of the logits

Heads, rotation bases and vocabularies are those of the package's decoder shapes.
Lengths follow the case's own `mix` number, everything else the seed.  Where `own` is
false, the same results are computed in their plain form, elementary torch operations.
"""
import math
import random

import torch

own = False

# heads, head dim, dtype, rotation base, norm epsilon and variant of the decoder shapes
HEADS = {"tiny_f32": (4, 4, 64, "f32", 1e4, 1e-5, ""), "tiny_bf16": (8, 2, 128, "bf16", 1e4, 1e-5, ""),
         "qwen25_1_5b": (12, 2, 128, "bf16", 1e6, 1e-6, "bias"), "llama8b": (32, 8, 128, "bf16", 5e5, 1e-5, ""),
         "qwen14b": (40, 8, 128, "bf16", 1e6, 1e-6, ""), "qwen3_8b": (32, 8, 128, "bf16", 1e6, 1e-6, "norm"),
         "qwen3_32b": (64, 8, 128, "bf16", 1e6, 1e-6, "norm")}
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
STD = 1.3


def listed():
    return [
        # one new token of every request of a decode batch, heads normed
        dict(name="append_step", kind="append", shape="qwen3_8b", rows=64, low=200, high=16000, block=16, mix=1),
        # drafted tokens of a few requests of a small model, biases
        dict(name="append_draft", kind="append", shape="qwen25_1_5b", rows=23, low=1, high=32768, block=32, mix=2),
        # a prompt's piece of a large model, far positions, an odd count
        dict(name="append_prompt", kind="append", shape="qwen14b", rows=8191, low=0, high=200000, block=16, mix=3),
        # a few answers to one short prompt, small model: latency
        dict(name="group_one", kind="group", shape="qwen25_1_5b", groups=1, each_low=4, each_high=4, prefix_low=171,
             prefix_high=171, tail_low=1, tail_high=60, query=1, block=16, mix=4),
        # the tiny fp32 decoder's heads, ragged groups
        dict(name="group_f32", kind="group", shape="tiny_f32", groups=7, each_low=1, each_high=6, prefix_low=1,
             prefix_high=200, tail_low=1, tail_high=150, query=1, block=24, mix=5),
        # a rollout batch: eight answers to each of eight prompts
        dict(name="group_rollout", kind="group", shape="llama8b", groups=8, each_low=8, each_high=8, prefix_low=500,
             prefix_high=2500, tail_low=100, tail_high=4000, query=1, block=16, mix=6),
        # one to four drafted tokens of each request checked in one pass
        dict(name="group_draft", kind="group", shape="qwen3_32b", groups=5, each_low=2, each_high=5, prefix_low=800,
             prefix_high=6000, tail_low=50, tail_high=1500, query=4, block=32, mix=7),
        # agents that share a long system prompt and repository context
        dict(name="group_long", kind="group", shape="qwen14b", groups=1, each_low=48, each_high=48, prefix_low=24011,
             prefix_high=24011, tail_low=200, tail_high=2000, query=1, block=16, mix=8),
        # one answer's tokens under the tiny decoder: latency
        dict(name="policy_one", kind="policy", rows=171, vocab=1024, dtype="f32", pad=0, grad=True, kl=0.05,
             scale=1.0, mix=9),
        # tokens scored without a gradient, rows on an odd stride
        dict(name="policy_forward", kind="policy", rows=384, vocab=128256, dtype="bf16", pad=1, grad=False, kl=0.0,
             scale=1.25, mix=10),
        # fp32 logits of a large vocabulary, gradient
        dict(name="policy_f32", kind="policy", rows=250, vocab=152064, dtype="f32", pad=0, grad=True, kl=0.01,
             scale=1.0, mix=11),
        # a training batch's piece, bf16 logits, gradient
        dict(name="policy_batch", kind="policy", rows=1024, vocab=151936, dtype="bf16", pad=0, grad=True, kl=0.02,
             scale=1.0, mix=12),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    """One more case of the same ranges."""
    while True:
        kind = rng.choice(["append", "append", "group", "group", "group", "policy", "policy"])
        c = dict(kind=kind, mix=rng.randrange(1 << 20))
        if kind == "policy":
            c.update(rows=_log_int(rng, 1, 1024), vocab=_log_int(rng, 1000, 152064),
                     dtype=rng.choice(["f32", "bf16"]), pad=rng.choice([0, 0, 1, 3, 8]),
                     grad=rng.random() < 0.75, kl=rng.choice([0.0, 0.01, 0.2]), scale=rng.choice([1.0, 1.25, 0.7]))
            if work(c)["bytes"] <= 6.3e8:
                return c
            continue
        c.update(shape=rng.choice(list(HEADS)), block=rng.choice([8, 16, 16, 24, 32, 64]))
        if kind == "append":
            c["rows"] = _log_int(rng, 1, 8192)
            c["high"] = _log_int(rng, 16, 1 << 20)
            c["low"] = int(c["high"] * rng.random())
            if work(c)["bytes"] <= 2.4e8:
                return c
            continue
        most = _log_int(rng, 1, 64)
        c.update(groups=_log_int(rng, 1, 64), each_low=max(1, int(most * rng.uniform(0.2, 1))), each_high=most)
        prefix, tail = _log_int(rng, 1, 32768), _log_int(rng, 1, 8192)
        c.update(prefix_low=max(1, int(prefix * rng.uniform(0.1, 1))), prefix_high=prefix,
                 tail_low=max(1, int(tail * rng.uniform(0.02, 1))), tail_high=tail,
                 query=rng.choice([1, 1, 1, 2, 4, 5]))
        # what the plain form spreads out: every context as long as the longest
        if c["groups"] * most * (prefix + tail) * 1024 <= 1.3e9 and work(c)["bytes"] <= 4.2e8:
            return c


# --------------------------------------------------------------------------
# Sizes of a case
# --------------------------------------------------------------------------
def _batch(case):
    """Of a group case: requests of each group, shared positions, lengths, query rows."""
    rng = random.Random(case["mix"])
    each = [rng.randint(case["each_low"], case["each_high"]) for _ in range(case["groups"])]
    prefix = [rng.randint(case["prefix_low"], case["prefix_high"]) for _ in each]
    lens = [p + rng.randint(case["tail_low"], case["tail_high"]) for n, p in zip(each, prefix) for _ in range(n)]
    shared = [p for n, p in zip(each, prefix) for _ in range(n)]
    rows = [min(n - p, rng.randint(1, case["query"])) for n, p in zip(lens, shared)]
    return each, prefix, shared, lens, rows


def _blocks(n, B):
    return (n + B - 1) // B


def work(case):
    kind = case["kind"]
    if kind == "policy":
        e = 4 if case["dtype"] == "f32" else 2
        n = case["rows"] * case["vocab"]
        return {"bytes": float(n * e * (2 if case["grad"] else 1) + 28 * case["rows"]),
                "flops": (10.0 if case["grad"] else 5.0) * n}
    nq, nkv, d, dt = HEADS[case["shape"]][:4]
    e = 4 if dt == "f32" else 2
    if kind == "append":
        n = case["rows"]
        return {"bytes": float(n * (2 * (nq + 2 * nkv) * d * e + 12)), "flops": 4.0 * n * (nq + nkv) * d}
    _, prefix, shared, lens, rows = _batch(case)
    held = sum(prefix) + sum(lens) - sum(shared)
    pairs = sum(m * n - m * (m - 1) // 2 for m, n in zip(rows, lens))
    return {"bytes": float(held * 2 * nkv * d * e + 2 * sum(rows) * nq * d * e), "flops": 4.0 * nq * d * pairs}


# --------------------------------------------------------------------------
# Inputs, from the seed alone
# --------------------------------------------------------------------------
class _State(dict):
    """A worker's handles; the binding is given back with it."""

    def __del__(self):
        for give_back, handle in self.pop("handles", ()):
            give_back(handle)


def _randn(g, *shape, std=1.0, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).to(dtype)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return dict(append=_append_inputs, group=_group_inputs, policy=_policy_inputs)[case["kind"]](case, seed, g)


def _append_inputs(case, seed, g):
    nq, nkv, d, dt, _, _, variant = HEADS[case["shape"]]
    dt, n, B = DTYPE[dt], case["rows"], case["block"]
    # the rows of one product: q, k and v side by side
    qkv = _randn(g, n, (nq + 2 * nkv) * d, std=STD, dtype=dt)
    blocks = _blocks(n + n // 4, B) + 2
    slots = torch.randperm(blocks * B, generator=g, device="cuda")[:n]
    positions = torch.randint(case["low"], case["high"] + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
    st = dict(case=case, qkv=qkv, slots=slots, positions=positions, blocks=blocks,
              arena=torch.zeros(1, 2, blocks * B, nkv, d, dtype=dt, device="cuda"),
              q_out=torch.empty(n, nq, d, dtype=dt, device="cuda"))
    if variant == "norm":
        st.update(q_norm=1 + _randn(g, d, std=0.1), k_norm=1 + _randn(g, d, std=0.1))
    if variant == "bias":
        st.update(bq=_randn(g, nq * d), bk=_randn(g, nkv * d), bv=_randn(g, nkv * d))
    for name in ("q_norm", "k_norm", "bq", "bk", "bv"):
        st[name] = st[name].to(dt) if name in st else None
    return st


def _group_inputs(case, seed, g):
    nq, nkv, d, dt = HEADS[case["shape"]][:4]
    dt, B = DTYPE[dt], case["block"]
    each, prefix, shared, lens, rows = _batch(case)
    # a group's whole blocks of the prefix are named by all its tables; the block in which
    # the prefix ends is each request's own copy
    own_blocks = [_blocks(n, B) - p // B for n, p in zip(lens, shared)]
    total = sum(p // B for p in prefix) + sum(own_blocks)
    total += max(2, total // 8)
    perm = torch.randperm(total, generator=torch.Generator().manual_seed(seed)).tolist()
    tables = torch.zeros(len(lens), max(_blocks(n, B) for n in lens), dtype=torch.int32)
    starts, r = [0], 0
    copies = [], []
    for n, p in zip(each, prefix):
        common = [perm.pop() for _ in range(p // B)]
        first = r
        for r in range(first, first + n):
            mine = [perm.pop() for _ in range(own_blocks[r])]
            tables[r, :_blocks(lens[r], B)] = torch.tensor(common + mine, dtype=torch.int32)
            for at in range(p - p % B, p):
                copies[0].append(int(tables[first, at // B]) * B + at % B)
                copies[1].append(int(tables[r, at // B]) * B + at % B)
        r = first + n
        starts.append(r)
    tables, lens_t = tables.cuda(), _int32(lens)
    pos = torch.arange(max(lens), device="cuda")
    slots = (tables.long()[:, pos // B] * B + pos % B)[pos < lens_t[:, None]]
    # slots outside the contexts hold no numbers
    arena = torch.full((1, 2, total * B, nkv, d), math.nan, dtype=dt, device="cuda")
    slots = slots.unique()
    for kv in range(2):
        arena[0, kv, slots] = _randn(g, len(slots), nkv, d, std=STD, dtype=dt)
    source, target = (torch.tensor(c, dtype=torch.int64, device="cuda") for c in copies)
    arena[0, :, target] = arena[0, :, source]
    off = torch.cat([torch.zeros(1, dtype=torch.int64), torch.tensor(rows).cumsum(0)])
    return dict(case=case, arena=arena, blocks=total, tables=tables, lens=lens_t, max_len=max(lens),
                offsets=off.to(torch.int32).cuda(), rows=sum(rows), max_query=max(rows), groups=_int32(starts),
                prefix=_int32(prefix), q=_randn(g, sum(rows), nq, d, std=STD, dtype=dt))


def _policy_inputs(case, seed, g):
    R, V, dt = case["rows"], case["vocab"], DTYPE[case["dtype"]]
    logits = _randn(g, R, V + case["pad"], std=2.0, dtype=dt)[:, :V]
    # sampled tokens of rows between flat and nearly certain
    logits[torch.arange(R, device="cuda"), torch.randint(0, V, (R,), generator=g, device="cuda")] += \
        torch.rand(R, generator=g, device="cuda").mul_(30).to(dt)
    tokens = torch.empty(R, dtype=torch.int64, device="cuda")
    logp = torch.empty(R, device="cuda")
    for i in range(0, R, 128):
        x = logits[i:i + 128].float() * case["scale"]
        noise = torch.rand(x.shape, generator=g, device="cuda").clamp_(1e-9, 1 - 1e-7)
        tokens[i:i + 128] = (x - torch.log(-torch.log(noise))).argmax(-1)
        logp[i:i + 128] = torch.log_softmax(x, -1).gather(1, tokens[i:i + 128, None])[:, 0]
    # the rollout's policy is some updates old, the reference further away
    old, ref = logp + _randn(g, R, std=0.15), logp + _randn(g, R, std=0.3)
    weights = torch.rand(R, generator=g, device="cuda").add_(0.5).div_(R)
    weights[torch.rand(R, generator=g, device="cuda") < 0.1] = 0  # padding and the environment's tokens
    weights[0] = 1.0 / R
    return dict(case=case, logits=logits, tokens=tokens.to(torch.int32), old=old.clamp(max=0), ref=ref.clamp(max=0),
                advantages=_randn(g, R), weights=weights)


CLIP_LOW, CLIP_HIGH = 0.2, 0.28


def prepare(case, seed):
    st = _State(_inputs(case, seed))
    if not own:
        return st
    import dataclasses

    from paper_2608_14635_amd import kvr
    from paper_2608_14635_amd import workloads as W

    st["kvr"], st["stream"], kind = kvr, torch.cuda.current_stream().cuda_stream, case["kind"]
    if kind == "policy":
        R, z = case["rows"], st["logits"]
        st["ws_bytes"] = kvr.kv_policy_loss_workspace_bytes(R, case["vocab"])
        st["ws"] = torch.empty(st["ws_bytes"], dtype=torch.uint8, device="cuda")
        st["total"] = torch.empty(1, device="cuda")
        st["losses"], st["logprobs"], st["kls"] = (torch.empty(R, device="cuda") for _ in range(3))
        st["grad"] = torch.empty(R, case["vocab"], dtype=z.dtype, device="cuda") if case["grad"] else None
        return st
    shape, arena = dataclasses.replace(W.SHAPES[case["shape"]], num_layers=1), st["arena"]
    st["arena_handle"] = kvr.kv_arena_bind(arena.data_ptr(), arena.numel() * arena.element_size(), shape,
                                           case["block"], st["blocks"])
    st["handles"] = [(kvr.kv_arena_release, st["arena_handle"])]
    if kind == "append":
        names = ("q_norm", "k_norm", "bq", "bk", "bv")
        st["layer"] = {k: st[k].data_ptr() for k in names if st[k] is not None}
        return st
    st["out"] = torch.empty_like(st["q"])
    st["ws_bytes"] = kvr.kv_group_attention_workspace_bytes(shape, len(st["lens"]), st["rows"], case["groups"],
                                                            st["max_query"], st["max_len"])
    st["ws"] = torch.empty(st["ws_bytes"], dtype=torch.uint8, device="cuda")
    return st


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------
def run(st):
    return (_run_own if own else _run_plain)[st["case"]["kind"]](st)


def _own_append(st):
    nq, nkv, d = HEADS[st["case"]["shape"]][:3]
    qkv, q_out = st["qkv"], st["q_out"]
    wide, at, e = qkv.stride(0), qkv.data_ptr(), qkv.element_size()
    st["kvr"].kv_append(st["arena_handle"], 0, st["layer"], at, wide, at + nq * d * e, wide, at + (nq + nkv) * d * e,
                        wide, st["positions"].data_ptr(), st["slots"].data_ptr(), st["case"]["rows"], q_out.data_ptr(),
                        q_out.stride(0), st["stream"])
    return {"q": q_out, "arena": st["arena"]}


def _own_group(st):
    q, out = st["q"], st["out"]
    st["kvr"].kv_group_attention(st["arena_handle"], 0, q.data_ptr(), q.stride(0), st["offsets"].data_ptr(),
                                 st["rows"], st["lens"].data_ptr(), st["tables"].data_ptr(), len(st["lens"]),
                                 st["tables"].shape[1], st["groups"].data_ptr(), st["prefix"].data_ptr(),
                                 st["case"]["groups"], st["max_query"], st["max_len"], out.data_ptr(), out.stride(0),
                                 st["ws"].data_ptr(), st["ws_bytes"], st["stream"])
    return {"out": out}


def _own_policy(st):
    c, z, kvr, grad = st["case"], st["logits"], st["kvr"], st["grad"]
    kvr.kv_policy_loss(z.data_ptr(), kvr.KV_F32 if c["dtype"] == "f32" else kvr.KV_BF16, c["rows"], c["vocab"],
                       z.stride(0), c["scale"], st["tokens"].data_ptr(), st["old"].data_ptr(),
                       st["ref"].data_ptr(), st["advantages"].data_ptr(), st["weights"].data_ptr(), CLIP_LOW,
                       CLIP_HIGH, c["kl"], st["total"].data_ptr(), st["losses"].data_ptr(), st["logprobs"].data_ptr(),
                       st["kls"].data_ptr(), grad.data_ptr() if c["grad"] else 0, c["vocab"], st["ws"].data_ptr(),
                       st["ws_bytes"], stream=st["stream"])
    out = {k: st[k] for k in ("total", "losses", "logprobs", "kls")}
    return {**out, "grad": grad} if c["grad"] else out


def _plain_append(st):
    nq, nkv, d, _, theta, eps, _ = HEADS[st["case"]["shape"]]
    x = st["qkv"].float()
    q, k, v = x.split([nq * d, nkv * d, nkv * d], 1)
    if st["bq"] is not None:
        q, k, v = q + st["bq"].float(), k + st["bk"].float(), v + st["bv"].float()
    q, k = q.unflatten(1, (nq, d)), k.unflatten(1, (nkv, d))
    if st["q_norm"] is not None:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + eps) * st["q_norm"].float()
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + eps) * st["k_norm"].float()
    inv = theta ** (-torch.arange(0, d, 2, dtype=torch.float64, device=x.device) / d)
    angle = st["positions"].double()[:, None] * inv
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def rotated(t):
        a, b = t[..., :d // 2], t[..., d // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(st["qkv"].dtype)
    arena, slots = st["arena"], st["slots"]
    arena[0, 0, slots], arena[0, 1, slots] = rotated(k), v.unflatten(1, (nkv, d)).to(arena.dtype)
    return {"q": rotated(q), "arena": arena}


def _plain_group(st):
    q, lens, B = st["q"], st["lens"].long(), st["case"]["block"]
    nq, nkv, d = HEADS[st["case"]["shape"]][:3]
    R, n, dev = len(lens), st["max_len"], q.device
    key = torch.arange(n, device=dev)
    inside = key < lens[:, None]
    slots = st["tables"].long()[:, key // B] * B + key % B
    k, v = (st["arena"][0, i, slots].masked_fill_(~inside[:, :, None, None], 0.0).transpose(1, 2).float().contiguous()
            for i in range(2))
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


def _plain_policy(st):
    c = st["case"]
    t = st["tokens"].long()[:, None]
    z = st["logits"].float()
    most = z.amax(-1, keepdim=True)
    e = torch.exp((z - most) * c["scale"])
    # the other tokens' share in 64 bits: next to certain tokens 1 - p is what remains
    mine = torch.exp((z.gather(1, t) - most).double() * c["scale"])
    rest = e.scatter(1, t, 0.0).sum(-1, keepdim=True, dtype=torch.float64)
    logp = -torch.log1p(rest / mine)[:, 0]
    w, a, ref = st["weights"].double(), st["advantages"].double(), st["ref"].double()
    ratio = torch.exp(logp - st["old"])
    kept, cut = ratio * a, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * a
    diff = ref - logp
    kl = torch.where(w != 0, torch.expm1(diff) - diff, 0.0)
    losses = torch.where(w != 0, w * (c["kl"] * kl - torch.minimum(kept, cut)), 0.0)
    out = {"total": losses.sum()[None].float(), "losses": losses.float(), "logprobs": logp.float(), "kls": kl.float()}
    if c["grad"]:
        slope = w * (-torch.where(kept <= cut, kept, 0.0) - c["kl"] * torch.expm1(diff)) * c["scale"]
        slope = torch.where(w != 0, slope, 0.0)[:, None]
        g = e.mul_((-slope / (rest + mine)).float())
        g.scatter_(1, t, (slope * rest / (rest + mine)).float())
        out["grad"] = g.to(st["logits"].dtype)
    return out


_run_own = dict(append=_own_append, group=_own_group, policy=_own_policy)
_run_plain = dict(append=_plain_append, group=_plain_group, policy=_plain_policy)


# --------------------------------------------------------------------------
# The same results in 64 bits, from the definitions
# --------------------------------------------------------------------------
def _exact_append(st):
    nq, nkv, d, _, theta, eps, _ = HEADS[st["case"]["shape"]]
    x, pos = st["qkv"].double(), st["positions"].double()
    heads = []
    for h in range(nq + 2 * nkv):
        y = x[:, h * d:(h + 1) * d]
        which, at = ("q", h) if h < nq else ("k", h - nq) if h < nq + nkv else ("v", h - nq - nkv)
        if st["b" + which] is not None:
            y = y + st["b" + which].double()[at * d:(at + 1) * d]
        if which != "v":
            if st[which + "_norm"] is not None:
                y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / d + eps) * st[which + "_norm"].double()
            # the pair (i, i + d/2) as one complex number, turned
            turn = torch.stack([torch.polar(torch.ones_like(pos), pos * theta ** (-2.0 * i / d)) for i in range(d // 2)], 1)
            y = torch.complex(y[:, :d // 2], y[:, d // 2:]) * turn
            y = torch.cat([y.real, y.imag], 1)
        heads.append(y)
    heads = torch.stack(heads, 1)
    arena = torch.zeros(st["arena"].shape, dtype=torch.float64, device="cuda")
    arena[0, 0, st["slots"]], arena[0, 1, st["slots"]] = heads[:, nq:nq + nkv], heads[:, nq + nkv:]
    return {"q": heads[:, :nq].contiguous(), "arena": arena}


def _exact_group(st):
    q, B = st["q"].double(), st["case"]["block"]
    nq, nkv, d = HEADS[st["case"]["shape"]][:3]
    g = nq // nkv
    off, out = st["offsets"].tolist(), torch.empty_like(q)
    for r, n in enumerate(st["lens"].tolist()):
        blocks = st["tables"][r, :_blocks(n, B)].long()
        rows, m = slice(off[r], off[r + 1]), off[r + 1] - off[r]
        late = torch.arange(n, device="cuda") > torch.arange(n - m, n, device="cuda")[:, None]
        k, v = (st["arena"][0, i].unflatten(0, (-1, B))[blocks].flatten(0, 1)[:n].double() for i in range(2))
        for h in range(nkv):
            s = torch.matmul(q[rows, h * g:(h + 1) * g].flatten(0, 1), k[:, h].t()) / math.sqrt(d)
            s = s.unflatten(0, (m, g)).masked_fill(late[:, None], -math.inf)
            out[rows, h * g:(h + 1) * g] = torch.matmul(torch.softmax(s, -1).flatten(0, 1), v[:, h]).unflatten(0, (m, g))
    return {"out": out}


def _exact_policy(st):
    """The loss as a function of the logits in 64 bits, the gradient by differentiation."""
    c, parts = st["case"], []
    for i in range(0, c["rows"], 64):
        part = slice(i, i + 64)
        z = st["logits"][part].double().requires_grad_(c["grad"])
        w, a = st["weights"][part].double(), st["advantages"][part].double()
        with torch.set_grad_enabled(c["grad"]):
            lp = torch.log_softmax(z * c["scale"], -1).gather(1, st["tokens"][part].long()[:, None])[:, 0]
            ratio = (lp - st["old"][part].double()).exp()
            gain = torch.where(a > 0, ratio.clamp(max=1 + CLIP_HIGH), ratio.clamp(min=1 - CLIP_LOW)) * a
            over = st["ref"][part].double() - lp
            kl = torch.where(w > 0, over.exp() - over - 1, 0.0)
            loss = w * (c["kl"] * kl - gain)
            if c["grad"]:
                loss.sum().backward()
        parts.append((loss.detach(), lp.detach(), kl.detach(), z.grad))
    losses, logp, kls = (torch.cat([p[i] for p in parts]) for i in range(3))
    out = {"total": losses.sum()[None], "losses": losses, "logprobs": logp, "kls": kls}
    return {**out, "grad": torch.cat([p[3] for p in parts])} if c["grad"] else out


@torch.no_grad()
def exact(case, seed):
    st = _inputs(case, seed)
    return dict(append=_exact_append, group=_exact_group, policy=_exact_policy)[case["kind"]](st)
