"""Log probabilities of given tokens, entropy and likeliest tokens (kv_logprobs,
include/kvr_logprob.h) against 64 bits; the likeliest tokens are whole numbers and
have to be equal, ties in index order.

Tolerances, u = 2^-24, x = scale (z - max z), X = sum p |x|: e^x carries the
rounding of its argument (2 |x| u) and of the exponential (2 u); a thread adds up to
64 of them and the rest is trees and up to 256 chunks in turn, at most 400 u
relative; logf and the last operations add 4 u of their values.  So log l is off by
at most (400 + 2 X) u + 4 u |log l| and a log probability by that and 3 u |x_t|; the
entropy by (800 + 4 X) u (1 + X) + 4 u (|log l| + X)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_14635_amd import kvr  # noqa: E402

U = 2.0 ** -24
KEPT = 77


def reference(z, scale, tokens, top):
    z = np.asarray(z, np.float64)
    R, V = z.shape
    lp, ent, tol_lp, tol_ent = np.zeros(R), np.zeros(R), np.zeros(R), np.zeros(R)
    tops, top_lp, tol_top = np.zeros((R, top), int), np.zeros((R, top)), np.zeros((R, top))
    for r in range(R):
        rank = np.where(np.isnan(z[r]), -np.inf, z[r])
        order = np.lexsort((np.arange(V), np.isnan(z[r]), -rank))[:top]
        tops[r] = order
        bad = np.isnan(z[r]).any() or (z[r] == np.inf).any()
        none = (z[r] == -np.inf).all()
        t = tokens[r]
        if bad:
            lp[r], ent[r], top_lp[r] = np.nan, np.nan, np.nan
            lp[r] = 0.0 if t < 0 else np.nan
            continue
        if none:
            lp[r], ent[r], top_lp[r] = (0.0 if t < 0 else -np.inf), 0.0, -np.inf
            continue
        x = scale * (z[r] - z[r].max())
        e = np.exp(x)
        l = e.sum()
        p = e / l
        ax = np.where(p > 0, np.abs(np.where(p > 0, x, 0)), 0)
        X = (p * ax).sum()
        ent[r] = np.log(l) + X
        base = (400 + 2 * X) * U + 4 * U * np.log(l)
        tol_ent[r] = (800 + 4 * X) * U * (1 + X) + 4 * U * (np.log(l) + X)
        lp[r] = 0.0 if t < 0 else -np.inf if t >= V else x[t] - np.log(l)
        top_lp[r] = x[order] - np.log(l)
        with np.errstate(invalid="ignore"):
            tol_lp[r] = base + (3 * U * abs(x[t]) if 0 <= t < V and np.isfinite(x[t]) else 0)
            tol_top[r] = base + 3 * U * np.where(np.isfinite(x[order]), np.abs(x[order]), 0)
    return lp, ent, tops, top_lp, tol_lp, tol_ent, tol_top


def near(got, want, tol):
    got, want = np.asarray(got, np.float64), np.asarray(want)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        bad = ~same & ~(np.abs(got - want) <= tol)
    assert not bad.any(), (got[bad][:5], want[bad][:5], np.asarray(tol)[bad][:5])


class Call:
    def __init__(self, z, scale=1.0, tokens=None, top=0, pad=0, lead=0, want=(True, True)):
        """z: a CPU tensor [R, V]; rows `pad` elements apart, the first `lead` behind an
        allocation's start."""
        R, V = z.shape
        flat = torch.full((lead + R * (V + pad) + 8,), float("nan"), dtype=z.dtype, device="cuda")
        self.z = flat[lead:lead + R * (V + pad)].view(R, V + pad)[:, :V]
        self.z.copy_(z)
        self.host, self.scale, self.top, self.want = z.float().numpy(), scale, top, want
        self.tokens = np.zeros(R, int) if tokens is None else np.asarray(tokens)
        self.d_tokens = torch.tensor(self.tokens, dtype=torch.int32, device="cuda")
        self.lp, self.ent = (torch.full((R + 2,), float(KEPT), device="cuda") for _ in range(2))
        self.top_lp = torch.full((R * top + 2,), float(KEPT), device="cuda")
        self.tops = torch.full((R * top + 2,), KEPT, dtype=torch.int32, device="cuda")
        self.bytes = kvr.kv_logprobs_workspace_bytes(R, V, top)
        self.ws = torch.full((self.bytes,), 255, dtype=torch.uint8, device="cuda")

    def run(self, ws=None):
        R, V = self.z.shape
        kvr.kv_logprobs(self.z.data_ptr(), kvr.KV_F32 if self.z.dtype == torch.float32 else kvr.KV_BF16, R, V,
                        self.z.stride(0), self.scale, self.d_tokens.data_ptr(), self.top,
                        self.lp.data_ptr() if self.want[0] else 0, self.ent.data_ptr() if self.want[1] else 0,
                        self.top_lp.data_ptr(), self.tops.data_ptr(), (self.ws if ws is None else ws).data_ptr(),
                        self.bytes, stream=torch.cuda.current_stream().cuda_stream)

    def check(self):
        R, n = len(self.tokens), self.top
        lp, ent, tops, top_lp, tol_lp, tol_ent, tol_top = reference(self.host, self.scale, self.tokens, n)
        got = [a.cpu().numpy() for a in (self.lp, self.ent, self.top_lp, self.tops)]
        for g, end, wanted in ((got[0], R, self.want[0]), (got[1], R, self.want[1]), (got[2], R * n, 1),
                               (got[3], R * n, 1)):
            assert (g[end if wanted else 0:] == KEPT).all()
        assert np.array_equal(got[3][:R * n].reshape(R, n), tops)
        near(got[2][:R * n].reshape(R, n), top_lp, tol_top)
        if self.want[0]:
            near(got[0][:R], lp, tol_lp)
        if self.want[1]:
            near(got[1][:R], ent, tol_ent)


def random_rows(R, V, dtype, seed, std=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(R, V, generator=g) * std).to(dtype), torch.randint(0, V, (R,), generator=g).numpy()


DT = {"f32": torch.float32, "bf16": torch.bfloat16}
# one entry, fewer than a workgroup's threads, both sides of whole chunks of 8192
VOCABS = [1, 5, 63, 255, 1000, 4097, 8191, 8192, 8193, 16385, 40001]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("V", VOCABS)
def test_vocabularies(V, dt):
    for top, pad, lead, scale in ((0, 0, 0, 1.0), (min(V, 5), 1, 1, 1.25), (min(V, 64), 3, 5, 0.5)):
        z, tok = random_rows(3, V, DT[dt], V + top)
        c = Call(z, scale, tok, top, pad, lead)
        c.run()
        c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("R,V,top", [(1, 152064, 64), (16, 128256, 20), (600, 4097, 3), (700, 333, 64), (513, 20000, 1)])
def test_rows(R, V, top, dt):
    z, tok = random_rows(R, V, DT[dt], R)
    c = Call(z, 1.0, tok, top, pad=1)
    c.run()
    c.check()


def special_rows(V, dtype):
    """Rows of one pattern each, and their tokens."""
    i = torch.arange(V, dtype=torch.float32)
    low = torch.finfo(dtype).min
    rows, tok = [], []

    def add(r, t):
        rows.append(r)
        tok.append(t)
    g = torch.Generator().manual_seed(V)
    base = torch.randn(V, generator=g) * 3
    add(torch.zeros(V), V - 1)                                  # all equal
    add(i / V, 0)                                               # rising
    add(-i / V, V // 2)                                         # falling
    add(torch.where(i % 2 == 0, -0.0, 0.0), 1)                  # two zeros: equal
    add((i % 7), 6)                                             # few values, ties across chunks
    add(torch.where(i < V - 3, 1.0, 2.0), 0)                    # a tie that ends the row
    add(torch.full((V,), -np.inf), 2)                           # nothing left
    add(torch.where(i == V // 3, 1.5, -np.inf), V // 3)         # one token left
    add(torch.where(i == V // 3, 1.5, -np.inf), 0)              # a masked token
    add(torch.where(i % 3 == 0, base, torch.tensor(low)), 3)    # masks of the lowest value
    add(torch.full((V,), low), 1)                               # that alone
    add(torch.where(i == 7, np.nan, base), 3)                   # a NaN
    add(torch.where(i == 7, np.nan, -np.inf), 3)                # NaN above nothing
    add(torch.full((V,), np.nan), 3)
    add(torch.where(i == V - 2, np.inf, base), 3)               # an infinity
    add(base * 1e4, 5)                                          # far apart
    add(base * 1e-4, 5)                                         # nearly equal
    add(base, -1)                                               # no token
    add(base, V)                                                # a token past the vocabulary
    add(base, 2 ** 31 - 1)
    add(torch.full((V,), -np.inf), -5)
    return torch.stack(rows).to(dtype), tok


@pytest.mark.gpu
@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("V,top", [(100, 64), (4100, 20), (17000, 64), (70000, 5)])
def test_special_rows(V, top, dt):
    z, tok = special_rows(V, DT[dt])
    c = Call(z, 1.0, tok, top)
    c.run()
    c.check()
    many = z.repeat(32, 1)  # enough rows for the wide chunks
    c = Call(many[:600] if V <= 17000 else z, 1.25, (tok * 32)[:600] if V <= 17000 else tok, min(top, 7))
    c.run()
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", list(DT))
def test_logits_of_any_size(dt):
    """Where scale log2 e times the largest logit has steps above 1, or no fp32 value."""
    V = 20000
    base = torch.randn(V, generator=torch.Generator().manual_seed(4)) * 3
    i = torch.arange(V)
    for size in (1e8, 1e10, 1e20, 1e37):
        rows = torch.stack([torch.full((V,), -size), torch.full((V,), size), base * size,
                            torch.where(i < V // 2, -size, -1.25 * size), torch.where(i == 5, size, base),
                            torch.where(i % 2 == 0, base, torch.tensor(-size))]).to(DT[dt])
        for scale in (1.0, 2.0 / size, 2.0 ** (20 if size < 1e30 else 0)):
            c = Call(rows, scale, [5, 7, 9, V - 1, 5, 6], 4)
            c.run()
            c.check()
    c = Call((base * 2.0 ** -100).to(DT[dt])[None], 2.0 ** 100, [3], 4)
    c.run()
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", list(DT))
def test_the_largest_vocabulary(dt):
    V = 1 << 21
    g = torch.Generator().manual_seed(9)
    z = torch.stack([torch.randn(V, generator=g) * 3, torch.randint(0, 5, (V,), generator=g).float(), torch.zeros(V)])
    c = Call(z.to(DT[dt]), 1.0, [V - 1, 0, V // 2], 64)
    c.run()
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", list(DT))
def test_equal_values_that_fill_the_list(dt):
    """Many equal entries of few threads, and of few ranks of many chunks: lists of a bound
    on the threads' values that are given up."""
    V = 64 * 8192
    i = torch.arange(V)
    low = -1 - torch.rand(V, generator=torch.Generator().manual_seed(11))
    per = 4 if dt == "f32" else 8  # consecutive entries of a thread
    rows = [torch.where(i % (256 * per) // per < 100, 2.0, low), torch.where(i % 8192 < 24, 2.0, low),
            torch.where(i % 8192 % (8 * per) < per, (i // 8192 % 2).float(), low)]
    c = Call(torch.stack(rows).to(DT[dt]), 1.0, [0, 5, V - 1], 64)
    c.run()
    c.check()


@pytest.mark.gpu
def test_more_rows_than_a_short_grid():
    R, V = (1 << 17) + 3, 37
    z, tok = random_rows(R, V, torch.float32, 10)
    c = Call(z, 1.0, tok)
    c.run()
    x = z.double() - z.double().amax(1, keepdim=True)
    lse = x.exp().sum(1).log()
    p = (x - lse[:, None]).exp()
    X = (p * x.abs()).sum(1)
    xt = x.gather(1, torch.as_tensor(tok)[:, None])[:, 0]
    base = (400 + 2 * X) * U + 4 * U * lse
    near(c.lp[:R].cpu().numpy(), (xt - lse).numpy(), (base + 3 * U * xt.abs()).numpy())
    near(c.ent[:R].cpu().numpy(), (lse + X).numpy(), ((800 + 4 * X) * U * (1 + X) + 4 * U * (lse + X)).numpy())
    assert (c.lp[R:] == KEPT).all()


@pytest.mark.gpu
def test_outputs_not_wanted():
    z, tok = random_rows(4, 5000, torch.float32, 3)
    for want, top in (((True, False), 0), ((False, True), 0), ((False, False), 4), ((True, False), 2)):
        c = Call(z, 1.0, tok, top, want=want)
        c.run()
        c.check()
    kvr.kv_logprobs(c.z.data_ptr(), kvr.KV_F32, 4, 5000, 5000, 1.0, 0, 0, 0, 0, 0, 0, 0, 0)  # nothing wanted
    kvr.kv_logprobs(0, kvr.KV_F32, 0, 5000, 5000, 1.0, 0, 0, 0, 0, 0, 0, 0, 0)               # no rows


@pytest.mark.gpu
def test_graphs_follow_the_logits_and_share_a_workspace():
    a, b = (Call(*random_rows(R, V, torch.float32, R)[:1], 1.0, [1] * R, top) for R, V, top in ((5, 9000, 20), (600, 700, 3)))
    ws = torch.full((max(a.bytes, b.bytes),), 255, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = []
    for c in (a, b):
        with torch.cuda.stream(s):
            c.run(ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            c.run(ws)
        graphs.append(g)
    for step in range(4):
        for c, g in zip((a, b), graphs):
            z, _ = random_rows(*c.z.shape, torch.float32, 50 + step)
            c.z.copy_(z)
            c.host = z.numpy()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            c.check()


@pytest.mark.gpu
def test_calls_on_two_streams_at_once():
    calls = [Call(*random_rows(40, 30000, torch.float32, i)[:1], 1.0, [i] * 40, 20) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip(calls, streams):
            with torch.cuda.stream(s):
                c.run()
    torch.cuda.synchronize()
    for c in calls:
        c.check()


# ---- sizes and refusals (no device access) -------------------------------------
def test_workspace_bytes():
    assert kvr.kv_logprobs_workspace_bytes(16, 128256, 0) > 0
    assert kvr.kv_logprobs_workspace_bytes((1 << 20) - 1, 131072, 0) > 0
    assert kvr.kv_logprobs_workspace_bytes(16, 128256, 20) > kvr.kv_logprobs_workspace_bytes(16, 128256, 0)
    for bad in ((0, 100, 0), (-1, 100, 0), (1 << 21, 100, 0), (1, 0, 0), (1, (1 << 21) + 1, 0), (1, 100, -1),
                (1, 100, 65), (1, 10, 11), (1 << 20, 131073, 0), (1 << 16, 1 << 21, 0)):
        assert kvr.kv_logprobs_workspace_bytes(*bad) == 0


def test_a_device_that_is_not_there():
    with pytest.raises(kvr.KvError) as e:
        kvr.kv_logprobs(0x1000, kvr.KV_F32, 4, 1000, 1000, 1.0, 0x2000, 0, 0x3000, 0, 0, 0, 0x10000, 1 << 20, device=4096)
    assert e.value.status == kvr.KV_EDEVICE and e.value.message


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=2), kvr.KV_EINVAL), (dict(rows=-1), kvr.KV_EINVAL), (dict(rows=(1 << 20) + 1), kvr.KV_EINVAL),
    (dict(vocab=0), kvr.KV_EINVAL), (dict(rows=1 << 20, vocab=131073, stride=131073), kvr.KV_EINVAL),
    (dict(vocab=(1 << 21) + 1, stride=1 << 22), kvr.KV_EINVAL),
    (dict(stride=999), kvr.KV_EINVAL), (dict(scale=0.0), kvr.KV_EINVAL), (dict(scale=-1.0), kvr.KV_EINVAL),
    (dict(scale=float("inf")), kvr.KV_EINVAL), (dict(scale=2.0 ** 127 * 1.5), kvr.KV_EINVAL), (dict(scale=float("nan")), kvr.KV_EINVAL),
    (dict(top_n=-1), kvr.KV_EINVAL), (dict(top_n=65), kvr.KV_EINVAL), (dict(vocab=3, top_n=4), kvr.KV_EINVAL),
    (dict(logits=0), kvr.KV_EINVAL), (dict(tokens=0), kvr.KV_EINVAL), (dict(top_tokens=0), kvr.KV_EINVAL),
    (dict(top_logprobs=0), kvr.KV_EINVAL), (dict(logits=0x1002), kvr.KV_EINVAL), (dict(tokens=0x2001), kvr.KV_EINVAL),
    (dict(workspace=0), kvr.KV_EINVAL), (dict(workspace=0x10004), kvr.KV_EINVAL),
    (dict(workspace_bytes=10), kvr.KV_ENOMEM)])
def test_refusals(bad, status):
    a = dict(logits=0x1000, dtype=kvr.KV_F32, rows=4, vocab=1000, stride=1000, scale=1.0, tokens=0x2000, top_n=5,
             logprobs=0x3000, entropy=0x4000, top_logprobs=0x5000, top_tokens=0x6000, workspace=0x10000,
             workspace_bytes=1 << 20)
    with pytest.raises(kvr.KvError) as e:
        kvr.kv_logprobs(**{**a, **bad})
    assert e.value.status == status and e.value.message
