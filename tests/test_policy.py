"""The clipped policy loss and its gradient (kv_policy_loss, include/kvr_policy.h) against
the formula in 64 bits, and the gradient against differences of the losses.

Tolerances, with u = 2^-24, T the largest |x_v - max x| / ln 2 that does not vanish (at most
150), p the token's probability:
  a term of the sum has the rounding of its exponent (u T), of the factor scale log2 e
  (u T) and of the exponential (2 u); a chunk's sum of them in fp32 has at most 32 + 10 steps:
  R = (50 + 2 T) u of the sum;
  lp = -log1p(rest / mine) then moves by (1 - p) R, and is rounded once;
  loss and kl by their slopes in lp times that, delta, and kl by e^D delta^2 besides: where D
  is 0 its slope is too, and kl(D + delta) = (e^D (e^delta - 1) - delta) + kl(D) differs from
  kl(D) + (e^D - 1) delta by e^D (e^delta - 1 - delta) <= e^D delta^2; grad by its row's slope, whose own slope in lp
  is w (rho |A| + kl_coef e^D), and by 2 R of its softmax; each rounded once to its type.
Rows are kept away from the clip bounds by far more than that."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_14635_amd import harness as Hn  # noqa: E402
from paper_2608_14635_amd import kvr  # noqa: E402

U = 2.0 ** -24
KEPT = 7.0
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def to64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Batch:
    def __init__(self, rows, vocab, dtype="f32", pad=0, lead=0, seed=0, std=2.0, scale=1.0, kl=0.05, old=True, ref=True,
                 weights=True, clip=(0.2, 0.3)):
        self.rows, self.vocab, self.scale, self.clip, self.kl = rows, vocab, scale, clip, kl
        self.dt = DT[dtype]
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        rand = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
        w = vocab + pad
        self.flat = rand(lead + rows * w).mul_(std).to(self.dt)
        self.z = self.flat[lead:].view(rows, w)[:, :vocab]
        self.tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
        self.advantages = rand(rows)
        lp = torch.log_softmax(self.z.double() * scale, -1).gather(1, self.tokens.long()[:, None])[:, 0]
        # ratios of e^-0.6 .. e^0.6, none within 0.02 of a bound
        steps = torch.tensor([-0.6, -0.3, -0.1, 0.0, 0.05, 0.2, 0.35, 0.6], device="cuda")
        pick = lambda: steps[torch.randint(0, 8, (rows,), generator=g, device="cuda")]  # noqa: E731
        self.old = (lp - pick()).float() if old else None
        self.ref = (lp + pick() + 0.3).float() if ref else None
        self.weights = torch.rand(rows, generator=g, device="cuda").add_(0.1) if weights else None
        f = lambda: torch.full((rows + 1,), KEPT, device="cuda")  # noqa: E731
        self.total, self.losses, self.logprobs = f()[:1].clone(), f(), f()
        self.kls = f() if ref else None
        self.grad = torch.full((rows * (w + 3) + lead,), KEPT, dtype=self.dt, device="cuda")
        self.g = self.grad[lead:].view(rows, w + 3)
        self.ws_bytes = kvr.kv_policy_loss_workspace_bytes(rows, vocab)
        self.ws = torch.full((self.ws_bytes,), 255, dtype=torch.uint8, device="cuda")

    def run(self, grad=True, in_place=False, ws=None, stream=None):
        p = lambda t: 0 if t is None else t.data_ptr()  # noqa: E731
        g, gs = (self.z, self.z.stride(0)) if in_place else (self.g, self.g.stride(0))
        kvr.kv_policy_loss(p(self.z), kvr.KV_F32 if self.dt == torch.float32 else kvr.KV_BF16, self.rows, self.vocab,
                           self.z.stride(0), self.scale, p(self.tokens), p(self.old), p(self.ref), p(self.advantages),
                           p(self.weights), self.clip[0], self.clip[1], self.kl, p(self.total), p(self.losses),
                           p(self.logprobs), p(self.kls), p(g) if grad else 0, gs, p(self.ws if ws is None else ws),
                           self.ws_bytes, stream=Hn.stream_ptr() if stream is None else stream)

    def reference(self):
        """{name: (value, tolerance)} of every output, 64 bits."""
        n, V, s = self.rows, self.vocab, self.scale
        z, t = to64(self.z), self.tokens.cpu().numpy()
        w = np.ones(n) if self.weights is None else to64(self.weights)
        a = to64(self.advantages)
        out = {k: np.zeros(n) for k in ("losses", "logprobs", "kls")}
        tol = {k: np.full(n, 1e-37) for k in out}
        grad, grad_tol = np.zeros((n, V)), np.full((n, V), 1e-36)
        half = torch.finfo(self.dt).eps / 2
        beta, (cl, ch) = self.kl, self.clip
        with np.errstate(all="ignore"):
            for i in range(n):
                if not 0 <= t[i] < V:
                    continue
                x = s * z[i]
                m = x.max()
                if m == -math.inf:
                    lp, p, rest, T = -math.inf, np.zeros(V), 1.0, 0
                else:
                    e = np.exp(x - m)
                    others = np.delete(e, t[i]).sum()
                    T = min(150, np.min(x, where=x > m - 104, initial=m) * -1 + m) / math.log(2) if np.isfinite(m) else 0
                    lp = -np.log1p(others / e[t[i]]) if e[t[i]] > others else x[t[i]] - m - np.log(e.sum())
                    rest, p = others / e.sum(), e / e.sum()
                R = (50 + 2 * T) * U
                out["logprobs"][i], tol["logprobs"][i] = lp, rest * R + U * abs(lp) + 1e-37
                if w[i] == 0:
                    continue
                rho = np.exp(lp - to64(self.old)[i]) if self.old is not None else np.exp(lp - lp) if lp > -math.inf else 1.0
                plain, cut = rho * a[i], np.clip(rho, 1 - cl, 1 + ch) * a[i]
                kept = not plain > cut
                D = to64(self.ref)[i] - lp if self.ref is not None else 0.0
                kl = math.inf if np.expm1(D) == math.inf else np.expm1(D) - D
                fall = beta * np.expm1(D) if beta else 0.0
                loss = w[i] * ((beta * kl if beta else 0.0) - (plain if kept else cut))
                slope = w[i] * (-(plain if kept else 0.0) - fall)
                bend = w[i] * (abs(plain if kept else 0.0) + beta * np.exp(D))
                second = np.exp(min(D, 80.0)) * (rest * R) ** 2
                # a term with coefficient 0 is not in the loss, nor is its rounding (0 times an infinite kl is NaN)
                far = beta * kl if beta else 0.0
                out["losses"][i], tol["losses"][i] = loss, w[i] * beta * second + abs(slope) * rest * R + 2 * U * w[i] * (abs(plain if kept else cut) + far)
                out["kls"][i], tol["kls"][i] = kl, abs(np.expm1(D)) * rest * R + U * kl + second
                shape = -p
                shape[t[i]] = rest
                grad[i] = s * slope * shape
                grad_tol[i] += np.abs(grad[i]) * (2 * R + 8 * U + half) + s * bend * rest * R * np.abs(shape)
        res = {k: (out[k], tol[k] + 1e-37) for k in out}
        res["total"] = (out["losses"].sum()[None], tol["losses"].sum()[None] + U * np.abs(out["losses"].sum()) + 1e-37)
        res["grad"] = (grad, grad_tol)
        return res

    def check(self, grad=True, want=None):
        want = want or self.reference()
        got = {"total": to64(self.total), "losses": to64(self.losses), "logprobs": to64(self.logprobs)}
        if self.kls is not None:
            got["kls"] = to64(self.kls)
        if grad:
            g = to64(self.g)
            assert (g[:, self.vocab:] == KEPT).all()
            got["grad"] = g[:, :self.vocab]
        for k, v in got.items():
            if k not in ("total", "grad"):
                assert v[-1] == KEPT
                v = v[:-1]
            w, tol = want[k]
            same = (v == w) | (np.isnan(v) & np.isnan(w))
            with np.errstate(invalid="ignore"):
                bad = ~same & ~(np.abs(v - w) <= tol)
            assert not bad.any(), (k, int(bad.sum()), v[bad][:4], w[bad][:4], tol[bad][:4])


SIZES = [(1, 1), (3, 2), (5, 7), (70, 301), (4, 8192), (3, 8193), (2, 20001), (5, 32769), (3, 131073), (1, 1 << 21)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_loss_and_gradient(dtype, rows, vocab):
    for i, (pad, lead) in enumerate([(0, 0), (3, 1), (5, 2)]):
        b = Batch(rows, vocab, dtype, pad, lead, seed=rows + vocab + i, scale=(1.0, 1.25, 0.7)[i])
        b.run()
        torch.cuda.synchronize()
        b.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [8193, 16385, 32768, 40003, 65537, 90001, 131073, 163839, 200001])
def test_many_rows(dtype, vocab):
    """Enough rows that each has a workgroup of its own, which takes several, one after the other;
    vocabularies that end within a thread's piece, at its border, and past what its registers hold."""
    b = Batch(300, vocab, dtype, pad=vocab % 5, lead=vocab % 3, seed=vocab)
    b.weights[[3, 290]] = 0
    b.tokens[7], b.tokens[299] = -1, vocab
    b.tokens[8], b.tokens[9], b.tokens[10], b.tokens[11] = 0, vocab - 1, vocab - 9, vocab // 2
    lp = torch.log_softmax(b.z[8:12].double(), -1).gather(1, b.tokens[8:12].long()[:, None])[:, 0]
    b.old[8:12], b.ref[8:12] = (lp + 0.1).float(), (lp - 0.2).float()
    b.z[5, 100:] = -math.inf
    b.tokens[5] = 60
    lp = float(torch.log_softmax(b.z[5].double(), -1)[60])
    b.old[5], b.ref[5] = lp - 0.1, lp + 0.3
    b.run()
    torch.cuda.synchronize()
    b.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(65, 9001), (7, 40001), (131, 33001)])
@pytest.mark.parametrize("what", [dict(kl=0.0, ref=False), dict(old=False), dict(weights=False), dict(kl=0.0),
                                  dict(clip=(0.0, 0.0)), dict(clip=(1.0, math.inf)),
                                  dict(old=False, ref=False, weights=False, kl=0.0)])
def test_what_may_be_left_out(dtype, what, rows, vocab):
    b = Batch(rows, vocab, dtype, seed=5, **what)
    if what.get("clip") == (0.0, 0.0):
        b.old += 0.01  # off the bounds that ratios of 1 are on
    b.run()
    torch.cuda.synchronize()
    b.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_alone(dtype):
    """The same results without a gradient, by the same tolerances (rows are summed in another
    order), and nothing written to it."""
    for rows, vocab in ((300, 10007), (5, 40000), (400, 900), (512, 17003), (513, 17003), (3, 32769), (256, 65536),
                        (130, 70001), (200, 200003), (257, 40000)):
        b = Batch(rows, vocab, dtype, pad=1, seed=6)
        b.run(grad=False)
        torch.cuda.synchronize()
        b.check(grad=False)
        assert bool((b.grad == KEPT).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(7, 5), (40, 20011), (600, 3001), (300, 90003), (270, 170001)])
def test_over_the_logits(dtype, rows, vocab):
    b = Batch(rows, vocab, dtype, pad=3, lead=1, seed=7)
    b.run()
    before = b.flat.clone()
    torch.cuda.synchronize()
    want = b.g[:, :vocab].clone()
    b.run(in_place=True)
    torch.cuda.synchronize()
    assert torch.equal(b.z, want)
    kept = torch.ones_like(b.flat, dtype=torch.bool)
    kept[1:].view(rows, vocab + 3)[:, :vocab] = False
    assert torch.equal(b.flat[kept], before[kept])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(40, 700), (40, 17000), (40, 50000), (140, 50000)])
def test_tokens_next_to_certain(dtype, rows, vocab):
    """Log probabilities of -1e-3 to -1e-20, to parts of themselves."""
    b = Batch(rows, vocab, dtype, seed=8, std=1.0)
    b.z[torch.arange(rows, device="cuda"), b.tokens.long()] = torch.linspace(8, 60, rows, device="cuda").to(b.dt)
    b.old.fill_(-0.1)
    b.ref.fill_(-0.05)
    want = b.reference()
    assert (want["logprobs"][0] < 0).all() and want["logprobs"][0][-1] > -1e-18
    b.run()
    torch.cuda.synchronize()
    b.check(want=want)
    for t in (b.total, b.losses, b.logprobs, b.kls):
        t.fill_(KEPT)
    b.run(grad=False)
    torch.cuda.synchronize()
    b.check(grad=False, want=want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(12, 64), (12, 9000), (12, 33000), (140, 33000)])
def test_masked_and_left_out(dtype, rows, vocab):
    """Masked logits, rows of nothing else, weights of 0 over NaN, tokens that are none."""
    b = Batch(rows, vocab, dtype, seed=9, kl=0.0)
    tok, inf, nan = b.tokens.long(), math.inf, math.nan
    keep = b.z[torch.arange(rows), tok].clone()
    b.z[0, ::2] = -inf
    b.z[1, :] = -inf
    b.z[2, :] = -inf                                  # the token's alone
    b.z[3, 1:vocab // 2] = torch.finfo(b.dt).min
    b.z[torch.tensor([0, 2, 3]), tok[[0, 2, 3]]] = keep[[0, 2, 3]]
    b.z[4] = torch.finfo(b.dt).min                    # a flat row of the least number
    b.z[5, 3] = nan
    b.z[6, 4] = inf
    b.weights[[7, 8]] = 0
    b.z[7, 5], b.advantages[8], b.old[8], b.ref[8] = nan, nan, inf, nan
    b.tokens[9], b.tokens[10], b.tokens[11] = -1, vocab, 2 ** 31 - 1
    b.z[9, :3], b.advantages[10] = nan, nan
    lp = torch.log_softmax(b.z.double(), -1)
    ok = [0, 2, 3, 4]
    b.old[ok] = lp[torch.tensor(ok), tok[ok]].float() + 0.1
    b.old[1] = -3.0
    want = b.reference()
    # the reference's own arithmetic where a row is not a number
    for row in (5, 6):
        for k in ("losses", "logprobs", "kls"):
            want[k][0][row] = nan
        want["grad"][0][row] = nan
    want["logprobs"][0][7], want["total"][0][:] = nan, nan
    b.run()
    torch.cuda.synchronize()
    b.check(want=want)
    g = to64(b.g)[:, :vocab]
    assert not g[[1, 7, 8, 9, 10, 11]].any()
    assert not g[0, torch.isinf(b.z[0]).cpu().numpy()].any()
    for t in (b.total, b.losses, b.logprobs, b.kls):
        t.fill_(KEPT)
    b.run(grad=False)
    torch.cuda.synchronize()
    b.check(grad=False, want=want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(12, 64), (12, 9000), (12, 33000), (140, 33000), (140, 170001)])
def test_steep_rows(dtype, rows, vocab):
    """Slopes that pass the largest number, by far policies and far references, over probabilities
    that make numbers of them again; masked logits and those of the least number beside them, at
    the row's token too.  An entry of probability 0 has gradient 0.  An entry's exponent has the
    roundings of its difference, of the scale and of the sum: 3 u of its size."""
    b = Batch(rows, vocab, dtype, pad=1, seed=21, kl=0.05)
    low, inf = torch.finfo(b.dt).min, math.inf
    at = [2, vocab // 2, vocab - 3]
    for i, (mine, others) in enumerate([(-64, -50), (-104, -100), (-304, -300), (-inf, -80), (0, -90), (0, -250), (0, -300),
                                        (low, -90), (0, -inf)]):
        b.z[i, at] = others
        b.z[i, [5, vocab - 9]], b.z[i, [6, vocab // 3]] = -inf, low
        if i == 8:
            b.z[i] = -inf
        b.tokens[i] = [0, vocab - 1, vocab // 4][i % 3]
        b.z[i, int(b.tokens[i])] = mine
    lp = torch.log_softmax(b.z[:9].double(), -1).gather(1, b.tokens[:9].long()[:, None])[:, 0]
    b.old[:9], b.ref[:9] = (lp + 0.1).float(), -2.0
    b.old[3], b.old[4], b.old[5], b.old[6], b.old[8] = -1.0, lp[4] - 100, lp[5] - 300, lp[6] - 300, -800.0
    b.advantages[[4, 5, 8]], b.advantages[6] = -1.5, 2.0
    b.run()
    torch.cuda.synchronize()
    want = b.reference()
    x = to64(b.z) - to64(b.z).max(-1, keepdims=True)
    with np.errstate(all="ignore"):
        for k, (v, tol) in want.items():
            tol = np.where(np.isfinite(tol), tol, 0.0)
            if k == "grad":
                none = np.exp(x[:9]) == 0
                none[8] = True  # its token's probability is 1
                none[np.arange(8), b.tokens[:8].cpu().numpy()] = False
                v[:9][none] = 0
                tol += 3 * U * np.abs(v) * np.minimum(np.abs(x), 1000) / math.log(2)
            # a rounding to the nearest is infinite from half a step above the largest number on
            eps = torch.finfo(b.dt if k == "grad" else torch.float32).eps
            want[k] = (np.where(np.abs(v) >= 2.0 ** 128 * (1 - eps / 4), np.sign(v) * inf, v), tol)
    assert np.isinf(want["losses"][0][[1, 2, 3, 4, 5, 7, 8]]).all() and np.isfinite(want["losses"][0][[0, 6]]).all()
    g = np.abs(want["grad"][0][:, at[0]])
    assert 0.01 < g[1] < 1 and 0.01 < g[2] < 1 and 1e12 < g[5] < 1e22 and np.isinf(g[[3, 7]]).all()
    b.check(want=want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(5, 4000), (5, 30011), (5, 40003), (130, 151936), (130, 500003)])
def test_equal_logits(dtype, rows, vocab):
    """Rows of one value, a third of them with a few larger ones: sums of equal terms, whose roundings
    all go one way."""
    b = Batch(rows, vocab, dtype, seed=17)
    b.z[:] = torch.linspace(-3, 3, rows, device="cuda")[:, None].to(b.dt)
    b.z[::3, ::1000] += 1.0 / 3.0
    lp = torch.log_softmax(b.z.double(), -1).gather(1, b.tokens.long()[:, None])[:, 0]
    b.old, b.ref = (lp + 0.1).float(), (lp - 0.2).float()
    b.run()
    torch.cuda.synchronize()
    want = b.reference()
    b.check(want=want)
    for t in (b.total, b.losses, b.logprobs, b.kls):
        t.fill_(KEPT)
    b.run(grad=False)
    torch.cuda.synchronize()
    b.check(grad=False, want=want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,std,scale", [("f32", 1e30, 1e-30), ("f32", 5e37, 4e-38), ("bf16", 1e37, 1e-37),
                                             ("f32", 3000.0, 1.0), ("f32", 1e-3, 2000.0)])
@pytest.mark.parametrize("rows,vocab", [(20, 3000), (20, 33000), (129, 33000)])
def test_logits_of_any_size(dtype, std, scale, rows, vocab):
    b = Batch(rows, vocab, dtype, seed=10, std=std, scale=scale)
    lp = torch.log_softmax(b.z.double() * scale, -1)
    b.tokens[:10] = lp[:10].argmax(-1).int()
    mine = lp.gather(1, b.tokens.long()[:, None])[:, 0]
    b.old, b.ref = (mine - 0.1).float(), (mine + 0.2).float()
    # differences of logits are of one sign and exact to 2 u of them: an error of the exponent
    want = b.reference()
    z = b.z.double() * scale
    spread = float(((z.amax(-1) - z.amin(-1)).clamp(max=150) + mine.abs().clamp(max=1e6)).max())
    extra = 4 * U * spread
    for k in ("logprobs", "losses", "kls", "total", "grad"):
        v, t = want[k]
        grow = {"logprobs": extra + U * np.abs(v), "kls": extra * 2, "losses": extra * 6 * np.ones_like(v),
                "total": extra * 6 * b.rows, "grad": extra * 8 * np.abs(v) + extra * scale * 6 * np.abs(v)}[k]
        want[k] = (v, t + grow)
    # old and ref are rounded to fp32: the ratio follows them, not lp
    b.run()
    torch.cuda.synchronize()
    b.check(want=want)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab,grad", [(6, 40000, False), (130, 90001, False), (130, 90001, True), (6, 90001, True),
                                             (6, 30011, True), (6, 9001, True)])
@pytest.mark.parametrize("sign", [1, -1])
def test_logits_of_two_bases(rows, vocab, grad, sign):
    """Logits in steps of 1/16 about 2^20 ln 2, where their multiples change from numbers that may be
    rounded to ones that may not: a row's first entries below its later ones, ones above them,
    all of one height, and steps at odd places.  Differences of logits are exact."""
    b = Batch(rows, vocab, seed=31, pad=1)
    g = torch.Generator(device="cuda")
    g.manual_seed(vocab)
    steps = torch.randint(-9, 3, b.z.shape, generator=g, device="cuda")  # 726817.5 is 2^20 ln 2 + 0.11
    at = torch.arange(vocab, device="cuda")
    steps[0::6] += 6 * (at >= min(8192, vocab // 2))
    steps[1::6] += 6 * (at < vocab // 2)
    steps[2::6] += 4 * (at // 4096)
    steps[4::6] = steps[4::6].clamp(max=-3) + 6 * (at >= 73728)  # past what a long row's registers hold
    steps[5::6] += 6 * (at % 7919 > 7000)
    b.z[:] = sign * 726817.5 + steps / 16.0
    lp = torch.log_softmax(b.z.double(), -1).gather(1, b.tokens.long()[:, None])[:, 0]
    b.old, b.ref = (lp + 0.1).float(), (lp - 0.2).float()
    b.run(grad=grad)
    torch.cuda.synchronize()
    b.check(grad=grad)


@pytest.mark.gpu
def test_gradient_against_differences():
    """Central differences with step h of the losses that the forward pass returns: off by
    h^2/6 of the third derivative, at most 2 (rho |A| + kl_coef (e^D + 1)), and by the losses' own
    tolerances over h."""
    b = Batch(24, 40, seed=11, kl=0.1, clip=(0.9, 20.0))  # nothing clipped within a step
    b.run()
    torch.cuda.synchronize()
    grad, h = to64(b.g)[:, :40], 2.0 ** -6
    w, a = to64(b.weights), to64(b.advantages)
    lp = to64(b.logprobs)[:-1]
    rho, e = np.exp(lp - to64(b.old)), np.exp(to64(b.ref) - lp)
    tol = w * (2 * 1.2 * (rho * np.abs(a) + 0.1 * (e + 1))) * h * h / 6 + 2 * b.reference()["losses"][1].max() / h
    for v in range(0, 40, 3):
        ends = []
        for step in (h, -h):
            z = b.z.clone()
            b.z[:, v] += step
            b.run(grad=False)
            torch.cuda.synchronize()
            ends.append(to64(b.losses)[:-1])
            # the step that was taken
            ends.append(to64(b.z[:, v]))
            b.z.copy_(z)
        d = (ends[0] - ends[2]) / (ends[1] - ends[3])
        assert (np.abs(d - grad[:, v]) <= tol).all(), v


@pytest.mark.gpu
def test_graphs_follow_their_arrays_and_share_a_workspace():
    batches = (Batch(33, 20000, seed=12), Batch(9, 500, "bf16", seed=13), Batch(131, 33001, "bf16", seed=15),
               Batch(5, 40000, seed=16))
    ws = torch.full((max(x.ws_bytes for x in batches),), 255, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    for x in batches:
        with torch.cuda.stream(side):
            x.run(ws=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            x.run(ws=ws)
        graphs.append(g)
    for step in range(3):
        for x, g in zip(batches, graphs):
            x.z.copy_(torch.randn(x.z.shape, device="cuda") * 2)
            x.tokens.copy_(torch.randint(-1, x.vocab, (x.rows,), device="cuda"))
            # rows may land near a bound: replay and eager are compared bit for bit
            for t in (x.g, x.losses, x.logprobs, x.kls, x.total):
                t.fill_(KEPT)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in (x.g, x.losses, x.logprobs, x.kls, x.total)]
            x.run()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(got, (x.g, x.losses, x.logprobs, x.kls, x.total)))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab", [(200, 30000), (300, 40000), (50, 40000)])
def test_two_streams_at_once(rows, vocab):
    b = Batch(rows, vocab, "bf16", seed=14)
    b.run()
    torch.cuda.synchronize()
    want, wsum = b.g.clone(), b.total.clone()
    outs = []
    streams = [torch.cuda.Stream() for _ in range(2)]
    wss = [torch.full_like(b.ws, 255) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(4):
        for s, ws in zip(streams, wss):
            with torch.cuda.stream(s):
                b.g, b.total = torch.full_like(want, KEPT), torch.full_like(wsum, KEPT)
                b.run(ws=ws, stream=s.cuda_stream)
                outs.append((b.g, b.total))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) and torch.equal(t, wsum) for g, t in outs)


@pytest.mark.gpu
def test_rows_past_four_gib():
    """The last rows of 5 GiB of logits and of their gradient, those before them with weight 0."""
    rows, vocab = 20000, 131072
    z = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    small = Batch(4, vocab, "bf16", seed=15)
    z[-4:] = small.z
    small.run()
    f = lambda t: torch.cat([torch.zeros(rows - 4, device="cuda", dtype=t.dtype), t])  # noqa: E731
    args = [f(t) for t in (small.tokens, small.old, small.ref, small.advantages, small.weights)]
    grad = torch.full((rows, vocab), KEPT, dtype=torch.bfloat16, device="cuda")
    n = kvr.kv_policy_loss_workspace_bytes(rows, vocab)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    out = torch.empty(rows, device="cuda")
    kvr.kv_policy_loss(z.data_ptr(), kvr.KV_BF16, rows, vocab, vocab, 1.0, *(t.data_ptr() for t in args), *small.clip,
                       small.kl, 0, out.data_ptr(), 0, 0, grad.data_ptr(), vocab, ws.data_ptr(), n,
                       stream=Hn.stream_ptr())
    torch.cuda.synchronize()
    assert not out[:-4].any() and not bool((grad[:-4] != 0).any())
    small.losses[:4], small.g[:, :vocab] = out[-4:], grad[-4:]  # by the formula, like the same rows alone
    small.check()


@pytest.mark.gpu
def test_no_rows():
    t = torch.full((1,), KEPT, device="cuda")
    kvr.kv_policy_loss(0, kvr.KV_F32, 0, 5, 5, 1.0, 0, 0, 0, 0, 0, 0.2, 0.2, 0.0, t.data_ptr(), 0, 0, 0, 0, 0, 0, 0,
                       stream=Hn.stream_ptr())
    torch.cuda.synchronize()
    assert float(t) == 0.0


# ---- sizes and refusals -----------------------------------------------------
def test_workspace_bytes():
    f = kvr.kv_policy_loss_workspace_bytes
    assert f(1, 1) > 0 and f(1 << 20, 8192 * 15) > 0
    for bad in ((0, 5), (5, 0), (-1, 5), ((1 << 20) + 1, 5), (5, (1 << 21) + 1), (1 << 20, 1 << 20)):
        assert f(*bad) == 0, bad
    rng = np.random.default_rng(3)
    for _ in range(2000):
        big = int(2 ** rng.uniform(0, 14)), int(2 ** rng.uniform(0, 20))
        small = tuple(int(rng.integers(1, n + 1)) for n in big)
        assert 0 < f(*small) <= f(*big)


def test_refusals():
    ok = dict(logits=0x1000, dtype=kvr.KV_F32, rows=4, vocab=100, stride=100, scale=1.0, tokens=0x2000,
              old_logprobs=0x3000, ref_logprobs=0x4000, advantages=0x5000, weights=0x6000, clip_low=0.2, clip_high=0.2,
              kl_coef=0.1, total=0x7000, losses=0x8000, logprobs=0x9000, kls=0xa000, grad=0xb000, grad_stride=100,
              workspace=0x10000, workspace_bytes=1 << 20)
    nan, inf = math.nan, math.inf
    for bad in (dict(dtype=2), dict(rows=-1), dict(rows=(1 << 20) + 1), dict(vocab=0), dict(vocab=(1 << 21) + 1),
                dict(rows=1 << 20, vocab=1 << 20, stride=1 << 20, grad_stride=1 << 20), dict(stride=99), dict(grad_stride=99),
                dict(stride=1 << 60), dict(scale=0.0), dict(scale=-1.0), dict(scale=nan), dict(scale=inf), dict(clip_low=-0.1),
                dict(clip_low=1.1), dict(clip_low=nan), dict(clip_high=-0.1), dict(clip_high=nan), dict(kl_coef=nan),
                dict(kl_coef=inf), dict(ref_logprobs=0), dict(ref_logprobs=0, kls=0), dict(ref_logprobs=0, kl_coef=0.0),
                dict(logits=0), dict(tokens=0), dict(advantages=0), dict(logits=0x1002), dict(tokens=0x2001),
                dict(old_logprobs=0x3002), dict(weights=0x6002), dict(total=0x7002), dict(grad=0xb002),
                dict(workspace=0), dict(workspace=0x10008), dict(grad=0x1000, grad_stride=104)):
        with pytest.raises(kvr.KvError) as e:
            kvr.kv_policy_loss(**{**ok, **bad})
        assert e.value.status == kvr.KV_EINVAL, bad
    need = kvr.kv_policy_loss_workspace_bytes(4, 100)
    with pytest.raises(kvr.KvError) as e:
        kvr.kv_policy_loss(**{**ok, "workspace_bytes": need - 1})
    assert e.value.status == kvr.KV_ENOMEM
    with pytest.raises(kvr.KvError) as e:
        kvr.kv_policy_loss(**{**ok, "device": 9999})
    assert e.value.status == kvr.KV_EDEVICE
    kvr.kv_policy_loss(**{**ok, "rows": 0, "total": 0})  # nothing to do
    kvr.kv_policy_loss(**{**ok, "total": 0, "losses": 0, "logprobs": 0, "kls": 0, "grad": 0})
