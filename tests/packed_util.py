"""The packed arena's format in numpy, 64 bits, from its definition (test-only)."""
import dataclasses

import numpy as np
import torch

from paper_2608_14635_amd import kvr
from paper_2608_14635_amd import workloads as W

MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
EVEN_FIRST = (0, 2, 4, 6, 1, 3, 5, 7)  # the order in which ties are settled
VALUES = np.concatenate([MAGNITUDES, -MAGNITUDES])

# heads of the decoders, cut to what the packed arena sees of them
BF16 = dataclasses.replace(W.TINY_BF16, num_layers=2, num_q_heads=32, num_kv_heads=8)
F32 = {d: dataclasses.replace(W.TINY_F32, num_layers=2, num_q_heads=8 * 128 // d, num_kv_heads=2 * 128 // d,
                              head_dim=d) for d in (32, 64, 128)}
SHAPES = {"bf16": BF16, "f32_32": F32[32], "f32_64": F32[64], "f32_128": F32[128]}


def quantise(x):
    """x [..., d] -> codes [..., d] of 0..15 and scale bytes [..., d/32], by trying every value."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, 32)
    most = np.abs(g).max(-1)
    finite = np.isfinite(g).all(-1)
    e = np.full(most.shape, -120)
    while True:
        over = finite & (most > 6 * np.exp2(e.astype(np.float64))) & (e < 125)
        if not over.any():
            break
        e = e + over
    with np.errstate(invalid="ignore"):
        y = np.abs(g) / np.exp2(e.astype(np.float64))[..., None]
        best, err = np.zeros(g.shape, np.int64), np.full(g.shape, np.inf)
        for c in EVEN_FIRST:
            diff = np.abs(y - MAGNITUDES[c])
            take = diff < err
            best, err = np.where(take, c, best), np.where(take, diff, err)
    codes = best + 8 * np.signbit(g)
    return codes.reshape(x.shape), np.where(finite, e + 127, 255)


def values(codes, scales):
    """What codes [..., d] and scale bytes [..., d/32] stand for, 64 bits."""
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    v = VALUES[codes].reshape(*scales.shape, 32) * s[..., None]
    return v.reshape(codes.shape)


def _split(raw, shape, blocks, B):
    L, nkv, d = shape.num_layers, shape.num_kv_heads, shape.head_dim
    rec = raw.reshape(L, blocks, nkv, B // 16, 17 * d)
    w = d // 32
    k, v = rec[..., :8 * d], rec[..., 8 * d:16 * d]
    ks, vs = rec[..., 16 * d:16 * d + 16 * w], rec[..., 16 * d + 16 * w:]
    v = v.reshape(*v.shape[:-1], 4, 16, 4, w).swapaxes(-3, -2)
    vs = vs.reshape(*vs.shape[:-1], 4, w, 4).swapaxes(-2, -1)

    def rows(a):  # [L, blocks, nkv, tiles, 16, n] -> [L, slots, nkv, n]
        a = a.reshape(L, blocks, nkv, B, -1)
        return a.swapaxes(2, 3).reshape(L, blocks * B, nkv, -1)
    return rows(k), rows(v), rows(ks), rows(vs)


def unpack(raw, shape, blocks, B):
    """The arena's bytes -> (k codes, v codes, k scale bytes, v scale bytes) by layer and slot."""
    k, v, ks, vs = _split(np.asarray(raw), shape, blocks, B)
    nib = lambda a: np.stack([a & 15, a >> 4], -1).reshape(*a.shape[:-1], -1)  # noqa: E731
    return nib(k), nib(v), ks, vs


class PackedArena:
    """A packed arena of arbitrary bytes on the device, bound."""

    def __init__(self, shape, B, blocks, seed=0):
        self.shape, self.B, self.blocks = shape, B, blocks
        n = kvr.kv_packed_bytes(shape, B, blocks)
        assert n == shape.num_layers * blocks * shape.num_kv_heads * (B // 16) * 17 * shape.head_dim
        rng = np.random.default_rng(seed)
        # a guard of 64 bytes behind the arena
        self.before = rng.integers(0, 256, size=n + 64).astype(np.uint8)
        self.raw = torch.from_numpy(self.before.copy()).cuda()
        self.handle = kvr.kv_packed_bind(self.raw.data_ptr(), n, shape, B, blocks)
        self.n = n

    def parts(self, before=False):
        raw = self.before if before else self.raw.cpu().numpy()
        assert np.array_equal(raw[self.n:], self.before[self.n:])
        return unpack(raw[:self.n], self.shape, self.blocks, self.B)

    def release(self):
        kvr.kv_packed_release(self.handle)


def torch_dtype(shape):
    return torch.bfloat16 if shape.dtype == W.BF16 else torch.float32
