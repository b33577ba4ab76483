"""Plain statements of the 4-bit cache and of attention over it, for the tests (numpy / torch on the CPU, 64 bits)."""
from __future__ import annotations

import numpy as np
import torch

PAGE, D, TILE = 16, 128, 2176


def bf16_round(x):
    """float32 array -> nearest bf16 value, as float32 (torch's conversion rounds to nearest, ties to even)."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).bfloat16().float().numpy().reshape(np.shape(x))


def encode(x):
    """x [..., 128] float (bf16 values) -> codes uint8, scale float64, z int, by the definition in include/isd.h.

    Quotients are taken in 64 bits and rounded to 32 where the definition has a 32-bit quotient (the 64-bit quotient of
    two 24-bit numbers, rounded once more to 24 bits, is the correctly rounded one: 53 >= 2 * 24 + 2)."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(all="ignore"):
        lo, hi = np.minimum(0.0, x.min(-1)), np.maximum(0.0, x.max(-1))
        t = ((hi.astype(np.float32) - lo.astype(np.float32)).astype(np.float64) / 15.0).astype(np.float32)
        s = bf16_round(t).astype(np.float64)
        bad = ~np.isfinite(s) | ~np.isfinite(x).all(-1)
        live = ~bad & (s > 0)
        safe = np.where(live, s, 1.0)
        z = np.where(live, np.clip(np.rint((-lo / safe).astype(np.float32)), 0, 15), 0)
        q = np.rint((x / safe[..., None]).astype(np.float32)).astype(np.float64)
        c = np.where(live[..., None], np.clip(np.nan_to_num(q) + z[..., None], 0, 15), 0)
    return c.astype(np.uint8), np.where(bad, np.nan, s), z.astype(np.int64)


class Cache:
    """A 4-bit pool as separate arrays; `tiles()` packs it."""

    def __init__(self, pages, heads):
        self.c = np.zeros((2, pages, heads, PAGE, D), np.uint8)
        self.s = np.zeros((2, pages, heads, PAGE), np.float64)
        self.z128 = np.full((2, pages, heads, PAGE), 128, np.int64)

    def store(self, page, off, k, v):
        """k, v [heads, 128] of one token"""
        for i, x in enumerate((k, v)):
            c, s, z = encode(x)
            self.c[i, page, :, off], self.s[i, page, :, off], self.z128[i, page, :, off] = c, s, z + 128

    def empty(self, page, off):
        self.s[:, page, :, off], self.z128[:, page, :, off] = 0.0, 128

    def values(self, page):
        """K, V [heads, 16, 128] of a page"""
        with np.errstate(invalid="ignore"):
            return [self.s[i, page][..., None] * (self.c[i, page].astype(np.float64) - (self.z128[i, page][..., None] - 128))
                    for i in range(2)]


def unpack(tiles):
    """uint8 [..., 2176] -> codes (K, V) [..., 16, 128], scales (K, V), zeros (K, V) [..., 16], nibble by nibble."""
    tiles = np.asarray(tiles)
    tok, dim = np.meshgrid(np.arange(PAGE), np.arange(D), indexing="ij")
    codes = []
    for word, e in (((dim // 32) * 64 + tok * 4 + (dim % 32) // 8, dim % 8), (256 + dim * 2 + tok // 8, tok % 8)):
        bit = 4 * (e // 2) + 16 * (e % 2)
        codes.append((tiles[..., word * 4 + bit // 8] >> (bit % 8).astype(np.uint8)) & 15)
    meta = np.ascontiguousarray(tiles[..., 2048:]).view(np.uint16).reshape(*tiles.shape[:-1], 4, 16)
    f = (meta.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    return codes, (f[..., 0, :], f[..., 2, :]), (f[..., 1, :], f[..., 3, :])


def pack(cache: Cache):
    """The pool bytes of a Cache."""
    _, pages, heads = cache.c.shape[:3]
    out = np.zeros((pages, heads, TILE), np.uint8)
    tok, dim = np.meshgrid(np.arange(PAGE), np.arange(D), indexing="ij")
    for i, (word, e) in enumerate((((dim // 32) * 64 + tok * 4 + (dim % 32) // 8, dim % 8), (256 + dim * 2 + tok // 8, tok % 8))):
        bit = 4 * (e // 2) + 16 * (e % 2)
        byte = (word * 4 + bit // 8).reshape(-1)
        val = (cache.c[i].reshape(pages, heads, -1) << (bit % 8).astype(np.uint8).reshape(-1)).astype(np.uint8)
        for half in (0, 4):  # two nibbles of a byte come from two elements
            at = (bit % 8).reshape(-1) == half
            out[:, :, byte[at]] |= val[:, :, at]
    meta = np.stack([cache.s[0], cache.z128[0], cache.s[1], cache.z128[1]], 2).astype(np.float32)
    out[:, :, 2048:] = (np.ascontiguousarray(meta).view(np.uint32) >> 16).astype(np.uint16).reshape(pages, heads, 64).view(np.uint8)
    return out


def random_cache(pages, heads, seed, sigma=0.5):
    """A filled cache: codes, scales and zeros as the codec makes them from normal rows (drawn directly, not encoded)."""
    rng = np.random.default_rng(seed)
    c = Cache(pages, heads)
    c.c[:] = rng.integers(0, 16, c.c.shape, dtype=np.uint8)
    c.s[:] = bf16_round(rng.uniform(0.6, 1.4, c.s.shape) * sigma * 5.2 / 15).astype(np.float64)
    c.z128[:] = 128 + rng.integers(5, 11, c.z128.shape)
    return c


def attention(q, K, V, ctx, scale):
    """q [n, Hq, 128], K / V [Hkv, >= ctx + n, 128] in 64 bits -> out [n, Hq, 128], lse [n, Hq], and for the tolerances
    the weights' mean of |v| [n, Hq, 128] and max_j scale * sum_d |q_d K_jd| [n, Hq]."""
    n, Hq, _ = q.shape
    G = Hq // K.shape[0]
    out, lse = np.zeros(q.shape), np.zeros((n, Hq))
    absv, mag = np.zeros(q.shape), np.zeros((n, Hq))
    with np.errstate(all="ignore"):
        for r in range(n):
            L = ctx + r + 1
            for g in range(K.shape[0]):
                k, v, x = K[g, :L], V[g, :L], q[r, g * G:(g + 1) * G]
                a = x @ k.T * scale
                m = a.max(-1, keepdims=True)
                e = np.exp(a - m)
                t = e.sum(-1, keepdims=True)
                sl = slice(g * G, (g + 1) * G)
                out[r, sl], lse[r, sl] = (e / t) @ v, (m + np.log(t))[:, 0]
                absv[r, sl], mag[r, sl] = (e / t) @ np.abs(v), (np.abs(x) @ np.abs(k).T).max(-1) * scale
    return out, lse, absv, mag


def attention_bounds(out, lse, absv, mag):
    """How far bf16 outputs and fp32 log sums may be from `attention`'s.

    Score: an fp32 sum of 128 products of bf16 numbers (each product exact), at most 128 roundings of 2^-24 of
    the sum of magnitudes; its scaling, its distance from the reference maximum and the base-2 exponential (2 ulp) add a few
    more of 2^-24 of at most twice the magnitude: together (128 + 16) * 2^-24 * mag + 2^-21.  A probability is off by that factor and its
    product with the value scale is rounded to bf16 (2^-8 at most); numerator and sum each carry the factor, the sums
    over the keys at most another 2^-13 (2^11 rounding steps of 2^-24 in one accumulator chain).  The output is rounded
    to bf16 once more."""
    ds = 144 * 2.0 ** -24 * mag + 2.0 ** -21
    tol_out = (2.0 ** -8 + 2 * ds[..., None] + 2.0 ** -12) * absv * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(out) + 1e-30
    tol_lse = ds + 2.0 ** -12 + 2.0 ** -22 * np.abs(lse)
    return tol_out, tol_lse
