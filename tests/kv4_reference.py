"""The 4-bit key/value cache in 64 bits, from the definitions in include/moe_kv.h: what its tests compare with.  Nothing here uses the library."""
from __future__ import annotations

import math

import numpy as np

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def value_of(codes: np.ndarray) -> np.ndarray:
    return np.where(codes & 8, -1.0, 1.0) * LEVELS[codes & 7]


def nearest(x: np.ndarray) -> np.ndarray:
    """The code nearest to x (|x| up to 6), of two as near the even one."""
    d = np.abs(np.abs(x)[..., None] - LEVELS)
    low = d.argmin(-1)
    tie = (low < 7) & (d[..., 0] >= 0) & (np.take_along_axis(d, np.minimum(low + 1, 7)[..., None], -1)[..., 0] == np.take_along_axis(d, low[..., None], -1)[..., 0])
    return np.where(tie & (low % 2 == 1), low + 1, low) | np.where(np.signbit(x), 8, 0)


def exponent(amax: np.ndarray) -> np.ndarray:
    """Of the smallest power of two, 2^-45 at least, of which six reach amax."""
    e = np.full(np.shape(amax), -45)
    for n in range(-45, 45):
        e = np.where(amax > 6 * 2.0 ** n, n + 1, e)
    return e


def quantized(x: np.ndarray, width: int, top: float):
    """(codes [..., n], exponents [..., n / width]) of groups of `width` along the last axis."""
    x = np.where(np.isnan(x), 0.0, np.clip(x, -top, top))
    g = x.reshape(*x.shape[:-1], -1, width)
    e = exponent(np.abs(g).max(-1))
    return nearest(g / np.exp2(e)[..., None]).reshape(x.shape), e


def unpack(b: np.ndarray) -> np.ndarray:
    return np.stack([b & 15, b >> 4], -1).reshape(*b.shape[:-1], -1)


def key_codes(k: np.ndarray) -> np.ndarray:
    """[..., page, D] of a cache's bytes [..., page, D/2]."""
    return unpack(k)


def key_exponents(b: np.ndarray) -> np.ndarray:
    """[..., page, D/32] of scale bytes [..., page/16, 4, D/32, 4]."""
    x = b.astype(np.int64) - 127
    x = np.moveaxis(x, -1, -3)                  # [..., page/16, 4 t, 4 r, D/32]
    return x.reshape(*x.shape[:-4], -1, x.shape[-1])


def value_codes(v: np.ndarray) -> np.ndarray:
    """[..., page, D] of a cache's bytes [..., page/16, D, 8]."""
    x = np.swapaxes(unpack(v), -1, -2)
    return x.reshape(*x.shape[:-3], -1, x.shape[-1])


def keys(k, kb) -> np.ndarray:
    c, e = key_codes(k), key_exponents(kb)
    return value_of(c) * np.repeat(np.exp2(e.astype(np.float64)), 32, -1)


def values(v, vb) -> np.ndarray:
    return value_of(value_codes(v)) * np.exp2(vb.astype(np.float64) - 127)[..., None]


def attend_head(q, k, v, vs, positions, n_keys, scale, causal, window):
    """(out, lse, what roundings may do to out, and to lse) of rows q [n][dim] with `positions`, in 64 bits.  vs: the values' scales."""
    j = np.arange(n_keys)
    pos = np.asarray(positions)[:, None]
    see = (j <= pos) if causal else np.ones((len(q), n_keys), bool)
    if window:
        see = see & (j > pos - window)
    k, v, vs = k[:n_keys], v[:n_keys], vs[:n_keys]
    with np.errstate(invalid="ignore"):
        z = np.where(see, scale * (q @ k.T), -np.inf)
    # A query's number is off by 2^-20 of the power of two above the largest of its 32 dims, twice that largest number at most: 2^-19 of it.
    blocks = np.repeat(np.abs(q).reshape(len(q), -1, 32).max(-1), 32, -1)
    # fp32 sums of D / 32 blocks of four digits (32 additions at heads of 256, each off by 2^-24 of what is there), and two products: 2^-19 of the terms' sizes
    noise = scale * (2.0 ** -19 * (np.abs(q) @ np.abs(k).T) + 2.0 ** -19 * (blocks @ np.abs(k).T))
    out, lse = np.zeros((len(q), v.shape[1])), np.full(len(q), -np.inf)
    slack, off = np.zeros((len(q), v.shape[1])), np.zeros(len(q))
    for i in range(len(q)):
        s = see[i]
        if not s.any():
            continue
        top = z[i][s].max()
        p = np.exp(z[i][s] - top)
        lse[i] = top + math.log(p.sum())
        p /= p.sum()
        out[i] = p @ v[s]
        # the exponent in powers of two, its scale's byte added: below 2^8 or the scores' own size, rounded three times by 2^-24 of that; exp2 by 2^-22
        wrong = noise[i][s].max() + 2.0 ** -21.4 * max(256.0, 1.5 * np.abs(z[i][s]).max()) * math.log(2) + 2.0 ** -22
        n = int(s.sum())
        # weights are rounded to fp16: by half a step, 2^-11, and below 2^-14 by 2^-25 where the largest is at least 1; sums of n in fp32
        sums = n * 2.0 ** -24 + 2.0 ** -20
        slack[i] = (2 * wrong + 2.0 ** -11 + 2 * sums) * (p @ np.abs(v[s])) + 2.0 ** -25 * 6 * n * (p * vs[s]).max()
        off[i] = wrong + sums + 2.0 ** -21 * abs(lse[i])
    return out, lse, slack, off
