"""The attention half of a decode step in 64 bits, one number after the other, from the definitions in include/moe_kv.h: what
the tests of the paged 8-bit cache compare with.  Nothing here uses the library."""
from __future__ import annotations

import math

import numpy as np
import torch

LARGEST = {"e4m3": 448.0, "int8": 127.0}
CODE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def e4m3_table():
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[c] = math.nan if c & 127 == 127 else -v if c & 128 else v
    return out


E4M3 = e4m3_table()


def code_values(codes: np.ndarray, fmt: str) -> np.ndarray:
    return E4M3[codes] if fmt == "e4m3" else codes.view(np.int8).astype(np.float64)


def nearest(x: np.ndarray, fmt: str) -> np.ndarray:
    """The format's value nearest to x (|x| within the largest), ties to even."""
    if fmt == "int8":
        return np.rint(x)
    _, e = np.frexp(x)
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)
    return np.rint(x / step) * step


def page_scale(amax: float, fmt: str) -> float:
    if amax == 0:
        return 2.0 ** -96
    e = -96
    while amax > LARGEST[fmt] * 2.0 ** e:
        e += 1
    return 2.0 ** e


def plan(ctx, new, table, free, room, *, n_tokens, max_new, n_pages, page):
    """What moe_kv_plan writes, request after request; `table` is changed."""
    width = table.shape[1]
    room = min(max(room, 0), n_pages)
    start, positions, slots, kv, status, asked, used, rows = [0], [-1] * n_tokens, [-1] * n_tokens, [], [], 0, 0, 0
    for r, (c, n) in enumerate(zip(ctx, new)):
        st = 3 if c < 0 or n < 0 or n > max_new else 0
        c, n = max(c, 0), min(max(n, 0), n_tokens + 1)
        rows += n
        if rows > n_tokens:
            st = 3
        held, total = -(-c // page), -(-(c + n) // page)
        if not st and total > width:
            st = 2
        pages = total - held if not st else 0
        asked += pages
        if pages and asked > room:
            st = 1
        start.append(min(rows, n_tokens))
        if not st:
            for b in range(held, total):
                table[r, b] = free[room - 1 - used]
                used += 1
            for i in range(n):
                p = c + i
                positions[start[-2] + i] = p
                t = int(table[r, p // page])
                slots[start[-2] + i] = t * page + p % page if 0 <= t < n_pages else -1
        kv.append(c if st else c + n)
        status.append(st)
    return start, positions, slots, kv, status, room - used


def turned(x: np.ndarray, positions, gamma, eps, freq, interleaved) -> np.ndarray:
    """Norm and rotation of [n][heads][dim] in 64 bits."""
    x = x.astype(np.float64).copy()
    if eps:
        with np.errstate(invalid="ignore", over="ignore"):
            x = x / np.sqrt((x * x).mean(-1, keepdims=True) + float(np.float32(eps)))
        x = x * (1.0 if gamma is None else gamma.astype(np.float64))
    if freq is not None:
        n = len(freq)
        a = np.asarray(positions, np.float64)[:, None] * freq.astype(np.float64)
        cos, sin = np.cos(a)[:, None], np.sin(a)[:, None]
        i, j = (np.arange(n) * 2, np.arange(n) * 2 + 1) if interleaved else (np.arange(n), np.arange(n) + n)
        u, w = x[..., i].copy(), x[..., j].copy()
        with np.errstate(invalid="ignore"):
            x[..., i], x[..., j] = u * cos - w * sin, u * sin + w * cos
    return x


def cache_values(codes: torch.Tensor, scale: torch.Tensor, fmt: str, values: bool, ids, head: int) -> np.ndarray:
    """[len(ids) * page][dim] of one head, from the cache's tensors."""
    c = codes.view(torch.uint8)[torch.as_tensor(ids, dtype=torch.long, device=codes.device), head].cpu().numpy()
    x = code_values(c, fmt)                     # keys [n][s][d/16][16][16], values [n][s][d][16]
    x = x.transpose(0, 1, 3, 2) if values else x.transpose(0, 1, 3, 2, 4)
    n, s = x.shape[:2]
    x = x.reshape(n, s * 16, -1)
    sc = scale[torch.as_tensor(ids, dtype=torch.long, device=scale.device), head].double().cpu().numpy()
    return (x * sc[:, None, None]).reshape(n * s * 16, -1)


def attend_head(q, k, v, positions, n_keys, scale, causal, window):
    """(out, lse, and a bound on what roundings may do to out) of rows q [n][dim] with `positions`, in 64 bits."""
    j = np.arange(n_keys)
    pos = np.asarray(positions)[:, None]
    see = (j <= pos) if causal else np.ones((len(q), n_keys), bool)
    if window:
        see = see & (j > pos - window)
    with np.errstate(invalid="ignore"):
        z = np.where(see, scale * (q @ k[:n_keys].T), -np.inf)
    noise = scale * (np.abs(q) @ np.abs(k[:n_keys]).T)
    out, lse, slack = np.zeros((len(q), v.shape[1])), np.full(len(q), -np.inf), np.zeros((len(q), v.shape[1]))
    for i in range(len(q)):
        s = see[i]
        if not s.any():
            continue
        top = z[i][s].max()
        p = np.exp(z[i][s] - top)
        lse[i] = top + math.log(p.sum())
        p /= p.sum()
        out[i] = p @ v[:n_keys][s]
        # fp32 scores: off by 2^-24 of their terms' sizes for each of a few roundings and of the 2^11 additions' tree; weights are
        # rounded to fp16 (half a step: 2^-12 each, 2^-25 of the largest below 2^-14); the rest is fp32
        wrong = 2.0 ** -20 * noise[i][s].max() + 2.0 ** -20
        slack[i] = (2 * wrong + 2.0 ** -12) * (p @ np.abs(v[:n_keys][s])) + 2.0 ** -24 * np.abs(v[:n_keys][s]).max() * s.sum() * p.max()
    return out, lse, slack
