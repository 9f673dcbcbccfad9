"""Attention of the paged cache at the ends of the ranges of its numbers, against the definition in 64 bits, in each of its forms: requests of one
row, of a few (tiles that several waves share), of many (a tile a wave), and rows whose cached tokens several blocks share."""
import math

import numpy as np
import pytest
import torch

from paper_2312_17238_amd import paged
from test_gpu_kv import DEV, Pool, check_attend, fill, i32

pytestmark = pytest.mark.gpu

# (tokens in all, new ones) of two requests, two query heads a kv head: 2 rows; 40 and 10; 140 and 80; a row over 9000 tokens
FORMS = [([300, 41], [1, 1]), ([300, 41], [20, 5]), ([300, 100], [70, 40]), ([9000, 7], [1, 1]), ([9000, 90], [20, 3]), ([9000, 90], [70, 40])]


def planned(pool, lens, new):
    """A step whose pages are those that the table names already."""
    s = paged.Step(len(lens), sum(new), max(new), pool.width, pool.n_pages, pool.page, pool.q_heads, pool.kv_heads, pool.dim, pool.causal, pool.window)
    table = pool.table.clone()
    free = [int(table[r, b]) for r, (n, m) in enumerate(zip(lens, new)) for b in range(-(-(n - m) // pool.page), -(-n // pool.page))][::-1]
    s.plan(i32([n - m for n, m in zip(lens, new)]), i32(new), pool.table, i32(free + [0]), i32([len(free)]))
    assert (pool.table == table).all() and s.status.tolist() == [0] * len(lens)
    return s


def pool_of(lens, **k):
    return Pool(len(lens), -(-max(lens) // 16) + 1, page=16, q_heads=4, kv_heads=2, seed=max(lens), **k)


@pytest.mark.parametrize("lens,new", FORMS)
@pytest.mark.parametrize("dim", [64, 256])
@pytest.mark.parametrize("size", [100, 114, 116, 120, 125])
def test_queries_of_any_size(lens, new, dim, size):
    """bf16 queries up to its largest numbers, with keys so small that the scores are a few."""
    p = pool_of(lens, dim=dim, dtype=torch.bfloat16, fmt="int8")
    fill(p, lens, scales="one")
    p.cache.k_scale.fill_(2.0 ** -96)
    s = planned(p, lens, new)
    q = p.rows(sum(new), 4, spread=0.0)
    q = torch.ldexp(q.float(), torch.tensor(size, device=DEV)).clamp(-3e38, 3e38).to(torch.bfloat16)
    if size == 125:
        q[0, 0, 3], q[-1, 2, 5] = torch.finfo(torch.bfloat16).max, torch.finfo(torch.bfloat16).min
    # codes of about 35 and dim of them: scores of about 2
    scale = 2.0 ** (96 - size) / (16 * math.sqrt(dim))
    out, lse = paged.attend(p.cache, s, q, scale, with_lse=True)
    assert np.isfinite(lse.cpu().numpy()).all()
    check_attend(p, s, q, out, lse, lens, new, scale, rows=6)


@pytest.mark.parametrize("lens,new", FORMS)
@pytest.mark.parametrize("dim,fmt", [(64, "int8"), (128, "e4m3"), (256, "int8")])
@pytest.mark.parametrize("size", [8, 31, 60, 92])
@pytest.mark.parametrize("order", ["zeros first", "zeros last", "every other", "any"])
def test_values_of_any_size(lens, new, dim, fmt, size, order):
    """Pages of zeros (scale 2^-96) beside pages of very large values, with scores of the same size: tokens of either have their share of the sum.
    'any': scales from one to the other, at random."""
    p = pool_of(lens, dim=dim, dtype=torch.bfloat16, fmt=fmt)
    fill(p, lens, scales="one")
    if order == "any":
        e = p.rng.integers(-96, size + 1, tuple(p.cache.v_scale.shape))
    else:
        e = np.full(tuple(p.cache.v_scale.shape), size)
        for r, n in enumerate(lens):
            pages = -(-n // 16)
            for b in range(pages):
                if {"zeros first": b < (pages + 1) // 2, "zeros last": b >= pages // 2, "every other": b % 2 == 0}[order]:
                    i = int(p.table[r, b])
                    e[i] = -96
                    p.cache.v.view(torch.uint8)[i] = 0
    p.cache.v_scale.copy_(torch.from_numpy(np.exp2(e.astype(np.float64)).astype(np.float32)))
    s = planned(p, lens, new)
    q = p.rows(sum(new), 4, spread=0.0)
    scale = 1 / math.sqrt(dim)
    out, lse = paged.attend(p.cache, s, q, scale, with_lse=True)
    check_attend(p, s, q, out, lse, lens, new, scale, rows=6)
