"""What a row of the paged cache's attention does to the others of its tile, block and request: a query of NaN or infinity spoils its own row alone, one
of large numbers gets what 64 bits make of it, a request that is turned down gets zeros; in every form that attention has."""
import math

import pytest
import torch

from paper_2312_17238_amd import binding as B
from paper_2312_17238_amd import paged
from test_gpu_kv import Pool, check_attend, fill, i32

pytestmark = pytest.mark.gpu

# (tokens in all, new ones) of three requests, of which the middle one is turned down; two query heads a kv head
FORMS = [([90, 1, 41], [1, 1, 1]), ([90, 5, 41], [5, 5, 3]), ([90, 20, 41], [20, 17, 10]), ([200, 20, 141], [25, 32, 31]), ([200, 70, 141], [70, 40, 33]),
         ([9000, 5, 300], [5, 5, 1]), ([9000, 20, 300], [20, 17, 1]), ([9000, 70, 300], [70, 70, 40])]


@pytest.mark.parametrize("lens,new", FORMS)
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_rows_keep_to_themselves(lens, new, dtype, dim):
    p = Pool(3, -(-max(lens) // 16) + 1, page=16, q_heads=4, kv_heads=2, dim=dim, dtype=dtype, seed=sum(lens))
    held = [lens[0], 0, lens[2]]
    fill(p, held, scales="one")
    s = paged.Step(3, sum(new), max(new), p.width, p.n_pages, 16, 4, 2, dim)
    free = [int(p.table[r, b]) for r in (0, 2) for b in range(-(-(lens[r] - new[r]) // 16), -(-lens[r] // 16))][::-1]
    s.plan(i32([lens[0] - new[0], 16 * p.width, lens[2] - new[2]]), i32(new), p.table, i32(free + [0]), i32([len(free)]))
    assert s.status.tolist() == [B.MOE_KV_SERVED, B.MOE_KV_TOO_LONG, B.MOE_KV_SERVED]
    q = p.rows(sum(new), 4)
    last = sum(new) - 1
    q[0, 3], q[last, 0] = 30000.0, -30000.0
    spoilt = q.clone()
    rows = [(0, 1, 5, math.nan), (0, 2, 6, math.inf), (new[0] - 1, 0, 0, -math.inf), (last, 3, dim - 1, math.nan)]
    for t, h, d, x in rows:
        spoilt[t, h, d] = x
    good, good_lse = paged.attend(p.cache, s, q, with_lse=True)
    out, lse = paged.attend(p.cache, s, spoilt, with_lse=True)
    for t, h, _, _ in rows:
        assert out[t, h].isnan().all() and good[t, h].isfinite().all()
        out[t, h], lse[t, h] = good[t, h], good_lse[t, h]
    down = slice(new[0], new[0] + new[1])
    assert (out[down] == 0).all() and (lse[down] == -math.inf).all()
    mine = [i for i in range(sum(new)) if not new[0] <= i < new[0] + new[1]]
    p.table[1].copy_(p.table[2])
    for o, l in ((good, good_lse), (out, lse)):
        check_attend(p, s, q[mine], o[mine], l[mine], [lens[0], lens[2]], [new[0], new[2]], 1 / math.sqrt(dim))
