"""Attention over the cache in 4 bits where numbers are far apart: blocks of a query, scores that are large, single tokens beside very many, and what is left of a score's
last bits. Every form of it: single tokens, tiles of few rows, tiles of many."""
import numpy as np
import pytest
import torch

import kv4_reference as R4
from paper_2312_17238_amd import paged
from test_gpu_kv4 import DEV, Pool, fill, half_step, planned

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,new", [([300, 41], [1, 1]), ([300, 41], [20, 5]), ([300, 100], [70, 40])])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("gap", [90, 100, 101, 120, 200])
def test_blocks_of_a_query_far_below_its_largest(lens, new, dim, gap):
    """A block of 32 dims 2^gap below the row's largest number, which meets keys of 0: the block counts for what it is, not for more."""
    p = Pool(2, -(-max(lens) // 16) + 1, page=16, q_heads=4, kv_heads=2, dim=dim, dtype=torch.bfloat16, seed=gap)
    fill(p, lens, k_exp=(-1, 0), v_exp=(-1, 1))
    p.cache.k.view(torch.uint8)[..., :16] = 0
    s = planned(p, lens, new)
    top = gap // 2
    q = p.rows(sum(new), 4, spread=0.0).float()
    q[..., 32:] = torch.ldexp(q[..., 32:], torch.tensor(top - gap, device=DEV))
    q[..., :32] = 2.0 ** top
    q = q.to(torch.bfloat16)
    scale = 2.0 ** (95 - top)
    out, lse = (x.double().cpu().numpy() for x in paged.attend(p.cache, s, q, scale, with_lse=True))
    # A number is off by 2^-20 of the power of two above its block's largest, or of 2^-99 of the row's largest if that is more; keys are 6 at most.
    # In scores: scale 2^-20 2^(top - 99) 6 (dim - 32); what attend_head allows counts the first.
    extra = 2.0 ** (95 - 20 - 99) * 6 * (dim - 32)
    k, kb, v, vb = p.tensors()
    qd, at = q.double().cpu().numpy(), 0
    for r, (n, m) in enumerate(zip(lens, new)):
        ids = p.table[r, :-(-n // 16)].cpu().numpy()
        for h in range(4):
            kh, vh = R4.keys(k[ids, h // 2], kb[ids, h // 2]).reshape(-1, dim), R4.values(v[ids, h // 2], vb[ids, h // 2]).reshape(-1, dim)
            vs = np.exp2(vb[ids, h // 2].astype(np.float64) - 127).reshape(-1)
            want, wl, slack, off = R4.attend_head(qd[at:at + m, h], kh, vh, vs, list(range(n - m, n)), n, scale, True, 0)
            # twice a score's error of the mean of |v|, 12 at most
            assert (np.abs(out[at:at + m, h] - want) <= slack + half_step(want, p.dtype) * 1.01 + 2 * extra * 12).all()
            assert (np.abs(lse[at:at + m, h] - wl) <= off + extra).all()
        at += m
