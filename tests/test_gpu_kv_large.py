"""Calls of the paged cache whose grids have more than 2^32 threads."""
import pytest
import torch

from paper_2312_17238_amd import paged

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_gather_of_a_million_tokens_of_256_heads():
    n, heads, dim, page = (1 << 20) + 5, 256, 64, 16
    g = torch.Generator(device=DEV).manual_seed(4)
    c = paged.Cache.empty(2, heads, dim, page, torch.int8)
    for t in (c.k, c.v):
        t.copy_(torch.randint(-127, 128, t.shape, dtype=torch.int8, device=DEV, generator=g))
    c.k_scale.copy_(torch.exp2(torch.randint(-9, 1, c.k_scale.shape, device=DEV, generator=g).float()))
    c.v_scale.copy_(torch.exp2(torch.randint(-9, 1, c.v_scale.shape, device=DEV, generator=g).float()))
    every = paged.gather(c, torch.arange(2 * page, dtype=torch.int32, device=DEV))
    slots = torch.randint(0, 2 * page, (n,), dtype=torch.int32, device=DEV, generator=g)
    got = paged.gather(c, slots)
    for x, values in zip(got, every):
        for at in range(0, n, 1 << 15):
            assert torch.equal(x[at:at + (1 << 15)], values[slots[at:at + (1 << 15)].long()]), at
