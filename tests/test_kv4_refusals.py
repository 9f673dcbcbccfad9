"""What the entry points refuse of a cache held in 4 bits, without a GPU: every refusal comes before anything is launched."""
import ctypes as C

import pytest
import torch

from paper_2312_17238_amd import binding as B
from paper_2312_17238_amd import paged
from test_kv_refusals import P, cache, query, refused, rows, step


def four(**k):
    return cache(**{"format": B.MOE_KV_E2M1, **k})


@pytest.mark.parametrize("k", [dict(n_pages=0), dict(page=17), dict(kv_heads=0), dict(head_dim=80), dict(head_dim=32), dict(format=3), dict(format=5), dict(reserved=3), dict(k=None),
                               dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(k=P + 8), dict(v=P + 1), dict(k_scale=P + 4), dict(v_scale=P + 8)], ids=str)
def test_bad_caches(k):
    c = four(**k)
    refused(B.moe_kv_write, c, step(), P, rows(), 0)
    refused(B.moe_kv_attend, c, step(), P, P, query(), None, 0, 0)
    refused(B.moe_kv_gather, c, P, 1, 0, P, P, 0)


@pytest.mark.parametrize("k", [dict(n_pages=33), dict(page=32), dict(kv_heads=4), dict(head_dim=128)], ids=str)
def test_a_step_for_another_cache(k):
    refused(B.moe_kv_write, four(**k), step(), P, rows(), 0)
    refused(B.moe_kv_attend, four(**k), step(), P, P, query(), None, 0, 0)


@pytest.mark.parametrize("k", [dict(dtype=2), dict(rot_dim=8), dict(rot_dim=80), dict(interleaved=2), dict(eps=-1.0), dict(eps=float("nan")), dict(q=None), dict(k=None), dict(v=None),
                               dict(q_out=None), dict(inv_freq=None), dict(q=P + 1), dict(q_stride=511), dict(k_stride=127), dict(v_stride=0), dict(q_out=P, q_out_stride=520)], ids=str)
def test_bad_rows(k):
    refused(B.moe_kv_write, four(), step(), P, rows(**k), 0)


@pytest.mark.parametrize("k", [dict(dtype=7), dict(scale=0.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(q=None), dict(out=None), dict(out=P), dict(q=P + 1), dict(lse=P + 2),
                               dict(q_stride=511), dict(out_stride=100)], ids=str)
def test_bad_queries(k):
    refused(B.moe_kv_attend, four(), step(), P, P, query(**k), None, 0, 0)


def test_the_scratch_has_to_be_there():
    s = step(max_blocks=1024)
    n = B.moe_kv_scratch_bytes(s)
    assert n > 0
    for at, size in ((None, n), (P, n - 1), (P + 8, n)):
        refused(B.moe_kv_attend, four(), s, P, P, query(), at, size, 0, code=B.MOE_ENOMEM)


@pytest.mark.parametrize("args", [(P, -1, 0, P, P), (P, (1 << 26) + 1, 0, P, P), (P, 1, 2, P, P), (None, 1, 0, P, P), (P, 1, 0, None, P), (P, 1, 0, P, P + 8), (P + 2, 1, 0, P, P)], ids=str)
def test_bad_lists(args):
    refused(B.moe_kv_gather, four(), *args, 0)
    B.moe_kv_gather(four(), None, 0, 0, None, None, 0)          # nothing to read


def test_the_tensor_layer_refuses_what_does_not_fit():
    code, byte = torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
    z = lambda t, *shape: torch.zeros(*shape, dtype=torch.uint8).view(t)  # noqa: E731
    k, v, ks, vs = z(code, 4, 2, 16, 32), z(code, 4, 2, 1, 64, 8), z(byte, 4, 2, 1, 4, 2, 4), z(byte, 4, 2, 16)
    with pytest.raises(ValueError, match="on one GPU"):
        paged.Cache(k, v, ks, vs)
    for a in ((k[0], v, ks, vs), (k, v[:, :, :, :48], ks, vs), (k, v.view(torch.uint8), ks, vs), (k, v, ks.view(torch.uint8), vs), (k, v, ks[:, :, :, :, :1], vs), (k, v, ks, vs[:3]),
              (k, v, torch.ones(4, 2), torch.ones(4, 2)), (k.view(torch.int8), v.view(torch.int8), ks, vs)):
        with pytest.raises(ValueError, match="Cache"):
            paged.Cache(*a)
    with pytest.raises(ValueError, match="multiple"):
        paged.Cache.empty(4, 2, 48, 16, code, "cpu")
    with pytest.raises(ValueError, match="multiples"):
        paged.Cache.empty(4, 2, 64, 24, code, "cpu")
    assert C.sizeof(B.KvCache) == 56
