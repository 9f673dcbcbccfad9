"""What the entry points of the paged cache refuse, without a GPU: every refusal comes before anything is launched."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2312_17238_amd import binding as B
from paper_2312_17238_amd import paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000             # a pointer that nothing follows: a refused call reads none


def step(**k):
    d = dict(n_requests=2, n_tokens=8, max_new=4, max_blocks=16, n_pages=32, page=16, kv_heads=2, head_dim=64, q_heads=8, causal=1, window=0, reserved=0)
    d.update(k)
    return B.KvStep(*(d[n] for n, _ in B.KvStep._fields_))


def cache(**k):
    d = dict(n_pages=32, page=16, kv_heads=2, head_dim=64, format=0, reserved=0, k=P, v=P, k_scale=P, v_scale=P)
    d.update(k)
    return B.KvCache(*(d[n] for n, _ in B.KvCache._fields_))


def rows(**k):
    d = dict(dtype=0, rot_dim=64, interleaved=0, eps=0.0, q=P, k=P, v=P, q_stride=512, k_stride=128, v_stride=128, q_gamma=None, k_gamma=None, inv_freq=P,
             q_out=P + 2, q_out_stride=512)
    d.update(k)
    return B.KvRows(*(d[n] for n, _ in B.KvRows._fields_))


def query(**k):
    d = dict(dtype=0, scale=0.125, q=P, q_stride=512, out=P + 2, out_stride=512, lse=None)
    d.update(k)
    return B.KvQuery(*(d[n] for n, _ in B.KvQuery._fields_))


def lists(**k):
    d = {n: P + 64 * i for i, (n, _) in enumerate(B.KvLists._fields_)}
    d.update(k)
    return B.KvLists(*(d[n] for n, _ in B.KvLists._fields_))


def refused(call, *args, code=B.MOE_EINVAL):
    with pytest.raises(B.MoeError) as e:
        call(*args)
    assert e.value.code == code and "moe_kv_" in str(e.value)


BAD_STEPS = [dict(n_requests=0), dict(n_requests=4097), dict(n_tokens=0), dict(n_tokens=1048577), dict(max_new=0), dict(max_blocks=0), dict(n_pages=0),
             dict(page=8), dict(page=24), dict(page=256), dict(kv_heads=0), dict(kv_heads=257, q_heads=257), dict(head_dim=96), dict(head_dim=32), dict(q_heads=9),
             dict(q_heads=0), dict(q_heads=1026), dict(causal=2), dict(window=-1), dict(reserved=1), dict(n_pages=2 ** 27, page=16), dict(max_blocks=2 ** 26)]


def test_library_exports_every_declared_symbol():
    with open(os.path.join(ROOT, "include", "moe_kv.h")) as f:
        src = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    declared = set(re.findall(r"\b(moe_kv_[a-z0-9_]+)\s*\(", src))
    assert declared == set(B.KV_EXPORTS)
    assert all(hasattr(B.lib(), n) for n in declared)


@pytest.mark.parametrize("k", BAD_STEPS, ids=str)
def test_bad_steps(k):
    s = step(**k)
    assert B.moe_kv_plan_bytes(s) == 0 and B.moe_kv_scratch_bytes(s) == 0
    refused(B.moe_kv_plan, s, lists(), P, 0)
    refused(B.moe_kv_write, cache(), s, P, rows(), 0)
    refused(B.moe_kv_attend, cache(), s, P, P, query(), P, 1 << 40, 0)


def test_sizes():
    for page, blocks, new, n in ((16, 16, 4, 8), (16, 64, 4, 8), (128, 1024, 4, 8), (64, 4096, 512, 4096)):
        s = step(page=page, max_blocks=blocks, max_new=new, n_tokens=n)
        # row positions, at least, and as much again for every bound that grows
        assert B.moe_kv_plan_bytes(s) % 64 == 0 and B.moe_kv_plan_bytes(s) >= 4 * n
        more = step(page=page, max_blocks=blocks, max_new=new, n_tokens=2 * n, n_requests=4)
        assert B.moe_kv_plan_bytes(more) >= B.moe_kv_plan_bytes(s) + 4 * n
    assert B.moe_kv_scratch_bytes(step()) == 0                              # 256 tokens at most: nothing is split
    few = B.moe_kv_scratch_bytes(step(max_blocks=1024))
    many = B.moe_kv_scratch_bytes(step(max_blocks=1024, max_new=64, n_tokens=64))
    assert 0 < few < many and few % (2 * 32 * 66 * 4) == 0                  # parts of two heads, 32 rows of 64 + 2 numbers
    assert B.moe_kv_plan_bytes(step(n_requests=4096, n_tokens=1048576, max_new=1048576, q_heads=1024)) > 32 * (1048576 * 512 // 256)


@pytest.mark.parametrize("k", [dict(n_pages=0), dict(page=17), dict(kv_heads=0), dict(head_dim=80), dict(format=2), dict(format=-1), dict(reserved=3), dict(k=None), dict(v=None),
                               dict(k_scale=None), dict(v_scale=None), dict(k=P + 8), dict(v=P + 1), dict(k_scale=P + 2)], ids=str)
def test_bad_caches(k):
    c = cache(**k)
    refused(B.moe_kv_write, c, step(), P, rows(), 0)
    refused(B.moe_kv_attend, c, step(), P, P, query(), None, 0, 0)
    refused(B.moe_kv_gather, c, P, 1, 0, P, P, 0)


@pytest.mark.parametrize("k", [dict(n_pages=33), dict(page=32), dict(kv_heads=4), dict(head_dim=128)], ids=str)
def test_a_step_for_another_cache(k):
    refused(B.moe_kv_write, cache(**k), step(), P, rows(), 0)
    refused(B.moe_kv_attend, cache(**k), step(), P, P, query(), None, 0, 0)


@pytest.mark.parametrize("k", [{n: None} for n, _ in B.KvLists._fields_] + [dict(ctx_len=P + 2), dict(slots=P + 1), dict(kv_len=P), dict(free_left=P + 64 * 4),
                                                                         dict(row_start=P + 64 * 2)], ids=str)
def test_bad_lists(k):
    refused(B.moe_kv_plan, step(), lists(**k), P, 0)


def test_bad_plans():
    for p in (None, P + 64):
        refused(B.moe_kv_plan, step(), lists(), p, 0)
        refused(B.moe_kv_write, cache(), step(), p, rows(), 0)
        refused(B.moe_kv_attend, cache(), step(), p, P, query(), None, 0, 0)


@pytest.mark.parametrize("k", [dict(dtype=2), dict(rot_dim=8), dict(rot_dim=80), dict(rot_dim=-16), dict(interleaved=2), dict(inv_freq=None), dict(eps=-1.0), dict(eps=float("nan")),
                               dict(eps=float("inf")), dict(q=None), dict(k=None), dict(v=None), dict(q_out=None), dict(q=P + 1), dict(k_gamma=P + 1), dict(inv_freq=P + 2),
                               dict(q_stride=511), dict(k_stride=127), dict(v_stride=0), dict(q_out_stride=64), dict(q_out=P, q_stride=520)], ids=str)
def test_bad_rows(k):
    refused(B.moe_kv_write, cache(), step(), P, rows(**k), 0)


@pytest.mark.parametrize("k", [dict(dtype=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(out=None), dict(out=P),
                               dict(q=P + 1), dict(lse=P + 2), dict(q_stride=256), dict(out_stride=511)], ids=str)
def test_bad_queries(k):
    refused(B.moe_kv_attend, cache(), step(), P, P, query(**k), None, 0, 0)
    refused(B.moe_kv_attend, cache(), step(), P, None, query(), None, 0, 0)


def test_scratch_too_small():
    s = step(max_blocks=1024)
    n = B.moe_kv_scratch_bytes(s)
    for p, b in ((P, n - 1), (None, n), (P + 8, n)):
        refused(B.moe_kv_attend, cache(), s, P, P, query(), p, b, 0, code=B.MOE_ENOMEM)


def test_bad_gathers_and_releases():
    for a in ((P, -1, 0, P, P), (P, 1, 2, P, P), (None, 1, 0, P, P), (P, 1, 0, None, P), (P, 1, 0, P, P + 8), (P + 2, 1, 0, P, P)):
        refused(B.moe_kv_gather, cache(), *a, 0)
    good = [P, 1, 4, 32, 16, 8, P, P, P, 32, P, 0]
    for i, v in ((0, None), (1, -1), (2, 0), (3, 0), (4, 20), (5, 0), (6, None), (7, None), (8, None), (9, 0), (10, None)):
        refused(B.moe_kv_release, *(good[:i] + [v] + good[i + 1:]))


def test_the_tensor_layer_refuses_what_does_not_fit():
    t = torch.zeros(4, 2, 1, 4, 16, 16, dtype=torch.int8)
    v = torch.zeros(4, 2, 1, 64, 16, dtype=torch.int8)
    s = torch.ones(4, 2)
    for a in ((t, v, s, s), (t[0], v, s, s), (t, v[:, :, :, :48], s, s), (t, v.view(torch.uint8), s, s), (t, v, s.double(), s), (t, v, s[:3], s)):
        with pytest.raises(ValueError):
            paged.Cache(*a)                     # the first: not on a GPU
    with pytest.raises(B.MoeError):
        paged.Step(1, 1, 1, 1, 1, 20, 1, 1, 64, device="cpu")
    st = paged.Step(1, 2, 2, 4, 8, 16, 4, 2, 64, device="cpu")
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="ctx_len"):
        st.plan(i, i, torch.zeros(1, 4, dtype=torch.int32), i, i)
    with pytest.raises(ValueError, match="no plan"):
        paged.attend(None, st, torch.zeros(2, 4, 64, dtype=torch.float16))
    with pytest.raises(ValueError, match="no plan"):
        st.advance()
    assert C.sizeof(B.KvCache) == 56 and C.sizeof(B.KvStep) == 48 and C.sizeof(B.KvRows) == 104 and C.sizeof(B.KvQuery) == 48
