"""Tensors around include/moe_kv.h: a paged 8-bit key/value cache and the attention half of a decode step.

    cache = Cache.empty(n_pages, kv_heads, head_dim)                    # one per layer
    step = Step(n_requests, n_tokens, max_new, max_blocks, n_pages, page, q_heads, kv_heads, head_dim)
    step.plan(ctx_len, new_len, block_table, free_pages, free_count)    # once per step of the model
    q = write(cache, step, q, k, v, inv_freq=f)                         # per layer: norm, rotation, store
    out = attend(cache, step, q)                                        # per layer
    step.advance()                                                      # the new tokens are cached ones now

Everything runs on torch's current stream and reads no length on the host.  All lists of numbers are int32 tensors on the device.
"""
from __future__ import annotations

import math
from typing import Optional, Tuple

import torch

from . import binding as B

DTYPES = {torch.float16: B.MOE_KV_F16, torch.bfloat16: B.MOE_KV_BF16}
FORMATS = {torch.float8_e4m3fn: B.MOE_KV_E4M3, torch.int8: B.MOE_KV_INT8}


def _stream(t: torch.Tensor) -> int:
    return torch.cuda.current_stream(t.device).cuda_stream


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _ints(t: torch.Tensor, shape, what: str) -> int:
    _need(t.dtype == torch.int32 and t.is_cuda and t.is_contiguous() and tuple(t.shape) == tuple(shape),
          f"{what}: a contiguous int32 tensor {tuple(shape)} on the GPU is needed, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _rows(t: torch.Tensor, n: int, heads: int, dim: int, dtype, what: str) -> Tuple[int, int]:
    """(pointer, elements between rows) of [n][heads][dim] whose heads follow each other."""
    _need(t.dtype == dtype and t.is_cuda, f"{what}: {t.dtype} on {t.device}, {dtype} on the GPU is needed")
    _need(tuple(t.shape) == (n, heads, dim), f"{what}: shape {tuple(t.shape)}, ({n}, {heads}, {dim}) is needed")
    _need(t.stride(2) == 1 and (heads == 1 or t.stride(1) == dim), f"{what}: the heads of a row have to follow each other")
    return t.data_ptr(), t.stride(0) if n > 1 else heads * dim


class Cache:
    """Keys and values of one layer: 8-bit codes in 16 x 16 tiles and a scale for each page and kv head.

    k: [n_pages, kv_heads, page/16, head_dim/16, 16 tokens, 16 dims], v: [n_pages, kv_heads, page/16, head_dim, 16 tokens]
    (float8_e4m3fn or int8); k_scale, v_scale: [n_pages, kv_heads] fp32."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor):
        _need(k.dim() == 6 and k.shape[4:] == (16, 16), f"Cache: k has shape {tuple(k.shape)}")
        p, h, s, d = k.shape[:4]
        _need(tuple(v.shape) == (p, h, s, 16 * d, 16), f"Cache: v has shape {tuple(v.shape)}")
        _need(k.dtype in FORMATS and v.dtype == k.dtype, f"Cache: codes of type {k.dtype} and {v.dtype}")
        for t, what in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            _need(tuple(t.shape) == (p, h) and t.dtype == torch.float32, f"Cache: {what} is {t.dtype} {tuple(t.shape)}")
        _need(all(t.is_cuda and t.is_contiguous() and t.device == k.device for t in (k, v, k_scale, v_scale)), "Cache: contiguous tensors on one GPU are needed")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.kv_heads, self.page, self.head_dim = p, h, 16 * s, 16 * d
        self.c = B.KvCache(p, 16 * s, h, 16 * d, FORMATS[k.dtype], 0, k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr())

    @classmethod
    def empty(cls, n_pages: int, kv_heads: int, head_dim: int, page: int = 64, dtype=torch.float8_e4m3fn, device="cuda:0") -> "Cache":
        """Uninitialised: a page's content counts from the first token that is written into it."""
        _need(page % 16 == 0 and head_dim % 16 == 0, "Cache: page and head_dim have to be multiples of 16")
        k = torch.empty(n_pages, kv_heads, page // 16, head_dim // 16, 16, 16, dtype=torch.uint8, device=device)
        v = torch.empty(n_pages, kv_heads, page // 16, head_dim, 16, dtype=torch.uint8, device=device)
        s = torch.empty(2, n_pages, kv_heads, dtype=torch.float32, device=device)
        return cls(k.view(dtype), v.view(dtype), s[0], s[1])


class Step:
    """A step of a ragged batch: its bounds, the lists that `plan` fills (row_start, positions, slots, kv_len, status,
    free_left) and the workspaces that its layers share.  Made once for bounds that hold for many steps."""

    def __init__(self, n_requests: int, n_tokens: int, max_new: int, max_blocks: int, n_pages: int, page: int, q_heads: int, kv_heads: int,
                 head_dim: int, causal: bool = True, window: int = 0, device="cuda:0"):
        self.s = B.KvStep(n_requests, n_tokens, max_new, max_blocks, n_pages, page, kv_heads, head_dim, q_heads, int(causal), window, 0)
        n = B.moe_kv_plan_bytes(self.s)
        if n == 0:
            raise B.MoeError(B.MOE_EINVAL, "Step: unsupported sizes")
        i32 = lambda *shape: torch.empty(*shape, dtype=torch.int32, device=device)  # noqa: E731
        self.row_start, self.positions, self.slots = i32(n_requests + 1), i32(n_tokens), i32(n_tokens)
        self.kv_len, self.status, self.free_left = i32(n_requests), i32(n_requests), i32(1)
        self.plan_dev = torch.empty(n, dtype=torch.uint8, device=device)
        self.scratch_bytes = B.moe_kv_scratch_bytes(self.s)
        self._scratch: Optional[torch.Tensor] = None
        self.block_table: Optional[torch.Tensor] = None

    def plan(self, ctx_len, new_len, block_table, free_pages, free_count) -> None:
        """Pages for the step's new tokens (block_table is updated in place, ctx_len and the stack stay until `advance`)."""
        s = self.s
        _need(free_pages.dim() == 1 and free_pages.numel() >= 1, "plan: free_pages is a list")
        lists = B.KvLists(_ints(ctx_len, (s.n_requests,), "ctx_len"), _ints(new_len, (s.n_requests,), "new_len"),
                          _ints(block_table, (s.n_requests, s.max_blocks), "block_table"),
                          _ints(free_pages, free_pages.shape, "free_pages"), _ints(free_count, (1,), "free_count"),
                          self.row_start.data_ptr(), self.positions.data_ptr(), self.slots.data_ptr(),
                          self.kv_len.data_ptr(), self.status.data_ptr(), self.free_left.data_ptr())
        B.moe_kv_plan(s, lists, self.plan_dev.data_ptr(), _stream(self.plan_dev))
        self.block_table, self._ctx, self._count = block_table, ctx_len, free_count

    def advance(self) -> None:
        """The step is done: its tokens count as cached, its pages as taken."""
        _need(self.block_table is not None, "advance: no plan has been made")
        self._ctx.copy_(self.kv_len)
        self._count.copy_(self.free_left)

    def scratch(self) -> torch.Tensor:
        if self._scratch is None:
            self._scratch = torch.empty(max(16, self.scratch_bytes), dtype=torch.uint8, device=self.plan_dev.device)
        return self._scratch


def _on(step: Step, what: str) -> None:
    _need(step.block_table is not None, f"{what}: the step has no plan yet")


def write(cache: Cache, step: Step, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_gamma: Optional[torch.Tensor] = None,
          k_gamma: Optional[torch.Tensor] = None, eps: float = 0.0, inv_freq: Optional[torch.Tensor] = None, interleaved: bool = False,
          q_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Norm (eps > 0) and rotation (inv_freq: fp32, one number a pair) of queries and keys; keys and values go into
    the cache.  q [n_tokens, q_heads, head_dim], k, v [n_tokens, kv_heads, head_dim], views of one packed tensor among them.
    Returns the queries: q_out (which may be q), a new tensor if it is None; rows that belong to no request are left as they are."""
    _on(step, "write")
    s = step.s
    _need(q.dtype in DTYPES, f"write: queries of type {q.dtype}")
    d, n = s.head_dim, s.n_tokens
    if q_out is None:
        q_out = torch.empty(n, s.q_heads, d, dtype=q.dtype, device=q.device)
    (qp, qs), (op, os_) = _rows(q, n, s.q_heads, d, q.dtype, "q"), _rows(q_out, n, s.q_heads, d, q.dtype, "q_out")
    (kp, ks), (vp, vs) = _rows(k, n, s.kv_heads, d, q.dtype, "k"), _rows(v, n, s.kv_heads, d, q.dtype, "v")
    for g, what in ((q_gamma, "q_gamma"), (k_gamma, "k_gamma")):
        _need(g is None or (tuple(g.shape) == (d,) and g.dtype == q.dtype and g.is_contiguous() and g.device == q.device), f"write: {what}: {d} contiguous numbers of type {q.dtype} are needed")
        _need(g is None or eps > 0, f"write: {what} without a norm (eps is 0)")
    rot = 0
    if inv_freq is not None:
        _need(inv_freq.dtype == torch.float32 and inv_freq.dim() == 1 and inv_freq.is_contiguous() and inv_freq.device == q.device, "write: inv_freq is a contiguous fp32 list")
        rot = 2 * inv_freq.numel()
    rows = B.KvRows(DTYPES[q.dtype], rot, int(interleaved), eps, qp, kp, vp, qs, ks, vs,
                    q_gamma.data_ptr() if q_gamma is not None else None, k_gamma.data_ptr() if k_gamma is not None else None,
                    inv_freq.data_ptr() if rot else None, op, os_)
    B.moe_kv_write(cache.c, s, step.plan_dev.data_ptr(), rows, _stream(q))
    return q_out


def attend(cache: Cache, step: Step, q: torch.Tensor, scale: Optional[float] = None, out: Optional[torch.Tensor] = None, with_lse: bool = False):
    """Attention of the step's rows over all that is cached for their requests (scale: 1/sqrt(head_dim) if None).  Returns out [n_tokens,
    q_heads, head_dim], or (out, lse [n_tokens, q_heads] fp32); rows that belong to no request are left as they are."""
    _on(step, "attend")
    s = step.s
    _need(q.dtype in DTYPES, f"attend: queries of type {q.dtype}")
    if out is None:
        out = torch.empty(s.n_tokens, s.q_heads, s.head_dim, dtype=q.dtype, device=q.device)
    (qp, qs), (op, os_) = _rows(q, s.n_tokens, s.q_heads, s.head_dim, q.dtype, "q"), _rows(out, s.n_tokens, s.q_heads, s.head_dim, q.dtype, "out")
    lse = torch.empty(s.n_tokens, s.q_heads, dtype=torch.float32, device=q.device) if with_lse else None
    query = B.KvQuery(DTYPES[q.dtype], 1.0 / math.sqrt(s.head_dim) if scale is None else scale, qp, qs, op, os_, lse.data_ptr() if with_lse else None)
    B.moe_kv_attend(cache.c, s, step.plan_dev.data_ptr(), step.block_table.data_ptr(), query, step.scratch().data_ptr(), step.scratch_bytes, _stream(q))
    return (out, lse) if with_lse else out


def gather(cache: Cache, slots: torch.Tensor, dtype=torch.float16) -> Tuple[torch.Tensor, torch.Tensor]:
    """The keys and values that the tokens in `slots` stand for, [n, kv_heads, head_dim] each; zeros for a slot of -1."""
    _need(dtype in DTYPES, f"gather: values of type {dtype}")
    _need(slots.dim() == 1, "gather: slots is a list")
    p, n = _ints(slots, slots.shape, "slots"), slots.numel()
    k = torch.empty(n, cache.kv_heads, cache.head_dim, dtype=dtype, device=slots.device)
    v = torch.empty_like(k)
    B.moe_kv_gather(cache.c, p, n, DTYPES[dtype], k.data_ptr(), v.data_ptr(), _stream(slots))
    return k, v


def release(requests: torch.Tensor, n_pages: int, page: int, ctx_len: torch.Tensor, block_table: torch.Tensor, free_pages: torch.Tensor,
            free_count: torch.Tensor) -> None:
    """Give back the pages of the requests whose ids `requests` holds; their ctx_len becomes 0."""
    _need(requests.dim() == 1 and block_table.dim() == 2 and free_pages.dim() == 1, "release: requests and free_pages are lists, block_table a table")
    r, m = block_table.shape
    B.moe_kv_release(_ints(requests, requests.shape, "requests"), requests.numel(), r, n_pages, page, m, _ints(ctx_len, (r,), "ctx_len"),
                     _ints(block_table, (r, m), "block_table"), _ints(free_pages, free_pages.shape, "free_pages"), free_pages.numel(),
                     _ints(free_count, (1,), "free_count"), _stream(block_table))
