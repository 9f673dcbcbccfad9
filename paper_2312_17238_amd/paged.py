"""Tensors around include/moe_kv.h: a paged 8-bit key/value cache and the attention half of a decode step.

    cache = Cache.empty(n_pages, kv_heads, head_dim)                    # one per layer
    step = Step(n_requests, n_tokens, max_new, max_blocks, n_pages, page, q_heads, kv_heads, head_dim)
    step.plan(ctx_len, new_len, block_table, free_pages, free_count)    # once per step of the model
    q = write(cache, step, q, k, v, inv_freq=f)                         # per layer: norm, rotation, store
    out = attend(cache, step, q)                                        # per layer
    step.advance()                                                      # the new tokens are cached ones now

The step, the cache and all tensors of a call are on one GPU; everything runs on torch's current stream of that GPU (which need not be the
current one) and reads no length on the host.  All lists of numbers are int32 tensors on the device.
"""
from __future__ import annotations

import ctypes as C
import math
import threading
from typing import Optional, Tuple

import torch

from . import binding as B

DTYPES = {torch.float16: B.MOE_KV_F16, torch.bfloat16: B.MOE_KV_BF16}
FORMATS = {torch.float8_e4m3fn: B.MOE_KV_E4M3, torch.int8: B.MOE_KV_INT8}

# A call costs the host a few microseconds, which for single tokens is what counts: structures and references to them are made once,
# messages only when something is refused.


def _call(fn, device: int, *args) -> None:
    """fn(*args, stream): on the device's current stream, with the device current, for a default stream is 0 on all of them."""
    stream = torch._C._cuda_getCurrentRawStream(device)
    if torch._C._cuda_getDevice() == device:
        rc = fn(*args, stream)
    else:
        with torch.cuda.device(device):
            rc = fn(*args, stream)
    if rc:
        B.check(rc)


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _index(t: torch.Tensor) -> int:
    """The GPU that a tensor is on, -2 for none: what other tensors are compared with."""
    return t.get_device() if t.is_cuda else -2


def _ints(t: torch.Tensor, shape, device: int, what: str) -> int:
    if t.dtype is not torch.int32 or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous int32 tensor {tuple(shape)} on {_gpu(device)} is needed, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _gpu(device: int) -> str:
    return f"GPU {device}" if device >= 0 else "the GPU"


def _rows(t: torch.Tensor, shape, dtype, device: int, what: str) -> Tuple[int, int]:
    """(pointer, elements between rows) of [n][heads][dim] whose heads follow each other."""
    n, heads, dim = shape
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device:
        raise ValueError(f"{what}: {t.dtype} {tuple(t.shape)} on {t.device}, {dtype} {shape} on {_gpu(device)} is needed")
    row, head, one = t.stride()
    if one != 1 or (head != dim and heads != 1):
        raise ValueError(f"{what}: the heads of a row have to follow each other")
    return t.data_ptr(), row if n > 1 else heads * dim


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
        self.ref = C.byref(self.c)
        self.device = _index(k)

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
    free_left) and the workspaces that its layers share.  Made once for bounds that hold for many steps, under the stream that they run on
    (torch gives its memory to that stream's next tensors when it is dropped).  Threads may share it, streams may not."""

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
        self.device = _index(self.plan_dev)
        self.scratch_bytes = B.moe_kv_scratch_bytes(self.s)
        self.scratch = torch.empty(max(16, self.scratch_bytes), dtype=torch.uint8, device=device)
        self.block_table: Optional[torch.Tensor] = None
        self._lists = B.KvLists(*[None] * 5, *(t.data_ptr() for t in (self.row_start, self.positions, self.slots, self.kv_len, self.status, self.free_left)))
        self._row, self._query = B.KvRows(), B.KvQuery()
        self._lock = threading.Lock()       # a call fills these structures in, and the interpreter's lock is off while the library reads them
        self._ref, self._lists_ref, self._row_ref, self._query_ref = (C.byref(x) for x in (self.s, self._lists, self._row, self._query))
        self._per_request, self._table = (n_requests,), (n_requests, max_blocks)
        self._q_shape, self._kv_shape = (n_tokens, q_heads, head_dim), (n_tokens, kv_heads, head_dim)
        self._scale = 1.0 / math.sqrt(head_dim)

    def plan(self, ctx_len, new_len, block_table, free_pages, free_count) -> None:
        """Pages for the step's new tokens (block_table is updated in place, ctx_len and the stack stay until `advance`).
        A free_count above the length of free_pages counts as that length."""
        x, at = self._lists, self.device
        with self._lock:
            x.ctx_len, x.new_len = _ints(ctx_len, self._per_request, at, "ctx_len"), _ints(new_len, self._per_request, at, "new_len")
            x.block_table = _ints(block_table, self._table, at, "block_table")
            room = free_pages.numel()
            x.free_pages, x.free_count = _ints(free_pages, (room or 1,), at, "free_pages"), _ints(free_count, (1,), at, "free_count")
            _call(B.lib().moe_kv_plan_within, at, self._ref, self._lists_ref, room, self.plan_dev.data_ptr())
            self.block_table, self._ctx, self._count = block_table, ctx_len, free_count

    def advance(self) -> None:
        """The step is done: its tokens count as cached, its pages as taken.  Lengths that are set back afterwards (refused drafts) have to stay
        within the request's last page: see moe_kv.h."""
        _need(self.block_table is not None, "advance: no plan has been made")
        self._ctx.copy_(self.kv_len)
        self._count.copy_(self.free_left)


def write(cache: Cache, step: Step, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_gamma: Optional[torch.Tensor] = None,
          k_gamma: Optional[torch.Tensor] = None, eps: float = 0.0, inv_freq: Optional[torch.Tensor] = None, interleaved: bool = False,
          q_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Norm (eps > 0) and rotation (inv_freq: fp32, one number a pair) of queries and keys; keys and values go into
    the cache.  q [n_tokens, q_heads, head_dim], k, v [n_tokens, kv_heads, head_dim], views of one packed tensor among them.
    Returns the queries: q_out (which may be q), a new tensor if it is None; rows that belong to no request are left as they are."""
    if step.block_table is None:
        raise ValueError("write: the step has no plan yet")
    dtype, x, at = q.dtype, step._row, step.device
    if dtype not in DTYPES:
        raise ValueError(f"write: queries of type {dtype}")
    if cache.device != at:
        raise ValueError(f"write: the cache is on {_gpu(cache.device)}, the step on {_gpu(at)}")
    if q_out is None:
        q_out = torch.empty(step._q_shape, dtype=dtype, device=q.device)
    with step._lock:
        x.q, x.q_stride = _rows(q, step._q_shape, dtype, at, "q")
        x.q_out, x.q_out_stride = _rows(q_out, step._q_shape, dtype, at, "q_out")
        x.k, x.k_stride = _rows(k, step._kv_shape, dtype, at, "k")
        x.v, x.v_stride = _rows(v, step._kv_shape, dtype, at, "v")
        x.dtype, x.eps, x.interleaved = DTYPES[dtype], eps, interleaved
        x.q_gamma, x.k_gamma = _gain(q_gamma, step, eps, dtype, "q_gamma"), _gain(k_gamma, step, eps, dtype, "k_gamma")
        x.rot_dim, x.inv_freq = 0, None
        if inv_freq is not None and inv_freq.numel():
            if inv_freq.dtype is not torch.float32 or inv_freq.dim() != 1 or not inv_freq.is_contiguous() or inv_freq.get_device() != at:
                raise ValueError(f"write: inv_freq is a contiguous fp32 list on {_gpu(at)}")
            x.rot_dim, x.inv_freq = 2 * inv_freq.numel(), inv_freq.data_ptr()
        _call(B.lib().moe_kv_write, at, cache.ref, step._ref, step.plan_dev.data_ptr(), step._row_ref)
    return q_out


def _gain(g: Optional[torch.Tensor], step: Step, eps: float, dtype, what: str) -> Optional[int]:
    if g is None:
        return None
    if g.shape != step._q_shape[2:] or g.dtype is not dtype or not g.is_contiguous() or g.get_device() != step.device:
        raise ValueError(f"write: {what}: {step._q_shape[2]} contiguous numbers of type {dtype} on {_gpu(step.device)} are needed")
    _need(eps > 0, "write: a gain without a norm (eps is 0)")
    return g.data_ptr()


def attend(cache: Cache, step: Step, q: torch.Tensor, scale: Optional[float] = None, out: Optional[torch.Tensor] = None, with_lse: bool = False):
    """Attention of the step's rows over all that is cached for their requests (scale: 1/sqrt(head_dim) if None).  Returns out [n_tokens,
    q_heads, head_dim], or (out, lse [n_tokens, q_heads] fp32); rows that belong to no request are left as they are."""
    table = step.block_table
    if table is None:
        raise ValueError("attend: the step has no plan yet")
    dtype, x, at = q.dtype, step._query, step.device
    if dtype not in DTYPES:
        raise ValueError(f"attend: queries of type {dtype}")
    if cache.device != at:
        raise ValueError(f"attend: the cache is on {_gpu(cache.device)}, the step on {_gpu(at)}")
    if out is None:
        out = torch.empty(step._q_shape, dtype=dtype, device=q.device)
    lse = torch.empty(step._q_shape[:2], dtype=torch.float32, device=q.device) if with_lse else None
    with step._lock:
        x.q, x.q_stride = _rows(q, step._q_shape, dtype, at, "q")
        x.out, x.out_stride = _rows(out, step._q_shape, dtype, at, "out")
        x.dtype, x.scale, x.lse = DTYPES[dtype], step._scale if scale is None else scale, lse.data_ptr() if with_lse else None
        _call(B.lib().moe_kv_attend, at, cache.ref, step._ref, step.plan_dev.data_ptr(), table.data_ptr(), step._query_ref, step.scratch.data_ptr(),
              step.scratch_bytes)
    return (out, lse) if with_lse else out


def gather(cache: Cache, slots: torch.Tensor, dtype=torch.float16) -> Tuple[torch.Tensor, torch.Tensor]:
    """The keys and values that the tokens in `slots` stand for, [n, kv_heads, head_dim] each; zeros for a slot of -1."""
    if dtype not in DTYPES:
        raise ValueError(f"gather: values of type {dtype}")
    _need(slots.dim() == 1, "gather: slots is a list")
    p, n = _ints(slots, slots.shape, cache.device, "slots"), slots.numel()
    k = torch.empty(n, cache.kv_heads, cache.head_dim, dtype=dtype, device=slots.device)
    v = torch.empty_like(k)
    _call(B.lib().moe_kv_gather, cache.device, cache.ref, p, n, DTYPES[dtype], k.data_ptr(), v.data_ptr())
    return k, v


def release(requests: torch.Tensor, n_pages: int, page: int, ctx_len: torch.Tensor, block_table: torch.Tensor, free_pages: torch.Tensor,
            free_count: torch.Tensor) -> None:
    """Give back the pages of the requests whose ids `requests` holds; their ctx_len becomes 0.  Not between a step's plan and its advance."""
    _need(requests.dim() == 1 and block_table.dim() == 2 and free_pages.dim() == 1, "release: requests and free_pages are lists, block_table a table")
    r, m = block_table.shape
    at = _index(block_table)
    _call(B.lib().moe_kv_release, at, _ints(requests, requests.shape, at, "requests"), requests.numel(), r, n_pages, page, m, _ints(ctx_len, (r,), at, "ctx_len"),
          _ints(block_table, (r, m), at, "block_table"), _ints(free_pages, free_pages.shape, at, "free_pages"), free_pages.numel(),
          _ints(free_count, (1,), at, "free_count"))
