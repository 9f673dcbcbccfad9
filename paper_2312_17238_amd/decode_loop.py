"""Whole decoder blocks over requests of any lengths: the paged 8-bit cache and its attention in front of the MoE step.

    python -m paper_2312_17238_amd.decode_loop [--layers 2] [--requests 4] [--prompt 37] [--tokens 16] [--hidden 256] [--ffn 512] ...

A block is  x += attention(norm(x)) Wo;  x = MoE step of x  (the library norms in front of its gate).  The requests' prompts go through in one
step, then every request gets a token a step; each step's pages are handed out on the GPU (paged.Step.plan), keys are turned and stored
(paged.write), rows attend to all that their request has cached (paged.attend), and finished requests give their pages back
(paged.release).  No length is read by the host.  Weights are seeded random numbers, so the "tokens" are hidden states that the last
block's output is fed back as.  Prints one JSON object.  Needs a GPU and the built library.
"""
from __future__ import annotations

import argparse
import contextlib
import json
import os
import sys
import time
from typing import List, Optional, Sequence

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import workload as W  # noqa: E402
from paper_2312_17238_amd import paged  # noqa: E402
from paper_2312_17238_amd.engine import Stack, layer_config  # noqa: E402


class Decoder:
    """`layers` blocks over a pool of `n_requests` requests.  Everything runs on the engine's compute stream, behind what the caller's current
    stream has been given so far; that stream waits for the results."""

    def __init__(self, layers: int, hidden: int, ffn: int, q_heads: int, kv_heads: int, head_dim: int, n_requests: int, max_len: int,
                 max_rows: int, page: int = 64, fmt=torch.float8_e4m3fn, window: int = 0, eps: float = 1e-5, theta: float = 1e6,
                 cache_slots: int = 8, seed: int = 0, device: str = "cuda:0", n_pages: Optional[int] = None):
        self.layers, self.hidden, self.q_heads, self.kv_heads, self.head_dim = layers, hidden, q_heads, kv_heads, head_dim
        self.n_requests, self.page, self.window, self.eps, self.device = n_requests, page, window, eps, device
        self.max_blocks = -(-max_len // page)
        self.n_pages = n_requests * self.max_blocks if n_pages is None else n_pages
        # The host makes the lengths, so it knows them without reading any: tokens and new tokens of each request, free pages, rows of a step.
        self._lens, self._new, self._free, self._rows = [0] * n_requests, [0] * n_requests, self.n_pages, 0
        cfg = layer_config(hidden, ffn, 8, 2, 4, 64, cache_slots, 2 if cache_slots < 8 else 0, eps, 1 if cache_slots == 8 else 0)
        self.stack = Stack([cfg] * layers, [W.gate_weight(seed, l, 8, hidden) for l in range(layers)], [W.rms_gamma(hidden)] * layers,
                           n_staging=0 if cache_slots == 8 else 4, max_batch=max_rows, device=device)
        for l in range(layers):
            for e in range(8):
                for m, mat in enumerate(W.quantized_expert(seed, l, e, hidden, ffn, 4, 64, device, 0)):
                    self.stack.load_expert(l, e, m, *mat)
        g = torch.Generator().manual_seed(seed)
        width = (q_heads + 2 * kv_heads) * head_dim
        self.wqkv = [(torch.randn(hidden, width, generator=g) * hidden ** -0.5).half().to(device) for _ in range(layers)]
        self.wo = [(torch.randn(q_heads * head_dim, hidden, generator=g) * (q_heads * head_dim) ** -0.5).half().to(device) for _ in range(layers)]
        self.inv_freq = (theta ** (-torch.arange(0, head_dim, 2, dtype=torch.float64) / head_dim)).float().to(device)
        self.caches = [paged.Cache.empty(self.n_pages, kv_heads, head_dim, page, fmt, device) for _ in range(layers)]
        i32 = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device=device)  # noqa: E731
        self.ctx_len, self.new_len, self.block_table = i32(n_requests), i32(n_requests), i32(n_requests, self.max_blocks)
        self.free_pages = torch.arange(self.n_pages, dtype=torch.int32, device=device)
        self.free_count = torch.full((1,), self.n_pages, dtype=torch.int32, device=device)
        torch.cuda.synchronize()

    def bounds(self, rows: int, most: int) -> paged.Step:
        """The workspaces of steps of `rows` rows in all and at most `most` of a request; made once for many steps."""
        with torch.cuda.stream(self.stack.compute):     # memory of the stream that uses it: it may be dropped while a step runs
            return paged.Step(self.n_requests, rows, most, self.max_blocks, self.n_pages, self.page, self.q_heads, self.kv_heads, self.head_dim,
                              window=self.window, device=self.device)

    @contextlib.contextmanager
    def _on_compute(self, *tensors: torch.Tensor):
        """The compute stream, behind the caller's, which then waits for it; `tensors` of the caller's are used there."""
        caller, compute = torch.cuda.current_stream(self.stack.device), self.stack.compute
        compute.wait_stream(caller)
        for t in tensors:
            t.record_stream(compute)
        try:
            with torch.cuda.stream(compute):
                yield caller
        finally:
            caller.wait_stream(compute)

    def attention_half(self, layer: int, step: paged.Step, x: torch.Tensor) -> torch.Tensor:
        """x + attention(norm(x)) Wo for the step's rows [rows, hidden]."""
        hq, hk, d = self.q_heads, self.kv_heads, self.head_dim
        f = x.float()
        h = (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + self.eps)).half()
        qkv = (h @ self.wqkv[layer]).view(-1, hq + 2 * hk, d)
        q = paged.write(self.caches[layer], step, qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:], inv_freq=self.inv_freq, q_out=qkv[:, :hq])
        # rows of no request are left alone by attention
        a = paged.attend(self.caches[layer], step, q, out=None if self._rows == len(x) else x.new_zeros(len(x), hq, d))
        return x + a.view(-1, hq * d) @ self.wo[layer]

    def _pages(self, tokens: int) -> int:
        return -(-tokens // self.page)

    def _check(self, step: paged.Step, new: List[int]) -> None:
        """Raises if the step would turn a request down, whose hidden state would go on without its token."""
        if len(new) != self.n_requests or min(new) < 0 or max(new) > step.s.max_new or sum(new) > step.s.n_tokens:
            raise ValueError(f"Decoder: {new} new tokens of {self.n_requests} requests do not fit a step of {step.s.n_tokens} rows, {step.s.max_new} of a request")
        for r, (c, n) in enumerate(zip(self._lens, new)):
            if n and self._pages(c + n) > self.max_blocks:
                raise ValueError(f"Decoder: request {r} has {c} tokens, {n} more are beyond {self.max_blocks} pages of {self.page}")
        need = sum(self._pages(c + n) - self._pages(c) for c, n in zip(self._lens, new))
        if need > self._free:
            raise ValueError(f"Decoder: {need} more pages are needed, {self._free} are free")

    def step(self, step: paged.Step, x: torch.Tensor, new: Optional[Sequence[int]] = None) -> torch.Tensor:
        """One step of all blocks for rows x [rows, hidden] (fp16); new: tokens of each request if they changed since the last step.  Rows past
        the requests' tokens come back as they are.  A step that cannot serve every request is refused (ValueError) before anything runs."""
        now = self._new if new is None else list(new)
        self._check(step, now)
        with self._on_compute(x) as caller:
            if new is not None:
                self.new_len.copy_(torch.tensor(now, dtype=torch.int32))
            self._new, self._rows = now, sum(now)
            step.plan(self.ctx_len, self.new_len, self.block_table, self.free_pages, self.free_count)
            for l in range(self.layers if self._rows else 0):
                x = self.attention_half(l, step, x)
                out = torch.empty_like(x)
                self.stack.step_layer(l, x[:self._rows], out[:self._rows])      # the others take no expert
                if self._rows < len(x):
                    out[self._rows:] = x[self._rows:]
                x = out
            step.advance()
            self._free -= sum(self._pages(c + n) - self._pages(c) for c, n in zip(self._lens, now))
            self._lens = [c + n for c, n in zip(self._lens, now)]
            x.record_stream(caller)
        return x

    def finish(self, requests: List[int]) -> None:
        """The requests' pages go back to the pool."""
        with self._on_compute():
            ids = torch.tensor(requests, dtype=torch.int32).to(self.device)
            paged.release(ids, self.n_pages, self.page, self.ctx_len, self.block_table, self.free_pages, self.free_count)
        for r in requests:
            if 0 <= r < self.n_requests:
                self._free += self._pages(self._lens[r])
                self._lens[r] = 0

    def close(self) -> None:
        self.stack.close()


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("layers", 2), ("requests", 4), ("prompt", 37), ("tokens", 16), ("hidden", 256), ("ffn", 512), ("q-heads", 4),
                          ("kv-heads", 2), ("head-dim", 64), ("page", 64), ("window", 0), ("cache-slots", 8), ("seed", 0)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--format", choices=("e4m3", "int8"), default="e4m3")
    a = ap.parse_args(argv)
    prompts = [max(1, a.prompt - 5 * r) for r in range(a.requests)]      # ragged
    rows = sum(prompts)
    d = Decoder(a.layers, a.hidden, a.ffn, a.q_heads, a.kv_heads, a.head_dim, a.requests, a.prompt + a.tokens, max(rows, a.requests), a.page,
                torch.float8_e4m3fn if a.format == "e4m3" else torch.int8, a.window, cache_slots=a.cache_slots, seed=a.seed)
    x = W.hidden_ar1(a.seed, 1, rows, a.hidden)[0].to(d.device)
    x = d.step(d.bounds(rows, max(prompts)), x, prompts)
    ends = torch.tensor(prompts).cumsum(0) - 1
    x = x[ends.to(d.device)].contiguous()
    one = d.bounds(a.requests, 1)
    x = d.step(one, x, [1] * a.requests)
    d.stack.synchronize()
    t = time.perf_counter()
    for _ in range(a.tokens - 1):
        x = d.step(one, x)
    d.stack.synchronize()
    t = time.perf_counter() - t
    lens = d.ctx_len.tolist()
    d.finish(list(range(a.requests)))
    d.stack.synchronize()
    result = {"layers": a.layers, "requests": a.requests, "cached_tokens": lens, "free_pages": int(d.free_count.item()), "pages": d.n_pages,
              "ms_per_step": 1e3 * t / max(1, a.tokens - 1), "tokens_per_s": a.requests * (a.tokens - 1) / t if a.tokens > 1 else None,
              "finite": bool(torch.isfinite(x).all()), "format": a.format}
    d.close()
    return result


if __name__ == "__main__":
    print(json.dumps(main()))
