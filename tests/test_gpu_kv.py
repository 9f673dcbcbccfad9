"""The paged 8-bit cache on the GPU against its definition in 64 bits: pages and slots from lengths, norm, rotation and store,
attention, the values read back."""
import math

import numpy as np
import pytest
import torch

import kv_reference as R
from paper_2312_17238_amd import binding as B
from paper_2312_17238_amd import paged

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def fenced(nbytes):
    """(a buffer, the bytes behind it, which nothing may touch)"""
    whole = torch.full((nbytes + 8192,), 0x5A, dtype=torch.uint8, device=DEV)
    return whole[:nbytes], whole[nbytes:]


# ---- pages and slots -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n_req,page,most_new,most_ctx,short", [
    (1, 16, 1, 0, False), (1, 64, 1, 700, False), (1, 128, 5000, 3, False), (7, 16, 9, 60, False), (8, 32, 1, 2000, True),
    (63, 16, 40, 100, False), (64, 64, 300, 300, True), (65, 128, 1, 1, False), (1000, 16, 20, 50, True), (1025, 16, 3, 5, False),
    (2049, 32, 30, 300, False), (4096, 16, 4, 64, True)])
@pytest.mark.parametrize("odd", [False, True])
def test_plan(n_req, page, most_new, most_ctx, short, odd):
    rng = np.random.default_rng(n_req * 7 + page + odd)
    ctx = rng.integers(0, most_ctx + 1, n_req).tolist()
    new = rng.integers(0 if n_req > 1 else 1, most_new + 1, n_req).tolist()
    width = max(-(-(c + n) // page) for c, n in zip(ctx, new)) + 1
    n_tokens = max(1, sum(new)) + int(rng.integers(0, 4))
    if odd:                     # lengths that no request can have, a table too narrow for some, rows for fewer than there are
        for i in rng.integers(0, n_req, 3):
            ctx[i] = int(rng.choice([-1, -2 ** 31, 2 ** 31 - 1, ctx[i]]))
        for i in rng.integers(0, n_req, 3):
            new[i] = int(rng.choice([-5, 2 ** 31 - 1 if n_req > 1 else -1, most_new + 1, new[i]]))
        width = max(1, width - 2)
        n_tokens = max(1, n_tokens - int(rng.integers(0, 6)))
    n_pages = n_req * width + 3
    table = rng.integers(-1, n_pages + 1, (n_req, width)).astype(np.int32)      # held pages: any, and such as do not exist
    free = rng.permutation(n_pages).astype(np.int32)
    need = sum(max(0, -(-(c + n) // page) - -(-c // page)) for c, n in zip(ctx, new) if c >= 0 and 0 <= n <= most_new)
    room = int(rng.integers(0, min(need, n_pages) + 1)) if short else n_pages
    step = paged.Step(n_req, n_tokens, most_new, width, n_pages, page, 8, 2, 64)
    step.plan_dev, fence = fenced(step.plan_dev.numel())
    tab = torch.from_numpy(table.copy()).to(DEV)
    step.plan(i32(ctx), i32(new), tab, torch.from_numpy(free).to(DEV), i32([room]))
    start, positions, slots, kv, status, left = R.plan(ctx, new, table, free, room, n_tokens=n_tokens, max_new=most_new, n_pages=n_pages, page=page)
    assert step.status.tolist() == status
    assert step.row_start.tolist() == start
    assert step.positions.tolist() == positions
    assert step.slots.tolist() == slots
    assert step.kv_len.tolist() == kv
    assert step.free_left.tolist() == [left]
    assert (tab.cpu().numpy() == table).all() and (fence == 0x5A).all()


def test_release_gives_pages_back_in_order():
    table = i32([[3, 4, 5, -1], [6, 99, 7, 8], [9, 10, 11, 12]])
    ctx, free, count = i32([33, 64, 1]), i32([0, 1, 2] + [-7] * 6), i32([3])
    paged.release(i32([1, 5, -1, 0, 1]), 16, 16, ctx, table, free, count)
    # request 1 holds four pages, of which 99 is none; request 0 three; ids 5 and -1 are nobody's, request 1 has nothing left
    assert ctx.tolist() == [0, 0, 1] and count.tolist() == [9]
    assert free.tolist() == [0, 1, 2, 6, 7, 8, 3, 4, 5]
    paged.release(i32([2]), 16, 16, ctx, table, free, count)                  # the stack is full
    assert ctx.tolist() == [0, 0, 0] and count.tolist() == [9] and free.tolist() == [0, 1, 2, 6, 7, 8, 3, 4, 5]


def test_release_many_pages():
    n = 1000
    table = torch.arange(n, dtype=torch.int32, device=DEV).view(1, n)
    ctx, free, count = i32([16 * n - 5]), torch.full((n + 5,), -1, dtype=torch.int32, device=DEV), i32([0])
    paged.release(i32([0]), n, 16, ctx, table, free, count)
    assert free[:n].tolist() == list(range(n)) and count.item() == n


# ---- a pool of requests, stepped --------------------------------------------------------------------------------------

class Pool:
    """Requests with pages of a cache, their tensors and what the definition says that the cache holds."""

    def __init__(self, n_req, width, *, q_heads=4, kv_heads=2, dim=64, page=16, fmt="e4m3", dtype=torch.float16, causal=True, window=0, seed=0, extra=3):
        self.rng = np.random.default_rng(seed)
        self.n_req, self.width, self.q_heads, self.kv_heads, self.dim, self.page, self.fmt, self.dtype = n_req, width, q_heads, kv_heads, dim, page, fmt, dtype
        self.causal, self.window = causal, window
        self.n_pages = n_req * width + extra
        self.cache = paged.Cache.empty(self.n_pages, kv_heads, dim, page, R.CODE[fmt], DEV)
        # whatever was there before: codes of every kind, NaN among them, and scales that are no numbers
        self.cache.k.view(torch.uint8).copy_(torch.from_numpy(self.rng.integers(0, 256, self.cache.k.shape, dtype=np.uint8)))
        self.cache.v.view(torch.uint8).copy_(torch.from_numpy(self.rng.integers(0, 256, self.cache.v.shape, dtype=np.uint8)))
        self.cache.k_scale.fill_(math.nan)
        self.cache.v_scale.fill_(math.nan)
        self.ctx = torch.zeros(n_req, dtype=torch.int32, device=DEV)
        self.table = torch.full((n_req, width), -1, dtype=torch.int32, device=DEV)
        self.free = torch.from_numpy(self.rng.permutation(self.n_pages).astype(np.int32)).to(DEV)
        self.count = i32([self.n_pages])
        self.lens = [0] * n_req
        # by request and head: pages of [tokens][dim] values, and their scales
        self.held = [[{} for _ in range(n_req)] for _ in range(2)]

    def step(self, new, spare=0):
        s = paged.Step(self.n_req, max(1, sum(new) + spare), max(1, max(new)), self.width, self.n_pages, self.page, self.q_heads, self.kv_heads, self.dim,
                       self.causal, self.window)
        s.plan(self.ctx, i32(new), self.table, self.free, self.count)
        assert s.status.tolist() == [0] * self.n_req
        return s

    def rows(self, n, heads, spread=1.0):
        x = self.rng.standard_normal((n, heads, self.dim)) * np.exp2(spread * self.rng.standard_normal((n, heads, 1)))
        return torch.from_numpy(x).to(self.dtype).to(DEV)

    def store(self, new, k, v):
        """Fills `held` with what k, v (64-bit numpy, rows in order) become."""
        at = 0
        for r, n in enumerate(new):
            for i in range(n):
                pos = self.lens[r] + i
                b, o = divmod(pos, self.page)
                for w, x in ((0, k), (1, v)):
                    self.held[w][r].setdefault(b, []).append(x[at + i])
            at += n

    def check_cache(self, new, k, v, top=65504.0):
        """The cache's tensors against the definition, page by page: what is new and what was there."""
        at, off, seen = 0, 0, 0
        limit = R.LARGEST[self.fmt]
        for r, n in enumerate(new):
            c = self.lens[r]
            for b in range(c // self.page, -(-(c + n) // self.page) if n else 0):
                lo, hi = max(c, b * self.page), min(c + n, (b + 1) * self.page)
                pid = int(self.table[r, b])
                for w, x, codes, scales in ((0, k, self.cache.k, self.cache.k_scale), (1, v, self.cache.v, self.cache.v_scale)):
                    for h in range(self.kv_heads):
                        y = x[at + lo - c:at + hi - c, h]
                        y = np.where(np.isnan(y), 0.0, np.clip(y, -top, top))
                        want = R.page_scale(np.abs(y).max(), self.fmt)
                        key = (b, h)
                        old, old_s = self.held[w][r].get(key, (np.zeros((0, self.dim)), 0.0))
                        s = max(want, old_s)
                        # a largest number at the border between two scales may be rounded to either side
                        got = float(scales[pid, h])
                        if got != s:
                            assert w == 0 and abs(np.abs(y).max() / (limit * min(s, got)) - 1) < 1e-5, (r, b, h, got, s)
                            s = got
                        val = np.concatenate([R.nearest(old / s, self.fmt) * s, R.nearest(y / s, self.fmt) * s])
                        have = R.cache_values(codes, scales, self.fmt, bool(w), [pid], h)[:hi - b * self.page]
                        # fp32 of a rotated key may lie on the other side of the middle between two codes
                        step = s if self.fmt == "int8" else np.maximum(np.abs(val) / 8, s * 2.0 ** -9)
                        d = np.abs(have - val)
                        assert (d <= (step * 1.001 if w == 0 else 0)).all(), (r, b, h, w)
                        off += int((d > 0).sum())
                        seen += val.size
                        self.held[w][r][key] = (have, s)
            at += n
            self.lens[r] += n
        assert off <= 2 + seen * 1e-3, f"{off} of {seen} codes are the neighbour of the right one"


def half_step(x, dtype):
    """Half a step of `dtype` at x, subnormal numbers included."""
    f = torch.finfo(dtype)
    return np.maximum(np.abs(x), f.tiny) * f.eps / 2


CASES = [
    dict(dim=64, page=16, fmt="e4m3", dtype=torch.float16),
    dict(dim=64, page=128, fmt="int8", dtype=torch.bfloat16, eps=1e-5, gain=True, rot=64, interleaved=True),
    dict(dim=128, page=16, fmt="int8", dtype=torch.float16, rot=128),
    dict(dim=128, page=32, fmt="e4m3", dtype=torch.bfloat16, eps=1e-6, rot=64, strided=True),
    dict(dim=128, page=64, fmt="e4m3", dtype=torch.float16, eps=1e-6, gain=True, rot=128, interleaved=True, odd=True),
    dict(dim=128, page=128, fmt="int8", dtype=torch.bfloat16, rot=48, odd=True),
    dict(dim=256, page=16, fmt="e4m3", dtype=torch.float16, rot=16, eps=1e-3),
    dict(dim=256, page=64, fmt="int8", dtype=torch.bfloat16, rot=256, gain=True, eps=1e-6),
    dict(dim=256, page=128, fmt="e4m3", dtype=torch.bfloat16, rot=128, interleaved=True, q_heads=6, kv_heads=3),
    dict(dim=64, page=64, fmt="e4m3", dtype=torch.float16, rot=64, q_heads=1, kv_heads=1, in_place=True),
]


def layer_inputs(pool, n, strided=False, odd=False, spread=1.0):
    """q, k, v of n rows: tensors of their own, views of one packed tensor, or views that are not 16-byte aligned."""
    hq, hk, d = pool.q_heads, pool.kv_heads, pool.dim
    x = pool.rows(n, hq + 2 * hk, spread)
    if odd:
        w = (hq + 2 * hk) * d
        flat = torch.zeros(n * (w + 3) + 1, dtype=pool.dtype, device=DEV)
        view = flat[1:].as_strided((n, hq + 2 * hk, d), (w + 3, d, 1))
        view.copy_(x)
        x = view
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    return (q, k, v) if strided or odd else (q.contiguous(), k.contiguous(), v.contiguous())


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v).replace("torch.", "") for v in c.values()))
def test_write(case):
    """Several steps of ragged requests, so that pages are begun, filled up and have their scales raised."""
    case = dict(case)
    eps, gain, rot, inter = case.pop("eps", 0.0), case.pop("gain", False), case.pop("rot", 0), case.pop("interleaved", False)
    strided, odd, in_place = case.pop("strided", False), case.pop("odd", False), case.pop("in_place", False)
    p = Pool(5, 4 if case["page"] == 128 else 24, seed=case["dim"] + case["page"], **case)
    g = torch.Generator().manual_seed(3)
    gq, gk = ((1 + 0.3 * torch.randn(2, p.dim, generator=g)).to(p.dtype).to(DEV)) if gain else (None, None)
    freq = (10000.0 ** (-torch.arange(0, rot, 2) / rot)).float().to(DEV) if rot else None
    for i, new in enumerate(([1, 0, 17, 130, 16], [1, 3, 1, 0, 1], [15, 1, 1, 1, 16], [1, 1, 1, 1, 1], [0, 40, 0, 33, 2])):
        s = p.step(new, spare=2)
        q, k, v = layer_inputs(p, sum(new) + 2, strided, odd, spread=0.5 * i)
        q_in = q.float().cpu().numpy()
        out = paged.write(p.cache, s, q, k, v, gq, gk, eps, freq, inter, q_out=q if in_place else None)
        pos = s.positions.tolist()[:sum(new)]
        np_ = lambda t: t.float().cpu().numpy()  # noqa: E731
        f = np_(freq) if rot else None
        n = sum(new)
        want_q = R.turned(q_in[:n], pos, np_(gq) if gain else None, eps, f, inter)
        want_k = R.turned(np_(k)[:n], pos, np_(gk) if gain else None, eps, f, inter)
        # one rounding to the type, and fp32 on the way: a dozen roundings of 2^-24 of the pair's size
        size = np.sqrt((want_q ** 2).max(-1, keepdims=True) * 2)
        err = np.abs(np_(out)[:n] - want_q)
        assert (err <= half_step(want_q, p.dtype) * 1.01 + 2.0 ** -20 * size).all(), err.max()
        if in_place:
            assert (np_(out)[n:] == q_in[n:]).all()
        p.check_cache(new, want_k, np_(v)[:n].astype(np.float64))
        s.advance()
    assert p.ctx.tolist() == p.lens


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_write_what_is_no_number_and_what_is_nothing(fmt, dtype):
    """Infinities are the largest number that is stored, NaN is 0, a page of zeros is zeros: no code is NaN, no scale unusable."""
    p = Pool(3, 2, fmt=fmt, dtype=dtype, kv_heads=1, q_heads=1, page=32)
    top = 65504.0 if dtype == torch.float16 else 2.0 ** 100
    for new in ([3, 5, 4], [2, 1, 30]):
        s = p.step(new)
        q, k, v = layer_inputs(p, sum(new))
        k, v = torch.zeros_like(k), torch.zeros_like(v)
        if new[0] == 2:
            k[0, 0, 0], v[1, 0, 5], v[2, 0, 7], k[2, 0, 3] = math.inf, -math.inf, math.nan, math.nan
            v[3:, :, :] = torch.finfo(dtype).smallest_normal
        paged.write(p.cache, s, q, k, v)
        p.check_cache(new, k.double().cpu().numpy(), v.double().cpu().numpy(), top=top)
        s.advance()
    for w, codes, sc in ((False, p.cache.k, p.cache.k_scale), (True, p.cache.v, p.cache.v_scale)):
        for r in range(3):
            for b in range(-(-p.lens[r] // p.page)):
                assert np.isfinite(R.cache_values(codes, sc, fmt, w, [int(p.table[r, b])], 0)[:max(0, p.lens[r] - b * 32)]).all()


def test_write_at_far_positions():
    """A rotation at position a million: the angle is worked out in 64 bits."""
    page, width = 16, 70000
    p = Pool(1, 4, fmt="int8", page=page, dim=128, q_heads=2, kv_heads=1)
    table = torch.zeros(1, width, dtype=torch.int32, device=DEV)
    freq = (10000.0 ** (-torch.arange(0, 128, 2) / 128)).float().to(DEV)
    for at in (0, 65535, 1000007, 16 * 69999):
        s = paged.Step(1, 1, 1, width, p.n_pages, page, 2, 1, 128)
        s.plan(i32([at]), i32([1]), table, p.free, p.count)
        q, k, v = layer_inputs(p, 1)
        out = paged.write(p.cache, s, q, k, v, inv_freq=freq).float().cpu().numpy()
        want = R.turned(q.float().cpu().numpy(), [at], None, 0.0, freq.cpu().numpy(), False)
        size = np.sqrt((want ** 2).max(-1, keepdims=True) * 2)
        assert (np.abs(out - want) <= half_step(want, torch.float16) * 1.01 + 2.0 ** -20 * size).all()


def test_gather_reads_what_is_stored():
    for fmt in ("e4m3", "int8"):
        for dtype in (torch.float16, torch.bfloat16):
            p = Pool(4, 5, fmt=fmt, dtype=dtype, dim=128, page=32, kv_heads=3, q_heads=3)
            new = [40, 1, 0, 77]
            s = p.step(new)
            q, k, v = layer_inputs(p, sum(new))
            paged.write(p.cache, s, q, k, v)
            slots = torch.cat([s.slots[torch.randperm(sum(new), device=DEV)], s.slots, i32([-1, p.n_pages * 32, 2 ** 31 - 1, -2 ** 31])])
            ko, vo = paged.gather(p.cache, slots, dtype)
            for w, got, codes, sc in ((False, ko, p.cache.k, p.cache.k_scale), (True, vo, p.cache.v, p.cache.v_scale)):
                for h in range(3):
                    every = R.cache_values(codes, sc, fmt, w, list(range(p.n_pages)), h)
                    want = np.stack([every[i] if 0 <= i < p.n_pages * 32 else np.zeros(128) for i in slots.tolist()])
                    assert (got[:, h].double().cpu().numpy() == want).all()     # 8 bits are exact in 16


# ---- attention ---------------------------------------------------------------------------------------------------------

def fill(pool, lens, codes_only=False, scales="powers"):
    """A cache with tokens already in it, straight into the tensors (finite codes), and their table."""
    rng = pool.rng
    table = np.full((pool.n_req, pool.width), -1, np.int32)
    ids = rng.permutation(pool.n_pages)
    at = 0
    for r, n in enumerate(lens):
        b = -(-n // pool.page)
        table[r, :b] = ids[at:at + b]
        at += b
    pool.table.copy_(torch.from_numpy(table))
    for codes in (pool.cache.k, pool.cache.v):
        c = codes.view(torch.uint8)
        if pool.fmt == "e4m3":
            x = torch.from_numpy(rng.standard_normal(tuple(c.shape), dtype=np.float32) * 20)
            c.copy_(x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
        else:
            c.copy_(torch.from_numpy(np.clip(np.rint(rng.standard_normal(tuple(c.shape), dtype=np.float32) * 35), -127, 127).astype(np.int8)).view(torch.uint8))
    unit = 1 / 20 if pool.fmt == "e4m3" else 1 / 35
    for sc in (pool.cache.k_scale, pool.cache.v_scale):
        e = rng.standard_normal(tuple(sc.shape)) * (0 if scales == "one" else 1 if scales == "powers" else 12)
        e = np.rint(e) if scales != "any" else e / 4
        sc.copy_(torch.from_numpy((unit * np.exp2(e)).astype(np.float32)))
    # beyond a request's last token: NaN codes in e4m3
    for r, n in enumerate(lens):
        if n % pool.page:
            pid, o = int(table[r, n // pool.page]), n % pool.page
            for t in range(o, pool.page):
                pool.cache.k.view(torch.uint8)[pid, :, t // 16, :, t % 16] = 0x7F
                pool.cache.v.view(torch.uint8)[pid, :, t // 16, :, t % 16] = 0x7F


def check_attend(pool, step, q, out, lse, lens, new, scale, rows=None, heads=None):
    """Rows of requests with `lens` cached tokens in all, the last `new` of them the step's."""
    at = 0
    g = pool.q_heads // pool.kv_heads
    qd, od, ld = q.double().cpu().numpy(), out.double().cpu().numpy(), lse.double().cpu().numpy()
    for r, (n, m) in enumerate(zip(lens, new)):
        pick = range(m) if rows is None or m <= rows else sorted(set([0, m - 1]) | set(pool.rng.integers(0, m, rows).tolist()))
        pick = list(pick)
        if pick:
            ids = [max(0, int(i)) for i in pool.table[r, :-(-n // pool.page)].tolist()]
            for h in heads or range(pool.kv_heads):
                k = R.cache_values(pool.cache.k, pool.cache.k_scale, pool.fmt, False, ids, h)
                v = R.cache_values(pool.cache.v, pool.cache.v_scale, pool.fmt, True, ids, h)
                k[n:] = 0
                v[n:] = 0
                for u in range(g):
                    head = h * g + u
                    want, wl, slack = R.attend_head(qd[[at + i for i in pick], head], k, v, [n - m + i for i in pick], n, scale, pool.causal, pool.window)
                    for x, i in enumerate(pick):
                        # a result beyond the type's largest number is infinite
                        over = np.abs(want[x]) > torch.finfo(pool.dtype).max
                        got = np.where(over & np.isinf(od[at + i, head]) & (np.sign(od[at + i, head]) == np.sign(want[x])), want[x], od[at + i, head])
                        err = np.abs(got - want[x])
                        allowed = slack[x] + half_step(want[x], pool.dtype) * 1.01
                        assert (err <= allowed).all(), (r, h, u, i, float((err / allowed).max()))
                        if wl[x] == -np.inf:
                            assert ld[at + i, head] == -np.inf
                        else:
                            assert abs(ld[at + i, head] - wl[x]) <= 2.0 ** -18 * (1 + abs(wl[x]) + np.abs(qd[at + i, head]).sum() * scale * np.abs(k[:n]).max() * 2.0 ** -4)
        at += m


ATTEND = [
    # requests' tokens (cached and new together), new ones
    dict(lens=[1], new=[1], dim=64),
    dict(lens=[17, 1, 31, 33], new=[1, 1, 1, 1], dim=128, page=16),
    dict(lens=[300, 64, 129], new=[1, 2, 3], dim=64, fmt="int8", dtype=torch.bfloat16, page=32),
    dict(lens=[1000, 5, 257], new=[5, 5, 5], dim=128, q_heads=14, kv_heads=2, dtype=torch.bfloat16),
    dict(lens=[700, 90], new=[1, 1], dim=256, fmt="int8", q_heads=8, kv_heads=1, page=128),
    dict(lens=[4000, 3], new=[1, 1], dim=128, page=16, q_heads=8, kv_heads=8),
    dict(lens=[20000], new=[1], dim=64, page=64, q_heads=2, kv_heads=1, fmt="int8"),
    dict(lens=[40, 200, 333], new=[40, 200, 100], dim=128, page=16, q_heads=4, kv_heads=2),
    dict(lens=[129, 65], new=[129, 33], dim=64, page=64, q_heads=1, kv_heads=1, dtype=torch.bfloat16),
    dict(lens=[500, 1, 90], new=[257, 1, 0], dim=256, page=32, q_heads=2, kv_heads=1, fmt="int8"),
    dict(lens=[2600, 700], new=[300, 1], dim=128, page=128, q_heads=16, kv_heads=2, fmt="int8", dtype=torch.bfloat16),
    dict(lens=[9000], new=[40], dim=64, page=16, q_heads=8, kv_heads=1),
    dict(lens=[90, 30], new=[3, 1], dim=64, q_heads=64, kv_heads=1, page=16),
    # windows
    dict(lens=[500, 40, 3], new=[1, 1, 1], dim=64, page=16, window=33),
    dict(lens=[2000, 100], new=[7, 2], dim=128, page=64, window=100, fmt="int8", q_heads=8, kv_heads=2),
    dict(lens=[700, 260], new=[300, 260], dim=64, page=16, window=70, dtype=torch.bfloat16),
    dict(lens=[700, 260], new=[300, 1], dim=128, page=32, window=1),
    # every token sees all
    dict(lens=[130, 33, 1], new=[50, 3, 1], dim=64, page=16, causal=False),
    dict(lens=[300, 90], new=[200, 90], dim=128, page=64, causal=False, window=50, fmt="int8"),
    # scales of very different sizes
    dict(lens=[900, 60], new=[1, 1], dim=128, page=16, scales="wide"),
    dict(lens=[900, 60], new=[90, 1], dim=64, page=16, scales="wide", dtype=torch.bfloat16, fmt="int8"),
    dict(lens=[300, 600], new=[1, 200], dim=128, page=32, scales="any"),
    # so many heads that a block has more steps than it knows the places of at a time
    dict(lens=[30000, 40], new=[1, 1], dim=64, page=64, kv_heads=128, q_heads=128, heads=[0, 77, 127]),
    dict(lens=[30000, 40], new=[20, 17], dim=64, page=64, kv_heads=128, q_heads=128, heads=[5, 127], fmt="int8"),
    dict(lens=[30000, 200], new=[70, 100], dim=64, page=64, kv_heads=128, q_heads=128, heads=[0, 126], dtype=torch.bfloat16),
    # many requests whose ends lie in the middle of blocks, some with nothing to do
    dict(lens=[37 * i % 701 + 1 for i in range(150)], new=[(i * 7) % 4 and 1 for i in range(150)], dim=64, page=16, q_heads=4, kv_heads=4, heads=[2]),
    dict(lens=[137 * i % 1701 + 9 for i in range(60)], new=[(i * 5) % 9 for i in range(60)], dim=128, page=32, q_heads=8, kv_heads=2, heads=[1], fmt="int8"),
    dict(lens=[1037 * i % 9001 + 60 for i in range(20)], new=[1 if i % 3 else 50 for i in range(20)], dim=64, page=128, q_heads=4, kv_heads=2, heads=[0]),
]


@pytest.mark.parametrize("case", ATTEND, ids=lambda c: "-".join(str(v).replace("torch.", "").replace(" ", "")[:40] for v in c.values()))
def test_attend(case):
    case = dict(case)
    lens, new, scales, heads = case.pop("lens"), case.pop("new"), case.pop("scales", "powers"), case.pop("heads", None)
    page = case.setdefault("page", 64)
    p = Pool(len(lens), -(-max(lens) // page) + 1, seed=sum(lens), **case)
    fill(p, lens, scales=scales)
    s = paged.Step(len(lens), sum(new) + 1, max(new), p.width, p.n_pages, page, p.q_heads, p.kv_heads, p.dim, p.causal, p.window)
    table = p.table.clone()
    need = [-(-n // page) - -(-(n - m) // page) for n, m in zip(lens, new)]
    free = [int(table[r, -(-(n - m) // page) + i]) for r, (n, m) in enumerate(zip(lens, new)) for i in range(need[r])][::-1]
    s.plan(i32([n - m for n, m in zip(lens, new)]), i32(new), p.table, i32(free + [0]), i32([len(free)]))
    assert (p.table == table).all() and s.status.tolist() == [0] * len(lens)
    q = p.rows(sum(new) + 1, p.q_heads, spread=0.5)
    scale = 1 / math.sqrt(p.dim)
    out = torch.full_like(q, 7.0)
    s.scratch, fence = fenced(max(16, s.scratch_bytes))
    out, lse = paged.attend(p.cache, s, q, scale, out=out, with_lse=True)
    assert (out[-1] == 7).all() and (fence == 0x5A).all()       # the last row is no request's
    check_attend(p, s, q, out, lse, lens, new, scale, rows=6, heads=heads)
    again, lse2 = paged.attend(p.cache, s, q, scale, with_lse=True)
    assert torch.equal(again[:-1], out[:-1]) and torch.equal(lse2[:-1], lse[:-1])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("new", [[1, 1, 1], [70, 1, 40]])
def test_attend_rows_that_see_nothing_and_rows_that_are_no_numbers(dtype, new):
    """Requests that were turned down give zeros; a query of NaN or infinity spoils its own rows alone; large scores do not overflow."""
    p = Pool(3, 8, dtype=dtype, page=16, q_heads=4, kv_heads=2)
    lens = [90, 100, 41]
    fill(p, lens, scales="one")
    s = paged.Step(3, sum(new), max(new), p.width, p.n_pages, 16, 4, 2, 64)
    s.plan(i32([lens[0] - new[0], 100000, lens[2] - new[2]]), i32(new), p.table, torch.flip(p.table[[0, 2]].reshape(-1), [0]).contiguous(), i32([0]))
    st = s.status.tolist()
    assert st[1] == B.MOE_KV_TOO_LONG
    served = [x == 0 for x in st]
    q = p.rows(sum(new), 4)
    clean = q.clone()
    q[0, 1, 5], q[0, 2, 6], q[0, 3] = math.nan, math.inf, 30000.0
    out, lse = paged.attend(p.cache, s, q, with_lse=True)
    ref, _ = paged.attend(p.cache, s, clean, with_lse=True)
    start = s.row_start.tolist()
    for r in range(3):
        o = out[start[r]:start[r + 1]]
        if not served[r]:
            assert (o == 0).all() and (lse[start[r]:start[r + 1]] == -math.inf).all()
        else:
            assert torch.equal(o[1:], ref[start[r]:start[r + 1]][1:]) and (o[1:].abs().sum() > 0 or new[r] == 1)
    if served[0]:
        assert torch.equal(out[0, 0], ref[0, 0]) and out[0, 1].isnan().all() and out[0, 2].isnan().all() and out[0, 3].isfinite().all()


def test_attend_skips_pages_that_do_not_exist():
    """Entries of the table outside the cache count as masked; with all of them there, the row sees nothing."""
    for new in (1, 40):
        p = Pool(2, 8, page=16, fmt="int8")
        lens = [100, 60]
        fill(p, lens, scales="one")
        s = paged.Step(2, 2 * new, new, p.width, p.n_pages, 16, 4, 2, 64)
        s.plan(i32([n - new for n in lens]), i32([new, new]), p.table.clone(), torch.zeros(16, dtype=torch.int32, device=DEV), i32([16]))
        bad = p.table.clone()
        bad[0, 1], bad[0, 3] = -1, p.n_pages
        bad[1] = 2 ** 31 - 1
        s.block_table = bad
        q = p.rows(2 * new, 4)
        out, lse = paged.attend(p.cache, s, q, with_lse=True)
        assert (out[new:] == 0).all() and (lse[new:] == -math.inf).all()
        ids = [max(0, min(int(i), p.n_pages - 1)) for i in p.table[0, :7].tolist()]
        for h in range(2):
            k = R.cache_values(p.cache.k, p.cache.k_scale, "int8", False, ids, h)
            v = R.cache_values(p.cache.v, p.cache.v_scale, "int8", True, ids, h)
            live = np.ones(112, bool)
            live[16:32] = live[48:64] = False
            for u in range(2):
                for i in range(new):
                    see = live.copy()
                    see[100 - new + i + 1:] = False
                    z = k[see] @ q[i, 2 * h + u].double().cpu().numpy() / 8
                    w = np.exp(z - z.max())
                    want = w @ v[see] / w.sum()
                    assert np.abs(out[i, 2 * h + u].double().cpu().numpy() - want).max() <= 2.0 ** -9 * np.abs(v[see]).max()


def test_attend_with_views_that_are_not_aligned():
    p = Pool(2, 8, page=16, dtype=torch.bfloat16, dim=64, q_heads=6, kv_heads=2)
    lens, new = [100, 120], [1, 50]
    fill(p, lens)
    s = paged.Step(2, 51, 50, p.width, p.n_pages, 16, 6, 2, 64)
    free = p.table[1, 5:8].flip(0).contiguous()
    s.plan(i32([99, 70]), i32(new), p.table, free, i32([3]))
    q = p.rows(51, 6)
    want, _ = paged.attend(p.cache, s, q, with_lse=True)
    store = torch.zeros(51 * 400 + 1, dtype=torch.bfloat16, device=DEV)
    odd = store[1:].as_strided((51, 6, 64), (397, 64, 1))
    odd.copy_(q)
    store2 = torch.full((51 * 400 + 1,), 3.0, dtype=torch.bfloat16, device=DEV)
    out = store2[1:].as_strided((51, 6, 64), (391, 64, 1))
    paged.attend(p.cache, s, odd, out=out)
    assert torch.equal(out, want)
    out.fill_(3.0)
    assert (store2 == 3).all()                      # nothing beside the rows


def test_far_pages_of_a_large_cache():
    """Codes beyond 4 GiB of a cache, and a table whose rows are far apart."""
    page, heads, dim = 128, 8, 128
    n_pages = (1 << 32) // (page * heads * dim) + 40
    c = paged.Cache(*(torch.zeros(n_pages, heads, page // 16, *t, dtype=torch.int8, device=DEV) for t in ((dim // 16, 16, 16), (dim, 16))),
                    *(torch.ones(n_pages, heads, device=DEV) for _ in range(2)))
    width = 40000
    table = torch.zeros(3, width, dtype=torch.int32, device=DEV)
    table[2, :3] = i32([n_pages - 1, 5, n_pages - 2])
    s = paged.Step(3, 300, 300, width, n_pages, page, heads, heads, dim)
    s.plan(i32([0, 0, 0]), i32([0, 0, 300]), table, i32([n_pages - 2, 5, n_pages - 1]), i32([3]))
    assert s.slots[:128].tolist() == list(range((n_pages - 1) * 128, n_pages * 128))
    g = torch.Generator(device=DEV).manual_seed(1)
    q, k, v = (torch.randn(300, heads, dim, device=DEV, generator=g).half() for _ in range(3))
    paged.write(c, s, q, k, v)
    ko, vo = paged.gather(c, s.slots)
    for got, want in ((ko, k), (vo, v)):            # half a step of 2^e, whose largest code is at least 64
        assert (got.float() - want.float()).abs().max() <= want.float().abs().max() / 127 + 1e-6
    out = paged.attend(c, s, q)
    qd, kd, vd = (x[:, 7].double().cpu() for x in (q, ko, vo))
    z = (qd @ kd.T / math.sqrt(dim)).masked_fill(torch.ones(300, 300).triu(1).bool(), -math.inf)
    want = torch.softmax(z, -1) @ vd
    assert (out[:, 7].double().cpu() - want).abs().max() <= 2.0 ** -10 * vd.abs().max()


# ---- streams and graphs ------------------------------------------------------------------------------------------------

def test_a_captured_step_serves_other_lengths():
    """One graph of plan, store, attention and the bookkeeping after it, replayed as a request grows, against the same calls one by one."""
    def make():
        p = Pool(3, 40, page=16, q_heads=4, kv_heads=2, fmt="int8", seed=5)
        s = paged.Step(3, 30, 20, 40, p.n_pages, 16, 4, 2, 64)
        t = {"new": i32([0, 0, 0]), "x": torch.zeros(30, 8, 64, dtype=torch.float16, device=DEV), "out": torch.zeros(30, 4, 64, dtype=torch.float16, device=DEV),
             "q": torch.zeros(30, 4, 64, dtype=torch.float16, device=DEV)}
        return p, s, t
    freq = (10000.0 ** (-torch.arange(0, 64, 2) / 64)).float().to(DEV)

    def body(p, s, t):
        s.plan(p.ctx, t["new"], p.table, p.free, p.count)
        x = t["x"]
        paged.write(p.cache, s, x[:, :4], x[:, 4:6], x[:, 6:], inv_freq=freq, q_out=t["q"])
        paged.attend(p.cache, s, t["q"], out=t["out"])
        s.advance()
    a, b = make(), make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        body(*b)                                     # lengths 0: nothing happens
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        body(*b)
    rng = np.random.default_rng(2)
    for i in range(12):
        new = [[20, 5, 5], [1, 1, 1], [0, 3, 0], [7, 1, 20]][i % 4]
        x = torch.from_numpy(rng.standard_normal((30, 8, 64))).half().to(DEV)
        for t in (a[2], b[2]):
            t["new"].copy_(i32(new))
            t["x"].copy_(x)
        body(*a)
        graph.replay()
        torch.cuda.synchronize()
        n = sum(new)
        assert torch.equal(a[2]["out"][:n], b[2]["out"][:n]) and a[0].ctx.tolist() == b[0].ctx.tolist() and a[0].count.item() == b[0].count.item()
        assert torch.equal(a[0].table, b[0].table) and a[2]["out"][:n].abs().sum() > 0


def test_calls_follow_the_current_stream():
    """Work on a stream that waits for a long one gives what it gives alone."""
    p = Pool(2, 8, page=32, dim=128)
    new = [100, 60]
    x = p.rows(160, 8)
    s = p.step(new)
    want_q = paged.write(p.cache, s, x[:, :4], x[:, 4:6], x[:, 6:])
    want = paged.attend(p.cache, s, want_q)
    late = torch.empty_like(x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        big = torch.randn(4096, 4096, device=DEV)
        for _ in range(20):
            big = big @ big * 1e-3
        late.copy_(x)
        p.cache.k.view(torch.uint8).zero_()
        q = paged.write(p.cache, s, late[:, :4], late[:, 4:6], late[:, 6:])
        out = paged.attend(p.cache, s, q)
    side.synchronize()
    assert torch.equal(q, want_q) and torch.equal(out, want)
