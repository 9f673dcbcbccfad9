"""The paged cache held in 4 bits on the GPU, against plain 64-bit code: what the store leaves in it, cached tokens read back, and attention over it in
each of its forms."""
import math

import numpy as np
import pytest
import torch

import kv4_reference as R4
import kv_reference as R
from paper_2312_17238_amd import binding as B
from paper_2312_17238_amd import paged

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FOUR = torch.float4_e2m1fn_x2


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def host(t):
    return t.view(torch.uint8).cpu().numpy()


def half_step(x, dtype):
    f = torch.finfo(dtype)
    return np.maximum(np.abs(x), f.tiny) * f.eps / 2


class Pool:
    """Requests with pages of a cache that holds random bytes wherever nothing was stored."""

    def __init__(self, n_req, width, *, q_heads=4, kv_heads=2, dim=64, page=16, dtype=torch.float16, causal=True, window=0, seed=0, extra=3):
        self.rng = np.random.default_rng(seed)
        self.n_req, self.width, self.q_heads, self.kv_heads, self.dim, self.page, self.dtype = n_req, width, q_heads, kv_heads, dim, page, dtype
        self.causal, self.window, self.n_pages = causal, window, n_req * width + extra
        self.cache = paged.Cache.empty(self.n_pages, kv_heads, dim, page, FOUR, DEV)
        for t in (self.cache.k, self.cache.v, self.cache.k_scale, self.cache.v_scale):
            t.view(torch.uint8).copy_(torch.from_numpy(self.rng.integers(0, 256, tuple(t.shape), dtype=np.uint8)))
        self.ctx = torch.zeros(n_req, dtype=torch.int32, device=DEV)
        self.table = torch.full((n_req, width), -1, dtype=torch.int32, device=DEV)
        self.free = torch.from_numpy(self.rng.permutation(self.n_pages).astype(np.int32)).to(DEV)
        self.count = i32([self.n_pages])

    def tensors(self):
        return [host(t).copy() for t in (self.cache.k, self.cache.k_scale, self.cache.v, self.cache.v_scale)]

    def step(self, new, spare=0):
        s = paged.Step(self.n_req, max(1, sum(new) + spare), max(1, max(new)), self.width, self.n_pages, self.page, self.q_heads, self.kv_heads, self.dim,
                       self.causal, self.window)
        s.plan(self.ctx, i32(new), self.table, self.free, self.count)
        assert s.status.tolist() == [0] * self.n_req
        return s

    def rows(self, n, heads, spread=1.0):
        x = self.rng.standard_normal((n, heads, self.dim)) * np.exp2(spread * self.rng.standard_normal((n, heads, 1)))
        return torch.from_numpy(x).to(self.dtype).to(DEV)


def fill(pool, lens, k_exp=(-3, 3), v_exp=(-3, 3)):
    """A cache with tokens already in it, straight into the tensors, and their table; what lies behind the last tokens stays random, scales of 0 and 255
    among it."""
    rng = pool.rng
    table = np.full((pool.n_req, pool.width), -1, np.int32)
    ids, at = rng.permutation(pool.n_pages), 0
    for r, n in enumerate(lens):
        b = -(-n // pool.page)
        table[r, :b] = ids[at:at + b]
        at += b
    pool.table.copy_(torch.from_numpy(table))
    kb, vb = host(pool.cache.k_scale).copy(), host(pool.cache.v_scale).copy()
    kb = np.moveaxis(kb, -1, -3)                        # in the tokens' order: [pages][heads][page/16][t][r][D/32]
    shape = (pool.n_pages, pool.kv_heads, pool.page)
    kb2, vb2 = kb.reshape(*shape, -1).copy(), vb
    for r, n in enumerate(lens):
        for b in range(-(-n // pool.page)):
            m = min(pool.page, n - b * pool.page)
            kb2[table[r, b], :, :m] = 127 + rng.integers(k_exp[0], k_exp[1] + 1, (pool.kv_heads, m, pool.dim // 32))
            vb2[table[r, b], :, :m] = 127 + rng.integers(v_exp[0], v_exp[1] + 1, (pool.kv_heads, m))
    back = kb2.reshape(*shape[:2], pool.page // 16, 4, 4, -1)
    pool.cache.k_scale.view(torch.uint8).copy_(torch.from_numpy(np.ascontiguousarray(np.moveaxis(back, -3, -1))))
    pool.cache.v_scale.view(torch.uint8).copy_(torch.from_numpy(vb2))


def planned(pool, lens, new, spare=0):
    """A step whose pages are those that the table names already."""
    s = paged.Step(len(lens), sum(new) + spare, max(1, max(new)), pool.width, pool.n_pages, pool.page, pool.q_heads, pool.kv_heads, pool.dim, pool.causal, pool.window)
    table = pool.table.clone()
    free = [int(table[r, b]) for r, (n, m) in enumerate(zip(lens, new)) for b in range(-(-(n - m) // pool.page), -(-n // pool.page))][::-1]
    s.plan(i32([n - m for n, m in zip(lens, new)]), i32(new), pool.table, i32(free + [0]), i32([len(free)]))
    assert (pool.table == table).all() and s.status.tolist() == [0] * len(lens)
    return s


def check_attend(pool, q, out, lse, lens, new, scale, rows=None, heads=None, table=None):
    """Rows of requests with `lens` cached tokens in all, the last `new` of them the step's."""
    at, g = 0, pool.q_heads // pool.kv_heads
    table = pool.table if table is None else table
    k, kb, v, vb = pool.tensors()
    qd, od, ld = q.double().cpu().numpy(), out.double().cpu().numpy(), lse.double().cpu().numpy()
    for r, (n, m) in enumerate(zip(lens, new)):
        pick = list(range(m)) if rows is None or m <= rows else sorted(set([0, m - 1]) | set(pool.rng.integers(0, m, rows).tolist()))
        if pick:
            ids = np.maximum(0, table[r, :-(-n // pool.page)].cpu().numpy())
            for h in heads or range(pool.kv_heads):
                kh = R4.keys(k[ids, h], kb[ids, h]).reshape(-1, pool.dim)
                vh = R4.values(v[ids, h], vb[ids, h]).reshape(-1, pool.dim)
                vs = np.exp2(vb[ids, h].astype(np.float64) - 127).reshape(-1)
                for u in range(g):
                    head = h * g + u
                    want, wl, slack, off = R4.attend_head(qd[[at + i for i in pick], head], kh, vh, vs, [n - m + i for i in pick], n, scale, pool.causal, pool.window)
                    for x, i in enumerate(pick):
                        err = np.abs(od[at + i, head] - want[x])
                        allowed = slack[x] + half_step(want[x], pool.dtype) * 1.01
                        assert (err <= allowed).all(), (r, h, u, i, float((err / allowed).max()))
                        if wl[x] == -np.inf:
                            assert ld[at + i, head] == -np.inf
                        else:
                            assert abs(ld[at + i, head] - wl[x]) <= off[x], (r, h, u, i, ld[at + i, head], wl[x], off[x])
        at += m


# ---- the store ---------------------------------------------------------------------------------------------------------

def expected(pool, before, s, n, k, v, top):
    """The cache's tensors after tokens k, v (64 bits, [n][heads][dim]) went into the step's slots; and where a value's byte may be anything."""
    kc, kb, vc, vb = [t.copy() for t in before]
    ck, ek = R4.quantized(k, 32, top)
    cv, ev = R4.quantized(v, v.shape[-1], top)
    free = np.zeros(vc.shape, np.uint8)         # halves of bytes behind the last token of a piece that was written
    last = {}
    for i, slot in enumerate(s.slots.tolist()[:n]):
        p, o = divmod(slot, pool.page)
        kc[p, :, o] = ck[i, :, 0::2] | (ck[i, :, 1::2] << 4)
        kb[p, :, o // 16, o % 4, :, o % 16 // 4] = ek[i] + 127
        vb[p, :, o] = ev[i][:, 0] + 127
        sh = 4 * (o % 2)
        b = vc[p, :, o // 16, :, o % 16 // 2]
        vc[p, :, o // 16, :, o % 16 // 2] = (b & ~np.uint8(15 << sh)) | (cv[i].astype(np.uint8) << sh)
        last[p, o // 16] = max(last.get((p, o // 16), -1), o % 16)
    for (p, sub), o in last.items():
        for t in range(o + 1, 16):
            free[p, :, sub, :, t // 2] |= 15 << (4 * (t % 2))
    return [kc, kb, vc, vb], free


CASES = [
    dict(dim=64, page=16, dtype=torch.float16),
    dict(dim=64, page=128, dtype=torch.bfloat16, eps=1e-5, gain=True, rot=64, interleaved=True),
    dict(dim=128, page=16, dtype=torch.float16, rot=128),
    dict(dim=128, page=32, dtype=torch.bfloat16, eps=1e-6, rot=64, strided=True),
    dict(dim=128, page=64, dtype=torch.float16, eps=1e-6, gain=True, rot=128, interleaved=True, odd=True),
    dict(dim=128, page=128, dtype=torch.bfloat16, rot=48, odd=True, q_heads=10, kv_heads=5),
    dict(dim=256, page=16, dtype=torch.float16, rot=16, eps=1e-3),
    dict(dim=256, page=64, dtype=torch.bfloat16, rot=256, gain=True, eps=1e-6),
    dict(dim=256, page=128, dtype=torch.bfloat16, rot=128, interleaved=True, q_heads=6, kv_heads=3),
    dict(dim=64, page=64, dtype=torch.float16, rot=64, q_heads=1, kv_heads=1, in_place=True),
    dict(dim=64, page=32, dtype=torch.float16, rot=32, eps=1e-6, gain=True, q_heads=37, kv_heads=37),
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
def test_store(case):
    """Several steps of ragged requests: every byte of the cache is what the definition makes of the new tokens, or what it was."""
    case = dict(case)
    eps, gain, rot, inter = case.pop("eps", 0.0), case.pop("gain", False), case.pop("rot", 0), case.pop("interleaved", False)
    strided, odd, in_place = case.pop("strided", False), case.pop("odd", False), case.pop("in_place", False)
    p = Pool(5, 4 if case["page"] == 128 else 24, seed=case["dim"] + case["page"], **case)
    g = torch.Generator().manual_seed(3)
    gq, gk = ((1 + 0.3 * torch.randn(2, p.dim, generator=g)).to(p.dtype).to(DEV)) if gain else (None, None)
    freq = (10000.0 ** (-torch.arange(0, rot, 2) / rot)).float().to(DEV) if rot else None
    np_ = lambda t: t.float().cpu().numpy()  # noqa: E731
    for i, new in enumerate(([1, 0, 17, 130, 16], [1, 3, 1, 0, 1], [15, 1, 1, 1, 16], [1, 1, 1, 1, 1], [0, 40, 0, 33, 2])):
        s = p.step(new, spare=2)
        q, k, v = layer_inputs(p, sum(new) + 2, strided, odd, spread=0.5 * i)
        q_in, before, n = q.float().cpu().numpy(), p.tensors(), sum(new)
        out = paged.write(p.cache, s, q, k, v, gq, gk, eps, freq, inter, q_out=q if in_place else None)
        pos = s.positions.tolist()[:n]
        f = np_(freq) if rot else None
        want_q = R.turned(q_in[:n], pos, np_(gq) if gain else None, eps, f, inter)
        want_k = R.turned(np_(k)[:n], pos, np_(gk) if gain else None, eps, f, inter)
        size = np.sqrt((want_q ** 2).max(-1, keepdims=True) * 2)
        assert (np.abs(np_(out)[:n] - want_q) <= half_step(want_q, p.dtype) * 1.01 + 2.0 ** -20 * size).all()
        if in_place:
            assert (np_(out)[n:] == q_in[n:]).all()
        want, free = expected(p, before, s, n, want_k, np_(v)[:n].astype(np.float64), 65504.0 if p.dtype == torch.float16 else 2.0 ** 47)
        got = p.tensors()
        for name, a, b in zip(("k", "k scales", "v", "v scales"), got, want):
            keep = ~free if name == "v" else np.uint8(255)
            assert ((a & keep) == (b & keep)).all(), (i, name, int(((a & keep) != (b & keep)).sum()))
        # and read back, with entries that name no token
        slots = s.slots.tolist()[:n] + [-1, p.n_pages * p.page, 2 ** 31 - 1, -2 ** 31]
        ko, vo = paged.gather(p.cache, i32(slots), p.dtype)
        for o, x in ((ko, R4.keys(want[0], want[1])), (vo, R4.values(want[2], want[3]))):
            o = o.double().cpu().numpy()
            assert (o[n:] == 0).all()
            for j, slot in enumerate(slots[:n]):
                assert (o[j] == x[slot // p.page, :, slot % p.page]).all(), (i, j)
        s.advance()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("values", [False, True])
def test_store_rounds_to_the_nearest_code(dtype, values):
    """Every number of the type up to 6 in size, beside a largest of 6: borders, ties and numbers that vanish."""
    n = 17
    p = Pool(1, 8, dim=64, page=128, q_heads=64, kv_heads=64, dtype=dtype)
    all_of_it = torch.arange(0, 65536, dtype=torch.int32).to(torch.int16).view(dtype)
    all_of_it = torch.where(all_of_it.abs() <= 6, all_of_it, torch.zeros((), dtype=dtype))
    x = torch.zeros(n * 64, 64, dtype=dtype)
    at = torch.tensor([d for d in range(64) if d % 32])
    flat = torch.zeros(n * 64 * 62, dtype=dtype)
    flat[:65536] = all_of_it[torch.from_numpy(np.random.default_rng(0).permutation(65536))]
    x[:, at] = flat.view(n * 64, 62)
    x[:, 0] = x[:, 32] = 6
    x = x.view(n, 64, 64).to(DEV)
    s = p.step([n])
    q = torch.zeros(n, 64, 64, dtype=dtype, device=DEV)
    paged.write(p.cache, s, q, x if not values else torch.zeros_like(x), x if values else torch.zeros_like(x))
    got = paged.gather(p.cache, s.slots, dtype)[values].double().cpu().numpy()
    want = R4.value_of(R4.nearest(x.double().cpu().numpy()))
    assert (got == want).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_store_of_what_is_no_number_and_what_is_nothing(dtype):
    """Infinities are the largest number that is stored, NaN is 0, zeros are zeros, all sizes have a scale."""
    p = Pool(1, 4, dim=64, page=32, q_heads=3, kv_heads=3, dtype=dtype)
    top = 65504.0 if dtype == torch.float16 else 2.0 ** 47
    x = p.rows(100, 3).float().cpu()
    x[0], x[1, 0, 5], x[1, 1, 6], x[1, 2, 40] = 0, math.inf, -math.inf, math.nan
    x[2, 0], x[2, 1] = math.nan, torch.finfo(dtype).max
    x[3, 0], x[3, 1, :32] = torch.finfo(dtype).tiny, 0
    for i in range(4, 100):
        x[i] *= 2.0 ** (i // 2 - 14 if dtype == torch.float16 and i < 60 else -60 + 1.3 * i if dtype == torch.bfloat16 else 0)
    x = x.to(dtype).to(DEV)
    s = p.step([100])
    before = p.tensors()
    paged.write(p.cache, s, torch.zeros(100, 3, 64, dtype=dtype, device=DEV), x, x)
    d = x.double().cpu().numpy()
    want, free = expected(p, before, s, 100, d, d, top)
    for a, b, keep in zip(p.tensors(), want, (255, 255, ~free, 255)):
        assert ((a & np.uint8(keep)) == (b & np.uint8(keep))).all()
    # fp16's largest number is stored as 4 times 2^14, which as fp16 is infinite: what is read back is the code's value, rounded to the type
    for got, x in zip(paged.gather(p.cache, s.slots, dtype), (R4.keys(*want[:2]), R4.values(*want[2:]))):
        for i, slot in enumerate(s.slots.tolist()):
            assert (got[i].cpu() == torch.from_numpy(x[slot // 32, :, slot % 32]).to(dtype)).all()
        assert (got[0] == 0).all() and not got.isnan().any()


def test_keys_far_out_are_turned_as_exactly_as_near_ones():
    """Positions of a million and more, with frequencies of any size: the same codes as from 64 bits."""
    page, width = 128, 131000
    table = torch.zeros(1, width, dtype=torch.int32, device=DEV)
    c = paged.Cache.empty(4, 2, 128, page, FOUR, DEV)
    rng = np.random.default_rng(0)
    freq = torch.from_numpy(np.concatenate([10000.0 ** (-np.arange(0, 120, 2) / 128), [3.7, 100.0, 1e-9, 0.0]]).astype(np.float32)).to(DEV)
    for at in (0, 128 * 1000, 128 * 8191, 128 * 130990):
        s = paged.Step(1, 100, 100, width, 4, page, 2, 2, 128)
        s.plan(i32([at]), i32([100]), table, i32([2]), i32([1]))
        k = torch.from_numpy(rng.standard_normal((100, 2, 128))).half().to(DEV)
        paged.write(c, s, k, k, k, inv_freq=freq)
        want = R.turned(k.float().cpu().numpy(), list(range(at, at + 100)), None, 0.0, freq.cpu().numpy(), False)
        codes, e = R4.quantized(want, 32, 65504.0)
        got = R4.key_codes(host(c.k)[2])[:, :100].swapaxes(0, 1)
        assert (got == codes).all() and (R4.key_exponents(host(c.k_scale)[2])[:, :100].swapaxes(0, 1) == e).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 15, 16, 17, 700])
def test_read(dim, dtype, n):
    """Any tokens in any order, some twice, some that do not exist."""
    p = Pool(3, 12, dim=dim, page=32, kv_heads=3, q_heads=3, dtype=dtype, seed=n)
    fill(p, [300, 17, 333], k_exp=(-14, 13), v_exp=(-14, 13))
    k, kb, v, vb = p.tensors()
    real = [int(p.table[r, t // 32]) * 32 + t % 32 for r, m in ((0, 300), (1, 17), (2, 333)) for t in range(m)]
    slots = p.rng.choice(real, n)
    slots[p.rng.random(n) < 0.1] = -1
    ko, vo = paged.gather(p.cache, i32(slots.tolist()), dtype)
    for o, x in ((ko, R4.keys(k, kb)), (vo, R4.values(v, vb))):
        o = o.double().cpu().numpy()
        for j, slot in enumerate(slots):
            want = x[slot // 32, :, slot % 32] if slot >= 0 else np.zeros((3, dim))
            assert (o[j] == torch.from_numpy(want).to(dtype).double().numpy()).all()


# ---- attention -----------------------------------------------------------------------------------------------------------

ATTEND = [
    # requests' tokens (cached and new together), new ones
    dict(lens=[1], new=[1], dim=64),
    dict(lens=[17, 1, 31, 33], new=[1, 1, 1, 1], dim=128, page=16),
    dict(lens=[300, 64, 129], new=[1, 2, 3], dim=64, dtype=torch.bfloat16, page=32),
    dict(lens=[1000, 5, 257], new=[5, 5, 5], dim=128, q_heads=14, kv_heads=2, dtype=torch.bfloat16),
    dict(lens=[700, 90], new=[1, 1], dim=256, q_heads=8, kv_heads=1, page=128),
    dict(lens=[4000, 3], new=[1, 1], dim=128, page=16, q_heads=8, kv_heads=8),
    dict(lens=[20000], new=[1], dim=64, page=64, q_heads=2, kv_heads=1),
    dict(lens=[9000, 8999], new=[1, 2], dim=256, page=64, q_heads=2, kv_heads=1, dtype=torch.bfloat16),
    dict(lens=[40, 200, 333], new=[40, 200, 100], dim=128, page=16, q_heads=4, kv_heads=2),
    dict(lens=[129, 65], new=[129, 33], dim=64, page=64, q_heads=1, kv_heads=1, dtype=torch.bfloat16),
    dict(lens=[500, 1, 90], new=[257, 1, 0], dim=256, page=32, q_heads=2, kv_heads=1),
    dict(lens=[2600, 700], new=[300, 1], dim=128, page=128, q_heads=16, kv_heads=2, dtype=torch.bfloat16),
    dict(lens=[9000], new=[40], dim=64, page=16, q_heads=8, kv_heads=1),
    dict(lens=[9000, 4100], new=[70, 129], dim=128, page=64, q_heads=3, kv_heads=1),
    dict(lens=[90, 30], new=[3, 1], dim=64, q_heads=64, kv_heads=1, page=16),
    # windows
    dict(lens=[500, 40, 3], new=[1, 1, 1], dim=64, page=16, window=33),
    dict(lens=[2000, 100], new=[7, 2], dim=128, page=64, window=100, q_heads=8, kv_heads=2),
    dict(lens=[700, 260], new=[300, 260], dim=64, page=16, window=70, dtype=torch.bfloat16),
    dict(lens=[700, 260], new=[300, 1], dim=128, page=32, window=1),
    dict(lens=[700, 260], new=[300, 1], dim=256, page=32, window=64),
    # every token sees all
    dict(lens=[130, 33, 1], new=[50, 3, 1], dim=64, page=16, causal=False),
    dict(lens=[300, 90], new=[200, 90], dim=128, page=64, causal=False, window=50),
    # scales from one end to the other
    dict(lens=[900, 60], new=[1, 1], dim=128, page=16, k_exp=(-8, 2), v_exp=(-45, 12), dtype=torch.bfloat16),
    dict(lens=[900, 60], new=[90, 1], dim=64, page=16, k_exp=(-8, 2), v_exp=(-45, 45), dtype=torch.bfloat16),
    dict(lens=[300, 600], new=[1, 200], dim=128, page=32, k_exp=(-8, 2), v_exp=(-45, 45), dtype=torch.bfloat16),
    dict(lens=[300, 600], new=[1, 20], dim=256, page=32, k_exp=(-8, 2), v_exp=(-45, 45), dtype=torch.bfloat16),
    dict(lens=[300, 600], new=[1, 20], dim=128, page=32, k_exp=(-45, -1), v_exp=(-2, 2)),
    # so many heads that a block has more steps than it knows the places of at a time
    dict(lens=[30000, 40], new=[1, 1], dim=64, page=64, kv_heads=128, q_heads=128, heads=[0, 77, 127]),
    dict(lens=[30000, 40], new=[20, 17], dim=64, page=64, kv_heads=128, q_heads=128, heads=[5, 127]),
    dict(lens=[30000, 200], new=[70, 100], dim=64, page=64, kv_heads=128, q_heads=128, heads=[0, 126], dtype=torch.bfloat16),
    # many requests whose ends lie in the middle of blocks, some with nothing to do
    dict(lens=[37 * i % 701 + 1 for i in range(150)], new=[(i * 7) % 4 and 1 for i in range(150)], dim=64, page=16, q_heads=4, kv_heads=4, heads=[2]),
    dict(lens=[137 * i % 1701 + 9 for i in range(60)], new=[(i * 5) % 9 for i in range(60)], dim=128, page=32, q_heads=8, kv_heads=2, heads=[1]),
    dict(lens=[1037 * i % 9001 + 60 for i in range(20)], new=[1 if i % 3 else 50 for i in range(20)], dim=64, page=128, q_heads=4, kv_heads=2, heads=[0]),
    dict(lens=[1037 * i % 9001 + 60 for i in range(20)], new=[1] * 20, dim=256, page=128, q_heads=4, kv_heads=2, heads=[1]),
]


def fenced(nbytes):
    """(a buffer, the bytes behind it, which nothing may touch)"""
    whole = torch.full((nbytes + 8192,), 0x5A, dtype=torch.uint8, device=DEV)
    return whole[:nbytes], whole[nbytes:]


@pytest.mark.parametrize("case", ATTEND, ids=lambda c: "-".join(str(v).replace("torch.", "").replace(" ", "")[:40] for v in c.values()))
def test_attend(case):
    case = dict(case)
    lens, new, heads = case.pop("lens"), case.pop("new"), case.pop("heads", None)
    exps = {k: case.pop(k) for k in ("k_exp", "v_exp") if k in case}
    page = case.setdefault("page", 64)
    p = Pool(len(lens), -(-max(lens) // page) + 1, seed=sum(lens), **case)
    fill(p, lens, **exps)
    s = planned(p, lens, new, spare=1)
    q = p.rows(sum(new) + 1, p.q_heads, spread=0.5)
    scale = 1 / math.sqrt(p.dim)
    out = torch.full_like(q, 7.0)
    s.scratch, fence = fenced(max(16, s.scratch_bytes))
    out, lse = paged.attend(p.cache, s, q, scale, out=out, with_lse=True)
    assert (out[-1] == 7).all() and (fence == 0x5A).all()       # the last row is no request's
    check_attend(p, q, out, lse, lens, new, scale, rows=6, heads=heads)
    again, lse2 = paged.attend(p.cache, s, q, scale, with_lse=True)
    assert torch.equal(again[:-1], out[:-1]) and torch.equal(lse2[:-1], lse[:-1])


# (tokens in all, new ones) of three requests, of which the middle one is turned down; two query heads a kv head
FORMS = [([90, 1, 41], [1, 1, 1]), ([90, 5, 41], [5, 5, 3]), ([90, 20, 41], [20, 17, 10]), ([200, 20, 141], [25, 32, 31]), ([200, 70, 141], [70, 40, 33]),
         ([9000, 5, 300], [5, 5, 1]), ([9000, 20, 300], [20, 17, 1]), ([9000, 70, 300], [70, 70, 40])]


@pytest.mark.parametrize("lens,new", FORMS)
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_rows_keep_to_themselves(lens, new, dtype, dim):
    """A query of NaN or infinity spoils its own row alone, one of large numbers gets what 64 bits make of it, a request that is turned down gets zeros."""
    p = Pool(3, -(-max(lens) // 16) + 1, page=16, q_heads=4, kv_heads=2, dim=dim, dtype=dtype, seed=sum(lens))
    fill(p, [lens[0], 0, lens[2]], k_exp=(-2, -2), v_exp=(-1, 1))
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
        assert out[t, h].isnan().all() and lse[t, h].isnan() and good[t, h].isfinite().all()
        out[t, h], lse[t, h] = good[t, h], good_lse[t, h]
    down = slice(new[0], new[0] + new[1])
    assert (out[down] == 0).all() and (lse[down] == -math.inf).all()
    mine = [i for i in range(sum(new)) if not new[0] <= i < new[0] + new[1]]
    for o, l in ((good, good_lse), (out, lse)):
        check_attend(p, q[mine], o[mine], l[mine], [lens[0], lens[2]], [new[0], new[2]], 1 / math.sqrt(dim), rows=8, table=p.table[[0, 2]])


@pytest.mark.parametrize("lens,new", [([300, 41], [1, 1]), ([300, 41], [20, 5]), ([300, 100], [70, 40]), ([9000, 7], [1, 1]), ([9000, 90], [70, 40])])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("size", [-120, -40, 40, 100, 120])
def test_queries_of_any_size(lens, new, dim, size):
    """bf16 queries from the smallest numbers to the largest, whose blocks of 32 dims are far apart in size too; scores are a few."""
    p = Pool(2, -(-max(lens) // 16) + 1, page=16, q_heads=4, kv_heads=2, dim=dim, dtype=torch.bfloat16, seed=max(lens))
    fill(p, lens, k_exp=(-1, 1), v_exp=(-1, 1))
    s = planned(p, lens, new)
    q = p.rows(sum(new), 4, spread=0.0).float()
    blocks = torch.ldexp(torch.ones(dim // 32), -3 * torch.arange(dim // 32)).repeat_interleave(32).to(DEV)
    q = torch.ldexp(q * blocks, torch.tensor(size, device=DEV)).to(torch.bfloat16)
    scale = 2.0 ** -size / 16 if size <= 100 else 2.0 ** -124
    out, lse = paged.attend(p.cache, s, q, scale, with_lse=True)
    check_attend(p, q, out, lse, lens, new, scale, rows=6)


def test_numbers_of_a_query_that_are_far_apart():
    """Beside one number of 2^15 others of a 32-dim block are taken to 2^-20 of 2^16; the other blocks' are not touched by it."""
    p = Pool(1, 8, dim=128, page=16, q_heads=1, kv_heads=1, seed=4)
    fill(p, [100], k_exp=(0, 0), v_exp=(0, 0))
    s = planned(p, [100], [1])
    q = p.rows(1, 1, spread=0.0)
    k, kb, v, vb = p.tensors()
    q[0, 0, 3] = 32768.0
    ids = p.table[0, :7].cpu().numpy()
    k[ids, 0, :, 1] &= 0x0F                         # dim 3 of every key is 0: the large number has no part in the scores
    p.cache.k.view(torch.uint8).copy_(torch.from_numpy(k))
    out, lse = paged.attend(p.cache, s, q, 0.1, with_lse=True)
    check_attend(p, q, out, lse, [100], [1], 0.1)
    assert abs(float(lse) - math.log(100)) < 10


# ---- neighbours, tables, streams and graphs -------------------------------------------------------------------------------

def test_what_a_table_does_not_name_is_masked():
    """Entries of -1 and beyond the cache inside a request count as tokens that nobody sees."""
    p = Pool(2, 24, dim=64, page=16, q_heads=4, kv_heads=2, seed=9)
    for new in ([1, 1], [20, 3], [70, 40]):
        lens = [333, 200]
        fill(p, lens)
        s = planned(p, lens, new)
        table = p.table.clone()
        for r, b, x in ((0, 2, -1), (0, 7, 2 ** 31 - 1), (1, 0, p.n_pages), (1, 5, -2 ** 31)):
            p.table[r, b] = x
        q = p.rows(sum(new), 4)
        out, lse = paged.attend(p.cache, s, q, with_lse=True)
        vb = host(p.cache.v_scale).copy()
        k, kb, v, _ = p.tensors()
        at = 0
        for r, (n, m) in enumerate(zip(lens, new)):
            seen = np.array([0 <= int(p.table[r, t // 16]) < p.n_pages for t in range(n)])
            ids = table[r, :-(-n // 16)].cpu().numpy()
            for i in (0, m - 1):
                live = np.nonzero(seen[:n - m + i + 1])[0]
                for h in range(2):
                    kh, vh = R4.keys(k[ids, h], kb[ids, h]).reshape(-1, 64)[live], R4.values(v[ids, h], vb[ids, h]).reshape(-1, 64)[live]
                    vs = np.exp2(vb[ids, h].astype(np.float64) - 127).reshape(-1)[live]
                    want, wl, slack, off = R4.attend_head(q[at + i, 2 * h].double().cpu().numpy()[None], kh, vh, vs, [len(live)], len(live), 0.125, True, 0)
                    assert (np.abs(out[at + i, 2 * h].double().cpu().numpy() - want[0]) <= slack[0] + half_step(want[0], p.dtype) * 1.01).all()
                    assert abs(float(lse[at + i, 2 * h]) - wl[0]) <= off[0]
            at += m


def test_strided_rows_give_the_same():
    p = Pool(2, 12, dim=64, page=16, q_heads=6, kv_heads=2, dtype=torch.bfloat16, seed=3)
    for new in ([1, 1], [5, 8], [50, 1]):
        fill(p, [150, 71])
        s = planned(p, [150, 71], new)
        n = sum(new)
        q = p.rows(n, 6)
        want, _ = paged.attend(p.cache, s, q, with_lse=True)
        store = torch.zeros(n * 400 + 1, dtype=torch.bfloat16, device=DEV)
        odd = store[1:].as_strided((n, 6, 64), (397, 64, 1))
        odd.copy_(q)
        store2 = torch.full((n * 400 + 1,), 3.0, dtype=torch.bfloat16, device=DEV)
        out = store2[1:].as_strided((n, 6, 64), (391, 64, 1))
        paged.attend(p.cache, s, odd, out=out)
        assert torch.equal(out, want)
        out.fill_(3.0)
        assert (store2 == 3).all()                  # nothing beside the rows


def test_far_pages_of_a_large_cache():
    """Codes beyond 4 GiB of keys, and a table whose rows are far apart."""
    page, heads, dim = 128, 16, 256
    n_pages = (1 << 32) // (page * heads * dim // 2) + 40
    c = paged.Cache.empty(n_pages, heads, dim, page, FOUR, DEV)
    width = 40000
    table = torch.zeros(3, width, dtype=torch.int32, device=DEV)
    table[2, :3] = i32([n_pages - 1, 5, n_pages - 2])
    s = paged.Step(3, 300, 300, width, n_pages, page, heads, heads, dim)
    s.plan(i32([0, 0, 0]), i32([0, 0, 300]), table, i32([n_pages - 2, 5, n_pages - 1]), i32([3]))
    g = torch.Generator(device=DEV).manual_seed(1)
    q, k, v = (torch.randn(300, heads, dim, device=DEV, generator=g).half() for _ in range(3))
    paged.write(c, s, q, k, v)
    ko, vo = paged.gather(c, s.slots)
    for got, x, w in ((ko, k, 32), (vo, v, dim)):
        codes, e = R4.quantized(x.double().cpu().numpy(), w, 65504.0)
        assert (got.double().cpu().numpy() == R4.value_of(codes) * np.repeat(np.exp2(e.astype(float)), w, -1)).all()
    for rows in (300, 1):
        if rows == 1:
            s = paged.Step(3, 1, 1, width, n_pages, page, heads, heads, dim)
            s.plan(i32([0, 0, 299]), i32([0, 0, 1]), table, i32([0]), i32([1]))
        out = paged.attend(c, s, q[300 - rows:])
        qd, kd, vd = (x[:, 15].double().cpu() for x in (q[300 - rows:], ko, vo))
        z = (qd @ kd.T / math.sqrt(dim)).masked_fill(torch.ones(300, 300).triu(1).bool()[300 - rows:], -math.inf)
        want = torch.softmax(z, -1) @ vd
        assert (out[:, 15].double().cpu() - want).abs().max() <= 2.0 ** -10 * vd.abs().max()


def test_a_captured_step_serves_other_lengths():
    """One graph of plan, store, attention and the bookkeeping after it, replayed as requests grow, against the same calls one by one."""
    def make():
        p = Pool(3, 40, page=16, q_heads=4, kv_heads=2, seed=5)
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
    want, read = paged.attend(p.cache, s, want_q), paged.gather(p.cache, s.slots)
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
        out, again = paged.attend(p.cache, s, q), paged.gather(p.cache, s.slots)
    side.synchronize()
    assert torch.equal(q, want_q) and torch.equal(out, want) and all(torch.equal(u, w) for u, w in zip(read, again))


def test_tokens_do_not_depend_on_their_step():
    """The cache after a prompt in one step is that after the same tokens one by one or in pieces."""
    freq = (10000.0 ** (-torch.arange(0, 128, 2) / 128)).float().to(DEV)
    caches = []
    x = None
    for pieces in ([90], [1] * 90, [7, 40, 1, 13, 29]):
        p = Pool(1, 4, page=32, dim=128, seed=1)
        for t in (p.cache.k, p.cache.v, p.cache.k_scale, p.cache.v_scale):
            t.view(torch.uint8).zero_()
        x = p.rows(90, 8) if x is None else x
        at = 0
        for n in pieces:
            s = p.step([n])
            paged.write(p.cache, s, x[at:at + n, :4], x[at:at + n, 4:6], x[at:at + n, 6:], inv_freq=freq, eps=1e-6)
            s.advance()
            at += n
        caches.append(p.tensors())
    for other in caches[1:]:
        assert all((a == b).all() for a, b in zip(caches[0], other))
