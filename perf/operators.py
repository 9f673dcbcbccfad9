"""Workloads of the attention half of a decode step that are timed: the pages of a step's tokens, the queries' and keys'
norm and rotation with the store into an 8-bit paged cache, and attention over that cache.

A case is a ragged batch of requests, each with tokens already cached and new ones. `run` computes it in plain torch
where `own` is false and with the framework's kernels where it is true; `exact` is the same in 64 bits.

The cache: k [pages][kv heads][page/16][D/16][16 tokens][16 dims], v [pages][kv heads][page/16][D][16 tokens], 8-bit codes,
and one fp32 scale per page and kv head for each of the two.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

EPS = 1e-6
THETA = 1e6
DEV = "cuda:0"


# ------------------------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------------------------

def _case(name, kind, requests, new, ctx, *, q_heads=32, kv_heads=8, head_dim=128, page=64, fmt="e4m3", dtype="float16", window=0,
          norm=False, interleaved=False, rot=0, spare=0, lengths=1):
    """new, ctx: (fewest, most) new and cached tokens of a request; spare: rows of the batch that belong to no request;
    rot: rotated dims of a head (0: all); lengths: which draw of the ragged lengths."""
    c = dict(kind=kind, requests=requests, new_lo=new[0], new_hi=new[1], ctx_lo=ctx[0], ctx_hi=ctx[1], q_heads=q_heads,
             kv_heads=kv_heads, head_dim=head_dim, page=page, fmt=fmt, dtype=dtype, window=window, norm=norm,
             interleaved=interleaved, rot=rot or head_dim, spare=spare, lengths=lengths)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the pages of a step of eight users' chats, one token each
        _case("plan_tokens8", "plan", 8, (1, 1), (1, 2000)),
        # a full server: two thousand requests, most with a token or a few drafts, some with a part of their prompt
        _case("plan_mixed2048", "plan", 2048, (1, 200), (0, 4000), page=16, spare=37),
        # one token of one chat with the head layout of the 4096-wide decode workloads: what a call costs
        _case("write_token", "write", 1, (1, 1), (700, 700)),
        # 256 chats decoded together; norms of queries and keys, neighbouring dims rotated, 8-bit integers
        _case("write_batch256", "write", 256, (1, 1), (1, 4000), page=16, fmt="int8", dtype="bfloat16", norm=True, interleaved=True),
        # three prompts of odd lengths, 8 thousand tokens in all
        _case("write_prompts", "write", 3, (1500, 3600), (0, 0), lengths=5),
        # one token of one short chat
        _case("attend_token", "attend", 1, (1, 1), (700, 700)),
        # 64 chats of very different lengths, a token each
        _case("attend_batch64", "attend", 64, (1, 1), (500, 8000)),
        # one token over a whole book
        _case("attend_long", "attend", 1, (1, 1), (131000, 131000), lengths=2),
        # five drafted tokens each to be verified; narrow heads, sliding window, small pages
        _case("attend_drafts24", "attend", 24, (5, 5), (100, 5000), q_heads=32, kv_heads=4, head_dim=64, page=16, fmt="int8",
              dtype="bfloat16", window=1024),
        # a prompt
        _case("attend_prompt4096", "attend", 1, (4096, 4096), (0, 0)),
        # parts of prompts onto what is cached, together with single tokens, at odd lengths
        _case("attend_chunks", "attend", 12, (1, 700), (0, 6000), fmt="int8", dtype="bfloat16", page=32, spare=3, lengths=3),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(max(hi, 1))))))))


def draw(rng):
    kind = rng.choice(["plan", "write", "write", "attend", "attend", "attend"])
    head_dim = rng.choice([64, 128, 128, 128, 256])
    group = rng.choice([1, 2, 4, 4, 7, 8, 16])
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    while group * kv_heads > 64:
        kv_heads //= 2
    more = dict(q_heads=group * kv_heads, kv_heads=kv_heads, head_dim=head_dim, page=rng.choice([16, 32, 64, 64, 128]),
                fmt=rng.choice(["e4m3", "int8"]), dtype=rng.choice(["float16", "bfloat16"]), norm=rng.random() < 0.5,
                interleaved=rng.random() < 0.5, rot=rng.choice([head_dim, head_dim, head_dim // 2]),
                spare=rng.choice([0, 0, 5]), lengths=rng.randrange(1000), window=rng.choice([0, 0, 0, 100, 1000]))
    if kind == "plan":
        return _case(None, kind, _log_int(rng, 1, 2048), (0, _log_int(rng, 1, 200)), (0, _log_int(rng, 1, 4000)), **more)
    if kind == "write":
        new = _log_int(rng, 1, 1500)
        most = 6000 * 48 * 128 // ((group + 2) * kv_heads * head_dim)
        return _case(None, kind, _log_int(rng, 1, max(1, min(256, most // new))), (rng.choice([0, 1, new]), new), (0, _log_int(rng, 1, 4000)), **more)
    new = rng.choice([1, 1, _log_int(rng, 2, 16), _log_int(rng, 17, 1500)])
    ctx = _log_int(rng, 1, 30000 if new <= 16 else 6000)
    one = kv_heads * group * head_dim * new * (new + ctx)
    while one > 2 ** 35:
        new, ctx, one = new // 2, ctx // 2, one // 4
    keys = 2 ** 27 // (kv_heads * head_dim * (new + ctx))
    return _case(None, kind, _log_int(rng, 1, max(1, min(64, 2 ** 35 // one, keys))), (rng.choice([0, 1, new]), new), (0, ctx), **more)


def _lengths(case):
    """(cached, new) tokens of each request: a matter of the case, not of the seed, so that a pass costs the same."""
    rng = random.Random(1000003 * case["lengths"] + case["requests"])
    pick = lambda lo, hi: lo if lo == hi or (lo == 0 and rng.random() < 0.1) else _log_int(rng, lo, hi)  # noqa: E731
    pairs = [(pick(case["ctx_lo"], case["ctx_hi"]), pick(case["new_lo"], case["new_hi"])) for _ in range(case["requests"])]
    ctx, new = [c for c, _ in pairs], [n for _, n in pairs]
    new[0] = new[0] if sum(new) else max(1, case["new_hi"])
    return ctx, new


def _blocks(n, page):
    return -(-n // page)


def _visible(case):
    """(row, key) pairs of one query head, and the keys of one kv head that any row of a request sees."""
    pairs = keys = 0
    for c, n in zip(*_lengths(case)):
        w = case["window"] or c + n
        pos = np.arange(c, c + n, dtype=np.int64)
        pairs += int(np.minimum(pos + 1, w).sum())
        keys += (c + n) - max(0, c + 1 - w) if n else 0
    return pairs, keys


def work(case):
    ctx, new = _lengths(case)
    t, r, d, hq, hk, page = sum(new) + case["spare"], case["requests"], case["head_dim"], case["q_heads"], case["kv_heads"], case["page"]
    fresh = sum(_blocks(c + n, page) - _blocks(c, page) for c, n in zip(ctx, new))
    if case["kind"] == "plan":
        return {"bytes": 8.0 * r + 4.0 * fresh + 4.0 * (2 * t + 3 * r + 2) + 4.0 * fresh, "flops": 0.0}
    if case["kind"] == "write":
        t = sum(new)
        old = sum(c % page for c, n in zip(ctx, new) if n)
        return {"bytes": 2.0 * t * (2 * hq + 2 * hk) * d + 2.0 * t * hk * d + 2.0 * old * hk * d + 4.0 * (t + old) * hk * d, "flops": 0.0}
    pairs, keys = _visible(case)
    t = sum(new)
    return {"bytes": 2.0 * keys * hk * d + 2.0 * 2 * t * hq * d + 4.0 * t * hq + 8.0 * hk * sum(_blocks(c + n, page) for c, n in zip(ctx, new) if n),
            "flops": 4.0 * pairs * hq * d}


# ------------------------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------------------------

def _qmax(fmt):
    return 448.0 if fmt == "e4m3" else 127.0


def _code_type(fmt):
    return torch.float8_e4m3fn if fmt == "e4m3" else torch.int8


def _encode(x, fmt):
    """x / scale, fp32, as codes."""
    return x.to(torch.float8_e4m3fn) if fmt == "e4m3" else x.round().to(torch.int8)


def _pow2(amax, qmax):
    """The smallest power of two that keeps amax within qmax codes, 2^-96 at least."""
    m, e = torch.frexp(amax / qmax)
    e = torch.where(amax > 0, torch.where(m > 0.5, e, e - 1), -96).clamp(-96, 120)
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _k_tiles(x):
    p, h, n, d = x.shape
    return x.view(p, h, n // 16, 16, d // 16, 16).permute(0, 1, 2, 4, 3, 5).contiguous()


def _v_tiles(x):
    p, h, n, d = x.shape
    return x.view(p, h, n // 16, 16, d).transpose(3, 4).contiguous()


def _k_rows(x):
    p, h, n, m = x.shape[:4]
    return x.permute(0, 1, 2, 4, 3, 5).reshape(p, h, n * 16, m * 16)


def _v_rows(x):
    p, h, n, d = x.shape[:4]
    return x.transpose(3, 4).reshape(p, h, n * 16, d)


def _filled(case, pages, gen):
    """Codes and scales of a cache of `pages` pages that holds keys or values of every size that heads have."""
    hk, d, page, fmt = case["kv_heads"], case["head_dim"], case["page"], case["fmt"]
    k, s = [], []
    spread = torch.exp2(torch.randn(1, hk, 1, d, device=DEV, generator=gen))     # some dims of a head are larger than others
    for at in range(0, pages, 1024):
        n = min(1024, pages - at)
        x = torch.randn(n, hk, page, d, device=DEV, generator=gen) * spread
        sc = _pow2(x.abs().amax(dim=(2, 3)), _qmax(fmt))
        k.append(_encode(x / sc[:, :, None, None], fmt))
        s.append(sc)
    return torch.cat(k), torch.cat(s)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rng = random.Random(seed)
    ctx, new = _lengths(case)
    page, r = case["page"], case["requests"]
    t = sum(new) + case["spare"]
    held = [_blocks(c, page) for c in ctx]
    total = [_blocks(c + n, page) for c, n in zip(ctx, new)]
    in_use, fresh = sum(held), sum(total) - sum(held)
    pages = sum(total) + 7
    order = list(range(pages))
    rng.shuffle(order)
    width = max(total) + 1 + case["lengths"] % 3
    table = np.full((r, width), -1, np.int32)
    at = 0
    for i, n in enumerate(held):
        table[i, :n] = order[at:at + n]
        at += n
    free = order[:at - 1 if at else None:-1]        # a stack: its end is handed out first
    if case["kind"] == "attend":                    # the step's pages have been handed out
        for i, (h, n) in enumerate(zip(held, total)):
            table[i, h:n] = order[at:at + n - h]
            at += n - h
    room = len(free)
    if case["kind"] == "plan" and case["lengths"] % 3 == 0 and fresh > 1:     # a pool that cannot serve everybody
        room = rng.randrange(fresh // 2, fresh)
        free = free[:room] + [-1] * (len(free) - room)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    s = {"kind": case["kind"], "page": page, "pages": pages, "tokens": t, "rows": sum(new), "max_new": max(new), 
         "window": case["window"], "q_heads": case["q_heads"], "kv_heads": case["kv_heads"], "head_dim": case["head_dim"], "fmt": case["fmt"],
         "ctx": i32(ctx), "new": i32(new), "table": i32(table.tolist()), "free": i32(free), "room": i32([room])}
    if case["kind"] == "plan":
        if own:
            from paper_2312_17238_amd import paged
            s["step"] = paged.Step(r, t, max(new), width, pages, page, case["q_heads"], case["kv_heads"], case["head_dim"], window=case["window"])
        return s
    dt = getattr(torch, case["dtype"])
    hq, hk, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    k, ks = _filled(case, pages, gen)
    v, vs = _filled(case, pages, gen)
    k, v = _k_tiles(k.view(torch.uint8)), _v_tiles(v.view(torch.uint8))
    for i, (c, n) in enumerate(zip(ctx, new)):      # what an earlier tenant left behind the last token
        have = c if case["kind"] == "write" else c + n
        if have % page:
            p, o = int(table[i, have // page]), have % page
            v[p, :, o // 16, :, o % 16:] = 0x7F
            v[p, :, o // 16 + 1:] = 0x7F
    s |= {"k": k.view(_code_type(case["fmt"])), "v": v.view(_code_type(case["fmt"])), "ks": ks, "vs": vs, "dtype": dt}
    rows = torch.randn(t, hq + 2 * hk, d, device=DEV, generator=gen)
    if case["kind"] == "write":
        rows *= torch.exp2(torch.randn(hq + 2 * hk, 1, device=DEV, generator=gen))
        s["qkv"] = rows.to(dt)
        s["gq"] = (1 + 0.2 * torch.randn(d, device=DEV, generator=gen)).to(dt) if case["norm"] else None
        s["gk"] = (1 + 0.2 * torch.randn(d, device=DEV, generator=gen)).to(dt) if case["norm"] else None
        s["eps"] = EPS if case["norm"] else 0.0
        s["freq"] = (THETA ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64) / case["rot"])).float().to(DEV)
        s["interleaved"] = case["interleaved"]
        s["touched"], s["slots"] = _touched(ctx, new, table, free, room, page)
        s["positions"] = i32([c + i for c, n in zip(ctx, new) for i in range(n)])
    else:
        s["q"] = rows[:, :hq].to(dt)
        s["scale"] = 1.0 / math.sqrt(d)
    if own:
        from paper_2312_17238_amd import paged
        s["cache"] = paged.Cache(s["k"], s["v"], s["ks"], s["vs"])
        s["step"] = paged.Step(r, t, max(new), width, pages, page, hq, hk, d, window=case["window"])
        s["step"].plan(s["ctx"], s["new"], s["table"], s["free"], s["room"])
    return s


def _touched(ctx, new, table, free, room, page):
    """Slots of the tokens that the pages of a step's new tokens hold afterwards, old ones and new ones; the new ones' alone."""
    out, mine, top = [], [], room
    for i, (c, n) in enumerate(zip(ctx, new)):
        if not n:
            continue
        b0, b1 = c // page, _blocks(c + n, page)
        ids = []
        for b in range(b0, b1):
            if b < _blocks(c, page):
                ids.append(int(table[i, b]))
            else:
                top -= 1
                ids.append(int(free[top]))
        pos = np.arange(b0 * page, c + n)
        out.append(np.asarray(ids, np.int64)[pos // page - b0] * page + pos % page)
        mine.append(out[-1][c - b0 * page:])
    return tuple(torch.from_numpy(np.concatenate(v).astype(np.int32)).to(DEV) for v in (out, mine))


# ------------------------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------------------------

def run(state):
    return {"plan": _run_plan, "write": _run_write, "attend": _run_attend}[state["kind"]](state)


def _run_plan(s):
    if own:
        st = s["step"]
        st.plan(s["ctx"], s["new"], s["table"], s["free"], s["room"])
        return {"row_start": st.row_start, "positions": st.positions, "slots": st.slots, "kv_len": st.kv_len, "status": st.status,
                "left": st.free_left, "table": s["table"]}
    return _plain_plan(s)


def _plain_plan(s):
    ctx, new, table, page, t = s["ctx"].long(), s["new"].long(), s["table"], s["page"], s["tokens"]
    free, room = s["free"].long(), s["room"].long()
    width, n_pages = table.shape[1], s["pages"]
    end = torch.cumsum(new, 0)
    held, total = (ctx + page - 1) // page, (ctx + new + page - 1) // page
    status = torch.where(total > width, 2, 0)
    status = torch.where(end > t, 3, status)
    need = torch.where(status == 0, total - held, 0)
    cum = torch.cumsum(need, 0)
    short = (need > 0) & (cum > room)
    status = torch.where(short, 1, status)
    ok = status == 0
    used = torch.where(ok & (need > 0), cum, 0).amax()
    col = torch.arange(width, device=DEV)
    fill = ok[:, None] & (col >= held[:, None]) & (col < total[:, None])
    nth = (cum - need)[:, None] + col - held[:, None]
    table.copy_(torch.where(fill, free[(room - 1 - nth).clamp(0, free.numel() - 1)].int(), table))
    tok = torch.arange(t, device=DEV)
    req = torch.searchsorted(end, tok, right=True)
    mine = req < new.numel()
    req = req.clamp(max=new.numel() - 1)
    pos = tok - (end - new)[req] + ctx[req]
    mine = mine & ok[req]
    blk = table[req, torch.where(mine, pos // page, 0)].long()
    slot = torch.where(mine & (blk >= 0) & (blk < n_pages), blk * page + pos % page, -1)
    return {"row_start": torch.cat([end.new_zeros(1), end.clamp(max=t)]).int(), "positions": torch.where(mine, pos, -1).int(), "slots": slot.int(),
            "kv_len": torch.where(ok, ctx + new, ctx).int(), "status": status.int(), "left": (room - used).int(), "table": table}


def _run_write(s):
    hq, hk = s["q_heads"], s["kv_heads"]
    q, k, v = s["qkv"][:, :hq], s["qkv"][:, hq:hq + hk], s["qkv"][:, hq + hk:]
    if own:
        from paper_2312_17238_amd import paged
        qo = paged.write(s["cache"], s["step"], q, k, v, q_gamma=s["gq"], k_gamma=s["gk"], eps=s["eps"], inv_freq=s["freq"],
                         interleaved=s["interleaved"])
        ko, vo = paged.gather(s["cache"], s["touched"], s["dtype"])
    else:
        qo, ko, vo = _plain_write(s, q, k, v)
    return {"q": qo[:s["rows"]], "k": ko, "v": vo}      # the spare rows belong to no request: nothing is computed for them


def _rotate(x, pos, freq, interleaved):
    ang = pos.double()[:, None] * freq.double()
    cos, sin = ang.cos().to(x.dtype)[:, None], ang.sin().to(x.dtype)[:, None]
    n = freq.numel()
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if interleaved else (x[..., :n], x[..., n:2 * n])
    u, w = a * cos - b * sin, a * sin + b * cos
    head = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([head, x[..., 2 * n:]], -1)


def _plain_write(s, q, k, v):
    page, fmt, qmax = s["page"], s["fmt"], _qmax(s["fmt"])
    n = s["rows"]
    pos, slot = s["positions"], s["slots"].long()
    q, k, v = q[:n].float(), k[:n].float(), v[:n].float()
    if s["eps"]:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + s["eps"]) * s["gq"].float()
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + s["eps"]) * s["gk"].float()
    q, k = _rotate(q, pos, s["freq"], s["interleaved"]), _rotate(k, pos, s["freq"], s["interleaved"])
    # the pages that get tokens, and from which of their tokens on
    hit, idx = torch.unique(slot // page, return_inverse=True)
    first = torch.full((hit.numel(),), page, device=DEV).scatter_reduce(0, idx, slot % page, "amin")
    out = []
    for x, codes, scales, rows, tiles in ((k, s["k"], s["ks"], _k_rows, _k_tiles), (v, s["v"], s["vs"], _v_rows, _v_tiles)):
        amax = torch.zeros(hit.numel(), x.shape[1], device=DEV).index_reduce_(0, idx, x.abs().amax(-1), "amax")
        old = torch.where(first[:, None] > 0, scales[hit], 0.0)
        sc = torch.maximum(old, _pow2(amax, qmax))
        have = rows(codes.view(torch.uint8)[hit]).view(codes.dtype).float()         # [pages][heads][tokens][dims]
        keep = (torch.arange(page, device=DEV) < first[:, None])[:, None, :, None]
        have = torch.where(keep, have * (old / sc)[:, :, None, None], 0.0)
        have[idx, :, slot % page] = x / sc[idx][:, :, None]
        new = _encode(have, fmt)
        codes.view(torch.uint8)[hit] = tiles(new.view(torch.uint8))
        scales[hit] = sc
        want = s["touched"].long()
        at = torch.searchsorted(hit, want // page)
        out.append((new.float()[at, :, want % page] * sc[at][:, :, None]).to(s["dtype"]))
    return q.to(s["dtype"]), out[0], out[1]


def _run_attend(s):
    if own:
        from paper_2312_17238_amd import paged
        out, lse = paged.attend(s["cache"], s["step"], s["q"], s["scale"], with_lse=True)
    else:
        out, lse = _plain_attend(s)
    return {"out": out[:s["rows"]], "lse": lse[:s["rows"]]}


def _plain_attend(s):
    """All requests at once, padded to the longest."""
    page, hk, d = s["page"], s["kv_heads"], s["head_dim"]
    g = s["q_heads"] // hk
    ctx, new, table = s["ctx"].long(), s["new"].long(), s["table"].long()
    r, most, t = ctx.numel(), s["max_new"], s["q"].shape[0]
    nb = table.shape[1]
    kv = ctx + new
    start = torch.cumsum(new, 0) - new
    i = torch.arange(most, device=DEV)
    row = (start[:, None] + i).clamp(max=t - 1)                                     # [r][most]
    real = i < new[:, None]
    q = s["q"][row].float().view(r, most, hk, g, d).permute(0, 2, 3, 1, 4).reshape(r, hk, g * most, d)
    ids = table.clamp(min=0)
    k = _k_rows(s["k"].view(torch.uint8)[ids].view(r * nb, hk, page // 16, d // 16, 16, 16)).view(s["k"].dtype).float()
    k = (k.view(r, nb, hk, page, d) * s["ks"][ids][:, :, :, None, None]).permute(0, 2, 1, 3, 4).reshape(r, hk, nb * page, d)
    j = torch.arange(nb * page, device=DEV)
    pos = ctx[:, None] + i
    see = (j <= pos[..., None]) & real[..., None]                                   # [r][most][keys]
    if s["window"]:
        see &= j > pos[..., None] - s["window"]
    z = torch.matmul(q, k.transpose(2, 3).contiguous()).view(r, hk, g, most, nb * page) * s["scale"]
    del k
    z = z.masked_fill(~see[:, None, None], float("-inf"))
    top = z.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    z = torch.exp(z - top)
    tot = z.sum(-1, keepdim=True)
    v = _v_rows(s["v"].view(torch.uint8)[ids].view(r * nb, hk, page // 16, d, 16)).view(s["v"].dtype).float()
    v = (v.view(r, nb, hk, page, d) * s["vs"][ids][:, :, :, None, None]).permute(0, 2, 1, 3, 4).reshape(r, hk, nb * page, d)
    v = torch.where((j < kv[:, None])[:, None, :, None], v, 0.0)
    o = torch.matmul(z.view(r, hk, g * most, nb * page), v).view(r, hk, g, most, d)
    o = torch.where(tot > 0, o / tot, 0.0)
    lse = (torch.log(tot) + top)[..., 0]
    out = torch.zeros(t, hk, g, d, device=DEV)
    out_l = torch.zeros(t, hk, g, device=DEV)
    flat = row[real]
    out[flat] = o.permute(0, 3, 1, 2, 4)[real]
    out_l[flat] = lse.permute(0, 3, 1, 2)[real]
    return out.view(t, hk * g, d).to(s["dtype"]), out_l.view(t, hk * g)


# ------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ------------------------------------------------------------------------------------------------------------------

def _e4m3_values():
    v = []
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v.append(math.nan if c & 127 == 127 else -x if c & 128 else x)
    return torch.tensor(v, dtype=torch.float64, device=DEV)


def _value_of(codes, fmt):
    if fmt == "int8":
        return codes.view(torch.int8).double()
    return _e4m3_values()[codes.view(torch.uint8).long()]


def _two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _nearest(x, fmt):
    """The format's value nearest to x, ties to the even code."""
    if fmt == "int8":
        return torch.round(x)
    _, e = torch.frexp(x)
    step = _two_to((e - 1).clamp(min=-6) - 3)
    return torch.round(x / step) * step


def _tokens_of(s, c, v_not_k, ids, head):
    """One head's cached tokens of the pages `ids`, 64 bits [tokens][dims]."""
    if v_not_k:
        x = s["v"].view(torch.uint8)[ids, head]         # [pages][page/16][D][16]
        x = _value_of(x, c["fmt"]).transpose(2, 3).reshape(-1, c["head_dim"])
        sc = s["vs"][ids, head]
    else:
        x = s["k"].view(torch.uint8)[ids, head]         # [pages][page/16][D/16][16][16]
        x = _value_of(x, c["fmt"]).permute(0, 1, 3, 2, 4).reshape(-1, c["head_dim"])
        sc = s["ks"][ids, head]
    return x * sc.double().repeat_interleave(c["page"])[:, None]


def _exact_plan(case, s):
    page, width, t = case["page"], s["table"].shape[1], s["tokens"]
    table, free, room = s["table"].cpu().numpy().copy(), s["free"].tolist(), int(s["room"][0])
    ctx, new = _lengths(case)
    start, pos, slot, kv, status, asked, used = [0], [-1] * t, [-1] * t, [], [], 0, 0
    for r, (c, n) in enumerate(zip(ctx, new)):
        first = start[-1]
        start.append(min(t, first + n))
        held, total = _blocks(c, page), _blocks(c + n, page)
        st = 3 if first + n > t else 2 if total > width else 0
        if not st and total > held:
            asked += total - held
            if asked > room:
                st = 1
            else:
                for b in range(held, total):
                    table[r, b] = free[room - 1 - used]
                    used += 1
        status.append(st)
        kv.append(c if st else c + n)
        for i in range(0 if st else n):
            p = c + i
            pos[first + i], slot[first + i] = p, int(table[r, p // page]) * page + p % page
    arr = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return {"row_start": arr(start), "positions": arr(pos), "slots": arr(slot), "kv_len": arr(kv), "status": arr(status),
            "left": arr([room - used]), "table": torch.from_numpy(table)}


def _exact_write(case, s):
    hq, hk, d, page, fmt = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"], case["fmt"]
    ctx, new = _lengths(case)
    pos = torch.tensor([c + i for c, n in zip(ctx, new) for i in range(n)], dtype=torch.float64, device=DEV)
    x = s["qkv"][:pos.numel()].double()
    f = s["freq"].double()
    z = torch.polar(torch.ones(pos.numel(), f.numel(), dtype=torch.float64, device=DEV), pos[:, None] * f)

    def turned(y, gamma):
        if s["eps"]:
            y = y / torch.sqrt(y.pow(2).sum(-1, keepdim=True) / d + s["eps"]) * gamma.double()
        n = f.numel()
        at = torch.arange(n, device=DEV)
        i, j = (2 * at, 2 * at + 1) if case["interleaved"] else (at, at + n)
        w = torch.complex(y[..., i], y[..., j]) * z[:, None]
        y = y.clone()
        y[..., i], y[..., j] = w.real, w.imag
        return y

    q, k, v = turned(x[:, :hq], s["gq"]), turned(x[:, hq:hq + hk], s["gk"]), x[:, hq + hk:]
    table, free, top = s["table"].cpu().numpy(), s["free"].tolist(), int(s["room"][0])
    outs, t0 = [[], []], 0
    for r, (c, n) in enumerate(zip(ctx, new)):
        for b in range(c // page, _blocks(c + n, page) if n else 0):
            if b < _blocks(c, page):
                pid = int(table[r, b])
            else:
                top -= 1
                pid = free[top]
            lo, hi = max(c, b * page), min(c + n, (b + 1) * page)
            had = lo - b * page
            ids = torch.tensor([pid], device=DEV)
            for which, src in ((0, k), (1, v)):
                y = src[t0 + lo - c:t0 + hi - c]
                m, e = torch.frexp(y.abs().amax(dim=(0, 2)) / _qmax(fmt))
                sc = _two_to(torch.where(m > 0.5, e, e - 1))
                if had:
                    sc = torch.maximum(sc, (s["vs"] if which else s["ks"])[pid].double())
                    old = torch.stack([_tokens_of(s, case, bool(which), ids, h)[:had] for h in range(hk)], 1)
                    y = torch.cat([old, y])
                outs[which].append(_nearest(y / sc[:, None], fmt) * sc[:, None])
        t0 += n
    return {"q": q, "k": torch.cat(outs[0]), "v": torch.cat(outs[1])}


def _exact_attend(case, s):
    hq, hk, d, page = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    ctx, new = _lengths(case)
    n_rows = sum(new)
    out = torch.zeros(n_rows, hq, d, dtype=torch.float64, device=DEV)
    lse = torch.zeros(n_rows, hq, dtype=torch.float64, device=DEV)
    t0 = 0
    for r, (c, n) in enumerate(zip(ctx, new)):
        if n:
            ids = s["table"][r, :_blocks(c + n, page)].long()
            p = torch.arange(c, c + n, device=DEV)[:, None]
            j = torch.arange(c + n, device=DEV)
            hidden = (j > p) | (j <= p - (case["window"] or c + n + 1))
            for h in range(hk):
                k, v = (_tokens_of(s, case, w, ids, h)[:c + n] for w in (False, True))
                for u in range(h * (hq // hk), (h + 1) * (hq // hk)):
                    z = s["scale"] * (s["q"][t0:t0 + n, u].double() @ k.T.contiguous())
                    z[hidden] = -math.inf
                    lse[t0:t0 + n, u] = torch.logsumexp(z, 1)
                    out[t0:t0 + n, u] = torch.exp(z - lse[t0:t0 + n, u, None]) @ v
        t0 += n
    return {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    return {"plan": _exact_plan, "write": _exact_write, "attend": _exact_attend}[case["kind"]](case, s)
