"""The 4-bit cache where it is used: under whole decoder blocks, beside layers that keep 8 bits, and handed from one cache to another."""
import math

import numpy as np
import pytest
import torch

import kv4_reference as R4
import kv_reference as R
from paper_2312_17238_amd import decode_loop, paged
from test_gpu_kv4 import DEV, FOUR, Pool, check_attend, host, i32

pytestmark = pytest.mark.gpu


def make(n_requests=3, max_rows=64, **k):
    return decode_loop.Decoder(2, 256, 512, 4, 2, 64, n_requests, 80, max_rows, page=16, fmt=FOUR, **k)


def test_attention_half_against_64_bits():
    """Prompts, single tokens and drafts of three requests through two blocks: what attention adds is what 64 bits make of the cache, and the cache is
    what 64 bits make of the hidden states' keys and values, but for codes at a border (the projections are fp16 products)."""
    d = make()
    g = torch.Generator().manual_seed(1)
    lens, apart, seen_codes = [0, 0, 0], 0, 0
    for new in ([20, 1, 33], [1, 1, 1], [1, 5, 0]):
        s = d.bounds(sum(new), max(new))
        x = torch.randn(sum(new), 256, generator=g).half().to(d.device)
        torch.cuda.synchronize()
        seen = {}

        def spy(layer, step, x):
            y = decode_loop.Decoder.attention_half(d, layer, step, x)
            seen[layer] = (x.clone(), y.clone())
            return y
        d.attention_half = spy
        d.step(s, x, new)
        d.stack.synchronize()
        lens = [c + n for c, n in zip(lens, new)]
        assert d.ctx_len.tolist() == lens
        freq = d.inv_freq.cpu().numpy()
        for l in range(2):
            c = d.caches[l]
            k, kb, v, vb = (host(t) for t in (c.k, c.k_scale, c.v, c.v_scale))
            xi, yi = (t.double().cpu().numpy() for t in seen[l])
            h = (xi / np.sqrt((xi * xi).mean(-1, keepdims=True) + 1e-5)).astype(np.float16).astype(np.float64)
            qkv = (h @ d.wqkv[l].double().cpu().numpy()).reshape(-1, 8, 64)
            at = 0
            for r, n in enumerate(new):
                pos = list(range(lens[r] - n, lens[r]))
                q = R.turned(qkv[at:at + n, :4], pos, None, 0.0, freq, False)
                ids = d.block_table[r, :-(-lens[r] // 16)].cpu().numpy()
                out = np.zeros((n, 4, 64))
                for w in range(2):
                    kh, vh = R4.keys(k[ids, w], kb[ids, w]).reshape(-1, 64), R4.values(v[ids, w], vb[ids, w]).reshape(-1, 64)
                    if not n:
                        continue
                    for u in (2 * w, 2 * w + 1):
                        out[:, u] = R4.attend_head(q[:, u], kh, vh, np.ones(len(vh)), pos, lens[r], 0.125, True, 0)[0]
                    for x64, have, width in ((R.turned(qkv[at:at + n, 4 + w:5 + w], pos, None, 0.0, freq, False)[:, 0], kh, 32), (qkv[at:at + n, 6 + w], vh, 64)):
                        codes, e = R4.quantized(x64, width, 65504.0)
                        want = R4.value_of(codes) * np.repeat(np.exp2(e.astype(float)), width, -1)
                        got = have[lens[r] - n:lens[r]]
                        apart += int((got != want).sum())
                        seen_codes += got.size
                        # a code next door, or a scale: two units of the coarser at most
                        assert (np.abs(got - want) <= 4 * np.repeat(np.exp2(e.astype(float)), width, -1)).all()
                want = xi[at:at + n] + out.reshape(n, 256) @ d.wo[l].double().cpu().numpy()
                # fp16 queries (2^-11 of scores of a few), fp16 attention, product and sum
                assert np.abs(yi[at:at + n] - want).max(initial=0) <= 2.0 ** -7
                at += n
    # a projection is rounded to fp16, 2^-11 of a number of about 2 steps' size: seven borders, each hit by about 2^-11 of the numbers, and scales now and then
    assert apart <= seen_codes * 0.03
    free = d.n_pages - sum(-(-n // 16) for n in lens)
    assert d.free_count.item() == free
    d.finish([0, 1, 2])
    d.stack.synchronize()
    assert d.free_count.item() == d.n_pages
    d.close()


@pytest.mark.parametrize("args", [[], ["--page", "16", "--window", "20", "--requests", "7", "--cache-slots", "3", "--head-dim", "128"]])
def test_command(args):
    r = decode_loop.main(args + ["--format", "e2m1"])
    n = r["requests"]
    assert r["finite"] and r["format"] == "e2m1" and r["cached_tokens"] == [max(1, 37 - 5 * i) + 16 for i in range(n)] and r["free_pages"] == r["pages"]


@pytest.mark.parametrize("new", [[1, 1], [9, 3], [70, 40]])
def test_layers_of_different_formats_share_a_step(new):
    """A plan and its scratch serve caches of 8 and of 4 bits in turn, again and again, with the results that each has alone."""
    p = Pool(2, 100, dim=128, page=64, q_heads=4, kv_heads=2, seed=3)
    eight = paged.Cache.empty(p.n_pages, 2, 128, 64, torch.float8_e4m3fn, DEV)
    first = [5200, 300]
    s = p.step(first)
    x = p.rows(sum(first), 8)
    for c in (p.cache, eight):
        paged.write(c, s, x[:, :4], x[:, 4:6], x[:, 6:])
    s.advance()
    lens = [a + b for a, b in zip(first, new)]
    s = p.step(new)
    x = p.rows(sum(new), 8)
    for c in (p.cache, eight):
        paged.write(c, s, x[:, :4], x[:, 4:6], x[:, 6:])
    q = x[:, :4].contiguous()
    results = [(paged.attend(p.cache, s, q, with_lse=True), paged.attend(eight, s, q, with_lse=True)) for _ in range(4)]
    for four_bits, eight_bits in results[1:]:
        for a, b in zip(four_bits + eight_bits, results[0][0] + results[0][1]):
            assert torch.equal(a, b)
    check_attend(p, q, *results[0][0], lens, new, 1 / math.sqrt(128), rows=4)
    # the two caches hold the same numbers to 4 bits (a quarter of a number) and 8: so much are the outputs alike
    a, b = (r[0].float() for r in results[0])
    assert (a - b).abs().max() <= 0.5 * b.abs().max()


def test_what_is_read_back_and_stored_again_is_the_same():
    """Tokens that move to another cache by way of their values keep them: the store of what a code stands for gives that code's value again."""
    p, to = (Pool(1, 8, dim=128, page=32, kv_heads=3, q_heads=3, dtype=torch.bfloat16, seed=i) for i in (1, 2))
    x = p.rows(200, 9)
    s = p.step([200])
    paged.write(p.cache, s, x[:, :3], x[:, 3:6], x[:, 6:])
    k, v = paged.gather(p.cache, s.slots, torch.bfloat16)
    t = to.step([200])
    paged.write(to.cache, t, torch.zeros_like(k), k, v)
    for a, b in zip(paged.gather(to.cache, t.slots, torch.bfloat16), (k, v)):
        assert torch.equal(a, b)
    # and their attention
    q = p.rows(200, 3)
    assert torch.allclose(paged.attend(p.cache, s, q).float(), paged.attend(to.cache, t, q).float(), atol=0.02)


@pytest.mark.parametrize("shape", [(300, 1), (1, 300)])
def test_requests_together_get_what_each_gets_alone(shape):
    """Two requests in one step and one after the other: the same cache bytes and the same rows of attention, to rounding."""
    x = None
    got = []
    for order in ([list(shape)], [[shape[0], 0], [0, shape[1]]]):
        p = Pool(2, 12, dim=64, page=32, seed=4)
        x = p.rows(sum(shape), 8) if x is None else x
        rows = {}
        for new in order:
            s = p.step(new)
            mine = torch.cat([x[:shape[0]] if new[0] else x[:0], x[shape[0]:] if new[1] else x[:0]])
            paged.write(p.cache, s, mine[:, :4], mine[:, 4:6], mine[:, 6:])
            out = paged.attend(p.cache, s, mine[:, :4].contiguous())
            k, v = paged.gather(p.cache, s.slots)
            at = 0
            for r, n in enumerate(new):
                if n:
                    rows[r] = (out[at:at + n].float(), k[at:at + n], v[at:at + n])
                at += n
            s.advance()
        got.append(rows)
    for r in (0, 1):
        a, b = got[0][r], got[1][r]
        assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
        # two ways to share the work out: each within fp16's half step and the weights' 2^-11 of 64 bits
        assert (a[0] - b[0]).abs().max() <= 2.0 ** -9 * b[2].float().abs().max()
