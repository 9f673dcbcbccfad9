"""Attention over the cache in 4 bits where numbers are far apart: blocks of a query, scores that are large, single tokens beside very many, and what is left of a score's
last bits; rows that see all tokens or none; what the format costs. Every form of it: single tokens, tiles of few rows, tiles of many."""
import math

import numpy as np
import pytest
import torch

import kv4_reference as R4
from paper_2312_17238_amd import paged
from test_gpu_kv4 import DEV, FOUR, Pool, check_attend, fill, half_step, i32, planned

pytestmark = pytest.mark.gpu


def pack(keys, values, heads):
    """A cache whose pages hold these codes [pages][page][dim] in all heads, all scales 1."""
    n, page, dim = keys.shape
    c = paged.Cache.empty(n, heads, dim, page, FOUR, DEV)
    k = keys[..., 0::2] | (keys[..., 1::2] << 4)
    v = values.reshape(n, page // 16, 16, dim).swapaxes(2, 3)
    v = v[..., 0::2] | (v[..., 1::2] << 4)
    for t, x in ((c.k, k), (c.v, v)):
        t.view(torch.uint8).copy_(torch.from_numpy(np.ascontiguousarray(x)).unsqueeze(1).expand(*t.shape))
    for t in (c.k_scale, c.v_scale):
        t.view(torch.uint8).fill_(127)
    return c


@pytest.mark.parametrize("lens,new", [([300, 41], [1, 1]), ([300, 41], [20, 5]), ([300, 100], [70, 40])])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("gap", [90, 100, 101, 120, 200])
def test_blocks_of_a_query_far_below_its_largest(lens, new, dim, gap):
    """A block of 32 dims 2^gap below the row's largest number, which meets keys of 0: the block counts for what it is, not for more."""
    p = Pool(2, -(-max(lens) // 16) + 1, page=16, q_heads=4, kv_heads=2, dim=dim, dtype=torch.bfloat16, seed=gap)
    fill(p, lens, k_exp=(-1, 0), v_exp=(-1, 1))
    p.cache.k.view(torch.uint8)[..., :16] = 0
    s = planned(p, lens, new)
    top = gap // 2
    q = p.rows(sum(new), 4, spread=0.0).float()
    q[..., 32:] = torch.ldexp(q[..., 32:], torch.tensor(top - gap, device=DEV))
    q[..., :32] = 2.0 ** top
    q = q.to(torch.bfloat16)
    scale = 2.0 ** (95 - top)
    out, lse = (x.double().cpu().numpy() for x in paged.attend(p.cache, s, q, scale, with_lse=True))
    # A number is off by 2^-20 of the power of two above its block's largest, or of 2^-99 of the row's largest if that is more; keys are 6 at most.
    # In scores: scale 2^-20 2^(top - 99) 6 (dim - 32); what attend_head allows counts the first.
    extra = 2.0 ** (95 - 20 - 99) * 6 * (dim - 32)
    k, kb, v, vb = p.tensors()
    qd, at = q.double().cpu().numpy(), 0
    for r, (n, m) in enumerate(zip(lens, new)):
        ids = p.table[r, :-(-n // 16)].cpu().numpy()
        for h in range(4):
            kh, vh = R4.keys(k[ids, h // 2], kb[ids, h // 2]).reshape(-1, dim), R4.values(v[ids, h // 2], vb[ids, h // 2]).reshape(-1, dim)
            vs = np.exp2(vb[ids, h // 2].astype(np.float64) - 127).reshape(-1)
            want, wl, slack, off = R4.attend_head(qd[at:at + m, h], kh, vh, vs, list(range(n - m, n)), n, scale, True, 0)
            # twice a score's error of the mean of |v|, 12 at most
            assert (np.abs(out[at:at + m, h] - want) <= slack + half_step(want, p.dtype) * 1.01 + 2 * extra * 12).all()
            assert (np.abs(lse[at:at + m, h] - wl) <= off + extra).all()
        at += m


FORMS = [([1], 1), ([3], 2), ([20], 1), ([70], 2), ([130], 1)]      # new tokens, query heads a kv head


@pytest.mark.parametrize("new,group", FORMS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("power", [20, 24, 26, 27, 28, 30])
def test_scores_whose_last_bit_is_large(new, group, dim, power):
    """Two tokens that one wave meets one after the other, with scores of 2^power (in powers of two) and one to four of such a number's last bits between
    them. Their values are alike, so the output is that value whatever the bits do."""
    step = 2.0 ** (power - 23)
    for first in range(4):
        for second in range(first + 1, 5):
            keys, values = np.zeros((6, 64, dim), np.uint8), np.zeros((6, 64, dim), np.uint8)
            values[0, 0] = values[4, 0] = 2
            keys[0, 0, 0] = keys[4, 0, 0] = 2
            keys[0, 0, 32], keys[4, 0, 32] = (0, 2, 4, 5, 6)[first], (0, 2, 4, 5, 6)[second]      # 0, 1, 2, 3, 4
            c = pack(keys, values, 2)
            n = sum(new)
            s = paged.Step(1, n, n, 6, 6, 64, 2 * group, 2, dim)
            table = torch.arange(6, dtype=torch.int32, device=DEV)[None].contiguous()
            s.plan(i32([384 - n]), i32(new), table, i32([5, 4, 3][:(384 - -(-(384 - n) // 64) * 64) // 64] + [0]), i32([6 - -(-(384 - n) // 64)]))
            assert s.status.tolist() == [0] and table.tolist() == [list(range(6))]
            q = torch.zeros(n, 2 * group, dim, dtype=torch.bfloat16, device=DEV)
            q[..., 0], q[..., 32] = 2.0 ** power, step
            out, lse = paged.attend(c, s, q, math.log(2), with_lse=True)
            late = torch.arange(384 - n, 384, device=DEV) >= 256           # rows that see the second token, too; the others see the first
            top = torch.where(late, float(second), float(first)).double() * step + 2.0 ** power
            # all other tokens' weights are 0; these two's are rounded to fp16 (2^-11), their sum is not, and bf16's half step is 2^-8 at 1
            assert ((out.double() - 1).abs() <= 2.0 ** -8).all(), (first, second)
            # in a score's last bits: the factor 1, what is added to it 1/2, the maximum 1/2, the logarithm added 1/2, ln 2 and the product 3/4, and the sum of
            # two weights is two at most
            assert ((lse.double() / math.log(2) - top[:, None]).abs() <= 4 * step + 1 + 2.0 ** -6).all(), (first, second)


@pytest.mark.parametrize("new,group", FORMS)
@pytest.mark.parametrize("dim,dtype", [(64, torch.float16), (128, torch.bfloat16), (256, torch.float16)])
def test_many_tokens_behind_one(new, group, dim, dtype):
    """131000 tokens with a score of 0 behind one of 17.5: each has e^-17.5 (2^-25.2) of its weight, all of them 0.3 % of the sum."""
    m, n, heads, peak = sum(new), 131000, 64, 17.5
    keys, values = np.zeros((2, 64, dim), np.uint8), np.zeros((2, 64, dim), np.uint8)
    keys[0, 0, 0] = 7                                   # 6 in the first dim of the first token
    values[:, :, :dim // 2] = 2                         # all others: 1 in the first half
    values[0, 0, :dim // 2], values[0, 0, dim // 2:] = 0, 2
    c = pack(keys, values, heads)
    width = -(-n // 64)
    table = torch.ones(1, width, dtype=torch.int32, device=DEV)
    table[0, 0] = 0
    s = paged.Step(1, m, m, width, 2, 64, heads * group, heads, dim)
    free = width - -(-(n - m) // 64)
    s.plan(i32([n - m]), i32(new), table, i32([1] * 4), i32([free]))
    assert s.status.tolist() == [0]
    q = torch.zeros(m, heads * group, dim, dtype=dtype, device=DEV)
    q[..., 0] = 1
    out, lse = (x.double().cpu().numpy() for x in paged.attend(c, s, q, peak / 6, with_lse=True))
    tail = np.arange(n - m, n, dtype=np.float64)[:, None, None]         # other tokens that a row sees
    want = np.broadcast_to(tail / (tail + math.exp(peak)), out[..., :dim // 2].shape)
    # Each weight is off by 2^-11 of itself or 2^-32 of the wave's largest, the score by three roundings of 26 (in powers of two), and sums of
    # n numbers in fp32 by n 2^-24, in the weights and in what they are divided by.
    allowed = tail * 2.0 ** -32 + want * (2.0 ** -11 + 3 * 26 * 2.0 ** -24 + 2 * n * 2.0 ** -24) + half_step(want, dtype) * 1.01
    err = np.abs(out[..., :dim // 2] - want)
    assert (err <= allowed).all(), float((err / allowed).max())
    one = 1 - want
    assert (np.abs(out[..., dim // 2:] - one) <= one * (2.0 ** -11 + 2.0 ** -17 + 2 * n * 2.0 ** -24) + half_step(one, dtype) * 1.01).all()
    assert (np.abs(lse - np.log(tail[..., 0] + math.exp(peak))) <= 2.0 ** -17 + n * 2.0 ** -24).all()


@pytest.mark.parametrize("new", [[1] * 300, [4] * 40, [20, 300, 40], [300, 1, 500]])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_the_sum_of_one_token_is_its_score(new, dim):
    """A window of one: lse is the row's own score, to fp32's rounding of numbers of its size, whatever the value's scale is."""
    p = Pool(len(new), -(-max(new) // 16) + 2, page=16, q_heads=4, kv_heads=2, dim=dim, window=1, seed=dim)
    lens = [n + 5 for n in new]
    fill(p, lens, k_exp=(-1, 1), v_exp=(1, 3))
    s = planned(p, lens, new)
    # multiples of 1/4 up to 2: four digits, products and sums are exact
    q = torch.from_numpy(p.rng.integers(-8, 9, (sum(new), 4, dim)) / 4.0).half().to(DEV)
    k, kb, _, _ = p.tensors()
    scores = np.zeros((sum(new), 4))
    qd, at = q.double().cpu().numpy(), 0
    for r, (n, m) in enumerate(zip(lens, new)):
        ids = p.table[r, :-(-n // 16)].cpu().numpy()
        for h in range(4):
            scores[at:at + m, h] = (qd[at:at + m, h] * R4.keys(k[ids, h // 2], kb[ids, h // 2]).reshape(-1, dim)[n - m:n]).sum(-1)
        at += m
    # the largest score becomes one power of two; the scale in fp32, as the call takes it
    scale = float(np.float32(math.log(2) / np.abs(scores).max()))
    _, lse = paged.attend(p.cache, s, q, scale, with_lse=True)
    # In units of 2^-24, in powers of two: the score's two products 2.5, the value's exponent (up to 3) added to it 2, the maximum lowered by 7 (half a step
    # below 16) 8, taken off 8, exp2 (a step of the result, 2 log2(e)) 3, its product with the value's inverse 1.5, log2 (a step of a number below 16) 16, the maximum added 8,
    # ln 2 and the product 2: 51.
    err = np.abs(lse.double().cpu().numpy() - scale * scores)
    assert err.max() <= 51 * 2.0 ** -24 * math.log(2), err.max()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 50])
@pytest.mark.parametrize("lens,new", [([300, 9000], [5, 3]), ([9000, 64, 1], [8, 2, 1]), ([2000, 33], [1, 1])])
def test_all_tokens_are_seen_by_few_rows(lens, new, window, dim):
    """Steps of at most sixteen rows a request without a causal mask, with and without a window."""
    p = Pool(len(lens), -(-max(lens) // 64) + 1, page=64, dim=dim, q_heads=4, kv_heads=2, causal=False, window=window, seed=sum(lens))
    fill(p, lens)
    s = planned(p, lens, new, spare=1)
    q = p.rows(sum(new) + 1, 4, spread=0.5)
    out, lse = paged.attend(p.cache, s, q, with_lse=True)
    check_attend(p, q, out, lse, lens, new, 1 / math.sqrt(dim))


@pytest.mark.parametrize("new", [[1, 1], [20, 3], [70, 40], [5, 70]])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("gone", [0, 1])
def test_a_request_that_is_served_and_sees_nothing(new, dim, gone):
    """Tables that name no page of the cache: rows get 0 and -inf, in one piece and in several that are joined, and the other request what it gets anyway."""
    lens = [9000, 200]
    p = Pool(2, 564, dim=dim, page=16, q_heads=4, kv_heads=2, seed=new[0])
    fill(p, lens)
    s = planned(p, lens, new)
    q = p.rows(sum(new), 4)
    want = paged.attend(p.cache, s, q, with_lse=True)
    p.table[gone] = torch.tensor([-1, p.n_pages, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=DEV).repeat(141)
    out, lse = paged.attend(p.cache, s, q, with_lse=True)
    mine = slice(0, new[0]) if gone == 0 else slice(new[0], sum(new))
    others = slice(new[0], sum(new)) if gone == 0 else slice(0, new[0])
    assert (out[mine] == 0).all() and (lse[mine] == -math.inf).all()
    assert torch.equal(out[others], want[0][others]) and torch.equal(lse[others], want[1][others])


@pytest.mark.parametrize("dim,value", [(64, 0.1191), (128, 0.1248), (256, 0.1335)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_what_four_bits_cost(dim, value, dtype):
    """Normally distributed numbers, as they are read back and as attention over them sees them, against the numbers themselves: root mean squares that follow from
    the definition (11.5 % for keys in blocks of 32, `value` for values), beside those of 8 bits."""
    g = torch.Generator().manual_seed(dim)
    n, m, heads = 700, 16, 8
    x = torch.randn(n, 3 * heads, dim, generator=g).to(dtype).to(DEV)
    q, k, v = x[:, :heads], x[:, heads:2 * heads], x[:, 2 * heads:]
    z = torch.matmul(q[n - m:].double().cpu().transpose(0, 1), k.double().cpu().permute(1, 2, 0).contiguous()) / math.sqrt(dim)
    want = torch.matmul(torch.softmax(z, -1), v.double().cpu().transpose(0, 1).contiguous()).transpose(0, 1)
    rms = lambda a, b: float((a.double().cpu() - b.double().cpu()).norm() / b.double().cpu().norm())  # noqa: E731
    off = {}
    for t in (FOUR, torch.float8_e4m3fn):
        c = paged.Cache.empty(11, heads, dim, 64, t, DEV)
        s = paged.Step(1, n, n, 11, 11, 64, heads, heads, dim)
        table = torch.zeros(1, 11, dtype=torch.int32, device=DEV)
        s.plan(i32([0]), i32([n]), table, i32(list(range(11))), i32([11]))
        paged.write(c, s, q, k, v)
        keys, values = paged.gather(c, s.slots, dtype)
        few = paged.Step(1, m, m, 11, 11, 64, heads, heads, dim, causal=False)
        few.plan(i32([n - m]), i32([m]), table, i32([0]), i32([0]))
        assert few.status.tolist() == [0]
        off[t] = rms(keys, k), rms(values, v), rms(paged.attend(c, few, q[n - m:]), want)
    # 358 thousand numbers and more: the figures hold to about 1 %. Scores are of size 1, so that a key's error is that of its weight, too; attention's figure, over
    # 128 rows, holds to a tenth.
    a, b, o = off[FOUR]
    assert abs(a - 0.1154) < 0.003 and abs(b - value) < 0.003 and abs(o - math.hypot(a, b)) < 0.02, off
    a, b, o = off[torch.float8_e4m3fn]
    assert abs(a - 0.0265) < 0.002 and abs(b - 0.0265) < 0.002 and 0.03 < o < 0.05, off
