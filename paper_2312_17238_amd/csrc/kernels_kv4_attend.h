// Attention of a step's rows over the paged cache held in 4 bits.
//
// As in kernels_kv_attend.h the cached tokens are the rows and the queries the columns of both products, and the probabilities go from the
// first to the second in the lane's own registers.  What differs:
//
// Scores.  Keys are e2m1 codes with a power-of-two scale for each 32 dims: what the scaled matrix instructions (32x32x64, 16x16x128)
// take as their first operand, so a key goes from memory to the matrix unit as it lies there, its scale byte beside it.  The second operand
// is the query, in a type of 6 bits at most if the instruction is to run at its full rate.  A query is therefore written as four
// digits for each 32 dims, q = 2^E (d0 + d1/32 + d2/1024 + d3/32768), each d a multiple of 1/8 from -2 to 2, which e2m3 holds exactly; the
// powers of 32 and 2^E are the second operand's scales.  Sums of 32 products of such digits are exact, those of the blocks are fp32: a query's number is
// off by at most 2^-20 of the power of two above the largest of its 32 dims, everything else of a score is fp32.  (As e4m3 numbers three parts would
// do, but a block's products are added with 13 bits or so below the largest, which numbers of very different sizes need more than: 2^-16 of the sum.)
//
// Values.  Twice a code becomes fp16 (exact), and its token has one scale, 2^(b - 127), half of which goes into the exponent: with t = scale log2(e) (q.k)
// + b - 128 the weight of a token's codes is 2^(t - m), m the running maximum of t less 7 (see LIFT), and the sum of the probabilities is that of the weights
// times 2^(128 - b).  b is from 82 to 172, so neither leaves fp32.  b - 128 is the byte with its highest bit turned over, as a signed one: t is of the size of the score
// and of the scale's exponent, and rounded as numbers of that size are (with b itself, which needs no turning over, by 2^-17 even where both are small).
//
// A prompt of 4096 (32 query and 8 kv heads of 128): 164 to 174 us, 0.8 PFLOP/s, 70 % of a large library product, by 8-bit codes the same.  Every wave reads
// its keys and values for itself, 133 bytes a token and head, out of the caches; nothing is shared through LDS and no wave waits for another.  By way of
// LDS (keys as they are, values converted once to fp16, scales as numbers) the same prompt took 174 us, with heads of 256 459 instead
// of 393.  Vector unit 69 % of the time, matrix unit 34 %: the two hardly overlap at two waves a SIMD, so what a step's 198 vector
// instructions are is what it costs: 32 conversions of values, 48 for bytes and inverses of scales, 16 each of scale, difference, exponential and sum.
#pragma once
#include "kernels_kv_attend.h"

namespace moe {
namespace kv {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef unsigned int v6u __attribute__((ext_vector_type(6)));
typedef float v32f __attribute__((ext_vector_type(32)));

constexpr int DIGITS = 4;

// Weights are taken relative to 2^-LIFT of the largest that a row had when its sums were last scaled, and may rise to 2^REACH before they are again:
// nearly all of what fp16 holds. A weight down to 2^-21 of that largest is rounded by 2^-11 of itself, a smaller one by 2^-32 of the largest, so
// that a million tokens behind one of a much higher score lose 2^-12 of the output at most (with weights of 1 for the largest: 2^-25 and 3 %).
constexpr float LIFT = 7.f, REACH = 15.f;

// Eight codes of a word as fp16 numbers, times two.
__device__ __forceinline__ v8h e2m1_to_half(uint32_t w)
{
    union { v8h v; v2h p[4]; } r;
    r.p[0] = __builtin_bit_cast(v2h, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 2.f, 0));
    r.p[1] = __builtin_bit_cast(v2h, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 2.f, 1));
    r.p[2] = __builtin_bit_cast(v2h, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 2.f, 2));
    r.p[3] = __builtin_bit_cast(v2h, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 2.f, 3));
    return r.v;
}

__device__ __forceinline__ v8i operand(uint4 k) { return v8i{(int)k.x, (int)k.y, (int)k.z, (int)k.w, 0, 0, 0, 0}; }
__device__ __forceinline__ v8i operand(v6u q) { return v8i{(int)q[0], (int)q[1], (int)q[2], (int)q[3], (int)q[4], (int)q[5], 0, 0}; }

// 32 numbers of a query as digits.  top: the largest of their bits without sign.  The digits' scale bytes, first digit lowest, are
// for numbers in units of 2^(row - 127), row the exponent of the query's largest number, times 2^-14.  A block is written in units of 2^-100 of
// that at least, so that its scales stay above 0: what is below has the small digits, or none, that it then comes to.
struct Digits {
    v6u d[DIGITS];
    int scale;
};

__device__ __forceinline__ Digits digits_of(float (&x)[32], uint32_t top, int row)
{
    Digits r;
    const int e = max(max((int)(top >> 23), 1), row - 100);
#pragma unroll
    for (int j = 0; j < 32; ++j) x[j] = ldexpf(x[j], 127 - e);      // below 2 in size
#pragma unroll
    for (int p = 0; p < DIGITS; ++p) {
        v16f even, odd;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            even[j] = x[2 * j];
            odd[j] = x[2 * j + 1];
        }
        // to the nearest eighth, and what is left of it times 32: 2 at most
        r.d[p] = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, 1.f);
        if (p + 1 < DIGITS) {
            const v32f n = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(r.d[p], 32.f);
#pragma unroll
            for (int j = 0; j < 32; ++j) x[j] = fmaf(x[j], 32.f, -n[j]);
        }
    }
    const int b = 127 + 14 + e - row;
    r.scale = b | (b - 5) << 8 | (b - 10) << 16 | (b - 15) << 24;
    return r;
}

// A number's bits without sign, for the largest; those of NaN and infinities are the largest of all.
__device__ __forceinline__ uint32_t size_bits(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7FFFFFFFu; }
constexpr uint32_t NO_NUMBER = 0x7F800000u;

// Bytes [lo, hi) of a lane's sixteen scales, those of the middle in the others' place.
__device__ __forceinline__ uint4 keep_scales(uint4 v, int lo, int hi)
{
    const uint4 k = keep_bytes(v, lo, hi), z = keep_bytes(make_uint4(0x7F7F7F7Fu, 0x7F7F7F7Fu, 0x7F7F7F7Fu, 0x7F7F7F7Fu), lo, hi);
    return make_uint4(k.x | (z.x ^ 0x7F7F7F7Fu), k.y | (z.y ^ 0x7F7F7F7Fu), k.z | (z.z ^ 0x7F7F7F7Fu), k.w | (z.w ^ 0x7F7F7F7Fu));
}

// b - 128 of byte i, from the word with every byte's highest bit turned over
__device__ __forceinline__ float exponent_of(uint32_t w, int i) { return (float)(int8_t)(w >> (8 * i)); }
// 2^(128 - b) of byte i, from the word's complement
__device__ __forceinline__ float inverse_of(uint32_t nw, int i) { return __builtin_bit_cast(float, ((nw >> (8 * i)) & 255u) << 23); }

// The queries of 32 rows: block 64 i + 32 h of a row's dims in lane (h, row).
template <int D>
struct Rows4 {
    Digits q[D / 64];
    float factor;       // of the scores: scale log2(e) and the row's power of two; NaN for a row that holds a NaN or an infinity
};

template <int DTYPE, int D>
__device__ __forceinline__ void load_rows4(const AttendArgs &a, const Item &it, int head, const Row &row, Rows4<D> &r)
{
    const int h = (threadIdx.x >> 5) & 1;
    const uint16_t *src = static_cast<const uint16_t *>(a.q.q) + (it.row0 + (row.real ? row.tok : 0)) * a.q.q_stride + (int64_t)(head * a.group + (row.real ? row.g : 0)) * D;
    uint32_t w[D / 64][16], top[D / 64], all = 0;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
        const uint16_t *p = src + 64 * i + 32 * h;
        if (!row.real) {
#pragma unroll
            for (int j = 0; j < 16; ++j) w[i][j] = 0;
        } else if (a.vec_q) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint4 u = reinterpret_cast<const uint4 *>(p)[j];
                w[i][4 * j] = u.x; w[i][4 * j + 1] = u.y; w[i][4 * j + 2] = u.z; w[i][4 * j + 3] = u.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) w[i][j] = p[2 * j] | ((uint32_t)p[2 * j + 1] << 16);
        }
        top[i] = 0;
#pragma unroll
        for (int j = 0; j < 16; ++j) top[i] = max(top[i], max(size_bits(from_bits<DTYPE>(w[i][j] & 0xFFFF)), size_bits(from_bits<DTYPE>(w[i][j] >> 16))));
        all = max(all, top[i]);
    }
    all = max(all, (uint32_t)__shfl_xor((int)all, 32));
    const int e = max((int)(all >> 23), 1);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
        float x[32];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            x[2 * j] = from_bits<DTYPE>(w[i][j] & 0xFFFF);
            x[2 * j + 1] = from_bits<DTYPE>(w[i][j] >> 16);
        }
        r.q[i] = digits_of(x, top[i], e);
    }
    r.factor = all >= NO_NUMBER ? __builtin_nanf("") : a.q.scale * LOG2E * ldexpf(1.f, e - 127 - 14);
}

// A row's state between steps.
template <int D>
struct State4 {
    v16f o[D / 32];     // O^T: column is the lane's row, row m = 8 (i/4) + 4 h + i%4 of tile n is dim 64 (n/2) + 2 m + n%2
    float m, l;
};

template <int D>
__device__ __forceinline__ void clear(State4<D> &s)
{
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) s.o[n][i] = 0.f;
    s.m = -INFINITY;
    s.l = 0.f;
}

template <int P>
__device__ __forceinline__ v16f score32(v8i k, int ks, const Digits &q, v16f z)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, operand(q.d[P]), z, 4, 2, 0, ks, P, q.scale);
}

// One step: 32 cached tokens against 32 rows.  k, ks: 32 dims of the lane's token and their scale, v: sixteen tokens of dims 64 n + 2 col
// and the next, vs: their scales.  edge: some row does not see some token, see: from which to which of the lane's sixteen this one does.
template <int D>
__device__ __forceinline__ void step4(State4<D> &s, const Rows4<D> &r, const uint4 (&k)[D / 64], const int (&ks)[D / 64], const uint4 (&v)[D / 64], uint4 vs, bool edge, Sees see)
{
    v16f z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
        const v8i op = operand(k[i]);
        z = score32<3>(op, ks[i], r.q[i], z);
        z = score32<2>(op, ks[i], r.q[i], z);
        z = score32<1>(op, ks[i], r.q[i], z);
        z = score32<0>(op, ks[i], r.q[i], z);
    }
    const uint32_t b[4] = {vs.x, vs.y, vs.z, vs.w};
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = fmaf(z[i], r.factor, exponent_of(b[i / 4] ^ 0x80808080u, i % 4));
    if (edge) {
        asm volatile("");               // a branch: as selections this would be worked out for every step
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = i >= see.lo && i < see.hi ? z[i] : -INFINITY;
    }
    float t = z[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) t = fmaxf(t, z[i]);
    t = max_halves(t);
    // the difference, which is exact where it matters: m + REACH is rounded up to 16 above m for scores of 2^27, and a weight of 2^16 is no fp16 number
    if (__any(t - s.m > REACH)) {
        const float m = fmaxf(s.m, t - LIFT);
        const float f = m == -INFINITY ? 1.f : exp2f(s.m - m);
        s.l = m == -INFINITY ? s.l : times_two_to(s.l, s.m - m);
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) s.o[n][i] *= f;
        s.m = m;
    }
    const float base = s.m == -INFINITY ? 0.f : s.m;
    v8h p[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float e = __builtin_amdgcn_exp2f(z[i] - base);
        s.l = fmaf(e, inverse_of(~b[i / 4], i % 4), s.l);
        p[i / 8][i % 8] = (_Float16)e;
    }
#pragma unroll
    for (int n = 0; n < D / 64; ++n) {
        s.o[2 * n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(e2m1_to_half(v[n].x), p[0], s.o[2 * n], 0, 0, 0);
        s.o[2 * n + 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(e2m1_to_half(v[n].z), p[0], s.o[2 * n + 1], 0, 0, 0);
        s.o[2 * n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(e2m1_to_half(v[n].y), p[1], s.o[2 * n], 0, 0, 0);
        s.o[2 * n + 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(e2m1_to_half(v[n].w), p[1], s.o[2 * n + 1], 0, 0, 0);
    }
}

// Which page a sub-block lies in; -1: none of the cache, or beyond what the request has.
__device__ __forceinline__ int page_of(const AttendArgs &a, const Item &it, int sub_block, int end_tok)
{
    const int blk = sub_block >> a.sub_shift;
    if (sub_block * SUB >= end_tok || blk >= a.max_blocks) return -1;
    const int id = a.table[(int64_t)it.req * a.max_blocks + blk];
    return (unsigned)id < (unsigned)a.c.n_pages ? id : -1;
}

// The steps kt0, kt0 + by, ... of 32 rows, straight from memory into registers.  PAIRS: pages of 32 tokens and more, in which a step's two sub-blocks
// follow each other: where a step lies is then a matter of scalars, and a lane's place in it the same in all steps.  A third of a step's vector
// instructions went into addresses without it: a prompt of 4096
// takes 165 us, 172 by the general way, 512 tokens onto 6000 103 and 106.
template <int D, bool PAIRS>
__device__ __forceinline__ void walk4(const AttendArgs &a, const Item &it, int head, const Rows4<D> &r, const Row &row, int pos_a, int pos_z, int kt0, int by, State4<D> &s)
{
    const int lane = threadIdx.x & 63, col = lane & 31, h = lane >> 5, heads = a.c.kv_heads;
    const Sees see = sees(a, it, row);
    // all rows see tokens [all_lo, all_hi); some see those in [any_lo, any_hi)
    const int end = it.ctx + it.n_new;
    const int any_lo = a.window > 0 ? max(0, pos_a + 1 - a.window) : 0, any_hi = a.causal ? pos_z + 1 : end;
    const int all_lo = a.window > 0 ? max(0, pos_z + 1 - a.window) : 0, all_hi = a.causal ? pos_a + 1 : end;
    const int kh = (col >> 2) & 1, ktok = 4 * (col >> 3) + (col & 3);     // row `col` of the scores is token 16 kh + ktok of the step
    const uint32_t lane_k = kh * (SUB * D / 2) + ktok * (D / 2) + 16 * h, lane_kb = kh * (SUB * D / 32) + (col & 3) * (D / 8) + 4 * h, lane_v = h * (SUB * D / 2) + col * 16;
    constexpr int BATCH = 32;       // steps whose pages the lanes hold, two sub-blocks a step
    for (int first = kt0; first < it.kt1; first += by * BATCH) {
        const int n = min(BATCH, div_up(it.kt1 - first, by));
        const int mine = (lane >> 1) < n ? page_of(a, it, 2 * (first + by * (lane >> 1)) + (lane & 1), end) : -1;
        uint4 k[2][D / 64], v[2][D / 64], vs[2];
        int ks[2][D / 64];
        auto fetch = [&](int j, int u) {
            const int sub = 2 * (first + by * j), in = (1 << a.sub_shift) - 1;
            const int id0 = max(__builtin_amdgcn_readlane(mine, 2 * j), 0);
            const uint64_t at0 = ((uint64_t)((uint32_t)id0 * heads + head) << a.sub_shift) + (sub & in);
            if constexpr (PAIRS) {
                const uint8_t *kp = static_cast<const uint8_t *>(a.c.k) + at0 * (SUB * D / 2), *vp = static_cast<const uint8_t *>(a.c.v) + at0 * (SUB * D / 2);
                const uint8_t *kb = a.c.k_byte + at0 * (SUB * D / 32), *vb = a.c.v_byte + at0 * SUB;
#pragma unroll
                for (int i = 0; i < D / 64; ++i) {
                    k[u][i] = *reinterpret_cast<const uint4 *>(kp + (lane_k + 32 * i));
                    ks[u][i] = *reinterpret_cast<const int *>(kb + (lane_kb + 8 * i));
                    v[u][i] = *reinterpret_cast<const uint4 *>(vp + (lane_v + 512 * i));
                }
                vs[u] = *reinterpret_cast<const uint4 *>(vb + (uint32_t)(SUB * h));
            } else {
                const int id1 = max(__builtin_amdgcn_readlane(mine, 2 * j + 1), 0);
                const uint64_t at1 = ((uint64_t)((uint32_t)id1 * heads + head) << a.sub_shift) + ((sub + 1) & in);
                const uint64_t ak = kh ? at1 : at0, av = h ? at1 : at0;
                const uint8_t *kp = static_cast<const uint8_t *>(a.c.k) + ak * (SUB * D / 2) + ktok * (D / 2) + 16 * h;
                const uint8_t *kb = a.c.k_byte + ak * (SUB * D / 32) + (col & 3) * (D / 8) + 4 * h;
                const uint8_t *vp = static_cast<const uint8_t *>(a.c.v) + av * (SUB * D / 2) + col * 16;
#pragma unroll
                for (int i = 0; i < D / 64; ++i) {
                    k[u][i] = *reinterpret_cast<const uint4 *>(kp + 32 * i);
                    ks[u][i] = *reinterpret_cast<const int *>(kb + 8 * i);
                    v[u][i] = *reinterpret_cast<const uint4 *>(vp + 512 * i);
                }
                vs[u] = *reinterpret_cast<const uint4 *>(a.c.v_byte + av * SUB);
            }
        };
        auto use = [&](int j, int u) {
            const int kt = first + by * j;
            if (kt * KT >= any_hi || (kt + 1) * KT <= any_lo) return;
            // of a pair the second sub-block may lie behind the request's end, where rows see nothing anyway
            const int id = __builtin_amdgcn_readlane(mine, 2 * j);
            const bool gone = PAIRS ? id < 0 : (h ? __builtin_amdgcn_readlane(mine, 2 * j + 1) : id) < 0;
            const bool edge = kt * KT < all_lo || (kt + 1) * KT > all_hi || __any(gone);
            const int tok0 = kt * KT + SUB * h;
            Sees mask{see.lo - tok0, gone ? 0 : see.hi - tok0};
            uint4 b = vs[u];
            if (edge) {
                asm volatile("");       // a branch, as in step4
                b = keep_scales(b, any_lo - tok0, gone ? 0 : end - tok0);
            }
            int sk[D / 64];
#pragma unroll
            for (int i = 0; i < D / 64; ++i) sk[i] = ks[u][i] >> (8 * (col >> 3));
            step4<D>(s, r, k[u], sk, v[u], b, edge, mask);
        };
        // no branch around a load: past the end the last step is requested again
        fetch(0, 0);
        for (int j = 0; j < n; j += 2) {
            fetch(min(j + 1, n - 1), 1);
            use(j, 0);
            fetch(min(j + 2, n - 1), 0);
            if (j + 1 < n) use(j + 1, 1);
        }
    }
    s.l += __shfl_xor(s.l, 32);
}

// ---- a tile of 32 rows: every wave takes every fourth step of the block's.
template <int DTYPE, int D, bool PAIRS>
__device__ __forceinline__ void attend4_few(const AttendArgs &a, const Item &it, int head, FewShared<D> &sh)
{
    constexpr int WAVES = ATTEND_WAVES;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 31, h = lane >> 5, heads = a.c.kv_heads;
    const int rows = it.n_new * a.group, row0 = it.tile * ROWS_FEW, here = min(ROWS_FEW, rows - row0);
    const Row row = row_at(a, row0, row0 + col, rows);
    Rows4<D> r;
    load_rows4<DTYPE, D>(a, it, head, row, r);
    State4<D> s;
    clear(s);
    walk4<D, PAIRS>(a, it, head, r, row, it.ctx + __builtin_amdgcn_readlane(row.tok, 0), it.ctx + __builtin_amdgcn_readlane(row.tok, here - 1), it.kt0 + wave, WAVES, s);
    // join the waves
    if (h == 0) {
        sh.m[wave][col] = s.m;
        sh.l[wave][col] = s.l;
    }
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = fmaxf(top, sh.m[w][col]);
    const float base = top == -INFINITY ? 0.f : top;
    const float l = sum_of_waves(sh.m, sh.l, col, base);
    float f = exp2f(s.m - base);
    const bool whole = it.part < 0;
    if (whole) f = l == 0.f ? 0.f : f / l;
    const int64_t part = ((int64_t)it.part * heads + head) * ROWS_FEW;
    float *ml = a.part_few + (int64_t)a.p.parts_few * heads * ROWS_FEW * D;
    if (tid < here) {
        if (!whole) put2(ml + (part + tid) * 2, top, l);
        else if (a.q.lse) a.q.lse[(int64_t)(it.row0 + row.tok) * heads * a.group + head * a.group + row.g] = LN2 * (top + log2f(l));
    }
    constexpr int STRIDE = D + 4, HOLD = sizeof(sh.o) / (WAVES * STRIDE * 4), QUADS = D / 4;
    for (int r0 = 0; r0 < here; r0 += HOLD) {
        if (r0) __syncthreads();
        if (col >= r0 && col < min(r0 + HOLD, here)) {
#pragma unroll
            for (int n = 0; n < D / 64; ++n)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    *reinterpret_cast<float4 *>(sh.o + (wave * HOLD + col - r0) * STRIDE + 64 * n + 16 * (i / 2) + 8 * h + 4 * (i % 2)) =
                        make_float4(s.o[2 * n][2 * i] * f, s.o[2 * n + 1][2 * i] * f, s.o[2 * n][2 * i + 1] * f, s.o[2 * n + 1][2 * i + 1] * f);
        }
        __syncthreads();
        for (int e = tid; e < min(HOLD, here - r0) * QUADS; e += 64 * WAVES) {
            const int rr = e / QUADS, d = (e % QUADS) * 4;
            float4 x = *reinterpret_cast<const float4 *>(sh.o + rr * STRIDE + d);
#pragma unroll
            for (int w = 1; w < WAVES; ++w) {
                const float4 y = *reinterpret_cast<const float4 *>(sh.o + (w * HOLD + rr) * STRIDE + d);
                x.x += y.x;
                x.y += y.y;
                x.z += y.z;
                x.w += y.w;
            }
            if (whole) {
                const Row out = row_at(a, row0, row0 + r0 + rr, rows);
                store4<DTYPE>(a.q.out, (it.row0 + out.tok) * a.q.out_stride + (int64_t)(head * a.group + out.g) * D + d, a.vec_out, x.x, x.y, x.z, x.w);
            } else {
                float *p = a.part_few + (part + r0 + rr) * D + d;
                put2(p, x.x, x.y);
                put2(p + 2, x.z, x.w);
            }
        }
    }
    if (!whole && all_parts_done(a.p.joins_few + it.join * heads + head, it.parts, sh.join.last)) join_parts<DTYPE, D>(a, it, head, a.part_few, ml, ROWS_FEW, sh.join);
}

// ---- tiles of 32 rows a wave: every wave has its own and takes all steps of the block's.
template <int DTYPE, int D, bool PAIRS>
__device__ __forceinline__ void attend4_many(const AttendArgs &a, const Item &it, int head, JoinShared &sh)
{
    constexpr int ROWS = 32 * ATTEND_WAVES;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 31, h = lane >> 5, heads = a.c.kv_heads;
    const int rows = it.n_new * a.group, tile0 = it.tile * ROWS, row0 = tile0 + wave * 32;
    const Row row = row_at(a, tile0, row0 + col, rows);
    State4<D> s;
    clear(s);
    if (row0 < rows) {
        Rows4<D> r;
        load_rows4<DTYPE, D>(a, it, head, row, r);
        walk4<D, PAIRS>(a, it, head, r, row, it.ctx + __builtin_amdgcn_readlane(row.tok, 0), it.ctx + __builtin_amdgcn_readlane(row.tok, min(31, rows - 1 - row0)), it.kt0, 1, s);
    }
    const bool whole = it.part < 0;
    float *ml = a.part_many + (int64_t)a.p.parts_many * heads * ROWS * D;
    const __amdgpu_buffer_rsrc_t parts = __builtin_amdgcn_make_buffer_rsrc(a.part_many, 0, (int)((uint32_t)(a.p.parts_many * heads * ROWS) * (D * 4u)), 0x00020000);
    if (row.real) {
        const int64_t part = ((int64_t)it.part * heads + head) * ROWS + wave * 32 + col;
        const uint32_t wave_at = (uint32_t)((it.part * heads + head) * ROWS + wave * 32) * D;
        const float f = whole ? (s.l == 0.f ? 0.f : 1.f / s.l) : 1.f;
        const int64_t out = (it.row0 + row.tok) * a.q.out_stride + (int64_t)(head * a.group + row.g) * D;
#pragma unroll
        for (int n = 0; n < D / 64; ++n)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = s.o[2 * n][2 * i] * f, y = s.o[2 * n + 1][2 * i] * f, z = s.o[2 * n][2 * i + 1] * f, w = s.o[2 * n + 1][2 * i + 1] * f;
                // dims 16 g + 8 h + 4 (i % 2) ..., where the join looks for 8 (2 g + h) + 4 (i % 2)
                const int g = 4 * n + i / 2;
                if (whole) store4<DTYPE>(a.q.out, out + 16 * g + 8 * h + 4 * (i % 2), a.vec_out, x, y, z, w);
                else put4(parts, wave_at + (2 * g + h) * 256 + (32 * (i % 2) + col) * 4, x, y, z, w);
            }
        if (h == 0) {
            if (!whole) put2(ml + part * 2, s.m, s.l);
            else if (a.q.lse) a.q.lse[(int64_t)(it.row0 + row.tok) * heads * a.group + head * a.group + row.g] = s.l == 0.f ? -INFINITY : LN2 * (s.m + log2f(s.l));
        }
    }
    if (!whole && all_parts_done(a.p.joins_many + it.join * heads + head, it.parts, sh.last)) join_tile<DTYPE, D, ROWS>(a, it, head, parts, ml, sh);
}

template <int DTYPE, int D, bool PAIRS>
__global__ void __launch_bounds__(64 * ATTEND_WAVES, D <= 128 ? 2 : 1) k_kv4_attend(AttendArgs a)
{
    __shared__ union {
        FewShared<D> few;
        JoinShared many;
    } sh;
    const int heads = a.c.kv_heads;
    if ((int)blockIdx.x < a.many_blocks) {
        const int i = blockIdx.x / heads;
        const Item it = item_at(a.p.many + i);
        if (i < a.p.head->many) attend4_many<DTYPE, D, PAIRS>(a, it, blockIdx.x - i * heads, sh.many);
    } else {
        const int b = blockIdx.x - a.many_blocks, i = b / heads;
        const int first = a.p.few_first[i], last = a.p.few_first[i + 1];
        if (i >= a.p.head->few_blocks) return;
        for (int k = first; k < last; ++k) {
            if (k > first) __syncthreads();          // the item before is done with LDS
            attend4_few<DTYPE, D, PAIRS>(a, item_at(a.p.few + k), b - i * heads, sh.few);
        }
    }
}

}  // namespace kv
}  // namespace moe
