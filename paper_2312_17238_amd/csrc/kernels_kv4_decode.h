// Attention over the cache held in 4 bits for steps whose requests bring no more than sixteen (token, query head of the group) rows each.
//
// The roles of lanes and waves, and what is requested ahead of its use, are those of kernels_kv_decode.h; the products those of
// kernels_kv4_attend.h on 16x16 instructions.  Row m of tile t of the scores stands for token 16 (m / 4) + 4 t + m % 4 of a step of 64, so that the
// lanes of four neighbouring rows read 4 x D / 2 bytes in one piece and a lane's four tiles have their scales in one word; output row m of
// tile 2 i + e is dim 32 i + 2 m + e.  A lane of quarter g holds 32 dims of a query: g's, of heads of 256 those of g + 4 too.  Heads of 64 have two
// blocks of dims, so that an instruction takes two digits at once, one in the lower half of its quarters and one in the upper.
//
// Memory is the bound, 133 bytes a token and kv head: 64 requests over 2000 tokens each 26.6 us (137 MB, 5.2 TB/s), 64 over 8000 98.8 (5.5 TB/s), one
// over 524000 106 (5.3 TB/s).  Below that it is starts and joins: 64 requests over 500 to 8000 50 us (176 MB; a plain read of as much 35.6, these
// loads without anything else 44), one over 131000 36.7 (139 MB; 29.9 and 38), of which a join of 64 parts is 4.  The 32-row kernel takes 59
// and 43 for these.  Two steps ahead instead of one: 66 and 45, for the registers.
#pragma once
#include "kernels_kv4_attend.h"
#include "kernels_kv_decode.h"

namespace moe {
namespace kv {

// Joining the parts of a tile's rows, in the parts' order.  What this costs is not its bytes but one wait behind the other, those for code that is not in
// the instruction cache among them: one short loop without a branch inside, which takes a part's maximum, sum and outputs in one go.  One token over 2000
// (3 parts) takes 11.3 us, 12.0 with join_parts, whose loops are unrolled; over 131000 (64 parts) 36.7 and 38.6; without any join 8.7 and 29.  SPAN, the parts
// that a thread asks for at once, as 8, 16 and 32: one token over 2000 10.3, 11.0 and 12.5 us, over 131000 38.5, 38.4 and 38.1, 64 uneven requests 50.0, 51.7
// and 55.7, 16 of heads of 256 21.2, 21.1 and 24.2.
struct Join4Shared {
    float4 sum[64 * DECODE_WAVES];      // of a thread
    float2 ml[64 * DECODE_WAVES];
    int last;
};

template <int DTYPE, int D>
__device__ __forceinline__ void join4(const AttendArgs &a, const Item &it, int head, const float *ml, Join4Shared &sh)
{
    constexpr int THREADS = 64 * DECODE_WAVES, QUADS = D / 4, SPAN = 16;
    const int tid = threadIdx.x, heads = a.c.kv_heads, rows = it.n_new * a.group, parts = it.parts;
    int pow2 = 4;
    while (pow2 < rows) pow2 *= 2;
    const __amdgpu_buffer_rsrc_t o = __builtin_amdgcn_make_buffer_rsrc(a.part_few, 0, (int)((uint32_t)(a.p.parts_few * heads * ROWS_FEW) * (D * 4u)), 0x00020000);
    // four dims a thread; where that leaves threads over, the parts are dealt out to groups of waves
    const int all = min(THREADS, pow2 * QUADS), groups = THREADS / all, g = __builtin_amdgcn_readfirstlane(tid / all);
    // 32 bits: at most 1024 parts of all heads, of 32 rows and 256 dims
    const uint32_t first = (uint32_t)(it.part0 * heads + head) * ROWS_FEW, stride = (uint32_t)heads * ROWS_FEW;
#pragma nounroll
    for (int e = tid % all; e < pow2 * QUADS; e += all) {
        const int r = min(e / QUADS, rows - 1), d = (e % QUADS) * 4;
        float top = -INFINITY, l = 0.f;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma nounroll
        for (int p0 = g; p0 < parts; p0 += SPAN * groups) {
            float4 x[SPAN];
            float2 v[SPAN];
            float high = top;
#pragma unroll
            for (int u = 0; u < SPAN; ++u) {            // past the last part that one again, which then does not count
                const uint32_t at = first + (uint32_t)min(p0 + u * groups, parts - 1) * stride;
                v[u] = get2(ml, (at + r) * 8);
                x[u] = __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(o, (r * D + d) * 4, (int)(at * (D * 4)), 16));
            }
#pragma unroll
            for (int u = 0; u < SPAN; ++u) high = fmaxf(high, v[u].x);
            const float base = high == -INFINITY ? 0.f : high, f = exp2f(top - base);
            top = high;
            l *= f;
            sum.x *= f;
            sum.y *= f;
            sum.z *= f;
            sum.w *= f;
#pragma unroll
            for (int u = 0; u < SPAN; ++u) {
                const float w = p0 + u * groups < parts ? exp2f(v[u].x - base) : 0.f;
                l = fmaf(w, v[u].y, l);
                sum.x = fmaf(w, x[u].x, sum.x);
                sum.y = fmaf(w, x[u].y, sum.y);
                sum.z = fmaf(w, x[u].z, sum.z);
                sum.w = fmaf(w, x[u].w, sum.w);
            }
        }
        if (groups > 1) {
            sh.sum[tid] = sum;
            sh.ml[tid] = make_float2(top, l);
            __syncthreads();
            float high = top;
            for (int w = 1; w < groups; ++w) high = fmaxf(high, sh.ml[w * all + e].x);
            const float base = high == -INFINITY ? 0.f : high;
            l = 0.f;
            sum = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int w = 0; w < groups; ++w) {
                const float2 v = sh.ml[w * all + e];
                const float4 x = sh.sum[w * all + e];
                const float f = exp2f(v.x - base);
                l = fmaf(f, v.y, l);
                sum.x = fmaf(f, x.x, sum.x);
                sum.y = fmaf(f, x.y, sum.y);
                sum.z = fmaf(f, x.z, sum.z);
                sum.w = fmaf(f, x.w, sum.w);
            }
            top = high;
        }
        if (g == 0 && e < rows * QUADS) {
            const float f = l == 0.f ? 0.f : 1.f / l;
            const int tok = r / a.group, gr = r - tok * a.group;
            store4<DTYPE>(a.q.out, (it.row0 + tok) * a.q.out_stride + (int64_t)(head * a.group + gr) * D + d, a.vec_out, sum.x * f, sum.y * f, sum.z * f, sum.w * f);
            if (a.q.lse && d == 0) a.q.lse[(int64_t)(it.row0 + tok) * heads * a.group + head * a.group + gr] = l == 0.f ? -INFINITY : LN2 * (top + log2f(l));
        }
    }
}

template <int D>
struct Decode4Shared {
    float m[DECODE_WAVES][ROWS_DECODE], l[DECODE_WAVES][ROWS_DECODE];
    __align__(16) float o[DECODE_WAVES * 8 * (D + 4)];
    Join4Shared join;
};

// What is known of an item before it is worked on: where the sub-blocks of its first sixteen steps lie, which of them are in the cache, queries.
template <int D>
struct Ahead4 {
    static constexpr int BLOCKS = D <= 128 ? 1 : 2;
    int id;             // page, as the table has it; -1 beyond what the part has
    uint32_t at;
    uint64_t there;     // lanes whose sub-block is in the cache
    uint32_t q[BLOCKS][16];
};

template <int DTYPE, int D>
struct Decode4 {
    static constexpr int BATCH = 16, BLOCKS = Ahead4<D>::BLOCKS, PASSES = D == 64 ? 2 : DIGITS;
    struct Keys { uint4 k[4][BLOCKS]; int scale[BLOCKS]; };
    struct Values { uint4 v[D / 32], scale; };

    const AttendArgs &a;
    Decode4Shared<D> &sh;
    const int head, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;

    __device__ __forceinline__ static int steps(const Item &it) { return div_up(it.kt1 - it.kt0, 2); }
    __device__ __forceinline__ int block_of(int i) const { return D == 64 ? g & 1 : g + 4 * i; }

    __device__ __forceinline__ int table(const Item &it, int first) const
    {
        const int s = first + DECODE_WAVES * (lane >> 2), sub = 2 * it.kt0 + 4 * s + (lane & 3), blk = sub >> a.sub_shift;
        if (s >= steps(it) || sub * SUB >= min(it.ctx + it.n_new, it.kt1 * KT) || blk >= a.max_blocks) return -1;
        return a.table[(int64_t)it.req * a.max_blocks + blk];
    }

    __device__ __forceinline__ void place(const Item &it, int first, Ahead4<D> &x) const
    {
        const int s = first + DECODE_WAVES * (lane >> 2), sub = 2 * it.kt0 + 4 * s + (lane & 3);
        const bool good = (unsigned)x.id < (unsigned)a.c.n_pages;
        const uint32_t p = (uint32_t)(good ? x.id : 0) * a.c.kv_heads + head;
        x.at = (p << a.sub_shift) + (sub & ((1 << a.sub_shift) - 1));
        x.there = __ballot(good);
    }

    __device__ __forceinline__ void queries(const Item &it, Ahead4<D> &x) const
    {
        const Row row = row_at(a, 0, col, it.n_new * a.group);
        const uint16_t *src = static_cast<const uint16_t *>(a.q.q) + (it.row0 + (row.real ? row.tok : 0)) * a.q.q_stride + (int64_t)(head * a.group + (row.real ? row.g : 0)) * D;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            const uint16_t *p = src + 32 * block_of(i);
            if (a.vec_q) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint4 u = reinterpret_cast<const uint4 *>(p)[j];
                    x.q[i][4 * j] = u.x; x.q[i][4 * j + 1] = u.y; x.q[i][4 * j + 2] = u.z; x.q[i][4 * j + 3] = u.w;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) x.q[i][j] = p[2 * j] | ((uint32_t)p[2 * j + 1] << 16);
            }
        }
    }

    // keys and values of the step whose four sub-blocks the lanes 4 j .. 4 j + 3 hold
    __device__ __forceinline__ void fetch_k(uint32_t at, int j, Keys &x) const
    {
        const uint64_t sub = __shfl(at, 4 * j + (col >> 2));
        const uint8_t *p = static_cast<const uint8_t *>(a.c.k) + sub * (SUB * D / 2) + (col & 3) * (D / 2);
        const uint8_t *b = a.c.k_byte + sub * (SUB * D / 32) + (col & 3) * (D / 8);
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
#pragma unroll
            for (int t = 0; t < 4; ++t) x.k[t][i] = *reinterpret_cast<const uint4 *>(p + t * (2 * D) + block_of(i) * 16);
            x.scale[i] = *reinterpret_cast<const int *>(b + block_of(i) * 4);
        }
    }
    __device__ __forceinline__ void fetch_v(uint32_t at, int j, Values &x) const
    {
        const uint64_t sub = __shfl(at, 4 * j + g);
        const uint8_t *p = static_cast<const uint8_t *>(a.c.v) + sub * (SUB * D / 2) + col * 16;
        x.scale = *reinterpret_cast<const uint4 *>(a.c.v_byte + sub * SUB);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) x.v[i] = *reinterpret_cast<const uint4 *>(p + i * 256);
    }

    __device__ __forceinline__ float *ml() const { return a.part_few + (int64_t)a.p.parts_few * a.c.kv_heads * ROWS_FEW * D; }

    template <int P>
    __device__ __forceinline__ static void scores(const Keys &x, int i, const v6u &q, int scale, v4f (&z)[4])
    {
        z[0] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(x.k[0][i]), operand(q), z[0], 4, 2, 0, x.scale[i], P, scale);
        z[1] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(x.k[1][i]), operand(q), z[1], 4, 2, 1, x.scale[i], P, scale);
        z[2] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(x.k[2][i]), operand(q), z[2], 4, 2, 2, x.scale[i], P, scale);
        z[3] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(x.k[3][i]), operand(q), z[3], 4, 2, 3, x.scale[i], P, scale);
    }

    // What a wave knows of its item while it walks over the tokens.
    struct Walk {
        Sees see;
        float factor;
        int any_lo, any_hi, all_lo, all_hi, part_hi;
    };

    // Step j of the n whose places `here` and `in_cache` hold, its tokens from `tok` on.  k, v: its keys and values, then the next step's: no
    // branch around a load, so behind the last step the next item's first one is requested (on), or the same step again, which the caches
    // still hold.
    __device__ __forceinline__ void step(const Walk &w, const v6u (&q)[BLOCKS][PASSES], const int (&qs)[BLOCKS], int j, int n, int tok, uint32_t here, uint64_t in_cache, bool on,
                                         uint32_t next_at, Keys &k, Values &v, v4f (&o)[D / 16], float &m, float &l) const
    {
        const uint32_t at = j + 1 < n || !on ? here : next_at;
        const int at_j = j + 1 < n ? j + 1 : on ? 0 : j;
        const int tok0 = tok + SUB * g;
        const uint32_t there = (uint32_t)(in_cache >> (4 * j)) & 15;
        const bool edge = tok < w.all_lo || tok + 64 > w.all_hi || there != 15;
        v4f z[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) z[t] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            if constexpr (D == 64) {
                scores<2>(k, i, q[i][1], qs[i], z);
                scores<0>(k, i, q[i][0], qs[i], z);
            } else {
                scores<3>(k, i, q[i][3], qs[i], z);
                scores<2>(k, i, q[i][2], qs[i], z);
                scores<1>(k, i, q[i][1], qs[i], z);
                scores<0>(k, i, q[i][0], qs[i], z);
            }
        }
        fetch_k(at, at_j, k);
        uint4 scale = v.scale;
        const bool dead = !(there >> g & 1);
        if (edge) {
            asm volatile("");       // a branch: as selections this would be worked out for every step
            scale = keep_scales(scale, w.any_lo - tok0, dead ? 0 : min(w.any_hi, w.part_hi) - tok0);
        }
        const uint32_t b[4] = {scale.x, scale.y, scale.z, scale.w};
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) z[t][i] = fmaf(z[t][i], w.factor, exponent_of(b[t] ^ 0x80808080u, i));
        if (edge) {
            asm volatile("");
            const int lo = w.see.lo - tok0, hi = dead ? 0 : min(w.see.hi, w.part_hi) - tok0;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) z[t][i] = 4 * t + i >= lo && 4 * t + i < hi ? z[t][i] : -INFINITY;
        }
        float s = fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3]));
#pragma unroll
        for (int t = 1; t < 4; ++t) s = fmaxf(fmaxf(s, fmaxf(z[t][0], z[t][1])), fmaxf(z[t][2], z[t][3]));
        s = max_quarters(s);
        if (__any(s - m > REACH)) {     // as in step4
            const float up = fmaxf(m, s - LIFT), f = up == -INFINITY ? 1.f : exp2f(m - up);
            l = up == -INFINITY ? l : times_two_to(l, m - up);
#pragma unroll
            for (int i = 0; i < D / 16; ++i) o[i] *= f;
            m = up;
        }
        const float base = m == -INFINITY ? 0.f : m;
        v8h p[2];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = __builtin_amdgcn_exp2f(z[t][i] - base);
                l = fmaf(e, inverse_of(~b[t], i), l);
                p[t / 2][4 * (t % 2) + i] = (_Float16)e;
            }
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            o[2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(e2m1_to_half(v.v[i].x), p[0], o[2 * i], 0, 0, 0);
            o[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(e2m1_to_half(v.v[i].z), p[0], o[2 * i + 1], 0, 0, 0);
            o[2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(e2m1_to_half(v.v[i].y), p[1], o[2 * i], 0, 0, 0);
            o[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(e2m1_to_half(v.v[i].w), p[1], o[2 * i + 1], 0, 0, 0);
        }
        fetch_v(at, at_j, v);
    }

    // One item; k, v: its first step's, on their way, and then the next item's (`after`).
    __device__ __forceinline__ void item(const Item &it, Ahead4<D> &x, const Item &next, bool more, Ahead4<D> &after, Keys &k, Values &v) const
    {
        const int tid = threadIdx.x, heads = a.c.kv_heads, rows = it.n_new * a.group;
        const Row row = row_at(a, 0, col, rows);
        uint32_t top[BLOCKS], largest = 0;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            top[i] = 0;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                x.q[i][j] = row.real ? x.q[i][j] : 0;
                top[i] = max(top[i], max(size_bits(from_bits<DTYPE>(x.q[i][j] & 0xFFFF)), size_bits(from_bits<DTYPE>(x.q[i][j] >> 16))));
            }
            largest = max(largest, top[i]);
        }
        largest = max(largest, (uint32_t)__shfl_xor((int)largest, 16));
        largest = max(largest, (uint32_t)__shfl_xor((int)largest, 32));
        const int exponent = max((int)(largest >> 23), 1);
        v6u q[BLOCKS][PASSES];
        int qs[BLOCKS];
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            float y[32];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                y[2 * j] = from_bits<DTYPE>(x.q[i][j] & 0xFFFF);
                y[2 * j + 1] = from_bits<DTYPE>(x.q[i][j] >> 16);
            }
            const Digits d = digits_of(y, top[i], exponent);
            if constexpr (D == 64) {
                q[i][0] = g & 2 ? d.d[1] : d.d[0];
                q[i][1] = g & 2 ? d.d[3] : d.d[2];
                qs[i] = g & 2 ? (int)((uint32_t)d.scale >> 8) : d.scale;       // bytes 0 and 2 are used
            } else {
#pragma unroll
                for (int p = 0; p < DIGITS; ++p) q[i][p] = d.d[p];
                qs[i] = d.scale;
            }
        }
        const float factor = largest >= NO_NUMBER ? __builtin_nanf("") : a.q.scale * LOG2E * ldexpf(1.f, exponent - 127 - 14);
        const int any_hi = it.ctx + it.n_new, part_hi = it.kt1 * KT;
        const int any_lo = a.window > 0 ? max(0, it.ctx + 1 - a.window) : 0;
        const int all_lo = a.window > 0 ? max(0, any_hi - a.window) : 0, all_hi = min(part_hi, a.causal ? it.ctx + 1 : any_hi);
        const Walk w{sees(a, it, row), factor, any_lo, any_hi, all_lo, all_hi, part_hi};

        v4f o[D / 16];
#pragma unroll
        for (int n = 0; n < D / 16; ++n) o[n] = v4f{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;
        const int all = steps(it);
        place(next, wave, after);
        for (int first = wave; first < all; first += DECODE_WAVES * BATCH) {
            if (first != wave) {
                x.id = table(it, first);
                place(it, first, x);
                fetch_k(x.at, 0, k);
                fetch_v(x.at, 0, v);
            }
            const int n = min(BATCH, div_up(all - first, DECODE_WAVES));
            const bool on = more && first + DECODE_WAVES * BATCH >= all;
            const uint32_t here = x.at, next_at = after.at;
            const uint64_t in_cache = x.there;
            for (int j = 0; j < n; ++j) step(w, q, qs, j, n, it.kt0 * KT + (first + DECODE_WAVES * j) * 64, here, in_cache, on, next_at, k, v, o, m, l);
        }
        if (more && all <= wave) {  // a wave without a step of this item
            fetch_k(after.at, 0, k);
            fetch_v(after.at, 0, v);
        }
        if (more) queries(next, after);

        // join the waves
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (g == 0) {
            sh.m[wave][col] = m;
            sh.l[wave][col] = l;
        }
        __syncthreads();
        float high = -INFINITY;
#pragma unroll
        for (int w = 0; w < DECODE_WAVES; ++w) high = fmaxf(high, sh.m[w][col]);
        const float base = high == -INFINITY ? 0.f : high;
        l = sum_of_waves(sh.m, sh.l, col, base);
        float f = exp2f(m - base);
        const bool whole = it.part < 0;
        if (whole) f = l == 0.f ? 0.f : f / l;
        const int64_t part = ((int64_t)it.part * heads + head) * ROWS_FEW;
        if (tid < ROWS_DECODE && row.real) {
            if (!whole) put2(ml() + (part + tid) * 2, high, l);
            else if (a.q.lse) a.q.lse[(int64_t)(it.row0 + row.tok) * heads * a.group + head * a.group + row.g] = LN2 * (high + log2f(l));
        }
        constexpr int STRIDE = D + 4, HOLD = 8, QUADS = D / 4;
        for (int r0 = 0; r0 < rows; r0 += HOLD) {
            if (r0) __syncthreads();
            if (col >= r0 && col < min(r0 + HOLD, rows)) {
#pragma unroll
                for (int i = 0; i < D / 32; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        *reinterpret_cast<float4 *>(sh.o + (wave * HOLD + col - r0) * STRIDE + 32 * i + 8 * g + 4 * e) =
                            make_float4(o[2 * i][2 * e] * f, o[2 * i + 1][2 * e] * f, o[2 * i][2 * e + 1] * f, o[2 * i + 1][2 * e + 1] * f);
            }
            __syncthreads();
            for (int e = tid; e < min(HOLD, rows - r0) * QUADS; e += 64 * DECODE_WAVES) {
                const int r = e / QUADS, d = (e % QUADS) * 4;
                float4 y = *reinterpret_cast<const float4 *>(sh.o + r * STRIDE + d);
#pragma unroll
                for (int w = 1; w < DECODE_WAVES; ++w) {
                    const float4 u = *reinterpret_cast<const float4 *>(sh.o + (w * HOLD + r) * STRIDE + d);
                    y.x += u.x;
                    y.y += u.y;
                    y.z += u.z;
                    y.w += u.w;
                }
                if (whole) {
                    const Row out = row_at(a, 0, r0 + r, rows);
                    store4<DTYPE>(a.q.out, (it.row0 + out.tok) * a.q.out_stride + (int64_t)(head * a.group + out.g) * D + d, a.vec_out, y.x, y.y, y.z, y.w);
                } else {
                    float *p = a.part_few + (part + r0 + r) * D + d;
                    put2(p, y.x, y.y);
                    put2(p + 2, y.z, y.w);
                }
            }
        }
    }

    __device__ __forceinline__ void join(const Item &it) const
    {
        if (all_parts_done(a.p.joins_few + it.join * a.c.kv_heads + head, it.parts, sh.join.last)) join4<DTYPE, D>(a, it, head, ml(), sh.join);
    }
};

template <int DTYPE, int D>
__global__ void __launch_bounds__(64 * DECODE_WAVES, decode_blocks(D)) k_kv4_decode(AttendArgs a)
{
    __shared__ Decode4Shared<D> sh;
    const int i = blockIdx.x / a.c.kv_heads;
    const int first = a.p.few_first[i], last = a.p.few_first[i + 1] - 1;
    if (i >= a.p.head->few_blocks) return;
    const Decode4<DTYPE, D> d{a, sh, (int)blockIdx.x - i * a.c.kv_heads};
    // The next item's way to its cached tokens (item, table and first step) goes on while this one is worked on.
    Item it = item_at(a.p.few + first), next = item_at(a.p.few + min(first + 1, last));
    Ahead4<D> x, after;
    x.id = d.table(it, d.wave);
    after.id = d.table(next, d.wave);
    d.queries(it, x);
    d.place(it, d.wave, x);
    typename Decode4<DTYPE, D>::Keys k;
    typename Decode4<DTYPE, D>::Values v;
    d.fetch_k(x.at, 0, k);
    d.fetch_v(x.at, 0, v);
    // Only a block's first and last item can have parts in other blocks: both are counted at the end, where the stores' way to
    // memory is waited for once.
    Item split = it;
    for (int n = first;; ++n) {
        uint4 third[3];           // not looked at before this item is done: a look would wait for it
#pragma unroll
        for (int u = 0; u < 3; ++u) third[u] = reinterpret_cast<const uint4 *>(a.p.few + min(n + 2, last))[u];
        d.item(it, x, next, n < last, after, k, v);
        if (n == last) break;
        it = next;
        next = item_of(third);
        x = after;
        after.id = d.table(next, d.wave);
        __syncthreads();          // the item before is done with LDS
    }
#pragma nounroll
    for (int u = first != last ? 0 : 1; u < 2; ++u) {
        const Item joined = u ? it : split;
        if (joined.part >= 0) d.join(joined);
        __syncthreads();          // done with LDS
    }
}

}  // namespace kv
}  // namespace moe
