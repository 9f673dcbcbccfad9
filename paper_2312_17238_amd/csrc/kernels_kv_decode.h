// Attention of steps whose requests bring no more than sixteen (token, query head of the group) rows each: single tokens, and a few
// drafted ones where the group is small.
//
// Memory is the bound (two bytes of cache for 4 x group operations a dim), and what stands in its way is latency: a block's first
// loads wait for its item, then for the block table, then for the scales, 2 to 5 us under load.  So a row's state is kept small, sixteen rows
// instead of the general kernel's thirty-two (16x16x32 instructions: half the outputs, scores and queries in registers), keys
// and values are requested anew as soon as they are used, and the next item's way to its tokens goes on under this one's work.
// D = 128, eight kv heads: one token over 131000 50 to 52 us by the machine (268 MB, 5.2 TB/s; a plain read of as much 43.7), 64 requests over 500 to 8000
// 69 (338 MB, 4.9 TB/s; 56.9).  The general kernel takes 53.8 and 73.6 for these, 9.4 instead of 7.4 for one over 700, 65 instead of 35 for one
// over 60000 with heads of 256.  The roles of lanes and tiles are those of kernels_kv_attend.h with four lane quarters for
// its two halves: row m of tile t of the scores stands for token 16 (m / 4) + 4 t + m % 4 of a step of 64, so that a lane of
// quarter g holds the scores of sub-block g in the order in which its sixteen bytes of a value tile hold their codes.
#pragma once
#include "kernels_kv_attend.h"

namespace moe {
namespace kv {

typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int ROWS_DECODE = 16;
constexpr int DECODE_WAVES = 4;

// Blocks of a compute unit, by their registers.  D = 128, one over 131000 and 64 over 500 to 8000: with one block 47 and 72 us, two 49
// and 69 (as they then were), three (fewer registers: an item's loads no longer ahead) 67 and 92.  D = 64: with two 29.9 and 42.5, three (whose registers spill) 36.9
// and 46.2, 512 over 300 39.1 and 50.9; D = 256 has registers for one.
__host__ __device__ constexpr int decode_blocks(int head_dim) { return head_dim <= 128 ? 2 : 1; }

template <int D>
struct DecodeShared {
    float m[DECODE_WAVES][ROWS_DECODE], l[DECODE_WAVES][ROWS_DECODE];
    __align__(16) float o[DECODE_WAVES * 8 * (D + 4)];
    JoinShared join;
};

// The largest of the four quarters' numbers of a row, in all four.
__device__ __forceinline__ float max_quarters(float x)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return max_halves(fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1])));
}

// One wave's view of an item: where the sub-blocks of its first sixteen steps lie (in units of sub-blocks of all pages and
// heads; a step of the wave is four sub-blocks, a lane holds one), their scales (ks = 0: nowhere) and its rows' queries as they are.
template <int D>
struct Ahead {
    int id;             // page, as the table has it; -1 beyond what the part has
    uint32_t at;
    float ks, vs;
    uint32_t q[D / 8];
};

template <int DTYPE, int FMT, int D>
struct Decode {
    const AttendArgs &a;
    DecodeShared<D> &sh;
    const int head, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
    static constexpr int BATCH = 16;

    __device__ __forceinline__ static int steps(const Item &it) { return div_up(it.kt1 - it.kt0, 2); }

    __device__ __forceinline__ int table(const Item &it, int first) const
    {
        const int s = first + DECODE_WAVES * (lane >> 2), sub = 2 * it.kt0 + 4 * s + (lane & 3), blk = sub >> a.sub_shift;
        if (s >= steps(it) || sub * SUB >= min(it.ctx + it.n_new, it.kt1 * KT) || blk >= a.max_blocks) return -1;
        return a.table[(int64_t)it.req * a.max_blocks + blk];
    }

    __device__ __forceinline__ void place(const Item &it, int first, Ahead<D> &x) const
    {
        const int s = first + DECODE_WAVES * (lane >> 2), sub = 2 * it.kt0 + 4 * s + (lane & 3);
        const bool good = (unsigned)x.id < (unsigned)a.c.n_pages;
        const uint32_t p = (uint32_t)(good ? x.id : 0) * a.c.kv_heads + head;
        x.at = (p << a.sub_shift) + (sub & ((1 << a.sub_shift) - 1));
    }

    __device__ __forceinline__ void scales(Ahead<D> &x) const
    {
        const uint32_t p = (uint32_t)((unsigned)x.id < (unsigned)a.c.n_pages ? x.id : 0) * a.c.kv_heads + head;
        x.ks = a.c.k_scale[p];
        x.vs = a.c.v_scale[p];
    }
    // ... and once they are there, as they are used
    __device__ __forceinline__ void settle(Ahead<D> &x) const
    {
        const bool good = (unsigned)x.id < (unsigned)a.c.n_pages;
        x.ks = good ? fmaxf(x.ks, LEAST_SCALE) : 0.f;
        x.vs = good ? fmaxf(x.vs, LEAST_SCALE) : 1.f;
    }

    __device__ __forceinline__ void queries(const Item &it, Ahead<D> &x) const
    {
        const Row row = row_at(a, 0, col, it.n_new * a.group);
        const uint16_t *src = static_cast<const uint16_t *>(a.q.q) + (it.row0 + (row.real ? row.tok : 0)) * a.q.q_stride + (int64_t)(head * a.group + (row.real ? row.g : 0)) * D;
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            const uint16_t *p = src + 16 * (4 * i + g);
            if (a.vec_q) {
                const uint4 u = reinterpret_cast<const uint4 *>(p)[0], v = reinterpret_cast<const uint4 *>(p)[1];
                x.q[8 * i] = u.x; x.q[8 * i + 1] = u.y; x.q[8 * i + 2] = u.z; x.q[8 * i + 3] = u.w;
                x.q[8 * i + 4] = v.x; x.q[8 * i + 5] = v.y; x.q[8 * i + 6] = v.z; x.q[8 * i + 7] = v.w;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) x.q[8 * i + j] = p[2 * j] | ((uint32_t)p[2 * j + 1] << 16);
            }
        }
    }

    // keys and values of the step whose four sub-blocks the lanes 4 j .. 4 j + 3 hold
    __device__ __forceinline__ void fetch_k(uint32_t at, int j, uint4 (&k)[4][D / 64]) const
    {
        const uint8_t *p = static_cast<const uint8_t *>(a.c.k) + g * 256 + (col & 3) * 16 + (uint64_t)__shfl(at, 4 * j + (col >> 2)) * (SUB * D);
#pragma unroll
        for (int i = 0; i < D / 64; ++i)
#pragma unroll
            for (int t = 0; t < 4; ++t) k[t][i] = *reinterpret_cast<const uint4 *>(p + i * 1024 + t * 64);
    }
    __device__ __forceinline__ void fetch_v(uint32_t at, int j, uint4 (&v)[D / 16]) const
    {
        const uint8_t *p = static_cast<const uint8_t *>(a.c.v) + col * 16 + (uint64_t)__shfl(at, 4 * j + g) * (SUB * D);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) v[i] = *reinterpret_cast<const uint4 *>(p + i * 256);
    }

    __device__ __forceinline__ float *ml() const { return a.part_few + (int64_t)a.p.parts_few * a.c.kv_heads * ROWS_FEW * D; }

    // One item; k, v: its first step's, on their way, and then the next item's (`after`).
    __device__ __forceinline__ void item(const Item &it, Ahead<D> &x, const Item &next, bool more, Ahead<D> &after, uint4 (&k)[4][D / 64], uint4 (&v)[D / 16]) const
    {
        const int tid = threadIdx.x, heads = a.c.kv_heads, rows = it.n_new * a.group;
        const Row row = row_at(a, 0, col, rows);
        // queries as the second operand: k-slot (step 2i + c, quarter g, j) is dim 16 (4i + g) + 8 c + j
        v8h q[D / 32];
        float unit = 1.f, by = 1.f;
        if constexpr (DTYPE == MOE_KV_BF16) {
            uint32_t top = 0;       // the row's largest exponent, to that of 2^14
#pragma unroll
            for (int i = 0; i < D / 8; ++i) top = max(top, max(x.q[i] & 0x7F80, (x.q[i] >> 16) & 0x7F80));
            top = max(top, (uint32_t)__shfl_xor((int)top, 16));
            top = max(top, (uint32_t)__shfl_xor((int)top, 32));
            const int e = max((int)(top >> 7) - 127 - 14, -100);
            by = ldexpf(1.f, -e);
            unit = ldexpf(1.f, e);
        }
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t u = row.real ? x.q[4 * i + j] : 0;
                if constexpr (DTYPE == MOE_KV_F16) {
                    const v2h p = __builtin_bit_cast(v2h, u);
                    q[i][2 * j] = p.x;
                    q[i][2 * j + 1] = p.y;
                } else {
                    q[i][2 * j] = (_Float16)(from_bits<DTYPE>(u & 0xFFFF) * by);
                    q[i][2 * j + 1] = (_Float16)(from_bits<DTYPE>(u >> 16) * by);
                }
            }
        const Sees see = sees(a, it, row);
        const float factor = a.q.scale * LOG2E * unit;
        const int any_hi = it.ctx + it.n_new, part_hi = it.kt1 * KT;
        const int any_lo = a.window > 0 ? max(0, it.ctx + 1 - a.window) : 0;
        const int all_lo = a.window > 0 ? max(0, any_hi - a.window) : 0, all_hi = min(part_hi, a.causal ? it.ctx + 1 : any_hi);

        v4f o[D / 16];
#pragma unroll
        for (int n = 0; n < D / 16; ++n) o[n] = v4f{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;
        bool rare = false;          // as in steps()
        const int all = steps(it);
        settle(x);
        place(next, wave, after);
        for (int first = wave; first < all; first += DECODE_WAVES * BATCH) {
            if (first != wave) {
                x.id = table(it, first);
                place(it, first, x);
                scales(x);
                fetch_k(x.at, 0, k);
                fetch_v(x.at, 0, v);
                settle(x);
            }
            const int n = min(BATCH, div_up(all - first, DECODE_WAVES));
            const bool on = more && first + DECODE_WAVES * BATCH >= all;
            for (int j = 0; j < n; ++j) {
                // no branch around a load: behind the last step the next item's first one is requested, or the same step
                // again, which the caches still hold
                const uint32_t at = j + 1 < n || !on ? x.at : after.at;
                const int at_j = j + 1 < n ? j + 1 : on ? 0 : j;
                const int tok = it.kt0 * KT + (first + DECODE_WAVES * j) * 64, tok0 = tok + SUB * g;
                const float ks = __shfl(x.ks, 4 * j + g), vs = __shfl(x.vs, 4 * j + g);
                const bool dead = ks == 0.f;
                const bool edge = tok < all_lo || tok + 64 > all_hi || __any(dead);
                v4f z[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) z[t] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < D / 64; ++i) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) z[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_half<FMT>(k[t][i].x, k[t][i].y), q[2 * i], z[t], 0, 0, 0);
#pragma unroll
                    for (int t = 0; t < 4; ++t) z[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_half<FMT>(k[t][i].z, k[t][i].w), q[2 * i + 1], z[t], 0, 0, 0);
                }
                fetch_k(at, at_j, k);
                if (edge) {
                    const int lo = see.lo - tok0, hi = dead ? 0 : min(see.hi, part_hi) - tok0;
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) z[t][i] = 4 * t + i >= lo && 4 * t + i < hi ? z[t][i] : -INFINITY;
                }
                const float sc = dead ? 1.f : factor * ks, lv = __builtin_amdgcn_logf(vs);
                float top = fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3]));
#pragma unroll
                for (int t = 1; t < 4; ++t) top = fmaxf(fmaxf(top, fmaxf(z[t][0], z[t][1])), fmaxf(z[t][2], z[t][3]));
                const float s = max_quarters(fmaf(top, sc, lv));
                if (__any(s > m + RISE)) {
                    const float up = fmaxf(m, s), f = up == -INFINITY ? 1.f : exp2f(m - up);
                    l = up == -INFINITY ? l : times_two_to(l, m - up);
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) o[i] *= f;
                    m = up;
                    rare |= __any(beyond_big(m));
                }
                const float off = lv - (m == -INFINITY ? 0.f : m);
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[t][i] = fmaf(z[t][i], sc, off);
                float iv = __builtin_amdgcn_rcpf(vs);
                // the batch's scales are looked at behind its first product, which does not wait for them
                if (j == 0) rare |= __any(fabsf(__builtin_amdgcn_logf(x.vs)) > WIDE);
                if (rare) {
                    iv = 0.f;
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            z[t][i] = z[t][i] > RISE ? RISE : z[t][i];
                            l += __builtin_amdgcn_exp2f(z[t][i] - lv);
                        }
                }
                v8h p[2];
                float sum = 0.f;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float e = __builtin_amdgcn_exp2f(z[t][i]);
                        sum += e;
                        p[t / 2][4 * (t % 2) + i] = (_Float16)e;
                    }
                l = fmaf(sum, iv, l);
                if (edge) {
                    const int lo = any_lo - tok0, hi = dead ? 0 : min(any_hi, part_hi) - tok0;
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) v[i] = keep_bytes(v[i], lo, hi);
                }
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    o[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_half<FMT>(v[i].x, v[i].y), p[0], o[i], 0, 0, 0);
                    o[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_half<FMT>(v[i].z, v[i].w), p[1], o[i], 0, 0, 0);
                }
                fetch_v(at, at_j, v);
            }
        }
        if (more && all <= wave) {  // a wave without a step of this item
            fetch_k(after.at, 0, k);
            fetch_v(after.at, 0, v);
        }
        if (more) {
            scales(after);
            queries(next, after);
        }

        // join the waves
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (g == 0) {
            sh.m[wave][col] = m;
            sh.l[wave][col] = l;
        }
        __syncthreads();
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < DECODE_WAVES; ++w) top = fmaxf(top, sh.m[w][col]);
        const float base = top == -INFINITY ? 0.f : top;
        l = sum_of_waves(sh.m, sh.l, col, base);
        float f = exp2f(m - base);
        const bool whole = it.part < 0;
        if (whole) f = l == 0.f ? 0.f : f / l;
        const int64_t part = ((int64_t)it.part * heads + head) * ROWS_FEW;
        if (tid < ROWS_DECODE && row.real) {
            if (!whole) put2(ml() + (part + tid) * 2, top, l);
            else if (a.q.lse) a.q.lse[(int64_t)(it.row0 + row.tok) * heads * a.group + head * a.group + row.g] = LN2 * (top + log2f(l));
        }
        constexpr int STRIDE = D + 4, HOLD = 8, QUADS = D / 4;
        for (int r0 = 0; r0 < rows; r0 += HOLD) {
            if (r0) __syncthreads();
            if (col >= r0 && col < min(r0 + HOLD, rows)) {
#pragma unroll
                for (int n = 0; n < D / 16; ++n)
                    *reinterpret_cast<float4 *>(sh.o + (wave * HOLD + col - r0) * STRIDE + 16 * n + 4 * g) = make_float4(o[n][0] * f, o[n][1] * f, o[n][2] * f, o[n][3] * f);
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
        if (all_parts_done(a.p.joins_few + it.join * a.c.kv_heads + head, it.parts, sh.join)) join_parts<DTYPE, D>(a, it, head, a.part_few, ml(), ROWS_FEW, sh.join);
    }
};

template <int DTYPE, int FMT, int D>
__global__ void __launch_bounds__(64 * DECODE_WAVES, decode_blocks(D)) k_kv_decode(AttendArgs a)
{
    __shared__ DecodeShared<D> sh;
    const int i = blockIdx.x / a.c.kv_heads;
    const int first = a.p.few_first[i], last = a.p.few_first[i + 1] - 1;
    if (i >= a.p.head->few_blocks) return;
    const Decode<DTYPE, FMT, D> d{a, sh, (int)blockIdx.x - i * a.c.kv_heads};
    // The next item's way to its cached tokens (item, table, scales and first step) goes on while this one is worked on.
    Item it = item_at(a.p.few + first), next = item_at(a.p.few + min(first + 1, last));
    Ahead<D> x, after;
    x.id = d.table(it, d.wave);
    after.id = d.table(next, d.wave);
    d.place(it, d.wave, x);
    uint4 k[4][D / 64], v[D / 16];
    d.fetch_k(x.at, 0, k);
    d.fetch_v(x.at, 0, v);
    d.scales(x);
    d.queries(it, x);
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
    if (first != last && split.part >= 0) d.join(split);
    if (it.part >= 0) d.join(it);
}

}  // namespace kv
}  // namespace moe
