// Attention of a step's rows over the paged 8-bit cache.
//
// A row is a (token, query head) pair of one kv head's group, so that all that read the same keys share them.  Both products run on
// 32x32x16 fp16 matrix instructions with the cached tokens as rows and the queries as columns:
//   S^T[32 tokens x 32 rows]  = K[32 x D] Q^T[D x 32],        O^T[D x 32 rows] += V^T[D x 32 tokens] P^T[32 x 32 rows].
// Codes of either format are exact in fp16, and the cache's tiles are laid out as the instructions read them: a lane's 16
// bytes of a key tile are 16 dims of a token, of a value tile 16 tokens of a dim, and a wave's loads are contiguous.  Row m of S^T stands for token
// 16 h + 4 a + b of the step (m = 8 a + 4 h + b): then the sixteen scores that lane (h, row) holds are those of the sixteen tokens
// of sub-block h, in order, which is the order in which the value tile gives that lane its sixteen codes.  The probabilities go
// from the first product to the second in the lane's own registers.
//
// A lane's sixteen tokens lie in one page, hence under one scale each for keys and values.  With t = scale log2(e) ks (q.k) + log2(vs)
// the weight of a value's code is 2^(t - m), m the running maximum of t over the row: scales cost one multiply-add a score, and
// the weights stay below one whatever the scales are, as fp16 wants it.  The sum of the probabilities is that of the weights, divided by vs page by page,
// in fp32 as are scores, maxima and outputs.  Weights are rounded to fp16 (2^-12 of a weight, half of what an fp16 output is rounded
// by); bf16 queries become fp16 after a power of two is taken off each row.
#pragma once
#include "kernels_kv_common.h"

namespace moe {
namespace kv {

constexpr int ATTEND_THREADS = 256;
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

struct AttendArgs {
    moe_kv_cache_t c;
    moe_kv_query_t q;
    Plan p;
    const int32_t *table;
    float *part_few, *part_many;    // [part][kv head][rows][D] outputs, then [part][kv head][rows] (m, l)
    int32_t group, max_blocks, causal, window;
    int32_t sub_shift;              // log2 of a page's sub-blocks
    int32_t many_blocks;            // blocks of the grid that take tiles of 128 rows; the others take requests of few rows
    int32_t vec_q, vec_out;
};

// What a row sees: tokens [lo, hi).
struct Sees {
    int lo, hi;
};

__device__ __forceinline__ Sees sees(const AttendArgs &a, const Item &it, int row, int rows)
{
    if (row >= rows) return {0, 0};
    const int pos = it.ctx + row / a.group;
    return {a.window > 0 ? max(0, pos + 1 - a.window) : 0, a.causal ? pos + 1 : it.ctx + it.n_new};
}

// A row's state between steps.
template <int D>
struct State {
    v16f o[D / 32];     // O^T: column is the lane's row, rows are dims 32 n + 8 (i/4) + 4 h + i%4
    float m, l;
    bool big;           // of any row of the wave: |m| is so large that fp32's steps there matter to an exponent
};

template <int D>
__device__ __forceinline__ void clear(State<D> &s)
{
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) s.o[n][i] = 0.f;
    s.m = -INFINITY;
    s.l = 0.f;
    s.big = false;
}

// Queries of 32 rows as the second operand of the first product.  k-slot (step 2i + c, lane half h, j) stands for dim
// 16 (2i + h) + 8 c + j, as the key tiles have it.  unit: what the scores have to be multiplied with.
template <int DTYPE, int D>
__device__ __forceinline__ void load_queries(const AttendArgs &a, const Item &it, int head, int row, int rows, v8h (&q)[D / 16], float &unit)
{
    const int h = (threadIdx.x >> 5) & 1;
    const bool real = row < rows;
    const int tok = real ? row / a.group : 0, g = real ? row - tok * a.group : 0;
    const uint16_t *src = static_cast<const uint16_t *>(a.q.q) + (it.row0 + tok) * a.q.q_stride + (int64_t)(head * a.group + g) * D;
    uint32_t w[D / 4];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        const uint16_t *p = src + 16 * (2 * i + h);
        if (!real) {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[8 * i + j] = 0;
        } else if (a.vec_q) {
            const uint4 u = reinterpret_cast<const uint4 *>(p)[0], v = reinterpret_cast<const uint4 *>(p)[1];
            w[8 * i] = u.x; w[8 * i + 1] = u.y; w[8 * i + 2] = u.z; w[8 * i + 3] = u.w;
            w[8 * i + 4] = v.x; w[8 * i + 5] = v.y; w[8 * i + 6] = v.z; w[8 * i + 7] = v.w;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[8 * i + j] = p[2 * j] | ((uint32_t)p[2 * j + 1] << 16);
        }
    }
    float by = 1.f;
    if constexpr (DTYPE == MOE_KV_BF16) {
        // the row's largest exponent to that of 2^14
#pragma unroll
        for (int i = 0; i < D / 4; ++i) top = max(top, max(w[i] & 0x7F80, (w[i] >> 16) & 0x7F80));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        const int e = min(max((int)(top >> 7) - 127 - 14, -100), 100);
        by = ldexpf(1.f, -e);
        unit = ldexpf(1.f, e);
    } else {
        unit = 1.f;
    }
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t u = w[4 * i + j];
            if constexpr (DTYPE == MOE_KV_F16) {
                const v2h p = __builtin_bit_cast(v2h, u);
                q[i][2 * j] = p.x;
                q[i][2 * j + 1] = p.y;
            } else {
                q[i][2 * j] = (_Float16)(from_bits<DTYPE>(u & 0xFFFF) * by);
                q[i][2 * j + 1] = (_Float16)(from_bits<DTYPE>(u >> 16) * by);
            }
        }
}

// Bytes [lo, hi) of a lane's sixteen, the others 0.
__device__ __forceinline__ uint64_t low_bytes(int n) { return n >= 8 ? ~0ull : n <= 0 ? 0ull : (1ull << (8 * n)) - 1; }

__device__ __forceinline__ uint4 keep_bytes(uint4 v, int lo, int hi)
{
    const uint64_t a = low_bytes(hi) & ~low_bytes(lo), b = low_bytes(hi - 8) & ~low_bytes(lo - 8);
    return make_uint4(v.x & (uint32_t)a, v.y & (uint32_t)(a >> 32), v.z & (uint32_t)b, v.w & (uint32_t)(b >> 32));
}

// One step: 32 cached tokens against 32 rows.  k, v: the lane's pieces of the two tiles.  sc: scale log2(e) ks of the lane's
// sub-block, lv: log2 vs, iv: 1 / vs.  edge: some row does not see some token of the step.
template <int FMT, int D>
__device__ __forceinline__ void step(State<D> &s, const v8h (&q)[D / 16], const uint4 (&k)[D / 32], const uint4 (&v)[D / 32],
                                     float sc, float lv, float iv, bool edge, int tok0, Sees see)
{
    v16f z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        z = __builtin_amdgcn_mfma_f32_32x32x16_f16(codes_to_half<FMT>(k[i].x, k[i].y), q[2 * i], z, 0, 0, 0);
        z = __builtin_amdgcn_mfma_f32_32x32x16_f16(codes_to_half<FMT>(k[i].z, k[i].w), q[2 * i + 1], z, 0, 0, 0);
    }
    if (edge) {
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = tok0 + i >= see.lo && tok0 + i < see.hi ? z[i] : -INFINITY;
    }
    float top = z[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, z[i]);
    float t = fmaf(top, sc, lv);
    t = fmaxf(t, __shfl_xor(t, 32));
    if (__any(t > s.m)) {
        const float m = fmaxf(s.m, t);
        const float f = m == -INFINITY ? 1.f : exp2f(s.m - m);
        s.l *= f;
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) s.o[n][i] *= f;
        s.m = m;
        s.big = __any(fabsf(m) > 0x1p20f && fabsf(m) < INFINITY);
    }
    const float off = lv - (s.m == -INFINITY ? 0.f : s.m);
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = fmaf(z[i], sc, off);
    // m is a rounded t, these are not: beyond 2^20 the difference shows as a weight above 1, at 2^28 one that fp16 does not hold
    if (s.big) {
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = z[i] > 0.f ? 0.f : z[i];
    }
    v8h p[2];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float e = __builtin_amdgcn_exp2f(z[i]);
        sum += e;
        p[i / 8][i % 8] = (_Float16)e;
    }
    s.l = fmaf(sum, iv, s.l);
#pragma unroll
    for (int n = 0; n < D / 32; ++n) {
        s.o[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(codes_to_half<FMT>(v[n].x, v[n].y), p[0], s.o[n], 0, 0, 0);
        s.o[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(codes_to_half<FMT>(v[n].z, v[n].w), p[1], s.o[n], 0, 0, 0);
    }
}

// Where a sub-block of sixteen tokens lies: its page (-1: not in the cache, or beyond what the request has) and scales.
struct Place {
    int id;
    float ks, vs;
};

__device__ __forceinline__ Place place_of(const AttendArgs &a, const Item &it, int head, int sub_block, int end_tok)
{
    Place p{-1, 1.f, 1.f};
    const int blk = sub_block >> a.sub_shift;
    if (sub_block * SUB < end_tok && blk < a.max_blocks) {
        const int id = a.table[(int64_t)it.req * a.max_blocks + blk];
        if ((unsigned)id < (unsigned)a.c.n_pages) {
            p.id = id;
            p.ks = fmaxf(a.c.k_scale[(int64_t)id * a.c.kv_heads + head], 0x1p-100f);
            p.vs = fmaxf(a.c.v_scale[(int64_t)id * a.c.kv_heads + head], 0x1p-100f);
        }
    }
    return p;
}

// Writes four neighbouring numbers of an output row.
template <int DTYPE>
__device__ __forceinline__ void store4(void *out, int64_t at, bool vec, float a, float b, float c, float d)
{
    uint16_t *p = static_cast<uint16_t *>(out) + at;
    if (vec) {
        *reinterpret_cast<uint2 *>(p) = make_uint2(pack2<DTYPE>(a, b), pack2<DTYPE>(c, d));
    } else {
        p[0] = (uint16_t)to_bits<DTYPE>(a);
        p[1] = (uint16_t)to_bits<DTYPE>(b);
        p[2] = (uint16_t)to_bits<DTYPE>(c);
        p[3] = (uint16_t)to_bits<DTYPE>(d);
    }
}

// ---- a request of few rows: every wave takes every fourth step of the block's, straight from memory into registers
template <int D>
struct FewShared {
    float m[4][ROWS_FEW], l[4][ROWS_FEW];
    float o[4][ROWS_FEW][33];
};

template <int DTYPE, int FMT, int D>
__device__ __forceinline__ void attend_few(const AttendArgs &a, const Item &it, int head, FewShared<D> &sh)
{
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 31, h = lane >> 5;
    const int rows = it.n_new * a.group;
    v8h q[D / 16];
    float unit;
    load_queries<DTYPE, D>(a, it, head, col, rows, q, unit);
    const Sees see = sees(a, it, col, rows);
    const float factor = a.q.scale * LOG2E * unit;
    // all rows see tokens [all_lo, all_hi); any row sees some of [any_lo, any_hi)
    const int any_lo = a.window > 0 ? max(0, it.ctx + 1 - a.window) : 0, any_hi = it.ctx + it.n_new;
    const int all_lo = a.window > 0 ? max(0, it.ctx + it.n_new - a.window) : 0, all_hi = a.causal ? it.ctx + 1 : any_hi;
    State<D> s;
    clear(s);

    const int sub_bytes = SUB * D, heads = a.c.kv_heads, subs = a.c.page / SUB;
    const int kh = (col >> 2) & 1, ktok = 4 * (col >> 3) + (col & 3);     // S^T row `col` is token 16 kh + ktok of the step
    const uint8_t *kbase = static_cast<const uint8_t *>(a.c.k), *vbase = static_cast<const uint8_t *>(a.c.v);
    constexpr int BATCH = 32;       // steps of a wave whose places the lanes hold, two sub-blocks a step
    for (int first = it.kt0 + wave; first < it.kt1; first += 4 * BATCH) {
        const int n = min(BATCH, (it.kt1 - first + 3) / 4);
        const Place mine = (lane >> 1) < n ? place_of(a, it, head, 2 * (first + 4 * (lane >> 1)) + (lane & 1), any_hi) : Place{-1, 1.f, 1.f};
        uint4 k[2][D / 32], v[2][D / 32];
        auto fetch = [&](int j, uint4 (&kk)[D / 32], uint4 (&vv)[D / 32]) {
            const int kt = first + 4 * j;
            const int id0 = max(__builtin_amdgcn_readlane(mine.id, 2 * j), 0), id1 = max(__builtin_amdgcn_readlane(mine.id, 2 * j + 1), 0);
            const int64_t at0 = (((int64_t)id0 * heads + head) * subs + ((2 * kt) & (subs - 1))) * sub_bytes;
            const int64_t at1 = (((int64_t)id1 * heads + head) * subs + ((2 * kt + 1) & (subs - 1))) * sub_bytes;
            const uint8_t *kp = kbase + (kh ? at1 : at0) + ktok * 16 + h * 256;
            const uint8_t *vp = vbase + (h ? at1 : at0) + col * 16;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) kk[i] = *reinterpret_cast<const uint4 *>(kp + i * 512);
#pragma unroll
            for (int i = 0; i < D / 32; ++i) vv[i] = *reinterpret_cast<const uint4 *>(vp + i * 512);
        };
        auto use = [&](int j, uint4 (&kk)[D / 32], uint4 (&vv)[D / 32]) {
            const int kt = first + 4 * j;
            const int src = 2 * j + h;
            const int id = __shfl(mine.id, src);
            const float ks = __shfl(mine.ks, src), vs = __shfl(mine.vs, src);
            const bool edge = kt * KT < all_lo || (kt + 1) * KT > all_hi || __any(id < 0);
            const int tok0 = kt * KT + SUB * h;
            Sees mask = see;
            if (edge) {
                if (id < 0) mask.hi = 0;
                const int lo = any_lo - tok0, hi = id < 0 ? 0 : any_hi - tok0;
#pragma unroll
                for (int i = 0; i < D / 32; ++i) vv[i] = keep_bytes(vv[i], lo, hi);
            }
            step<FMT, D>(s, q, kk, vv, factor * ks, __builtin_amdgcn_logf(vs), __builtin_amdgcn_rcpf(vs), edge, tok0, mask);
        };
        fetch(0, k[0], v[0]);
        for (int j = 0; j < n; j += 2) {
            if (j + 1 < n) fetch(j + 1, k[1], v[1]);
            use(j, k[0], v[0]);
            if (j + 1 < n) {
                if (j + 2 < n) fetch(j + 2, k[0], v[0]);
                use(j + 1, k[1], v[1]);
            }
        }
    }
    // join the waves
    s.l += __shfl_xor(s.l, 32);
    if (h == 0) {
        sh.m[wave][col] = s.m;
        sh.l[wave][col] = s.l;
    }
    __syncthreads();
    const float top = fmaxf(fmaxf(sh.m[0][col], sh.m[1][col]), fmaxf(sh.m[2][col], sh.m[3][col]));
    const float base = top == -INFINITY ? 0.f : top;
    float l = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) l += sh.l[w][col] * exp2f(sh.m[w][col] - base);
    float f = exp2f(s.m - base);
    const bool whole = it.part < 0;
    if (whole) f = l == 0.f ? 0.f : f / l;
    const int64_t part = ((int64_t)it.part * heads + head) * ROWS_FEW;
    if (tid < ROWS_FEW && tid < rows) {
        if (!whole) {
            float *ml = a.part_few + (int64_t)a.p.parts_few * heads * ROWS_FEW * D + (part + tid) * 2;
            ml[0] = top;
            ml[1] = l;
        } else if (a.q.lse) {
            a.q.lse[(int64_t)(it.row0 + tid / a.group) * heads * a.group + head * a.group + tid % a.group] = LN2 * (top + log2f(l));
        }
    }
#pragma unroll
    for (int n = 0; n < D / 32; ++n) {
        if (n) __syncthreads();
#pragma unroll
        for (int i = 0; i < 16; ++i) sh.o[wave][col][8 * (i / 4) + 4 * h + i % 4] = s.o[n][i] * f;
        __syncthreads();
        const int r = tid >> 3, d = (tid & 7) * 4;
        if (r < rows) {
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = (sh.o[0][r][d + i] + sh.o[1][r][d + i]) + (sh.o[2][r][d + i] + sh.o[3][r][d + i]);
            if (whole) {
                const int tok = r / a.group, g = r - tok * a.group;
                store4<DTYPE>(a.q.out, (it.row0 + tok) * a.q.out_stride + (int64_t)(head * a.group + g) * D + n * 32 + d, a.vec_out, x[0], x[1], x[2], x[3]);
            } else {
                *reinterpret_cast<float4 *>(a.part_few + (part + r) * D + n * 32 + d) = make_float4(x[0], x[1], x[2], x[3]);
            }
        }
    }
}

// ---- tiles of 128 rows: every wave has 32 of them, all waves share the block's steps through LDS, two steps at a time
template <int D>
struct ManyShared {
    static constexpr int PLACES = 256;      // sub-blocks whose places are known at a time
    uint4 k[2][4 * D], v[2][4 * D];         // [buffer][sub-block of the two steps][pieces]
    Place place[PLACES];
};

template <int DTYPE, int FMT, int D>
__device__ __forceinline__ void attend_many(const AttendArgs &a, const Item &it, int head, ManyShared<D> &sh)
{
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 31, h = lane >> 5;
    const int rows = it.n_new * a.group, row0 = it.tile * ROWS_MANY + wave * 32, row = row0 + col;
    v8h q[D / 16];
    float unit;
    load_queries<DTYPE, D>(a, it, head, row, rows, q, unit);
    const Sees see = sees(a, it, row, rows);
    const float factor = a.q.scale * LOG2E * unit;
    const int pos_a = it.ctx + min(row0, rows - 1) / a.group, pos_z = it.ctx + min(row0 + 31, rows - 1) / a.group;
    const int end = it.ctx + it.n_new;
    const int any_lo = a.window > 0 ? max(0, pos_a + 1 - a.window) : 0, any_hi = row0 >= rows ? 0 : a.causal ? pos_z + 1 : end;
    const int all_lo = a.window > 0 ? max(0, pos_z + 1 - a.window) : 0, all_hi = a.causal ? pos_a + 1 : end;
    // values before this one may lie in pages that the request has given back
    const int tile_lo = a.window > 0 ? max(0, it.ctx + it.tile * ROWS_MANY / a.group + 1 - a.window) : 0;
    State<D> s;
    clear(s);

    const int heads = a.c.kv_heads, subs = a.c.page / SUB;
    const int kh = (col >> 2) & 1, ktok = 4 * (col >> 3) + (col & 3);
    const uint4 *kbase = static_cast<const uint4 *>(a.c.k), *vbase = static_cast<const uint4 *>(a.c.v);
    constexpr int PER = 4 * D / ATTEND_THREADS;     // pieces of 16 bytes of a thread: two steps hold 4 D of each kind
    for (int batch = it.kt0; batch < it.kt1; batch += ManyShared<D>::PLACES / 2) {
        const int last = min(it.kt1, batch + ManyShared<D>::PLACES / 2);
        __syncthreads();
        for (int i = tid; i < 2 * (last - batch) + 2; i += ATTEND_THREADS)
            if (i < ManyShared<D>::PLACES) sh.place[i] = place_of(a, it, head, 2 * batch + i, end);
        __syncthreads();
        uint4 rk[PER], rv[PER];
        auto fetch = [&](int kt) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int piece = tid + i * ATTEND_THREADS, sb = piece / D, in = piece - sb * D;
                const int idx = 2 * (kt - batch) + sb;
                const int id = idx < ManyShared<D>::PLACES && kt + sb / 2 < last ? max(sh.place[idx].id, 0) : 0;
                const int64_t at = (((int64_t)id * heads + head) * subs + ((2 * kt + sb) & (subs - 1))) * D + in;
                rk[i] = kbase[at];
                rv[i] = vbase[at];
            }
        };
        auto put = [&](int buf) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                sh.k[buf][tid + i * ATTEND_THREADS] = rk[i];
                sh.v[buf][tid + i * ATTEND_THREADS] = rv[i];
            }
        };
        fetch(batch);
        put(0);
        __syncthreads();
        int buf = 0;
        for (int kt = batch; kt < last; kt += 2) {
            const bool more = kt + 2 < last;
            if (more) fetch(kt + 2);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int tok = (kt + u) * KT;
                if (kt + u < last && tok < any_hi && tok + KT > any_lo) {
                    const Place pl = sh.place[2 * (kt + u - batch) + h];
                    const bool edge = tok < all_lo || tok + KT > all_hi || __any(pl.id < 0);
                    uint4 kk[D / 32], vv[D / 32];
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) {
                        kk[i] = sh.k[buf][(2 * u + kh) * D + (2 * i + h) * 16 + ktok];
                        vv[i] = sh.v[buf][(2 * u + h) * D + i * 32 + col];
                    }
                    Sees mask = see;
                    if (edge) {
                        if (pl.id < 0) mask.hi = 0;
                        const int tok0 = tok + SUB * h, lo = tile_lo - tok0, hi = pl.id < 0 ? 0 : end - tok0;
#pragma unroll
                        for (int i = 0; i < D / 32; ++i) vv[i] = keep_bytes(vv[i], lo, hi);
                    }
                    step<FMT, D>(s, q, kk, vv, factor * pl.ks, __builtin_amdgcn_logf(pl.vs), __builtin_amdgcn_rcpf(pl.vs), edge, tok + SUB * h, mask);
                }
            }
            if (more) put(buf ^ 1);
            __syncthreads();
            buf ^= 1;
        }
    }
    s.l += __shfl_xor(s.l, 32);
    if (row >= rows) return;
    const bool whole = it.part < 0;
    const int tok = row / a.group, g = row - tok * a.group;
    const int64_t part = ((int64_t)it.part * heads + head) * ROWS_MANY + wave * 32 + col;
    const float f = whole ? (s.l == 0.f ? 0.f : 1.f / s.l) : 1.f;
    const int64_t out = (it.row0 + tok) * a.q.out_stride + (int64_t)(head * a.group + g) * D;
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = 32 * n + 8 * i + 4 * h;
            const float x = s.o[n][4 * i] * f, y = s.o[n][4 * i + 1] * f, z = s.o[n][4 * i + 2] * f, w = s.o[n][4 * i + 3] * f;
            if (whole) store4<DTYPE>(a.q.out, out + d, a.vec_out, x, y, z, w);
            else *reinterpret_cast<float4 *>(a.part_many + part * D + d) = make_float4(x, y, z, w);
        }
    if (h == 0) {
        if (!whole) {
            float *ml = a.part_many + (int64_t)a.p.parts_many * heads * ROWS_MANY * D + part * 2;
            ml[0] = s.m;
            ml[1] = s.l;
        } else if (a.q.lse) {
            a.q.lse[(int64_t)(it.row0 + tok) * heads * a.group + head * a.group + g] = s.l == 0.f ? -INFINITY : LN2 * (s.m + log2f(s.l));
        }
    }
}

template <int DTYPE, int FMT, int D>
__global__ void __launch_bounds__(ATTEND_THREADS, D <= 128 ? 2 : 1) k_kv_attend(AttendArgs a)
{
    __shared__ union {
        FewShared<D> few;
        ManyShared<D> many;
    } sh;
    const int heads = a.c.kv_heads;
    if ((int)blockIdx.x < a.many_blocks) {
        const int i = blockIdx.x / heads;
        if (i >= a.p.head->many) return;
        attend_many<DTYPE, FMT, D>(a, a.p.many[i], blockIdx.x % heads, sh.many);
    } else {
        const int b = blockIdx.x - a.many_blocks, i = b / heads;
        if (i >= a.p.head->few) return;
        attend_few<DTYPE, FMT, D>(a, a.p.few[i], b % heads, sh.few);
    }
}

// Joins the partial results of rows that were split: JOIN_ROWS rows of one tile and head a block.
constexpr int JOIN_THREADS = 512, JOIN_ROWS = 4;

template <int DTYPE>
__global__ void __launch_bounds__(JOIN_THREADS) k_kv_join(AttendArgs a, int many, int tile_rows, int chunks)
{
    __shared__ float red_m[JOIN_ROWS][2], red_l[JOIN_ROWS][2];
    __shared__ float4 red_o[JOIN_THREADS];
    const int tid = threadIdx.x, heads = a.c.kv_heads, D = a.c.head_dim;
    const int chunk = blockIdx.x % chunks, head = (blockIdx.x / chunks) % heads, i = blockIdx.x / chunks / heads;
    if (i >= (many ? a.p.head->joins_many : a.p.head->joins_few)) return;
    const Join j = (many ? a.p.joins_many : a.p.joins_few)[i];
    const int rows = min(tile_rows, j.n_new * a.group - j.tile * tile_rows), r0 = chunk * JOIN_ROWS;
    if (r0 >= rows) return;
    const float *o = many ? a.part_many : a.part_few;
    const float2 *ml = reinterpret_cast<const float2 *>(o + (int64_t)(many ? a.p.parts_many : a.p.parts_few) * heads * tile_rows * D);
    auto at = [&](int p, int r) { return ((int64_t)(j.part0 + p) * heads + head) * tile_rows + r; };
    // maximum and sum of each row: 128 threads a row
    {
        const int rr = tid >> 7, r = min(r0 + rr, rows - 1);
        float m = -INFINITY, l = 0.f;
        for (int p = tid & 127; p < j.parts; p += 128) {
            const float2 x = ml[at(p, r)];
            const float n = fmaxf(m, x.x);
            if (n > -INFINITY) l = l * exp2f(m - n) + x.y * exp2f(x.x - n);
            else l += x.y;              // 0, or NaN
            m = n;
        }
        for (int d = 32; d > 0; d >>= 1) {
            const float m2 = __shfl_xor(m, d), l2 = __shfl_xor(l, d), n = fmaxf(m, m2);
            l = n > -INFINITY ? l * exp2f(m - n) + l2 * exp2f(m2 - n) : l + l2;
            m = n;
        }
        if ((tid & 63) == 0) {
            red_m[rr][(tid >> 6) & 1] = m;
            red_l[rr][(tid >> 6) & 1] = l;
        }
    }
    __syncthreads();
    const int quads = D / 4, per = JOIN_ROWS * quads, groups = JOIN_THREADS / per;     // D = 64, 128, 256: 8, 4, 2 groups
    const int e = tid % per, g = tid / per, rr = e / quads, d = (e % quads) * 4, r = min(r0 + rr, rows - 1);
    const float top = fmaxf(red_m[rr][0], red_m[rr][1]), base = top == -INFINITY ? 0.f : top;
    const float l = red_l[rr][0] * exp2f(red_m[rr][0] - base) + red_l[rr][1] * exp2f(red_m[rr][1] - base);
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int p = g; p < j.parts; p += groups) {
        const int64_t k = at(p, r);
        const float w = exp2f(ml[k].x - base);
        const float4 x = *reinterpret_cast<const float4 *>(o + k * D + d);
        sum.x += w * x.x;
        sum.y += w * x.y;
        sum.z += w * x.z;
        sum.w += w * x.w;
    }
    red_o[tid] = sum;
    __syncthreads();
    if (tid < per && r0 + rr < rows) {
        for (int w = 1; w < groups; ++w) {
            const float4 x = red_o[w * per + tid];
            sum.x += x.x;
            sum.y += x.y;
            sum.z += x.z;
            sum.w += x.w;
        }
        const float f = l == 0.f ? 0.f : 1.f / l;
        const int row = j.tile * tile_rows + r0 + rr, tok = row / a.group, q = head * a.group + row % a.group;
        store4<DTYPE>(a.q.out, (j.row0 + tok) * a.q.out_stride + (int64_t)q * D + d, a.vec_out, sum.x * f, sum.y * f, sum.z * f, sum.w * f);
        if (a.q.lse && d == 0) a.q.lse[(int64_t)(j.row0 + tok) * heads * a.group + q] = l == 0.f ? -INFINITY : LN2 * (top + log2f(l));
    }
}

}  // namespace kv
}  // namespace moe
