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
// the weights stay below 2^8 (see RISE) whatever the scales are, as fp16 wants it.  The sum of the probabilities is that of the weights, divided by vs page
// by page, in fp32 as are scores, maxima and outputs; where value scales lie so far apart that a weight may be too small for fp32 and its
// probability matter, the probabilities' exponentials are worked out for themselves (see WIDE).  Weights are rounded to fp16 (2^-11 of a weight, as an fp16 output is, or 2^-25 of the largest if that is more);
// bf16 queries become fp16 after a power of two is taken off each row.
#pragma once
#include "kernels_kv_common.h"

namespace moe {
namespace kv {

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

struct AttendArgs {
    moe_kv_cache_t c;
    moe_kv_query_t q;
    Plan p;
    const int32_t *table;
    float *part_few, *part_many;    // [part][kv head][rows][D] outputs, then [part][kv head][rows] (m, l)
    int32_t group, max_blocks, causal, window;
    int32_t sub_shift;              // log2 of a page's sub-blocks
    float per_group;                // 1 / group
    int32_t many_blocks;            // blocks of the grid that take tiles of requests of many rows; the others those of few
    int32_t vec_q, vec_out;
};

// An item, in scalar registers.
__device__ __forceinline__ Item item_of(const uint4 (&u)[3])
{
    union { Item it; uint4 u[3]; int w[12]; } r;
#pragma unroll
    for (int i = 0; i < 3; ++i) r.u[i] = u[i];
#pragma unroll
    for (int i = 0; i < 12; ++i) r.w[i] = __builtin_amdgcn_readfirstlane(r.w[i]);
    return r.it;
}

// A row of an item: its token and query head of the group, counted from the first of the tile, at most 256 rows in all.
struct Row {
    int tok, g;
    bool real;
};

__device__ __forceinline__ Row row_at(const AttendArgs &a, int first, int row, int rows)
{
    // first / group is the same for all lanes; what is added to it is small enough for fp32's product to be exact after rounding down
    const int t0 = first / a.group, in = first - t0 * a.group + row - first;
    const int t = (int)(((float)in + 0.5f) * a.per_group);
    return {t0 + t, in - t * a.group, row < rows};
}

__device__ __forceinline__ Item item_at(const Item *p)
{
    uint4 u[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) u[i] = reinterpret_cast<const uint4 *>(p)[i];
    return item_of(u);
}

// What a row sees: tokens [lo, hi).
struct Sees {
    int lo, hi;
};

__device__ __forceinline__ Sees sees(const AttendArgs &a, const Item &it, const Row &row)
{
    if (!row.real) return {0, 0};
    const int pos = it.ctx + row.tok;
    return {a.window > 0 ? max(0, pos + 1 - a.window) : 0, a.causal ? pos + 1 : it.ctx + it.n_new};
}

// A row's state between steps.
template <int D>
struct State {
    v16f o[D / 32];     // O^T: column is the lane's row, rows are dims 32 n + 8 (i/4) + 4 h + i%4
    float m, l;
    bool rare;          // a value scale beyond WIDE has been met, or a row of the wave has had an |m| beyond BIG
};

// Smaller scales count as this one, the least that the store writes: sums of 2^24 probabilities, each up to 2^8 / vs, stay within fp32.
constexpr float LEAST_SCALE = 0x1p-96f;

// Value scales from 2^-WIDE to 2^WIDE are 90 powers of two apart at most: a weight below 2^-126, which the exponential takes for 0, then belongs
// to a probability below 2^-28 of the largest (the maximum may be 8 too low).  From the first scale outside on, the sum's exponentials do without
// the scales.  A page of zeros, whose scale is 2^-96, is such a page; other than that, values beyond 2^45 or below 2^-36 are.
constexpr float WIDE = 45.f;
// Where fp32's steps of a maximum matter to an exponent: m is a rounded t, the others' exponents are rounded once, after m is taken off.
// Beyond 2^20 the difference shows in a weight, at 2^28 as one that fp16 does not hold.
constexpr float BIG = 0x1p20f;

__device__ __forceinline__ bool beyond_big(float m) { return fabsf(m) > BIG && fabsf(m) < INFINITY; }

// l 2^d, d <= 0, also where 2^d is less than fp32 holds.
__device__ __forceinline__ float times_two_to(float l, float d)
{
    const float f = exp2f(d), h = __builtin_amdgcn_exp2f(0.5f * d);
    return f < 0x1p-126f ? l * h * h : l * f;
}

// The waves' sums of a row, taken to `base`.  Where a sum's power of two is below what fp32 holds is looked for, not worked out: 64
// requests took 74.5 us instead of 73 with times_two_to alone.
template <int WAVES, int ROWS>
__device__ __forceinline__ float sum_of_waves(const float (&m)[WAVES][ROWS], const float (&l)[WAVES][ROWS], int row, float base)
{
    float sum = 0.f;
    bool low = false;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const float d = m[w][row] - base;
        sum += l[w][row] * exp2f(d);
        low |= d < -126.f && l[w][row] > 0.f;
    }
    if (__any(low)) {
        sum = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) sum += times_two_to(l[w][row], m[w][row] - base);
    }
    return sum;
}

template <int D>
__device__ __forceinline__ void clear(State<D> &s)
{
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) s.o[n][i] = 0.f;
    s.m = -INFINITY;
    s.l = 0.f;
    s.rare = false;
}

// Queries of 32 rows as the second operand of the first product.  k-slot (step 2i + c, lane half h, j) stands for dim
// 16 (2i + h) + 8 c + j, as the key tiles have it.  unit: what the scores have to be multiplied with.
template <int DTYPE, int D>
__device__ __forceinline__ void load_queries(const AttendArgs &a, const Item &it, int head, const Row &row, v8h (&q)[D / 16], float &unit)
{
    const int h = (threadIdx.x >> 5) & 1;
    const bool real = row.real;
    const int tok = real ? row.tok : 0, g = real ? row.g : 0;
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
        const int e = max((int)(top >> 7) - 127 - 14, -100);
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

// The larger of lane l's and lane l ^ 32's number, in both.
__device__ __forceinline__ float max_halves(float x)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);      // the lower lanes' in both, the upper lanes' in both
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}

// How far (in powers of two) a row's maximum may rise before its sums are scaled down to it: a new maximum is common while few
// tokens have been seen, and scaling is 64 multiplies a lane.  Weights stay below 2^8, well within fp16.
constexpr float RISE = 8.f;

// N steps: 32 N cached tokens against 32 rows.  kf(u, i, c), vf(u, n, c): the first operands of step u, dims 16 (2 i + h) + 8 c ...
// of the keys, tokens 8 c ... of dims 32 n ... of the values.  For the lane's sub-block of each step, sc: scale log2(e) ks, lv: log2 vs,
// iv: 1 / vs.  edge: some row does not see some token.
template <int D, int N, class KF, class VF>
__device__ __forceinline__ void steps(State<D> &s, const v8h (&q)[D / 16], KF kf, VF vf, const float (&sc)[N], const float (&lv)[N], const float (&iv)[N],
                                      bool edge, const int (&tok0)[N], Sees see)
{
    v16f z[N];
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) z[u][i] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int u = 0; u < N; ++u) z[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf(u, i, c), q[2 * i + c], z[u], 0, 0, 0);
    if constexpr (N == 2) {
        // six operands ahead of the matrix instruction that takes them: left alone, the compiler keeps two and waits for LDS
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
        for (int i = 0; i < D / 8 - 6; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 6, 0);
    }
    if (edge) {
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) z[u][i] = tok0[u] + i >= see.lo && tok0[u] + i < see.hi ? z[u][i] : -INFINITY;
    }
    float t = -INFINITY;
#pragma unroll
    for (int u = 0; u < N; ++u) {
        float top = z[u][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, z[u][i]);
        t = fmaxf(t, fmaf(top, sc[u], lv[u]));
    }
    t = max_halves(t);
    if (__any(t > s.m + RISE)) {
        const float m = fmaxf(s.m, t);
        const float f = m == -INFINITY ? 1.f : exp2f(s.m - m);
        s.l = m == -INFINITY ? s.l : times_two_to(s.l, s.m - m);
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) s.o[n][i] *= f;
        s.m = m;
        s.rare |= __any(beyond_big(m));
    }
    const float base = s.m == -INFINITY ? 0.f : s.m;
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) z[u][i] = fmaf(z[u][i], sc[u], lv[u] - base);
    float w[N];
#pragma unroll
    for (int u = 0; u < N; ++u) w[u] = iv[u];
    if (s.rare) {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            w[u] = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                z[u][i] = z[u][i] > RISE ? RISE : z[u][i];
                s.l += __builtin_amdgcn_exp2f(z[u][i] - lv[u]);
            }
        }
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
        v8h p[2];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float e = __builtin_amdgcn_exp2f(z[u][i]);
            sum += e;
            p[i / 8][i % 8] = (_Float16)e;
        }
        s.l = fmaf(sum, w[u], s.l);
        // neighbouring instructions into different outputs: one into the same waits for it
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int n = 0; n < D / 32; ++n) s.o[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf(u, n, c), p[c], s.o[n], 0, 0, 0);
    }
    if constexpr (N == 2) {
        // the second step's exponentials beside the first one's products
        constexpr int M = D / 8;
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 1);
        __builtin_amdgcn_sched_group_barrier(0x400, 16, 1);
#pragma unroll
        for (int i = 0; i < M; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
            if (i < M - 6) __builtin_amdgcn_sched_group_barrier(0x100, 1, 1);
            if (i < M / 2) __builtin_amdgcn_sched_group_barrier(0x400, 32 / M, 1);
        }
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
            p.ks = fmaxf(a.c.k_scale[(int64_t)id * a.c.kv_heads + head], LEAST_SCALE);
            p.vs = fmaxf(a.c.v_scale[(int64_t)id * a.c.kv_heads + head], LEAST_SCALE);
        }
    }
    return p;
}

// The same as the steps use it: in units of sub-blocks of all pages and heads, ks = 0 for nowhere, log2 vs, 1 / vs.
struct __align__(16) Spot {
    uint32_t at;
    float ks, lv, iv;
};

__device__ __forceinline__ Spot spot_of(const AttendArgs &a, const Item &it, int head, int sub_block, int end_tok)
{
    const Place p = place_of(a, it, head, sub_block, end_tok);
    const uint32_t page = (uint32_t)max(p.id, 0) * a.c.kv_heads + head;
    return {(page << a.sub_shift) + (sub_block & ((1 << a.sub_shift) - 1)), p.id < 0 ? 0.f : p.ks, __builtin_amdgcn_logf(p.vs), __builtin_amdgcn_rcpf(p.vs)};
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

// ---- joining the parts of rows whose cached tokens several blocks share
// Each block leaves its outputs (scaled by 2^-m) and (m, l) in the scratch; the one that finds all others of its tile and head done
// puts them together, in the parts' order, so that the result does not depend on which one that is.  What crosses blocks goes
// past the dies' caches: stores and loads of agent scope, a wait for the stores' acknowledgement before the count.  A fence of
// that scope would write back a die's whole cache for each of a thousand blocks; a second launch instead costs 4 to 10 us
// on the GPU and 3.5 us of the host's time a layer.
__device__ __forceinline__ void put2(float *p, float x, float y)
{
    const uint64_t w = __builtin_bit_cast(uint32_t, x) | ((uint64_t)__builtin_bit_cast(uint32_t, y) << 32);
    __hip_atomic_store(reinterpret_cast<uint64_t *>(p), w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Four numbers, through a descriptor of all parts' outputs.  16: of agent scope.
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ void put4(__amdgpu_buffer_rsrc_t rs, uint32_t at, float x, float y, float z, float w)
{
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, make_float4(x, y, z, w)), rs, (int)(at * 4), 0, 16);
}

__device__ __forceinline__ float4 get4(__amdgpu_buffer_rsrc_t rs, uint32_t at)
{
    return __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)(at * 4), 0, 16));
}

// (the address of all lanes, a lane's own bytes from there)
__device__ __forceinline__ float get1(const float *p, uint32_t at)
{
    return __hip_atomic_load(reinterpret_cast<const float *>(reinterpret_cast<const char *>(p) + at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ float2 get2(const float *p, uint32_t at)
{
    const uint64_t w = __hip_atomic_load(reinterpret_cast<const uint64_t *>(reinterpret_cast<const char *>(p) + at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__builtin_bit_cast(float, (uint32_t)w), __builtin_bit_cast(float, (uint32_t)(w >> 32)));
}

struct JoinShared {
    float m[256], l[256];           // of a row
    float4 sum[512];                // of a thread
    int last;
};

// Counts this block's part; true in the block that came last.  Every thread's stores are acknowledged before the count.
__device__ __forceinline__ bool all_parts_done(int32_t *count, int parts, int &last)
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        last = __hip_atomic_fetch_add(count, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
        if (last) __hip_atomic_store(count, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);     // for the next layer
    }
    __syncthreads();
    return last;
}

// (m, l) of two parts of a row.
__device__ __forceinline__ void join_sum(float &m, float &l, float m2, float l2)
{
    const bool up = m2 > m;
    const float n = up ? m2 : m;
    l = n > -INFINITY ? (up ? l2 : l) + times_two_to(up ? l : l2, (up ? m : m2) - n) : l + l2;      // the latter 0, or NaN
    m = n;
}

// Maximum and sum of each row, into LDS; 1 to 64 lanes a row.
__device__ __forceinline__ void join_sums(const AttendArgs &a, const Item &it, int head, const float *ml, int tile_rows, int threads, JoinShared &sh)
{
    const int tid = threadIdx.x, heads = a.c.kv_heads, rows = min(tile_rows, it.n_new * a.group - it.tile * tile_rows);
    int pow2 = 4;
    while (pow2 < rows) pow2 *= 2;
    const int lanes = min(64, max(1, threads / pow2)), r = min(tid / lanes, rows - 1);
    float top = -INFINITY, l = 0.f;
    for (int p = tid % lanes; p < it.parts; p += lanes) {
        const float2 v = get2(ml, (((it.part0 + p) * heads + head) * tile_rows + r) * 8u);
        join_sum(top, l, v.x, v.y);
    }
    for (int d = lanes / 2; d > 0; d >>= 1) {
        const float m2 = __shfl_xor(top, d), l2 = __shfl_xor(l, d);
        join_sum(top, l, m2, l2);
    }
    if (tid % lanes == 0 && tid / lanes < rows) {
        sh.m[r] = top == -INFINITY ? 0.f : top;
        sh.l[r] = l;
        if (a.q.lse) {
            const int row = it.tile * tile_rows + r, tok = row / a.group;
            a.q.lse[(int64_t)(it.row0 + tok) * heads * a.group + head * a.group + row - tok * a.group] = l == 0.f ? -INFINITY : LN2 * (top + log2f(l));
        }
    }
}

// o: outputs [part][kv head][tile_rows][D], ml: [part][kv head][tile_rows][2]
template <int DTYPE, int D>
__device__ __forceinline__ void join_parts(const AttendArgs &a, const Item &it, int head, const float *o, const float *ml, int tile_rows, JoinShared &sh)
{
    constexpr int THREADS = 64 * ATTEND_WAVES;
    const int tid = threadIdx.x, heads = a.c.kv_heads;
    const int rows = min(tile_rows, it.n_new * a.group - it.tile * tile_rows);
    int pow2 = 4;
    while (pow2 < rows) pow2 *= 2;
    // 32 bits: two parts a block and head (see target_blocks), at most 1024 of all heads, of 32 rows and 256 dims
    auto at = [&](int p, int r) { return (uint32_t)(((it.part0 + p) * heads + head) * tile_rows + r); };
    // Four dims a thread; where that leaves threads over, the parts are dealt out to groups of threads.  The loads are past the
    // caches, one or two microseconds each: the first parts' are on their way before the maxima are known.
    constexpr int QUADS = D / 4, AHEAD = D == 64 ? 8 : 16;
    const int all = pow2 * QUADS, groups = max(1, THREADS / all);
    const int e_first = groups > 1 ? tid % all : tid, g = groups > 1 ? tid / all : 0;
    float m[AHEAD];
    float2 x[AHEAD], y[AHEAD];
    auto fetch = [&](int e, int p0) {
        const int r = min(e / QUADS, rows - 1), d = (e % QUADS) * 4;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (p0 - g + u * groups >= it.parts) break;
            const uint32_t k = at(min(p0 + u * groups, it.parts - 1), r);
            m[u] = get1(ml, k * 8);
            x[u] = get2(o, (k * D + d) * 4);
            y[u] = get2(o, (k * D + d + 2) * 4);
        }
    };
    fetch(e_first, g);
    join_sums(a, it, head, ml, tile_rows, THREADS, sh);
    __syncthreads();
    for (int e0 = 0; e0 < rows * QUADS; e0 += THREADS) {
        const int e = e0 + e_first, r = min(e / QUADS, rows - 1), d = (e % QUADS) * 4;
        const float top = sh.m[r];
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int p0 = g; p0 < it.parts; p0 += AHEAD * groups) {
            if (e0 || p0 != g) fetch(e, p0);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (p0 - g + u * groups >= it.parts) break;
                const float w = p0 + u * groups < it.parts ? exp2f(m[u] - top) : 0.f;
                sum.x = fmaf(w, x[u].x, sum.x);
                sum.y = fmaf(w, x[u].y, sum.y);
                sum.z = fmaf(w, y[u].x, sum.z);
                sum.w = fmaf(w, y[u].y, sum.w);
            }
        }
        if (groups > 1) {
            sh.sum[tid] = sum;
            __syncthreads();
            for (int w = 1; w < groups && g == 0; ++w) {
                const float4 z = sh.sum[w * all + e];
                sum.x += z.x;
                sum.y += z.y;
                sum.z += z.z;
                sum.w += z.w;
            }
        }
        if (g == 0 && e < rows * QUADS) {
            const float l = sh.l[r], f = l == 0.f ? 0.f : 1.f / l;
            const int row = it.tile * tile_rows + r, tok = row / a.group;
            store4<DTYPE>(a.q.out, (it.row0 + tok) * a.q.out_stride + (int64_t)(head * a.group + row - tok * a.group) * D + d, a.vec_out, sum.x * f, sum.y * f, sum.z * f, sum.w * f);
        }
    }
}

// The same for tiles of 32 rows a wave: [part][kv head][wave][D / 8][64 lanes][4 dims], as the waves hold them (lane (h, row) has dims
// 8 i + 4 h + (0..3)).  By rows, as above, a wave's store went to 64 places, eight bytes each: 128 tokens onto 8000 took 94 us,
// 68 this way.  One block joins it all, so what counts is how many loads are on their way at once: those of SPAN parts of
// each of ROUNDS rounds over the tile.
template <int DTYPE, int D, int ROWS, int SPAN>
__device__ __forceinline__ void join_tile_spans(const AttendArgs &a, const Item &it, int head, __amdgpu_buffer_rsrc_t o, const float *ml, JoinShared &sh)
{
    constexpr int THREADS = 64 * ATTEND_WAVES, WAVE = 8 * D, AHEAD = 16, ROUNDS = AHEAD / SPAN;
    const int tid = threadIdx.x, heads = a.c.kv_heads;
    // 32 bits: at most 1024 parts of all heads, of 128 rows and 256 dims
    const int rows = min(ROWS, it.n_new * a.group - it.tile * ROWS), quads = div_up(rows, 32) * WAVE;
    auto row_of = [&](int e) { return e / WAVE * 32 + e % 32; };
    float m[AHEAD];
    float4 x[AHEAD];
    auto fetch = [&](int e0, int p0) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (p0 + u % SPAN >= it.parts) continue;
            const int e = min(e0 + u / SPAN * THREADS, quads - 1);
            const uint32_t at = (uint32_t)(((it.part0 + p0 + u % SPAN) * heads + head) * ROWS);
            m[u] = get1(ml, (at + min(row_of(e), rows - 1)) * 8);
            x[u] = get4(o, at * D + e * 4);
        }
    };
    fetch(tid, 0);
    join_sums(a, it, head, ml, ROWS, THREADS, sh);
    __syncthreads();
    for (int e0 = tid; e0 < quads; e0 += THREADS * ROUNDS) {
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int p0 = 0; p0 < it.parts; p0 += SPAN) {
            if (e0 != tid || p0) fetch(e0, p0);
#pragma unroll
            for (int v = 0; v < ROUNDS; ++v) {
                const int e = e0 + v * THREADS, r = min(row_of(e), rows - 1), d = e / 64 % (D / 8) * 8 + (e >> 5 & 1) * 4;
                const float top = sh.m[r];
#pragma unroll
                for (int u = v * SPAN; u < (v + 1) * SPAN; ++u) {
                    if (p0 + u % SPAN >= it.parts) continue;
                    const float w = exp2f(m[u] - top);
                    sum.x = fmaf(w, x[u].x, sum.x);
                    sum.y = fmaf(w, x[u].y, sum.y);
                    sum.z = fmaf(w, x[u].z, sum.z);
                    sum.w = fmaf(w, x[u].w, sum.w);
                }
                if (p0 + SPAN < it.parts) continue;
                if (row_of(e) < rows) {
                    const float l = sh.l[r], f = l == 0.f ? 0.f : 1.f / l;
                    const int row = it.tile * ROWS + r, tok = row / a.group;
                    store4<DTYPE>(a.q.out, (it.row0 + tok) * a.q.out_stride + (int64_t)(head * a.group + row - tok * a.group) * D + d, a.vec_out, sum.x * f, sum.y * f, sum.z * f, sum.w * f);
                }
                sum = make_float4(0.f, 0.f, 0.f, 0.f);
            }
        }
    }
}

template <int DTYPE, int D, int ROWS>
__device__ __forceinline__ void join_tile(const AttendArgs &a, const Item &it, int head, __amdgpu_buffer_rsrc_t o, const float *ml, JoinShared &sh)
{
    if (it.parts <= 4) join_tile_spans<DTYPE, D, ROWS, 4>(a, it, head, o, ml, sh);
    else join_tile_spans<DTYPE, D, ROWS, 16>(a, it, head, o, ml, sh);
}

// ---- a tile of 32 rows: every wave takes every fourth step of the block's, straight from memory into registers.  24 requests of 40 rows
// that see 1024 tokens take 13.4 us of launch, table, scales, loads and join one behind the other; the cache alone would be 2 us.
template <int D>
struct FewShared {
    float m[ATTEND_WAVES][ROWS_FEW], l[ATTEND_WAVES][ROWS_FEW];
    __align__(16) float o[ATTEND_WAVES * 8 * (D + 4)];
    JoinShared join;
};

template <int DTYPE, int FMT, int D>
__device__ __forceinline__ void attend_few(const AttendArgs &a, const Item &it, int head, FewShared<D> &sh)
{
    constexpr int WAVES = ATTEND_WAVES;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 31, h = lane >> 5;
    const int rows = it.n_new * a.group, row0 = it.tile * ROWS_FEW, here = min(ROWS_FEW, rows - row0);
    const Row row = row_at(a, row0, row0 + col, rows);
    v8h q[D / 16];
    float unit;
    load_queries<DTYPE, D>(a, it, head, row, q, unit);
    const Sees see = sees(a, it, row);
    const float factor = a.q.scale * LOG2E * unit;
    // all rows see tokens [all_lo, all_hi); values below any_lo may lie in pages that the request has given back
    const int pos_a = it.ctx + __builtin_amdgcn_readlane(row.tok, 0), pos_z = it.ctx + __builtin_amdgcn_readlane(row.tok, here - 1), any_hi = it.ctx + it.n_new;
    const int any_lo = a.window > 0 ? max(0, pos_a + 1 - a.window) : 0;
    const int all_lo = a.window > 0 ? max(0, pos_z + 1 - a.window) : 0, all_hi = a.causal ? pos_a + 1 : any_hi;
    State<D> s;
    clear(s);

    const int sub_bytes = SUB * D, heads = a.c.kv_heads, subs = a.c.page / SUB;
    const int kh = (col >> 2) & 1, ktok = 4 * (col >> 3) + (col & 3);     // S^T row `col` is token 16 kh + ktok of the step
    const uint8_t *kbase = static_cast<const uint8_t *>(a.c.k), *vbase = static_cast<const uint8_t *>(a.c.v);
    constexpr int BATCH = 32;       // steps of a wave whose places the lanes hold, two sub-blocks a step
    for (int first = it.kt0 + wave; first < it.kt1; first += WAVES * BATCH) {
        const int n = min(BATCH, div_up(it.kt1 - first, WAVES));
        const Place mine = (lane >> 1) < n ? place_of(a, it, head, 2 * (first + WAVES * (lane >> 1)) + (lane & 1), any_hi) : Place{-1, 1.f, 1.f};
        uint4 k[2][D / 32], v[2][D / 32];
        auto fetch = [&](int j, uint4 (&kk)[D / 32], uint4 (&vv)[D / 32]) {
            const int kt = first + WAVES * j;
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
            const int kt = first + WAVES * j;
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
            steps<D, 1>(s, q, [&](int, int i, int c) { return c ? codes_to_half<FMT>(kk[i].z, kk[i].w) : codes_to_half<FMT>(kk[i].x, kk[i].y); },
                        [&](int, int i, int c) { return c ? codes_to_half<FMT>(vv[i].z, vv[i].w) : codes_to_half<FMT>(vv[i].x, vv[i].y); },
                        {factor * ks}, {__builtin_amdgcn_logf(vs)}, {__builtin_amdgcn_rcpf(vs)}, edge, {tok0}, mask);
        };
        // No branch around a load (past the end the last step is requested again): the compiler then waits for the step it
        // needs alone, with the next one's loads in flight.
        fetch(0, k[0], v[0]);
        s.rare |= __any(fabsf(__builtin_amdgcn_logf(mine.vs)) > WIDE);
        for (int j = 0; j < n; j += 2) {
            fetch(min(j + 1, n - 1), k[1], v[1]);
            use(j, k[0], v[0]);
            fetch(min(j + 2, n - 1), k[0], v[0]);
            if (j + 1 < n) use(j + 1, k[1], v[1]);
        }
    }
    // join the waves
    s.l += __shfl_xor(s.l, 32);
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
    // as many rows at a time as the waves' outputs of them fit into LDS: all of a token's where its group has eight heads or fewer
    constexpr int STRIDE = D + 4, HOLD = sizeof(sh.o) / (WAVES * STRIDE * 4), QUADS = D / 4;
    for (int r0 = 0; r0 < here; r0 += HOLD) {
        if (r0) __syncthreads();
        if (col >= r0 && col < min(r0 + HOLD, here)) {
#pragma unroll
            for (int n = 0; n < D / 32; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<float4 *>(sh.o + (wave * HOLD + col - r0) * STRIDE + 32 * n + 8 * i + 4 * h) =
                        make_float4(s.o[n][4 * i] * f, s.o[n][4 * i + 1] * f, s.o[n][4 * i + 2] * f, s.o[n][4 * i + 3] * f);
        }
        __syncthreads();
        for (int e = tid; e < min(HOLD, here - r0) * QUADS; e += 64 * WAVES) {
            const int r = e / QUADS, d = (e % QUADS) * 4;
            float4 x = *reinterpret_cast<const float4 *>(sh.o + r * STRIDE + d);
#pragma unroll
            for (int w = 1; w < WAVES; ++w) {
                const float4 y = *reinterpret_cast<const float4 *>(sh.o + (w * HOLD + r) * STRIDE + d);
                x.x += y.x;
                x.y += y.y;
                x.z += y.z;
                x.w += y.w;
            }
            if (whole) {
                const Row out = row_at(a, row0, row0 + r0 + r, rows);
                store4<DTYPE>(a.q.out, (it.row0 + out.tok) * a.q.out_stride + (int64_t)(head * a.group + out.g) * D + d, a.vec_out, x.x, x.y, x.z, x.w);
            } else {
                float *p = a.part_few + (part + r0 + r) * D + d;
                put2(p, x.x, x.y);
                put2(p + 2, x.z, x.w);
            }
        }
    }
    if (!whole && all_parts_done(a.p.joins_few + it.join * heads + head, it.parts, sh.join.last)) join_parts<DTYPE, D>(a, it, head, a.part_few, ml, ROWS_FEW, sh.join);
}

// ---- tiles of 32 rows a wave: every wave has its own, all waves share the block's steps through LDS, two at a time.  The codes
// become fp16 numbers once, on their way into LDS: left to the waves, the conversion was a third of their vector instructions, which
// are the bound here: a prompt of 4096 took 255 us that way, 181 with the codes converted once, parts of prompts 47 and 36.  Places and
// scales read once for all steps and products of neighbouring steps into different outputs made it 163 to 173 by the machine: 0.80 to 0.84
// PFLOP/s, 70 % of a large library product.  Matrix unit 35 % of the time, vector unit 43 %, waves waiting 35 % of theirs, no bank conflicts: no
// unit is full, two waves a SIMD do not cover a step's chain of product, maximum, exponential and product and its barrier.  Both roles' registers
// come to 256 at D = 128, of which 4 to 5 spill, and 49 to 61 spill at D = 256 (a prompt of 4096: 420 us, floor 237).  The scores of
// the next step beside the exponentials of this one, orders and priorities asked of the compiler: 0 to 4 % slower.
template <int D>
struct ManyShared {
    static constexpr int PLACES = 256;      // sub-blocks whose places are known at a time
    v8h k[2][2][4 * D], v[2][2][4 * D];     // [buffer][half of a piece][sub-block of the two steps][piece of 16 codes]
    Spot place[PLACES];
    JoinShared join;
};

template <int DTYPE, int FMT, int D>
__device__ __forceinline__ void attend_many(const AttendArgs &a, const Item &it, int head, ManyShared<D> &sh)
{
    constexpr int THREADS = 64 * ATTEND_WAVES, ROWS = 32 * ATTEND_WAVES;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 31, h = lane >> 5;
    const int rows = it.n_new * a.group, tile0 = it.tile * ROWS, row0 = tile0 + wave * 32;
    const Row row = row_at(a, tile0, row0 + col, rows);
    v8h q[D / 16];
    float unit;
    load_queries<DTYPE, D>(a, it, head, row, q, unit);
    const Sees see = sees(a, it, row);
    const float factor = a.q.scale * LOG2E * unit;
    const int pos_a = it.ctx + __builtin_amdgcn_readlane(row.tok, 0), pos_z = it.ctx + __builtin_amdgcn_readlane(row.tok, max(0, min(31, rows - 1 - row0)));
    const int end = it.ctx + it.n_new, part_hi = min(end, it.kt1 * KT);
    const int any_lo = a.window > 0 ? max(0, pos_a + 1 - a.window) : 0, any_hi = row0 >= rows ? 0 : a.causal ? pos_z + 1 : end;
    const int all_lo = a.window > 0 ? max(0, pos_z + 1 - a.window) : 0, all_hi = min(part_hi, a.causal ? pos_a + 1 : end);
    // values before this one may lie in pages that the request has given back
    const int tile_lo = a.window > 0 ? max(0, it.ctx + tile0 / a.group + 1 - a.window) : 0;
    State<D> s;
    clear(s);

    const int heads = a.c.kv_heads;
    const int kh = (col >> 2) & 1, ktok = 4 * (col >> 3) + (col & 3);
    const uint4 *kbase = static_cast<const uint4 *>(a.c.k), *vbase = static_cast<const uint4 *>(a.c.v);
    constexpr int PER = div_up(4 * D, THREADS);     // pieces of 16 bytes of a thread: two steps hold 4 D of each kind
    for (int batch = it.kt0; batch < it.kt1; batch += ManyShared<D>::PLACES / 2) {
        const int last = min(it.kt1, batch + ManyShared<D>::PLACES / 2), places = 2 * (last - batch);
        __syncthreads();
        for (int i = tid; i < places; i += THREADS) sh.place[i] = spot_of(a, it, head, 2 * batch + i, end);
        __syncthreads();
        uint4 rk[PER], rv[PER];
        bool gone[PER];
        auto fetch = [&](int kt) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int piece = tid + i * THREADS, sb = piece / D, in = piece - sb * D;
                const Spot sp = sh.place[min(2 * (kt - batch) + sb, places - 1)];
                gone[i] = sp.ks == 0.f;
                const uint64_t at = (uint64_t)sp.at * D + in;
                rk[i] = kbase[at];
                rv[i] = vbase[at];
            }
        };
        auto put = [&](int kt, int buf) {
            const bool whole = kt * KT >= tile_lo && (kt + 2) * KT <= part_hi;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int piece = tid + i * THREADS;
                if (!whole || gone[i]) {            // bytes that may be anything: before the window, behind the last token, of no page
                    const int tok0 = kt * KT + piece / D * SUB;
                    rv[i] = keep_bytes(rv[i], tile_lo - tok0, gone[i] ? 0 : part_hi - tok0);
                }
                sh.k[buf][0][piece] = codes_to_half<FMT>(rk[i].x, rk[i].y);
                sh.k[buf][1][piece] = codes_to_half<FMT>(rk[i].z, rk[i].w);
                sh.v[buf][0][piece] = codes_to_half<FMT>(rv[i].x, rv[i].y);
                sh.v[buf][1][piece] = codes_to_half<FMT>(rv[i].z, rv[i].w);
            }
        };
        fetch(batch);
        bool wide = false;
        for (int i = lane; i < places; i += 64) wide |= fabsf(sh.place[i].lv) > WIDE;
        s.rare |= __any(wide);
        put(batch, 0);
        __syncthreads();
        int buf = 0;
        for (int kt = batch; kt < last; kt += 2) {
            const bool more = kt + 2 < last;
            fetch(more ? kt + 2 : kt);              // no branch around a load
            const int tok = kt * KT;
            if (tok < any_hi && tok + 2 * KT > any_lo) {
                float sc[2], lv[2], iv[2];
                int tok0[2];
                bool none = false;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const Spot sp = sh.place[min(2 * (kt + u - batch) + h, places - 1)];
                    const bool dead = sp.ks == 0.f;
                    sc[u] = dead ? 1.f : factor * sp.ks;
                    lv[u] = sp.lv;
                    iv[u] = sp.iv;
                    tok0[u] = dead ? 0x40000000 : tok + u * KT + SUB * h;       // nowhere: as if behind all that the row sees
                    none |= dead;
                }
                const bool edge = tok < all_lo || tok + 2 * KT > all_hi || __any(none);
                const Sees mask{see.lo, min(see.hi, part_hi)};
                steps<D, 2>(s, q, [&](int u, int i, int c) { return sh.k[buf][c][(2 * u + kh) * D + (2 * i + h) * 16 + ktok]; },
                            [&](int u, int n, int c) { return sh.v[buf][c][(2 * u + h) * D + n * 32 + col]; }, sc, lv, iv, edge, tok0, mask);
            }
            if (more) put(kt + 2, buf ^ 1);
            __syncthreads();
            buf ^= 1;
        }
    }
    s.l += __shfl_xor(s.l, 32);
    const bool whole = it.part < 0;
    float *ml = a.part_many + (int64_t)a.p.parts_many * heads * ROWS * D;
    const __amdgpu_buffer_rsrc_t parts = __builtin_amdgcn_make_buffer_rsrc(a.part_many, 0, (int)((uint32_t)(a.p.parts_many * heads * ROWS) * (D * 4u)), 0x00020000);
    if (row.real) {
        const int tok = row.tok, g = row.g;
        const int64_t part = ((int64_t)it.part * heads + head) * ROWS + wave * 32 + col;
        const uint32_t lane_at = (uint32_t)((it.part * heads + head) * ROWS + wave * 32) * D + lane * 4;
        const float f = whole ? (s.l == 0.f ? 0.f : 1.f / s.l) : 1.f;
        const int64_t out = (it.row0 + tok) * a.q.out_stride + (int64_t)(head * a.group + g) * D;
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = 32 * n + 8 * i + 4 * h;
                const float x = s.o[n][4 * i] * f, y = s.o[n][4 * i + 1] * f, z = s.o[n][4 * i + 2] * f, w = s.o[n][4 * i + 3] * f;
                if (whole) {
                    store4<DTYPE>(a.q.out, out + d, a.vec_out, x, y, z, w);
                } else {
                    put4(parts, lane_at + (4 * n + i) * 256, x, y, z, w);
                }
            }
        if (h == 0) {
            if (!whole) put2(ml + part * 2, s.m, s.l);
            else if (a.q.lse) a.q.lse[(int64_t)(it.row0 + tok) * heads * a.group + head * a.group + g] = s.l == 0.f ? -INFINITY : LN2 * (s.m + log2f(s.l));
        }
    }
    if (!whole && all_parts_done(a.p.joins_many + it.join * heads + head, it.parts, sh.join.last)) join_tile<DTYPE, D, ROWS>(a, it, head, parts, ml, sh.join);
}

template <int DTYPE, int FMT, int D>
__global__ void __launch_bounds__(64 * ATTEND_WAVES, D <= 128 ? 2 : 1) k_kv_attend(AttendArgs a)
{
    __shared__ union {
        FewShared<D> few;
        ManyShared<D> many;
    } sh;
    // kv heads follow each other: blocks of one head, which share cached tokens, come to the same die where there are eight
    const int heads = a.c.kv_heads;
    if ((int)blockIdx.x < a.many_blocks) {
        const int i = blockIdx.x / heads;
        const Item it = item_at(a.p.many + i);      // in flight with the list's length; past it it is whatever was there
        if (i < a.p.head->many) attend_many<DTYPE, FMT, D>(a, it, blockIdx.x - i * heads, sh.many);
    } else {
        const int b = blockIdx.x - a.many_blocks, i = b / heads;
        const int first = a.p.few_first[i], last = a.p.few_first[i + 1];
        if (i >= a.p.head->few_blocks) return;
        for (int k = first; k < last; ++k) {
            if (k > first) __syncthreads();          // the item before is done with LDS
            attend_few<DTYPE, FMT, D>(a, item_at(a.p.few + k), b - i * heads, sh.few);
        }
    }
}

}  // namespace kv
}  // namespace moe
