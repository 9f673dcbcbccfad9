// Norm and rotation of queries and keys, and the store of keys and values as codes of 4 bits; cached tokens read back.
//
// A token's codes depend on that token alone: a key has a scale for each 32 dims, a value one for its head, and nothing that is cached changes
// when tokens follow.  With so few codes a border between two is what a rounding on the way may cross, and the neighbour is a third of the number
// away; so keys are normed and turned in fp64 and go to fp32 by way of the odd one of the two neighbours, which keeps them on their side of
// every border: the code is that of the exact number but for one in 2^50 or so.  Values are 16-bit numbers and exact as they are.  Queries
// take the fp32 path of the 8-bit cache.
//
// A block takes the new tokens of sixteen (which lie in one piece of a page), keys or values, of as many heads as give it 64 rows of a
// head.  Keys lie as rows and leave as four bytes a thread; values have sixteen tokens of a dim side by side and go through LDS.
//
// Prompts of 8 thousand tokens (165 MB, 32 and 8 heads of 128) 54 us, 3.1 TB/s where a large copy has 5.1; 256 tokens 7, one 4.  Queries are 41 of the
// 54 (fp64's registers leave them half the waves), keys 15.  Queries in a launch of their own, of twice the waves: 30 + 28.6.  Keys in fp32 with a
// bound on its error, and fp64 only where a code or a scale is in doubt: no faster (the sums of both ends cost what fp64 does), 256 tokens 10.  Registers
// limited to 80 and 64: 57 and 69.  32, 64 and 128 rows a block that stores: 8 thousand tokens stored and read back 68.5, 66.7 and 67.0, 256 and one the same.
#pragma once
#include "kernels_kv_write.h"

namespace moe {
namespace kv {

constexpr int WRITE4_ROWS = 64;

struct Write4Args {
    WriteArgs w;            // heads: of a block that stores; kv_blocks: blocks that store
    int32_t subs;           // pieces of sixteen that a segment's tokens can lie in
    int32_t groups;         // blocks that share a piece's heads
    uint32_t blocks;        // of the whole grid, fewer than 2^32
};

// Cosine and sine of pos * freq in fp64.  The product is exact (24 bits each).  The nearest quarter turn is taken off with pi/2 in two parts; the
// rest, pi / 4 at most, goes through the two series up to terms of 2^-54.
__device__ __forceinline__ double2 angle64(int pos, float freq)
{
    const double a = (double)pos * (double)freq, n = rint(a * 0.63661977236758134308);
    const double y = fma(-n, 6.123233995736766036e-17, fma(-n, 1.57079632679489661923, a)), z = y * y;
    double s = -1. / 1307674368000., c = 1. / 20922789888000.;
    s = fma(z, s, 1. / 6227020800.);
    c = fma(z, c, -1. / 87178291200.);
    s = fma(z, s, -1. / 39916800.);
    c = fma(z, c, 1. / 479001600.);
    s = fma(z, s, 1. / 362880.);
    c = fma(z, c, -1. / 3628800.);
    s = fma(z, s, -1. / 5040.);
    c = fma(z, c, 1. / 40320.);
    s = fma(z, s, 1. / 120.);
    c = fma(z, c, -1. / 720.);
    s = fma(z, s, -1. / 6.);
    c = fma(z, c, 1. / 24.);
    s = fma(y * z, s, y);
    c = fma(z, fma(z, c, -0.5), 1.);
    const int k = (int)(n - 4. * floor(n * 0.25));
    const double u = k & 1 ? s : c, v = k & 1 ? c : s;
    return make_double2(k == 1 || k == 2 ? -u : u, k & 2 ? -v : v);
}

// To fp32, of the two neighbours of a number that lies between the odd one: later roundings to fewer bits are those of the number itself.
__device__ __forceinline__ float to_odd(double d)
{
    const float f = (float)d;
    const double b = f;
    uint32_t u = __builtin_bit_cast(uint32_t, f);
    if (b != d && !(u & 1)) u += fabs(b) < fabs(d) ? 1u : 0xFFFFFFFFu;
    return __builtin_bit_cast(float, u);
}

// The exponent of the smallest power of two of which six reach amax, -45 at least, 127 added.  amax: 2^47 at most, no NaN.
__device__ __forceinline__ int scale_byte(float amax)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, amax);
    const int e = (int)(u >> 23) - ((u & 0x7FFFFFu) > 0x400000u ? 1 : 2);       // amax <= 1.5 2^(e - 125)
    return max(e, 127 - 45);
}

__device__ __forceinline__ float power_of(int byte) { return __builtin_bit_cast(float, (uint32_t)byte << 23); }

// Eight numbers within six times the scale as codes, the first lowest.
__device__ __forceinline__ uint32_t floats_to_e2m1(const float (&x)[8], float scale)
{
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}

// NaN is 0, what lies beyond `huge` that; the largest size of the eight.
__device__ __forceinline__ float tame8(float (&x)[8], float huge)
{
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = x[i] == x[i] ? fminf(fmaxf(x[i], -huge), huge) : 0.f;
        most = fmaxf(most, fabsf(x[i]));
    }
    return most;
}

__device__ __forceinline__ uint4 load_raw8(const void *base, int64_t at, bool vec)
{
    const uint16_t *p = static_cast<const uint16_t *>(base) + at;
    if (vec) return *reinterpret_cast<const uint4 *>(p);
    return make_uint4(p[0] | (uint32_t)p[1] << 16, p[2] | (uint32_t)p[3] << 16, p[4] | (uint32_t)p[5] << 16, p[6] | (uint32_t)p[7] << 16);
}

template <int DTYPE>
__device__ __forceinline__ void floats_of(uint4 r, float (&x)[8])
{
    const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = from_bits<DTYPE>(u[i] & 0xFFFF);
        x[2 * i + 1] = from_bits<DTYPE>(u[i] >> 16);
    }
}

template <int DTYPE>
__global__ void __launch_bounds__(WRITE_THREADS) k_kv4_write(Write4Args b)
{
    const WriteArgs &a = b.w;
    const int D = a.c.head_dim, shift = 31 - __builtin_clz(D), L = D / 8, tid = threadIdx.x, rot = a.r.rot_dim, half = rot / 2;
    const int sub = tid & (L - 1), mine = tid >> (shift - 3), per_pass = WRITE_THREADS >> (shift - 3), d0 = sub * 8;
    extern __shared__ __align__(16) uint8_t write4_lds[];
    // blocks that store are spread evenly among those of queries: these wait for memory, those for their fp64 sums (8 thousand tokens 54 us, 58 with
    // all that store in front)
    const uint32_t index = a.first + blockIdx.x, before = (uint32_t)((uint64_t)index * a.kv_blocks / b.blocks), through = (uint32_t)((uint64_t)(index + 1) * a.kv_blocks / b.blocks);
    if (through == before) {
        turn_queries<DTYPE>(a, (int)(index - before) * a.q_tokens, write4_lds);
        return;
    }
    const int block = (int)before;
    const int which = block & 1, unit = (block >> 1) / b.groups, h0 = ((block >> 1) - unit * b.groups) * a.heads, si = unit / b.subs;
    const int heads = a.c.kv_heads, page = a.c.page, hg = min(a.heads, heads - h0);
    const Segment s = a.p.segments[si];         // in flight with the list's length
    if (si >= a.p.head->segments || s.page_id < 0) return;
    const int piece = s.offset / SUB + unit - si * b.subs, lo = max(s.offset, piece * SUB), n = min(s.offset + s.count, piece * SUB + SUB) - lo, in0 = lo - piece * SUB;
    if (n <= 0) return;
    // tokens [in0, in0 + n) of the piece; the first of them:
    const int row0 = s.row0 + lo - s.offset, pos0 = s.pos0 + lo - s.offset, rows = n * hg;
    const int64_t place0 = (int64_t)s.page_id * heads + h0;
    const uint32_t per_hg = 0xFFFF / (uint32_t)hg + 1;
    auto token_of = [&](int r) { return (int)((uint32_t)r * per_hg >> 16); };       // r / hg, for r < 512 and hg <= 32
    // numbers beyond these are clamped: scales are 2^45 at most
    const float huge = DTYPE == MOE_KV_F16 ? 65504.f : 0x1p47f;
    const void *src = which ? a.r.v : a.r.k;
    const int64_t stride = which ? a.r.v_stride : a.r.k_stride;
    const bool vec = which ? a.vec_v : a.vec_k;
    // lanes past the end repeat the last row, without storing it
    auto fetch = [&](int r) {
        r = min(r, rows - 1);
        const int t = token_of(r), hh = r - t * hg;
        return load_raw8(src, (row0 + t) * stride + (int64_t)(h0 + hh) * D + d0, vec);
    };
    uint4 next = fetch(mine);

    if (!which) {
        // a token's angles: 8 j + i at [i][j], so that neighbouring threads, eight dims each, find theirs side by side (in order 63 us instead of 58)
        double2 *cs = reinterpret_cast<double2 *>(write4_lds);
        const int eighth = half / 8;
        const float per_half = 1.f / (float)half;
        for (int i = tid; i < n * half; i += WRITE_THREADS) {
            const int u = (int)(((float)i + 0.5f) * per_half), k = i - u * half;
            cs[u * half + (k & 7) * eighth + (k >> 3)] = angle64(pos0 + u, a.r.inv_freq[k]);
        }
        if (half) __syncthreads();
        // a dim's partner in its pair: itself's neighbour, or half of the rotated dims away
        const bool turns = d0 < rot, second = d0 >= half;
        const int away = a.r.interleaved || !turns ? 0 : second ? -half / 8 : half / 8, from = (tid & 63) + away, p0 = d0 + 8 * away;
        const uint32_t one = to_bits<DTYPE>(1.f) * 0x10001u;
        uint4 gain = make_uint4(one, one, one, one), pgain = gain;      // of the dims and of their partners
        if (a.r.eps > 0.f && a.r.k_gamma) {
            gain = load_raw8(a.r.k_gamma, d0, false);
            pgain = load_raw8(a.r.k_gamma, p0, false);
        }
        for (int r0 = 0; r0 < rows; r0 += per_pass) {
            const uint4 raw = next;
            next = fetch(r0 + per_pass + mine);
            const int r = min(r0 + mine, rows - 1), t = token_of(r), hh = r - t * hg;
            float x[8];
            floats_of<DTYPE>(raw, x);
            if (a.r.eps > 0.f || rot) {
                double f = 1.;
                if (a.r.eps > 0.f) {
                    double sum = 0.;
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum = fma((double)x[i], (double)x[i], sum);
                    for (int m = L / 2; m > 0; m >>= 1) sum += __shfl_xor(sum, m);
                    f = 1. / sqrt(sum / (double)D + (double)a.r.eps);
                }
                float y[8];
                if (rot && !a.r.interleaved)
                    floats_of<DTYPE>(make_uint4(__shfl((int)raw.x, from), __shfl((int)raw.y, from), __shfl((int)raw.z, from), __shfl((int)raw.w, from)), y);
                const double2 *at = cs + t * half;
                float g[8], pg[8];
                floats_of<DTYPE>(gain, g);
                floats_of<DTYPE>(pgain, pg);
                if (turns && a.r.interleaved) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const double2 w = at[((sub & 1) * 4 + i) * eighth + (sub >> 1)];
                        const double u = (double)x[2 * i] * f * g[2 * i], v = (double)x[2 * i + 1] * f * g[2 * i + 1];
                        x[2 * i] = to_odd(u * w.x - v * w.y);
                        x[2 * i + 1] = to_odd(u * w.y + v * w.x);
                    }
                } else if (turns) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const double2 w = at[i * eighth + (second ? sub - eighth : sub)];
                        const double u = (double)x[i] * f * g[i], v = (double)y[i] * f * pg[i];
                        x[i] = to_odd(second ? v * w.y + u * w.x : u * w.x - v * w.y);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = to_odd((double)x[i] * f * g[i]);
                }
            }
            float most = tame8(x, huge);
            most = fmaxf(most, __shfl_xor(most, 1));
            most = fmaxf(most, __shfl_xor(most, 2));
            const int byte = scale_byte(most);
            const uint32_t w = floats_to_e2m1(x, power_of(byte));
            if (r0 + mine < rows) {
                const int tok = lo + t;
                const int64_t place = place0 + hh;
                *reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(a.c.k) + (place * page + tok) * (D / 2) + d0 / 2) = w;
                if (sub % 4 == 0) a.c.k_byte[(place * page + piece * SUB) * (D / 32) + (tok & 3) * (D / 8) + d0 / 8 + (tok >> 2 & 3)] = (uint8_t)byte;
            }
        }
        return;
    }

    // ---- values: [row][D / 2] codes of pairs of dims in LDS
    const int row_bytes = D / 2 + 4;
    const bool old = in0 > 0;
    for (int r0 = 0; r0 < rows; r0 += per_pass) {
        const uint4 raw = next;
        next = fetch(r0 + per_pass + mine);
        const int r = min(r0 + mine, rows - 1), t = token_of(r), hh = r - t * hg;
        float x[8];
        floats_of<DTYPE>(raw, x);
        float most = tame8(x, huge);
        for (int m = L / 2; m > 0; m >>= 1) most = fmaxf(most, __shfl_xor(most, m));
        const int byte = scale_byte(most);
        const uint32_t w = floats_to_e2m1(x, power_of(byte));
        if (r0 + mine < rows) {
            *reinterpret_cast<uint32_t *>(write4_lds + r * row_bytes + d0 / 2) = w;
            if (sub == 0) a.c.v_byte[(place0 + hh) * page + lo + t] = (uint8_t)byte;
        }
    }
    __syncthreads();
    for (int e = tid; e < hg * (D / 2); e += WRITE_THREADS) {
        const int hh = e >> (shift - 1), pair = e & (D / 2 - 1);
        uint4 *p = reinterpret_cast<uint4 *>(static_cast<uint8_t *>(a.c.v) + ((place0 + hh) * page + piece * SUB) * (D / 2) + pair * 16);
        uint64_t u = 0, v = 0;
        if (old) {
            const uint4 have = *p;
            const uint64_t keep = (1ull << (4 * in0)) - 1;      // in0 is 15 at most
            u = (have.x | (uint64_t)have.y << 32) & keep;
            v = (have.z | (uint64_t)have.w << 32) & keep;
        }
        for (int t = 0; t < n; ++t) {
            const uint64_t c = write4_lds[(t * hg + hh) * row_bytes + pair];
            u |= (c & 15) << (4 * (in0 + t));
            v |= (c >> 4) << (4 * (in0 + t));
        }
        *p = make_uint4((uint32_t)u, (uint32_t)(u >> 32), (uint32_t)v, (uint32_t)(v >> 32));
    }
}

// Eight codes as 16-bit numbers.
template <int DTYPE>
__device__ __forceinline__ uint4 e2m1_to_16bit(uint32_t w, float s)
{
    const auto p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), q = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
    const auto r = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2), t = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3);
    return make_uint4(pack2<DTYPE>(p[0], p[1]), pack2<DTYPE>(q[0], q[1]), pack2<DTYPE>(r[0], r[1]), pack2<DTYPE>(t[0], t[1]));
}

// Sixteen entries of the list and one head.  A thread takes eight dims: of an entry's key (four bytes in, sixteen out), and of the values of
// as many entries as there are turns for, whose pieces of sixteen tokens it loads anew only where the next entry lies in another one.  Prefixes of 25 thousand
// tokens (105 MB) 20.8 us, 5.05 TB/s, which is a copy's rate; with 32 dims of a key and two of a value a thread 30.6.
template <int DTYPE>
__global__ void __launch_bounds__(256) k_kv4_gather(moe_kv_cache_t c, uint32_t first, const int32_t *slots, int n, void *k_out, void *v_out)
{
    const int D = c.head_dim, shift = 31 - __builtin_clz(D), L = D / 8, page_shift = 31 - __builtin_clz(c.page), page = c.page, heads = c.kv_heads;
    const uint32_t block = first + blockIdx.x;      // of the whole grid
    const int head = block % heads, e0 = (block / heads) * SUB, tid = threadIdx.x & 127, sub = tid & (L - 1), mine = tid >> (shift - 3), at_once = 128 >> (shift - 3);
    const int m = min(SUB, n - e0);
    const uint32_t limit = (uint32_t)c.n_pages * page;
    if (threadIdx.x < 128) {
        for (int e = mine; e < m; e += at_once) {
            const int slot = slots[e0 + e];
            const bool good = (uint32_t)slot < limit;
            const int id = good ? slot >> page_shift : 0, tok = good ? slot & (page - 1) : 0;
            const int64_t place = (int64_t)id * heads + head;
            uint32_t w = *reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(c.k) + (place * page + tok) * (D / 2) + sub * 4);
            float s = power_of(c.k_byte[(place * page + (tok & ~15)) * (D / 32) + (tok & 3) * (D / 8) + (sub & ~3) + (tok >> 2 & 3)]);
            if (!good) {
                w = 0;
                s = 1.f;
            }
            *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(k_out) + ((int64_t)(e0 + e) * heads + head) * D + sub * 8) = e2m1_to_16bit<DTYPE>(w, s);
        }
        return;
    }
    // neighbouring entries, which mostly lie in the same piece
    const int each = SUB / at_once;
    int have = -1;
    uint64_t x[8];
    for (int f = mine * each; f < min(m, (mine + 1) * each); ++f) {
        const int slot = slots[e0 + f];
        uint4 out = make_uint4(0, 0, 0, 0);
        if ((uint32_t)slot < limit) {
            const int64_t place = (int64_t)(slot >> page_shift) * heads + head;
            if ((slot >> 4) != have) {
                have = slot >> 4;
                const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(c.v) + (place * page + (slot & (page - 1) & ~15)) * (D / 2) + sub * 64);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint4 u = p[i];
                    x[2 * i] = u.x | (uint64_t)u.y << 32;
                    x[2 * i + 1] = u.z | (uint64_t)u.w << 32;
                }
            }
            uint32_t w = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) w |= ((uint32_t)(x[i] >> (4 * (slot & 15))) & 15) << (4 * i);
            out = e2m1_to_16bit<DTYPE>(w, power_of(c.v_byte[place * page + (slot & (page - 1))]));
        }
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(v_out) + ((int64_t)(e0 + f) * heads + head) * D + sub * 8) = out;
    }
}

}  // namespace kv
}  // namespace moe
