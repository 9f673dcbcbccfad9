// Norm and rotation of queries and keys, and the store of keys and values as 8-bit codes.
//
// A step's queries, keys and values are read once and written once: memory is what it costs.  Prompts of 8 thousand tokens (207 MB,
// 32 and 8 heads of 128) take 49 us, 4.2 TB/s where a large copy has 5.1; 256 single tokens 10 us, one token 5.8: launch, plan and
// positions one behind the other.  Queries and the cache share a launch.  A query block takes one
// token's heads (or several tokens'): its angles are worked out once, in fp64 (position * inv_freq, its whole
// quarter turns dropped, then the series in fp32: at a position of a million a 32-bit angle would be off by 0.03), and kept in LDS for all heads.  A cache block takes the new tokens of one page, keys or values: the scale
// belongs to the page, so all of a page's new tokens have to be known before the first is rounded; a thread keeps its numbers in
// registers meanwhile, eight neighbouring dims of a token in each of ITER passes.  It takes one head where the requests bring a page's
// worth of tokens, and as many as fill one pass where they bring few (a block a head for one token left 15 of 16
// threads idle and worked the angles out eight times).  The codes then go through LDS, from which
// 16-byte pieces leave in either tile order (a token's 16 dims, a dim's 16 tokens).
#pragma once
#include "kernels_kv_common.h"

namespace moe {
namespace kv {

constexpr int WRITE_THREADS = 256, WRITE_HEADS = 32;

struct WriteArgs {
    moe_kv_cache_t c;
    moe_kv_rows_t r;
    Plan p;
    int32_t q_heads, n_tokens;
    int32_t first;          // block of the whole grid that this launch begins with
    int32_t kv_blocks;      // blocks that store; the others turn queries
    int32_t q_tokens;       // tokens of a query block
    int32_t heads;          // heads of a block that stores, and rows of codes that its LDS holds
    int32_t lds_rows;
    int32_t vec_q, vec_k, vec_v, vec_qo;   // rows that can be moved 16 bytes at a time
};

template <int DTYPE>
__device__ __forceinline__ void load8(const void *base, int64_t at, bool vec, float (&x)[8])
{
    const uint16_t *p = static_cast<const uint16_t *>(base) + at;
    if (vec) {
        const uint4 w = *reinterpret_cast<const uint4 *>(p);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = from_bits<DTYPE>(u[i] & 0xFFFF);
            x[2 * i + 1] = from_bits<DTYPE>(u[i] >> 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = from_bits<DTYPE>(p[i]);
    }
}

template <int DTYPE>
__device__ __forceinline__ void store8(void *base, int64_t at, bool vec, const float (&x)[8])
{
    uint16_t *p = static_cast<uint16_t *>(base) + at;
    if (vec) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(pack2<DTYPE>(x[0], x[1]), pack2<DTYPE>(x[2], x[3]), pack2<DTYPE>(x[4], x[5]), pack2<DTYPE>(x[6], x[7]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = (uint16_t)to_bits<DTYPE>(x[i]);
    }
}

// Cosine and sine of pos * freq.  The nearest quarter turn is taken off in fp64; the rest (pi / 4 at most, rounded by 2^-26 at most) goes
// through the first terms of the two series, whose next ones are below 2^-28: both within 2^-23.7 (4 million points).  The
// hardware's functions, whose argument is in turns, are off by 2^-22.9, which now and then takes a key to the neighbouring code: prompts of 8
// thousand tokens in 49.4 us this way, 47.1 with those.
__device__ __forceinline__ float2 angle(int pos, float freq)
{
    const double quarters = (double)pos * (double)freq * 0.63661977236758134308;   // 2 / pi
    const double n = rint(quarters), turn = n * 0.25 - floor(n * 0.25);             // 0, 1/4, 1/2 or 3/4
    const float y = (float)((quarters - n) * 1.57079632679489661923), z = y * y;
    const float s = fmaf(y * z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), y);
    const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
    const int k = (int)(turn * 4);
    const float a = k & 1 ? s : c, b = k & 1 ? c : s;
    return make_float2(k == 1 || k == 2 ? -a : a, k & 2 ? -b : b);
}

// Norm of one head: `lanes` neighbouring threads hold it, eight dims each.
template <int DTYPE>
__device__ __forceinline__ void norm8(float (&x)[8], float eps, const void *gamma, int d0, int D)
{
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += x[i] * x[i];
    for (int m = D / 16; m > 0; m >>= 1) s += __shfl_xor(s, m);
    const float f = 1.f / sqrtf(s / (float)D + eps);
    if (gamma) {
        float g[8];
        load8<DTYPE>(gamma, d0, false, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * f * g[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= f;
    }
}

// Rotation of one head held the same way; cs: the token's rot/2 (cos, sin).  Every lane of the head takes part.
__device__ __forceinline__ void rotate8(float (&x)[8], const float2 *cs, int rot, bool interleaved, int d0)
{
    if (interleaved) {
        if (d0 < rot) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 t = cs[d0 / 2 + i];
                const float u = x[2 * i], w = x[2 * i + 1];
                x[2 * i] = u * t.x - w * t.y;
                x[2 * i + 1] = u * t.y + w * t.x;
            }
        }
    } else {
        const int half = rot / 2;
        const bool second = d0 >= half;
        const int lane = threadIdx.x & 63;
        const int partner = d0 >= rot ? lane : second ? lane - half / 8 : lane + half / 8;
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __shfl(x[i], partner);
        if (d0 < rot) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 t = cs[(second ? d0 - half : d0) + i];
                x[i] = second ? y[i] * t.y + x[i] * t.x : x[i] * t.x - y[i] * t.y;
            }
        }
    }
}

// 2^e, the smallest with amax <= largest * 2^e, 2^-96 at least
template <int FMT>
__device__ __forceinline__ float page_scale(float amax)
{
    int e = -96;
    if (amax > 0.f) {
        const float m = frexpf(amax / largest_code<FMT>(), &e);
        if (m <= 0.5f) e -= 1;
        e = max(e, -96);
    }
    return ldexpf(1.f, e);
}

// Queries: lds holds (cos, sin) of q_tokens tokens, the first of them t0.
template <int DTYPE>
__device__ __forceinline__ void turn_queries(const WriteArgs &a, int t0, uint8_t *lds)
{
    const int D = a.c.head_dim, shift = 31 - __builtin_clz(D), L = D / 8, tid = threadIdx.x, rot = a.r.rot_dim, half = rot / 2;
    const int sub = tid & (L - 1), mine = tid >> (shift - 3), per_pass = WRITE_THREADS >> (shift - 3), d0 = sub * 8;
    const float per_half = 1.f / (float)half;
    auto over_half = [&](int i) { return (int)(((float)i + 0.5f) * per_half); };       // i / half
    const bool rope = rot > 0;
    float2 *cs = reinterpret_cast<float2 *>(lds);
    const int n = min(a.q_tokens, a.n_tokens - t0), rows = n * a.q_heads;
    // lanes past the end repeat the last head, without storing it
    auto place = [&](int r, int &t, int &h) {
        r = min(r, rows - 1);
        t = a.q_tokens == 1 ? 0 : r / a.q_heads;
        h = r - t * a.q_heads;
    };
    int t, h;
    float x[8], y[8];
    place(mine, t, h);
    load8<DTYPE>(a.r.q, (t0 + t) * a.r.q_stride + h * D + d0, a.vec_q, x);
    if (rope) {
        for (int i = tid; i < n * half; i += WRITE_THREADS) {
            const int u = over_half(i);
            cs[i] = angle(max(a.p.positions[t0 + u], 0), a.r.inv_freq[i - u * half]);
        }
        __syncthreads();
    }
    for (int r0 = 0; r0 < rows; r0 += per_pass) {
        const int tt = t, hh = h;
        place(r0 + per_pass + mine, t, h);
        load8<DTYPE>(a.r.q, (t0 + t) * a.r.q_stride + h * D + d0, a.vec_q, y);     // the next one's, before this one is stored
        if (a.r.eps > 0.f) norm8<DTYPE>(x, a.r.eps, a.r.q_gamma, d0, D);
        if (rope) rotate8(x, cs + tt * half, rot, a.r.interleaved, d0);
        if (r0 + mine < rows && a.p.positions[t0 + tt] >= 0) store8<DTYPE>(a.r.q_out, (t0 + tt) * a.r.q_out_stride + hh * D + d0, a.vec_qo, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = y[i];
    }
}

template <int DTYPE, int FMT, int ITER>
__global__ void __launch_bounds__(WRITE_THREADS) k_kv_write(WriteArgs a)
{
    // Heads are 64, 128 or 256 wide and quotients small: shifts, and products with a reciprocal, in the place of divisions.
    const int D = a.c.head_dim, shift = 31 - __builtin_clz(D), L = D / 8, tid = threadIdx.x, rot = a.r.rot_dim, half = rot / 2;
    const int sub = tid & (L - 1), mine = tid >> (shift - 3), per_pass = WRITE_THREADS >> (shift - 3), d0 = sub * 8;
    const float per_half = 1.f / (float)half;
    auto over_half = [&](int i) { return (int)(((float)i + 0.5f) * per_half); };       // i / half
    extern __shared__ __align__(16) uint8_t write_lds[];
    uint8_t *lds = write_lds;
    const bool rope = rot > 0;
    const int block = a.first + blockIdx.x;

    if (block >= a.kv_blocks) {
        turn_queries<DTYPE>(a, (block - a.kv_blocks) * a.q_tokens, lds);
        return;
    }

    // ---- keys or values of a page, of hg heads
    const int heads = a.c.kv_heads, page = a.c.page, groups = div_up(heads, a.heads);
    constexpr bool ONE = ITER > 1;              // several passes: one head
    const int which = block & 1, si = (block >> 1) / groups, h0 = ((block >> 1) - si * groups) * a.heads, hg = ONE ? 1 : min(a.heads, heads - h0);
    const uint32_t per_hg = ONE ? 0 : 0xFFFF / (uint32_t)hg + 1;
    auto over_hg = [&](int i) { return ONE ? i : (int)((uint32_t)i * per_hg >> 16); };     // i / hg, for i < 2048 and hg <= 32
    const Segment s = a.p.segments[si];         // in flight with the list's length
    if (si >= a.p.head->segments || s.page_id < 0) return;
    float *scales = (which ? a.c.v_scale : a.c.k_scale) + (int64_t)s.page_id * heads + h0;
    uint8_t *codes = static_cast<uint8_t *>(which ? a.c.v : a.c.k) + ((int64_t)s.page_id * heads + h0) * page * D;
    __shared__ uint32_t amax[WRITE_HEADS];
    __shared__ float new_scale[WRITE_HEADS], again[WRITE_HEADS];
    const int stride = D + 16;                                   // bytes of a row's codes in LDS
    float2 *cs = reinterpret_cast<float2 *>(lds + a.lds_rows * stride);    // (cos, sin) of a pass's tokens
    // numbers beyond these are clamped: a code's value may be rounded up from its number, and bf16's largest would not fit in fp32
    const float huge = DTYPE == MOE_KV_F16 ? 65504.f : 0x1p100f;
    if (tid < WRITE_HEADS) amax[tid] = 0;
    const float old = tid < hg && s.offset ? scales[tid] : 0.f;

    // values: the sixteen-token pieces that old and new tokens share, requested before they are needed
    const int end = s.offset + s.count, sub0 = s.offset / SUB, subs = div_up(end, SUB) - sub0;
    const bool shared_piece = which && s.offset % SUB;
    constexpr int KEEP = ONE ? 1 : 4;
    uint4 piece[KEEP];
    if (shared_piece) {
#pragma unroll
        for (int k = 0; k < KEEP; ++k) {
            const int e = min(tid + k * WRITE_THREADS, hg * D - 1), hh = e >> shift;
            piece[k] = *reinterpret_cast<const uint4 *>(codes + (int64_t)hh * page * D + (sub0 * D + e - hh * D) * 16);
        }
    }

    // rows: one head's tokens in ITER passes, or all heads of so few tokens that they are one pass
    float x[ITER][8];
    const int rows = s.count * hg;
    auto place = [&](int it, int &t, int &hh) {
        const int r = min(it * per_pass + mine, rows - 1);
        t = over_hg(r);
        hh = r - t * hg;
    };
    const void *src = which ? a.r.v : a.r.k;
    const int64_t src_stride = which ? a.r.v_stride : a.r.k_stride;
    const bool vec = which ? a.vec_v : a.vec_k;
#pragma unroll
    for (int it = 0; it < ITER; ++it) {
        if (it * per_pass < rows) {
            int t, hh;
            place(it, t, hh);
            load8<DTYPE>(src, (s.row0 + t) * src_stride + (h0 + hh) * D + d0, vec, x[it]);
        }
    }
    __syncthreads();                            // amax is cleared
#pragma unroll
    for (int it = 0; it < ITER; ++it) {
        if (it * per_pass < rows) {
            int t, hh;
            place(it, t, hh);
            if (!which) {
                if (rope) {
                    const int first = hg == 1 ? it * per_pass : 0, n = min(per_pass, s.count - first);
                    if (it) __syncthreads();
                    for (int i = tid; i < n * half; i += WRITE_THREADS) {
                        const int u = over_half(i);
                        cs[i] = angle(s.pos0 + first + u, a.r.inv_freq[i - u * half]);
                    }
                    __syncthreads();
                    if (a.r.eps > 0.f) norm8<DTYPE>(x[it], a.r.eps, a.r.k_gamma, d0, D);
                    rotate8(x[it], cs + (t - first) * half, rot, a.r.interleaved, d0);
                } else if (a.r.eps > 0.f) {
                    norm8<DTYPE>(x[it], a.r.eps, a.r.k_gamma, d0, D);
                }
            }
            float most = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float v = x[it][i];
                x[it][i] = v == v ? fminf(fmaxf(v, -huge), huge) : 0.f;
                most = fmaxf(most, fabsf(x[it][i]));
            }
            for (int m = L / 2; m > 0; m >>= 1) most = fmaxf(most, __shfl_xor(most, m));
            if (sub == 0) atomicMax(&amax[hh], __builtin_bit_cast(uint32_t, most));     // not negative: ordered as its bits are
        }
    }
    __syncthreads();
    if (tid < hg) {
        const float scale = fmaxf(page_scale<FMT>(__builtin_bit_cast(float, amax[tid])), old);
        const bool grew = s.offset && scale > old;
        new_scale[tid] = scale;
        again[tid] = grew ? old / scale : 1.f;
        if (grew || !s.offset) scales[tid] = scale;
    }
    __syncthreads();
    const float lim = largest_code<FMT>();
#pragma unroll
    for (int it = 0; it < ITER; ++it) {
        const int r = it * per_pass + mine;
        if (r < rows) {
            int t, hh;
            place(it, t, hh);
            // a power of two has an exact inverse; a scale that something else stored may be no such power
            const float scale = new_scale[hh], inv = 1.f / scale;
            const bool power = (__builtin_bit_cast(uint32_t, scale) & 0x7FFFFF) == 0;
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = fminf(fmaxf(power ? x[it][i] * inv : x[it][i] / scale, -lim), lim);
            *reinterpret_cast<uint2 *>(lds + r * stride + d0) = make_uint2(floats_to_codes<FMT>(y[0], y[1], y[2], y[3]), floats_to_codes<FMT>(y[4], y[5], y[6], y[7]));
        }
    }
    __syncthreads();

    // codes of old tokens rounded again, from scale to scale; bytes past the last token may be anything
    auto rescale = [&](uint4 &u, float f) {
        uint32_t *w = reinterpret_cast<uint32_t *>(&u);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float y[4];
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const float c = code_to_float<FMT>((w[j] >> (8 * b)) & 255) * f;
                y[b] = c == c ? c : 0.f;
            }
            w[j] = floats_to_codes<FMT>(y[0], y[1], y[2], y[3]);
        }
    };
    if (!which) {
        const int tiles = D / 16;
        if constexpr (ONE) {
            // neighbouring threads: tokens of a tile, so that what they store is in one piece
            for (int e = tid; e < subs * D; e += WRITE_THREADS) {
                const int in = e & (D - 1), sb = e >> shift, t = (sub0 + sb) * SUB + (in & 15) - s.offset, dt = in >> 4;
                if (t >= 0 && t < s.count)
                    *reinterpret_cast<uint4 *>(codes + ((sub0 + sb) * D + in) * 16) = *reinterpret_cast<const uint4 *>(lds + t * stride + dt * 16);
            }
        } else {
            for (int e = tid; e < rows * tiles; e += WRITE_THREADS) {
                const int r = e >> (shift - 4), dt = e & (tiles - 1), t = over_hg(r), hh = r - t * hg, tok = s.offset + t;
                *reinterpret_cast<uint4 *>(codes + (int64_t)hh * page * D + (tok / SUB) * SUB * D + dt * 256 + (tok % SUB) * 16) =
                    *reinterpret_cast<const uint4 *>(lds + r * stride + dt * 16);
            }
        }
        for (int hh = 0; hh < hg; ++hh) {
            const float f = again[hh];
            if (f == 1.f) continue;
            for (int e = tid; e < s.offset * tiles; e += WRITE_THREADS) {
                const int tok = e >> (shift - 4), dt = e & (tiles - 1);
                uint4 *p = reinterpret_cast<uint4 *>(codes + (int64_t)hh * page * D + (tok / SUB) * SUB * D + dt * 256 + (tok % SUB) * 16);
                uint4 u = *p;
                rescale(u, f);
                *p = u;
            }
        }
        return;
    }
    // a piece: a dim's sixteen tokens, old ones, new ones and none
    auto fill = [&](int hh, int sb, int d, uint4 u) {
        uint32_t *w = reinterpret_cast<uint32_t *>(&u);
        const int t0 = sb * SUB - s.offset;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int t = t0 + j;
            if (t >= 0) {
                const uint32_t c = t < s.count ? lds[(t * hg + hh) * stride + d] : 0;
                w[j / 4] = (w[j / 4] & ~(255u << (8 * (j % 4)))) | (c << (8 * (j % 4)));
            }
        }
        *reinterpret_cast<uint4 *>(codes + (int64_t)hh * page * D + (sb * D + d) * 16) = u;
    };
    if (shared_piece) {
#pragma unroll
        for (int k = 0; k < KEEP; ++k) {
            const int e = tid + k * WRITE_THREADS, hh = e >> shift;
            if (e < hg * D) {
                if (again[hh] != 1.f) rescale(piece[k], again[hh]);
                fill(hh, sub0, e - hh * D, piece[k]);
            }
        }
        for (int e = tid + KEEP * WRITE_THREADS; e < hg * D; e += WRITE_THREADS) {
            const int hh = e >> shift;
            uint4 u = *reinterpret_cast<const uint4 *>(codes + (int64_t)hh * page * D + (sub0 * D + e - hh * D) * 16);
            if (again[hh] != 1.f) rescale(u, again[hh]);
            fill(hh, sub0, e - hh * D, u);
        }
    }
    const int skip = shared_piece ? 1 : 0;
    for (int e = tid; e < (subs - skip) * hg * D; e += WRITE_THREADS) {
        const int g = e >> shift, sb = over_hg(g), hh = g - sb * hg;
        fill(hh, sub0 + skip + sb, e - g * D, make_uint4(0, 0, 0, 0));
    }
    for (int hh = 0; hh < hg; ++hh) {
        const float f = again[hh];
        if (f == 1.f) continue;
        for (int e = tid; e < sub0 * D; e += WRITE_THREADS) {
            uint4 *p = reinterpret_cast<uint4 *>(codes + (int64_t)hh * page * D + e * 16);
            uint4 u = *p;
            rescale(u, f);
            *p = u;
        }
    }
}

// Sixteen entries of the list and one head.  Two waves take the keys, a token's 16 dims a thread; two the values, two dims of all
// sixteen tokens a thread, whose pieces of sixteen tokens are loaded anew only where the next entry lies in another one.
template <int DTYPE, int FMT>
__global__ void __launch_bounds__(256) k_kv_gather(moe_kv_cache_t c, uint32_t first, const int32_t *slots, int n, void *k_out, void *v_out)
{
    const int D = c.head_dim, page_shift = 31 - __builtin_clz(c.page), page = c.page, heads = c.kv_heads;
    const uint32_t block = first + blockIdx.x;      // of the whole grid
    const int head = block % heads, e0 = (block / heads) * SUB, tid = threadIdx.x & 127;
    const int m = min(SUB, n - e0);
    const uint32_t limit = (uint32_t)c.n_pages * page;
    const int mine = slots[min(e0 + (int)(threadIdx.x & 15), n - 1)];
    const int tiles = D / 16;
    if (threadIdx.x < 128) {
        for (int i = tid; i < m * tiles; i += 128) {
            const int e = i / tiles, dt = i - e * tiles;
            const int slot = slots[e0 + e];
            const bool good = (uint32_t)slot < limit;
            const int id = good ? slot >> page_shift : 0, tok = good ? slot & (page - 1) : 0;
            const int64_t place = (int64_t)id * heads + head;
            const float s = good ? c.k_scale[place] : 0.f;
            uint4 u = *reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(c.k) + place * page * D + (tok / SUB) * SUB * D + dt * 256 + (tok % SUB) * 16);
            if (!good) u = make_uint4(0, 0, 0, 0);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
            uint4 o[2];
            uint32_t *ow = reinterpret_cast<uint32_t *>(o);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                ow[j] = pack2<DTYPE>(code_to_float<FMT>((w[j / 2] >> (16 * (j % 2))) & 255) * s, code_to_float<FMT>((w[j / 2] >> (16 * (j % 2) + 8)) & 255) * s);
            uint4 *dst = reinterpret_cast<uint4 *>(static_cast<uint16_t *>(k_out) + ((int64_t)(e0 + e) * heads + head) * D + dt * 16);
            dst[0] = o[0];
            dst[1] = o[1];
        }
        return;
    }
    for (int i = tid; i < D / 2; i += 128) {
        int have = -1;
        uint4 piece[2] = {};
        float s = 0.f;
        for (int f = 0; f < m; ++f) {
            const int slot = __builtin_amdgcn_readlane(mine, f);
            uint32_t out = 0;
            if ((uint32_t)slot < limit) {
                if ((slot >> 4) != have) {
                    have = slot >> 4;
                    const int64_t place = (int64_t)(slot >> page_shift) * heads + head;
                    s = c.v_scale[place];
                    const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(c.v) + place * page * D + ((slot & (page - 1)) / SUB) * SUB * D + i * 32);
                    piece[0] = src[0];
                    piece[1] = src[1];
                }
                const int b = slot % SUB, w = b >> 2, at = 8 * (b & 3);
                const uint32_t x = w == 0 ? piece[0].x : w == 1 ? piece[0].y : w == 2 ? piece[0].z : piece[0].w;
                const uint32_t y = w == 0 ? piece[1].x : w == 1 ? piece[1].y : w == 2 ? piece[1].z : piece[1].w;
                out = pack2<DTYPE>(code_to_float<FMT>((x >> at) & 255) * s, code_to_float<FMT>((y >> at) & 255) * s);
            }
            reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(v_out) + ((int64_t)(e0 + f) * heads + head) * D)[i] = out;
        }
    }
}

}  // namespace kv
}  // namespace moe
