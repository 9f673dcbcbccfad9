// Norm and rotation of queries and keys, and the store of keys and values as 8-bit codes.
//
// A step's queries, keys and values are read once and written once: memory is what it costs.  Queries and
// the cache share a launch.  A query block takes one token's heads (or several tokens'): its angles are worked out once, in fp64 (position * inv_freq
// in turns, its whole turns dropped, then sine and cosine in fp32: at a position of a million a 32-bit angle would be
// off by 0.03), and kept in LDS for all heads.  A cache block takes the new tokens of one page for one head, keys or values: the scale
// belongs to the page, so all of a page's new tokens have to be known before the first is rounded; a thread keeps its numbers in
// registers meanwhile, eight neighbouring dims of a token in each of ITER passes.  The codes then go through LDS, from which
// 16-byte pieces leave in either tile order (a token's 16 dims, a dim's 16 tokens).
#pragma once
#include "kernels_kv_common.h"

namespace moe {
namespace kv {

constexpr int WRITE_THREADS = 256;

struct WriteArgs {
    moe_kv_cache_t c;
    moe_kv_rows_t r;
    Plan p;
    int32_t q_heads, n_tokens;
    int32_t kv_blocks;      // blocks that store; the others turn queries
    int32_t q_tokens;       // tokens of a query block
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

__device__ __forceinline__ float2 angle(int pos, float freq)
{
    double turns = (double)pos * (double)freq * 0.15915494309189533577;   // 1 / 2 pi
    turns -= rint(turns);
    float sn, cs;
    sincospif((float)(2.0 * turns), &sn, &cs);
    return make_float2(cs, sn);
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

template <int DTYPE, int FMT, int ITER>
__global__ void __launch_bounds__(WRITE_THREADS) k_kv_write(WriteArgs a)
{
    const int D = a.c.head_dim, L = D / 8, tid = threadIdx.x, rot = a.r.rot_dim, half = rot / 2;
    const int sub = tid % L, per_pass = WRITE_THREADS / L, d0 = sub * 8;
    extern __shared__ __align__(16) uint8_t write_lds[];
    uint8_t *lds = write_lds;
    const bool rope = rot > 0;

    if ((int)blockIdx.x >= a.kv_blocks) {
        // ---- queries: lds holds (cos, sin) of q_tokens tokens
        float2 *cs = reinterpret_cast<float2 *>(lds);
        const int t0 = (blockIdx.x - a.kv_blocks) * a.q_tokens;
        const int n = min(a.q_tokens, a.n_tokens - t0);
        if (rope) {
            for (int i = tid; i < n * half; i += WRITE_THREADS) cs[i] = angle(max(a.p.positions[t0 + i / half], 0), a.r.inv_freq[i % half]);
            __syncthreads();
        }
        const int rows = n * a.q_heads;
        for (int r0 = 0; r0 < rows; r0 += per_pass) {
            const int r = min(r0 + tid / L, rows - 1);      // lanes past the end repeat the last head, without storing it
            const int t = r / a.q_heads, h = r - t * a.q_heads;
            float x[8];
            load8<DTYPE>(a.r.q, (t0 + t) * a.r.q_stride + h * D + d0, a.vec_q, x);
            if (a.r.eps > 0.f) norm8<DTYPE>(x, a.r.eps, a.r.q_gamma, d0, D);
            if (rope) rotate8(x, cs + t * half, rot, a.r.interleaved, d0);
            if (r0 + tid / L < rows && a.p.positions[t0 + t] >= 0) store8<DTYPE>(a.r.q_out, (t0 + t) * a.r.q_out_stride + h * D + d0, a.vec_qo, x);
        }
        return;
    }

    // ---- keys or values of a page
    const int heads = a.c.kv_heads, page = a.c.page;
    const int which = blockIdx.x & 1, head = (blockIdx.x >> 1) % heads, si = (blockIdx.x >> 1) / heads;
    if (si >= a.p.head->segments) return;
    const Segment s = a.p.segments[si];
    if (s.page_id < 0) return;
    float *scales = which ? a.c.v_scale : a.c.k_scale;
    const int64_t place = (int64_t)s.page_id * heads + head;
    const float old = s.offset ? scales[place] : 0.f;
    __shared__ float red[WRITE_THREADS / 64];
    const int stride = D + 16;                                   // bytes of a token's codes in LDS
    float2 *cs = reinterpret_cast<float2 *>(lds + page * stride);    // (cos, sin) of a pass's tokens
    const float huge = DTYPE == MOE_KV_F16 ? 65504.f : 0x1p100f;    // a code's value may be rounded up from its number: bf16's largest would not fit in fp32

    float x[ITER][8];
    float amax = 0.f;
#pragma unroll
    for (int it = 0; it < ITER; ++it) {
        const int first = it * per_pass;
        if (first < s.count) {
            const int t = min(first + tid / L, s.count - 1);
            if (which) {
                load8<DTYPE>(a.r.v, (s.row0 + t) * a.r.v_stride + head * D + d0, a.vec_v, x[it]);
            } else {
                if (rope) {
                    if (it) __syncthreads();
                    const int n = min(per_pass, s.count - first);
                    for (int i = tid; i < n * half; i += WRITE_THREADS) cs[i] = angle(s.pos0 + first + i / half, a.r.inv_freq[i % half]);
                    __syncthreads();
                }
                load8<DTYPE>(a.r.k, (s.row0 + t) * a.r.k_stride + head * D + d0, a.vec_k, x[it]);
                if (a.r.eps > 0.f) norm8<DTYPE>(x[it], a.r.eps, a.r.k_gamma, d0, D);
                if (rope) rotate8(x[it], cs + (t - first) * half, rot, a.r.interleaved, d0);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float v = x[it][i];
                x[it][i] = v == v ? fminf(fmaxf(v, -huge), huge) : 0.f;
                amax = fmaxf(amax, fabsf(x[it][i]));
            }
        }
    }
    for (int m = 32; m > 0; m >>= 1) amax = fmaxf(amax, __shfl_xor(amax, m));
    if ((tid & 63) == 0) red[tid >> 6] = amax;
    __syncthreads();
    amax = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float scale = fmaxf(page_scale<FMT>(amax), old);
    const bool grew = s.offset && scale > old;
    const float again = grew ? old / scale : 1.f;
    // a power of two has an exact inverse; a scale that something else stored may be no such power
    const bool power = (__builtin_bit_cast(uint32_t, scale) & 0x7FFFFF) == 0;
    const float inv = 1.f / scale;
    const float lim = largest_code<FMT>();
#pragma unroll
    for (int it = 0; it < ITER; ++it) {
        const int t = it * per_pass + tid / L;
        if (t < s.count) {
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = fminf(fmaxf(power ? x[it][i] * inv : x[it][i] / scale, -lim), lim);
            *reinterpret_cast<uint2 *>(lds + (s.offset + t) * stride + d0) =
                make_uint2(floats_to_codes<FMT>(y[0], y[1], y[2], y[3]), floats_to_codes<FMT>(y[4], y[5], y[6], y[7]));
        }
    }
    __syncthreads();

    // Pieces of 16 bytes: of the new tokens, and of the old ones too where the scale grew.
    const int end = s.offset + s.count;
    const int sub0 = grew ? 0 : s.offset / SUB, sub1 = div_up(end, SUB);
    uint8_t *codes = static_cast<uint8_t *>(which ? a.c.v : a.c.k) + place * page * D;
    for (int i = sub0 * D + tid; i < sub1 * D; i += WRITE_THREADS) {
        const int sb = i / D, in = i - sb * D;          // D pieces a sub-block: (tile of 16 dims, token) or one dim
        uint8_t *dst = codes + (int64_t)i * 16;
        uint32_t w[4];
        if (!which) {
            const int tok = sb * SUB + (in & 15), dim = (in >> 4) * 16;
            if (tok >= s.offset && tok < end) {
                const uint4 u = *reinterpret_cast<const uint4 *>(lds + tok * stride + dim);
                *reinterpret_cast<uint4 *>(dst) = u;
                continue;
            }
            if (tok >= end || !grew) continue;          // past the last token, or an old one that stays
        }
        uint4 u = make_uint4(0, 0, 0, 0);
        if (sb * SUB < s.offset) u = *reinterpret_cast<const uint4 *>(dst);
        w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (grew && sb * SUB < s.offset) {
                float y[4];
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const float c = code_to_float<FMT>((w[j] >> (8 * b)) & 255) * again;
                    y[b] = c == c ? c : 0.f;            // bytes past the last token may be anything
                }
                w[j] = floats_to_codes<FMT>(y[0], y[1], y[2], y[3]);
            }
            if (which) {
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const int tok = sb * SUB + 4 * j + b;
                    if (tok >= s.offset) {
                        const uint32_t c = tok < end ? lds[tok * stride + in] : 0;
                        w[j] = (w[j] & ~(255u << (8 * b))) | (c << (8 * b));
                    }
                }
            }
        }
        *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (tid == 0 && (grew || !s.offset)) scales[place] = scale;
}

// Sixteen entries of the list and one head: a thread takes a token's 16 dims (keys) and a dim of all sixteen tokens
// (values, whose piece of sixteen tokens is loaded anew only where the next entry lies in another one).
template <int DTYPE, int FMT>
__global__ void __launch_bounds__(256) k_kv_gather(moe_kv_cache_t c, const int32_t *slots, int n, void *k_out, void *v_out)
{
    const int D = c.head_dim, page = c.page, heads = c.kv_heads;
    const int head = blockIdx.x % heads, e0 = (blockIdx.x / heads) * SUB;
    const int m = min(SUB, n - e0);
    const int limit = c.n_pages * page;
    for (int i = threadIdx.x; i < D; i += 256) {
        const int e = i / (D / 16), dt = i % (D / 16);
        if (e < m) {
            const int slot = slots[e0 + e];
            float x[16] = {};
            if ((unsigned)slot < (unsigned)limit) {
                const int id = slot / page, tok = slot % page;
                const int64_t place = (int64_t)id * heads + head;
                const float s = c.k_scale[place];
                const uint4 u = *reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(c.k) + place * page * D + (tok / SUB) * SUB * D + dt * 256 + (tok % SUB) * 16);
                const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int j = 0; j < 16; ++j) x[j] = code_to_float<FMT>((w[j / 4] >> (8 * (j % 4))) & 255) * s;
            }
            uint4 o[2];
            uint32_t *ow = reinterpret_cast<uint32_t *>(o);
#pragma unroll
            for (int j = 0; j < 8; ++j) ow[j] = pack2<DTYPE>(x[2 * j], x[2 * j + 1]);
            uint4 *dst = reinterpret_cast<uint4 *>(static_cast<uint16_t *>(k_out) + ((int64_t)(e0 + e) * heads + head) * D + dt * 16);
            dst[0] = o[0];
            dst[1] = o[1];
        }
        int have = -1;
        uint64_t piece[2] = {0, 0};
        float s = 0.f;
        for (int f = 0; f < m; ++f) {
            const int slot = slots[e0 + f];
            float x = 0.f;
            if ((unsigned)slot < (unsigned)limit) {
                if (slot / SUB != have) {
                    have = slot / SUB;
                    const int64_t place = (int64_t)(slot / page) * heads + head;
                    s = c.v_scale[place];
                    const uint64_t *src = reinterpret_cast<const uint64_t *>(static_cast<const uint8_t *>(c.v) + place * page * D + ((slot % page) / SUB) * SUB * D + i * 16);
                    piece[0] = src[0];
                    piece[1] = src[1];
                }
                const int b = slot % SUB;
                x = code_to_float<FMT>((uint32_t)((b < 8 ? piece[0] : piece[1]) >> (8 * (b & 7))) & 255) * s;
            }
            static_cast<uint16_t *>(v_out)[((int64_t)(e0 + f) * heads + head) * D + i] = (uint16_t)to_bits<DTYPE>(x);
        }
    }
}

}  // namespace kv
}  // namespace moe
