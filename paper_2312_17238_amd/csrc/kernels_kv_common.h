// Shared by the kernels of the paged 8-bit cache: what a plan holds, conversions between codes and numbers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/moe_kv.h"

namespace moe {
namespace kv {

typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));

constexpr int SUB = 16;            // tokens of a 16 x 16 tile of codes
constexpr int KT = 32;             // tokens of a step of the attention kernels: the rows of one matrix instruction
constexpr int ATTEND_WAVES = 4;    // of a block of the attention, two blocks a compute unit; heads of 256 take the registers of both for one
constexpr int ROWS_FEW = 32;       // (token, query head of the group) rows of a block whose waves share out the cached tokens
// Requests of up to this many rows are made of such blocks; the others of blocks whose waves share out the rows, 32 to each.  At
// 32, 64 and 128: 40 rows of 24 requests 17.1, 13.4 and 13.4 us; 96 rows of 16 requests 60.8, 60.8 and 40.7, but the pages of 2048
// requests 12.6, 12.6 and 17.1, as the plan then holds four tiles of a request in registers.
constexpr int FEW_MOST = 64;
constexpr int COMPUTE_UNITS = 256;
// Blocks that cached tokens are shared out to.  With 256 for the many, 512 tokens onto 6000 take 102.6 us instead of 99, with 1024 a
// prompt of 4096 takes 200 instead of 165 (its tiles are split then); for the few, the decode kernel says.
constexpr int BLOCKS_FEW = 2 * COMPUTE_UNITS;
constexpr int BLOCKS_MANY = 2 * COMPUTE_UNITS;
// Steps of a block at least.  Few: one token onto 4000 takes 13.0, 10.5 and 15.4 us at 4, 16 and 64, 11.1 at 24; 8 requests of a token onto
// 2000 to 2600 14.6 at 16, 13.5 at 24, 8 of 4 tokens onto 3000 18.8 and 16.9.  Many: 128 tokens onto 8000 take 68.5 us at 16, 52.7 at 32; 2
// requests of 24 tokens onto 3000 32.4 and 36.2.
constexpr int MIN_KT_FEW = 24, MIN_KT_MANY = 32;
// What joining a tile's parts costs, in steps of a block, and what a block's second tile costs besides.  SPLIT_STEPS at 8, 32 and 128: 24 requests
// of 40 rows that see 1024 tokens 24.9, 13.4 and 13.4 us, one of a token onto 4000 10.7, 10.5 and 18.6.  LINE_STEPS at 0, 64
// and 128: 8 requests of a token onto 2000 to 2600 20.5, 14.6 and 14.8, 64 of a token onto 500 to 8000 67.7, 68.0 and 75.0.
constexpr int SPLIT_STEPS = 32, LINE_STEPS = 64;

// A piece of work, for each kv head: rows [tile * ROWS, ...) of a request against the cached tokens [kt0, kt1) * KT.
struct __align__(16) Item {
    int32_t req, row0, n_new, ctx;      // row0: first packed row of the request; ctx: position of its token
    int32_t tile, kt0, kt1, part;       // part: which partial result, -1: the block holds all and writes the output
    int32_t part0, parts, join, pad;    // the parts that belong together, and where those that are done are counted
};
// New tokens of one page.
struct __align__(16) Segment {
    int32_t row0, count, page_id, offset;
    int32_t pos0, pad[3];
};
struct Header {
    int32_t segments, few_blocks, many, pad[13];
};

// Where a plan's lists lie in its buffer, and how long they can get.
struct Plan {
    Header *head;
    int32_t *positions;
    Segment *segments;
    Item *few, *many;
    int32_t *few_first;                 // [few_blocks + 1]: the items of a block of small requests are [few_first[b], few_first[b + 1])
    int32_t *joins_few, *joins_many;    // [join][kv head]: parts that are done; 0 between launches
    int32_t max_segments, blocks_few, max_few, max_many, max_joins_few, max_joins_many, parts_few, parts_many;
};

__host__ __device__ constexpr int div_up(int a, int b) { return (a + b - 1) / b; }

// a new float from its sixteen bits
template <int DTYPE>
__device__ __forceinline__ float from_bits(uint32_t b)
{
    if constexpr (DTYPE == MOE_KV_F16) return (float)__builtin_bit_cast(_Float16, (uint16_t)b);
    else return __builtin_bit_cast(float, b << 16);
}

// nearest, ties to even; NaN stays NaN
template <int DTYPE>
__device__ __forceinline__ uint32_t to_bits(float x)
{
    if constexpr (DTYPE == MOE_KV_F16) return __builtin_bit_cast(uint16_t, (_Float16)x);
    else return __builtin_bit_cast(uint16_t, (__bf16)x);
}

template <int DTYPE>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    return to_bits<DTYPE>(a) | (to_bits<DTYPE>(b) << 16);
}

template <int FMT>
constexpr float largest_code() { return FMT == MOE_KV_E4M3 ? 448.f : 127.f; }

// Eight codes as fp16 numbers, exact in both formats.
template <int FMT>
__device__ __forceinline__ v8h codes_to_half(uint32_t lo, uint32_t hi)
{
    union { v8h v; v2h p[4]; uint32_t u[4]; } r;
    if constexpr (FMT == MOE_KV_E4M3) {
        r.p[0] = __builtin_bit_cast(v2h, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false));
        r.p[1] = __builtin_bit_cast(v2h, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true));
        r.p[2] = __builtin_bit_cast(v2h, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false));
        r.p[3] = __builtin_bit_cast(v2h, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true));
    } else {
        // code + 128 as the low bits of 1024 .. 1279, then 1152 off
        const v2h bias = {(_Float16)1152.f, (_Float16)1152.f};
        lo ^= 0x80808080u;
        hi ^= 0x80808080u;
        r.u[0] = __builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u);
        r.u[1] = __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u);
        r.u[2] = __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u);
        r.u[3] = __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u);
        for (int i = 0; i < 4; ++i) r.p[i] = r.p[i] - bias;
    }
    return r.v;
}

template <int FMT>
__device__ __forceinline__ float code_to_float(uint32_t byte)
{
    if constexpr (FMT == MOE_KV_E4M3) return __builtin_amdgcn_cvt_f32_fp8((int)byte, 0);
    else return (float)(int8_t)byte;
}

// Four numbers within the largest code (or NaN: 0) as codes, nearest, ties to even.
template <int FMT>
__device__ __forceinline__ uint32_t floats_to_codes(float a, float b, float c, float d)
{
    if constexpr (FMT == MOE_KV_E4M3) {
        int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
    } else {
        const int i = (int)rintf(a), j = (int)rintf(b), k = (int)rintf(c), l = (int)rintf(d);
        return (uint32_t)(i & 255) | ((uint32_t)(j & 255) << 8) | ((uint32_t)(k & 255) << 16) | ((uint32_t)l << 24);
    }
}

}  // namespace kv
}  // namespace moe
