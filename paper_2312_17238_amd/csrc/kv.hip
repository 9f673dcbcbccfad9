// C ABI of the paged 8-bit key/value cache (see include/moe_kv.h for the contract): argument checks, where a plan's and the
// scratch's parts lie, launches.  Nothing here waits, allocates on the device or keeps state between calls.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/moe_kv.h"
#include "errors.h"
#include "kernels_kv_attend.h"
#include "kernels_kv_decode.h"
#include "kernels_kv_plan.h"
#include "kernels_kv_write.h"

using namespace moe;
using namespace moe::kv;

static int32_t bad(const char *fmt, ...)
{
    char text[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(text, sizeof(text), fmt, ap);
    va_end(ap);
    return report_error(MOE_EINVAL, 0, text);
}

static int32_t launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return MOE_OK;
    char text[256];
    snprintf(text, sizeof(text), "%s: launch failed: %s", what, hipGetErrorString(e));
    return report_error(MOE_EHIP, (int32_t)e, text);
}

static bool geometry_ok(int32_t n_pages, int32_t page, int32_t kv_heads, int32_t head_dim)
{
    return n_pages >= 1 && (page == 16 || page == 32 || page == 64 || page == 128) && (int64_t)n_pages * page < (1ll << 31) &&
           kv_heads >= 1 && kv_heads <= 256 && (int64_t)n_pages * kv_heads * (page / 16) < (1ll << 32) && (head_dim == 64 || head_dim == 128 || head_dim == 256);
}

static bool step_ok(const moe_kv_step_t *s)
{
    return s && s->n_requests >= 1 && s->n_requests <= MOE_KV_MAX_REQUESTS && s->n_tokens >= 1 && s->n_tokens <= MOE_KV_MAX_TOKENS &&
           s->max_new >= 1 && s->max_blocks >= 1 && geometry_ok(s->n_pages, s->page, s->kv_heads, s->head_dim) &&
           (int64_t)s->max_blocks * s->page <= (1ll << 24) - KT && s->q_heads >= 1 && s->q_heads <= 1024 && s->q_heads % s->kv_heads == 0 &&
           (s->causal == 0 || s->causal == 1) && s->window >= 0 && s->reserved == 0;
}

static bool cache_ok(const moe_kv_cache_t *c)
{
    return c && geometry_ok(c->n_pages, c->page, c->kv_heads, c->head_dim) && (c->format == MOE_KV_E4M3 || c->format == MOE_KV_INT8) &&
           c->reserved == 0 && c->k && c->v && c->k_scale && c->v_scale && !((uintptr_t)c->k & 15) && !((uintptr_t)c->v & 15) &&
           !((uintptr_t)c->k_scale & 3) && !((uintptr_t)c->v_scale & 3);
}

static bool same_geometry(const moe_kv_cache_t *c, const moe_kv_step_t *s)
{
    return c->n_pages == s->n_pages && c->page == s->page && c->kv_heads == s->kv_heads && c->head_dim == s->head_dim;
}

static int log2_of(int v)
{
    int n = 0;
    while ((1 << n) < v) ++n;
    return n;
}

struct Sizes {
    int rows_many;
    int group, new_most;        // new_most: rows that one request can bring
    bool decode;                // none can have more than ROWS_DECODE
    bool many;                  // some request can have more than ROWS_FEW rows
    uint64_t segments, positions, few, few_first, many_at, joins, total;
    Plan p;                     // counts only
};

static int target_blocks(int blocks, int heads) { return std::max(1, blocks / heads); }

static Sizes sizes_of(const moe_kv_step_t *s)
{
    Sizes z{};
    z.rows_many = 32 * ATTEND_WAVES;
    z.group = s->q_heads / s->kv_heads;
    z.new_most = std::min(s->max_new, s->n_tokens);
    z.many = (int64_t)z.new_most * z.group > FEW_MOST;
    z.decode = (int64_t)z.new_most * z.group <= ROWS_DECODE;
    const int R = s->n_requests, T = s->n_tokens;
    const int steps = div_up(s->max_blocks * s->page, KT);          // of one request at most
    Plan &p = z.p;
    p.max_segments = (int)std::min<int64_t>(T, (int64_t)T / s->page + 2ll * R);
    const bool split_many = z.many && steps > MIN_KT_MANY;
    const int tf = target_blocks(z.decode ? COMPUTE_UNITS * decode_blocks(s->head_dim) : BLOCKS_FEW, s->kv_heads), tm = target_blocks(BLOCKS_MANY, s->kv_heads);
    // tiles: of no request more than its rows, or the most rows of one, fill
    const int tiles_few = (int)std::min<int64_t>((int64_t)std::min(R, T) * div_up((int)std::min<int64_t>(FEW_MOST, (int64_t)z.new_most * z.group), ROWS_FEW),
                                                 (int64_t)T * z.group / ROWS_FEW + std::min(R, T));
    const bool split_few = (int64_t)tiles_few * steps > MIN_KT_FEW;     // more than one block
    p.blocks_few = split_few ? tf : tiles_few;
    p.max_few = tiles_few + p.blocks_few;
    const int tiles = z.many ? (int)((int64_t)T * z.group / z.rows_many) + std::min(R, T) : 0;
    p.max_many = tiles + (split_many ? tm : 0);
    p.parts_few = split_few ? 2 * tf : 0;
    p.parts_many = split_many ? 2 * tm : 0;
    p.max_joins_few = std::min(tiles_few, p.parts_few / 2);
    p.max_joins_many = std::min(tiles, p.parts_many / 2);
    uint64_t at = sizeof(Header);
    auto take = [&](uint64_t bytes) {
        const uint64_t here = at;
        at = (at + bytes + 63) & ~63ull;
        return here;
    };
    z.positions = take((uint64_t)T * 4);
    z.segments = take((uint64_t)p.max_segments * sizeof(Segment));
    z.few = take((uint64_t)p.max_few * sizeof(Item));
    z.few_first = take((uint64_t)(p.blocks_few + 1) * 4);
    z.many_at = take((uint64_t)p.max_many * sizeof(Item));
    z.joins = take((uint64_t)(p.max_joins_few + p.max_joins_many) * s->kv_heads * 4);
    z.total = at;
    return z;
}

static Plan plan_at(const Sizes &z, int kv_heads, const void *plan_dev)
{
    uint8_t *b = static_cast<uint8_t *>(const_cast<void *>(plan_dev));
    Plan p = z.p;
    p.head = reinterpret_cast<Header *>(b);
    p.positions = reinterpret_cast<int32_t *>(b + z.positions);
    p.segments = reinterpret_cast<Segment *>(b + z.segments);
    p.few = reinterpret_cast<Item *>(b + z.few);
    p.few_first = reinterpret_cast<int32_t *>(b + z.few_first);
    p.many = reinterpret_cast<Item *>(b + z.many_at);
    p.joins_few = reinterpret_cast<int32_t *>(b + z.joins);
    p.joins_many = p.joins_few + (int64_t)p.max_joins_few * kv_heads;
    return p;
}

static uint64_t part_bytes(int parts, int heads, int rows, int D) { return (uint64_t)parts * heads * rows * (D + 2) * 4; }

extern "C" uint64_t moe_kv_plan_bytes(const moe_kv_step_t *step) { return step_ok(step) ? sizes_of(step).total : 0; }

extern "C" uint64_t moe_kv_scratch_bytes(const moe_kv_step_t *step)
{
    if (!step_ok(step)) return 0;
    const Sizes z = sizes_of(step);
    return part_bytes(z.p.parts_few, step->kv_heads, ROWS_FEW, step->head_dim) + part_bytes(z.p.parts_many, step->kv_heads, z.rows_many, step->head_dim);
}

extern "C" int32_t moe_kv_plan(const moe_kv_step_t *step, const moe_kv_lists_t *io, void *plan_dev, void *stream)
{
    return moe_kv_plan_within(step, io, step ? step->n_pages : 1, plan_dev, stream);
}

extern "C" int32_t moe_kv_plan_within(const moe_kv_step_t *step, const moe_kv_lists_t *io, int32_t free_capacity, void *plan_dev, void *stream)
{
    if (!step_ok(step)) return bad("moe_kv_plan: bad or unsupported step");
    if (free_capacity < 1) return bad("moe_kv_plan: a stack of %d free pages", free_capacity);
    if (!io || !plan_dev || ((uintptr_t)plan_dev & 255)) return bad("moe_kv_plan: null lists, or a plan that is null or not 256-byte aligned");
    const void *in[] = {io->ctx_len, io->new_len, io->free_pages, io->free_count, io->block_table};
    const void *out[] = {io->row_start, io->positions, io->slots, io->kv_len, io->status, io->free_left};
    for (const void *p : in)
        if (!p || ((uintptr_t)p & 3)) return bad("moe_kv_plan: a null or misaligned list");
    for (const void *p : out) {
        if (!p || ((uintptr_t)p & 3)) return bad("moe_kv_plan: a null or misaligned list");
        for (const void *q : in)
            if (p == q) return bad("moe_kv_plan: an output is an input");
    }
    const Sizes z = sizes_of(step);
    PlanArgs a{*step, *io, plan_at(z, step->kv_heads, plan_dev), std::min(free_capacity, step->n_pages), z.group, log2_of(step->page), z.p.blocks_few, target_blocks(BLOCKS_MANY, step->kv_heads), z.rows_many, std::min(8, std::max(1, div_up(z.p.max_many, PLAN_MOST_THREADS)))};
    const int R = step->n_requests, threads = R <= 64 ? 64 : R <= 256 ? 256 : PLAN_MOST_THREADS;
    const dim3 grid(1 + a.many_blocks + std::min(240, div_up(std::max(step->n_tokens, z.p.max_segments), threads)));
    const size_t lds = (size_t)R * 12;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (threads == 64) hipLaunchKernelGGL((k_kv_plan<64, 1>), grid, dim3(64), lds, st, a);
    else if (threads == 256) hipLaunchKernelGGL((k_kv_plan<256, 1>), grid, dim3(256), lds, st, a);
    else hipLaunchKernelGGL((k_kv_plan<PLAN_MOST_THREADS, MOE_KV_MAX_REQUESTS / PLAN_MOST_THREADS>), grid, dim3(PLAN_MOST_THREADS), lds, st, a);
    return launched("moe_kv_plan");
}

extern "C" int32_t moe_kv_release(const int32_t *requests, int32_t n, int32_t n_requests, int32_t n_pages, int32_t page, int32_t max_blocks,
                                  int32_t *ctx_len, const int32_t *block_table, int32_t *free_pages, int32_t capacity,
                                  int32_t *free_count, void *stream)
{
    if (n < 0 || n_requests < 1 || max_blocks < 1 || capacity < 1 || !geometry_ok(n_pages, page, 1, 64)) return bad("moe_kv_release: a bad size");
    if (n == 0) return MOE_OK;
    for (const void *p : {(const void *)requests, (const void *)ctx_len, (const void *)block_table, (const void *)free_pages, (const void *)free_count})
        if (!p || ((uintptr_t)p & 3)) return bad("moe_kv_release: a null or misaligned list");
    hipLaunchKernelGGL(k_kv_release, dim3(1), dim3(256), 0, static_cast<hipStream_t>(stream), requests, n, n_requests, n_pages, page, max_blocks, ctx_len, block_table,
                       free_pages, capacity, free_count);
    return launched("moe_kv_release");
}

// A launch has fewer than 2^32 threads: `launch(first, blocks)` for pieces of a grid of blocks of 256.
constexpr int64_t MOST_BLOCKS = (1ll << 24) - 1;

template <class F>
static void in_pieces(int64_t blocks, F launch)
{
    for (int64_t first = 0; first < blocks; first += MOST_BLOCKS) launch((uint32_t)first, (unsigned)std::min(MOST_BLOCKS, blocks - first));
}

static bool rows16(const void *p, int64_t stride) { return !((uintptr_t)p & 15) && stride % 8 == 0; }

template <int DTYPE, int FMT>
static void launch_write(const WriteArgs &a, int iter, dim3 grid, size_t lds, hipStream_t s)
{
    switch (iter) {
    case 1: hipLaunchKernelGGL((k_kv_write<DTYPE, FMT, 1>), grid, dim3(WRITE_THREADS), lds, s, a); break;
    case 2: hipLaunchKernelGGL((k_kv_write<DTYPE, FMT, 2>), grid, dim3(WRITE_THREADS), lds, s, a); break;
    case 4: hipLaunchKernelGGL((k_kv_write<DTYPE, FMT, 4>), grid, dim3(WRITE_THREADS), lds, s, a); break;
    case 8: hipLaunchKernelGGL((k_kv_write<DTYPE, FMT, 8>), grid, dim3(WRITE_THREADS), lds, s, a); break;
    default: hipLaunchKernelGGL((k_kv_write<DTYPE, FMT, 16>), grid, dim3(WRITE_THREADS), lds, s, a); break;
    }
}

extern "C" int32_t moe_kv_write(const moe_kv_cache_t *cache, const moe_kv_step_t *step, const void *plan_dev, const moe_kv_rows_t *rows, void *stream)
{
    if (!cache_ok(cache)) return bad("moe_kv_write: bad or unsupported cache");
    if (!step_ok(step) || !same_geometry(cache, step)) return bad("moe_kv_write: bad step, or one for another cache");
    if (!plan_dev || ((uintptr_t)plan_dev & 255)) return bad("moe_kv_write: the plan is null or not 256-byte aligned");
    if (!rows || !rows->q || !rows->k || !rows->v || !rows->q_out) return bad("moe_kv_write: null rows");
    const moe_kv_rows_t &r = *rows;
    const int D = cache->head_dim;
    if (r.dtype != MOE_KV_F16 && r.dtype != MOE_KV_BF16) return bad("moe_kv_write: unknown type %d", r.dtype);
    if (r.rot_dim < 0 || r.rot_dim > D || r.rot_dim % 16 || (r.interleaved != 0 && r.interleaved != 1)) return bad("moe_kv_write: rot_dim %d is no multiple of 16 up to %d", r.rot_dim, D);
    if (r.rot_dim && !r.inv_freq) return bad("moe_kv_write: a rotation needs inv_freq");
    if (!(r.eps >= 0.f) || std::isinf(r.eps)) return bad("moe_kv_write: eps is negative or no number");
    if (((uintptr_t)r.q | (uintptr_t)r.k | (uintptr_t)r.v | (uintptr_t)r.q_out | (uintptr_t)r.q_gamma | (uintptr_t)r.k_gamma) & 1 || ((uintptr_t)r.inv_freq & 3))
        return bad("moe_kv_write: a misaligned pointer");
    if (r.q_stride < (int64_t)step->q_heads * D || r.q_out_stride < (int64_t)step->q_heads * D || r.k_stride < (int64_t)cache->kv_heads * D || r.v_stride < (int64_t)cache->kv_heads * D)
        return bad("moe_kv_write: rows overlap");
    if (r.q == r.q_out && r.q_stride != r.q_out_stride) return bad("moe_kv_write: q_out is q with another stride");
    const Sizes z = sizes_of(step);
    WriteArgs a{};
    a.c = *cache;
    a.r = r;
    a.p = plan_at(z, step->kv_heads, plan_dev);
    a.q_heads = step->q_heads;
    a.n_tokens = step->n_tokens;
    const int per_pass = WRITE_THREADS / (D / 8), angles = r.rot_dim / 2 * 8, most = std::min(cache->page, z.new_most);
    // heads of a block that stores: as many as fill a pass where requests bring few tokens (256 of one token: 9.6 us, a head a block 15.4)
    a.heads = std::max(1, std::min(std::min(cache->kv_heads, WRITE_HEADS), per_pass / most));
    a.lds_rows = std::max(most, a.heads * most);
    a.kv_blocks = z.p.max_segments * div_up(cache->kv_heads, a.heads) * 2;
    // Two tokens of a query block once there are blocks enough: 8 thousand tokens 47.9 us, with four 48.6; one fills more of the GPU before that.
    a.q_tokens = step->n_tokens >= 2048 ? 2 : 1;
    a.vec_q = rows16(r.q, r.q_stride);
    a.vec_k = rows16(r.k, r.k_stride);
    a.vec_v = rows16(r.v, r.v_stride);
    a.vec_qo = rows16(r.q_out, r.q_out_stride);
    // queries that neither turn nor move need no block
    const bool turn = r.rot_dim || r.eps > 0.f || r.q != r.q_out;
    const int64_t blocks = (int64_t)z.p.max_segments * div_up(cache->kv_heads, a.heads) * 2 + (turn ? div_up(step->n_tokens, a.q_tokens) : 0);
    const size_t lds = std::max<size_t>((size_t)a.lds_rows * (D + 16) + per_pass * angles, (size_t)a.q_tokens * angles);
    int iter = 1;
    while (iter * per_pass < a.lds_rows) iter *= 2;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    in_pieces(blocks, [&](uint32_t first, unsigned n) {
        a.first = (int32_t)first;
        if (r.dtype == MOE_KV_F16) {
            if (cache->format == MOE_KV_E4M3) launch_write<MOE_KV_F16, MOE_KV_E4M3>(a, iter, dim3(n), lds, s);
            else launch_write<MOE_KV_F16, MOE_KV_INT8>(a, iter, dim3(n), lds, s);
        } else {
            if (cache->format == MOE_KV_E4M3) launch_write<MOE_KV_BF16, MOE_KV_E4M3>(a, iter, dim3(n), lds, s);
            else launch_write<MOE_KV_BF16, MOE_KV_INT8>(a, iter, dim3(n), lds, s);
        }
    });
    return launched("moe_kv_write");
}

template <int DTYPE, int FMT>
static void launch_attend(const AttendArgs &a, int D, bool decode, dim3 grid, hipStream_t s)
{
    if (decode) {
        switch (D) {
        case 64: hipLaunchKernelGGL((k_kv_decode<DTYPE, FMT, 64>), grid, dim3(64 * DECODE_WAVES), 0, s, a); break;
        case 128: hipLaunchKernelGGL((k_kv_decode<DTYPE, FMT, 128>), grid, dim3(64 * DECODE_WAVES), 0, s, a); break;
        default: hipLaunchKernelGGL((k_kv_decode<DTYPE, FMT, 256>), grid, dim3(64 * DECODE_WAVES), 0, s, a); break;
        }
        return;
    }
    switch (D) {
    case 64: hipLaunchKernelGGL((k_kv_attend<DTYPE, FMT, 64>), grid, dim3(64 * ATTEND_WAVES), 0, s, a); break;
    case 128: hipLaunchKernelGGL((k_kv_attend<DTYPE, FMT, 128>), grid, dim3(64 * ATTEND_WAVES), 0, s, a); break;
    default: hipLaunchKernelGGL((k_kv_attend<DTYPE, FMT, 256>), grid, dim3(64 * ATTEND_WAVES), 0, s, a); break;
    }
}

extern "C" int32_t moe_kv_attend(const moe_kv_cache_t *cache, const moe_kv_step_t *step, const void *plan_dev, const int32_t *block_table,
                                 const moe_kv_query_t *query, void *scratch, uint64_t scratch_bytes, void *stream)
{
    if (!cache_ok(cache)) return bad("moe_kv_attend: bad or unsupported cache");
    if (!step_ok(step) || !same_geometry(cache, step)) return bad("moe_kv_attend: bad step, or one for another cache");
    if (!plan_dev || ((uintptr_t)plan_dev & 255)) return bad("moe_kv_attend: the plan is null or not 256-byte aligned");
    if (!block_table || ((uintptr_t)block_table & 3)) return bad("moe_kv_attend: null or misaligned block table");
    if (!query || !query->q || !query->out) return bad("moe_kv_attend: null query or output");
    const moe_kv_query_t &q = *query;
    const int D = cache->head_dim;
    if (q.dtype != MOE_KV_F16 && q.dtype != MOE_KV_BF16) return bad("moe_kv_attend: unknown type %d", q.dtype);
    if (!(q.scale > 0.f) || std::isinf(q.scale)) return bad("moe_kv_attend: the scale has to be a positive number");
    if (((uintptr_t)q.q | (uintptr_t)q.out) & 1 || ((uintptr_t)q.lse & 3)) return bad("moe_kv_attend: a misaligned pointer");
    if (q.q == q.out) return bad("moe_kv_attend: the output is the query");
    if (q.q_stride < (int64_t)step->q_heads * D || q.out_stride < (int64_t)step->q_heads * D) return bad("moe_kv_attend: rows overlap");
    const uint64_t need = moe_kv_scratch_bytes(step);
    if (scratch_bytes < need || (need && (!scratch || ((uintptr_t)scratch & 15))))
        return report_error(MOE_ENOMEM, 0, "moe_kv_attend: the scratch is null, not 16-byte aligned or smaller than moe_kv_scratch_bytes");
    const Sizes z = sizes_of(step);
    AttendArgs a{};
    a.c = *cache;
    a.q = q;
    a.p = plan_at(z, step->kv_heads, plan_dev);
    a.table = block_table;
    a.part_few = static_cast<float *>(scratch);
    a.part_many = scratch ? reinterpret_cast<float *>(static_cast<uint8_t *>(scratch) + part_bytes(z.p.parts_few, cache->kv_heads, ROWS_FEW, D)) : nullptr;
    a.group = z.group;
    a.max_blocks = step->max_blocks;
    a.causal = step->causal;
    a.window = step->window;
    a.per_group = 1.f / z.group;
    a.sub_shift = log2_of(cache->page / SUB);
    a.vec_q = rows16(q.q, q.q_stride);
    a.vec_out = rows16(q.out, q.out_stride);
    // below 2^24: a million rows of 1024 query heads are 2^23 tiles, 4096 requests of 256 heads have 2^20 more
    const int64_t many = (int64_t)z.p.max_many * cache->kv_heads, blocks = many + (int64_t)z.p.blocks_few * cache->kv_heads;
    a.many_blocks = (int32_t)many;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)blocks);
    if (q.dtype == MOE_KV_F16) {
        if (cache->format == MOE_KV_E4M3) launch_attend<MOE_KV_F16, MOE_KV_E4M3>(a, D, z.decode, grid, s);
        else launch_attend<MOE_KV_F16, MOE_KV_INT8>(a, D, z.decode, grid, s);
    } else {
        if (cache->format == MOE_KV_E4M3) launch_attend<MOE_KV_BF16, MOE_KV_E4M3>(a, D, z.decode, grid, s);
        else launch_attend<MOE_KV_BF16, MOE_KV_INT8>(a, D, z.decode, grid, s);
    }
    return launched("moe_kv_attend");
}

extern "C" int32_t moe_kv_gather(const moe_kv_cache_t *cache, const int32_t *slots, int32_t n, int32_t dtype, void *k_out, void *v_out, void *stream)
{
    if (!cache_ok(cache)) return bad("moe_kv_gather: bad or unsupported cache");
    if (n < 0 || n > (1 << 26) || (dtype != MOE_KV_F16 && dtype != MOE_KV_BF16)) return bad("moe_kv_gather: bad count or type");
    if (n == 0) return MOE_OK;
    if (!slots || !k_out || !v_out || (((uintptr_t)k_out | (uintptr_t)v_out) & 15) || ((uintptr_t)slots & 3)) return bad("moe_kv_gather: a null or misaligned pointer");
    const hipStream_t s = static_cast<hipStream_t>(stream);
    in_pieces((int64_t)div_up(n, SUB) * cache->kv_heads, [&](uint32_t first, unsigned blocks) {
        const dim3 grid(blocks);
        if (dtype == MOE_KV_F16) {
            if (cache->format == MOE_KV_E4M3) hipLaunchKernelGGL((k_kv_gather<MOE_KV_F16, MOE_KV_E4M3>), grid, dim3(256), 0, s, *cache, first, slots, n, k_out, v_out);
            else hipLaunchKernelGGL((k_kv_gather<MOE_KV_F16, MOE_KV_INT8>), grid, dim3(256), 0, s, *cache, first, slots, n, k_out, v_out);
        } else {
            if (cache->format == MOE_KV_E4M3) hipLaunchKernelGGL((k_kv_gather<MOE_KV_BF16, MOE_KV_E4M3>), grid, dim3(256), 0, s, *cache, first, slots, n, k_out, v_out);
            else hipLaunchKernelGGL((k_kv_gather<MOE_KV_BF16, MOE_KV_INT8>), grid, dim3(256), 0, s, *cache, first, slots, n, k_out, v_out);
        }
    });
    return launched("moe_kv_gather");
}
