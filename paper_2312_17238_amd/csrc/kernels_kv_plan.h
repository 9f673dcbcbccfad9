// The pages of a step and how its attention is shared out, from the requests' lengths.
//
// Everything follows from prefix sums over the requests: rows (where a request's rows lie), pages needed (which free pages
// it gets), pages touched (the segments that the store works on), tiles of rows and steps over cached tokens (the attention's
// blocks).  Up to 4096 requests are 16 KB of lengths, so every block of the launch makes the sums it needs by
// itself, in LDS, and there is no exchange between blocks: block 0 writes what is per request and shares out the requests of
// few rows, the next ones those of many, the others look up rows and pages with a binary search in the sums.  Latency is all there is
// to it: 2048 requests with 77 thousand rows move 0.7 MB.
#pragma once
#include "kernels_common.h"
#include "kernels_kv_common.h"

namespace moe {
namespace kv {

constexpr int PLAN_MOST_THREADS = 1024;

struct PlanArgs {
    moe_kv_step_t s;
    moe_kv_lists_t io;
    Plan p;
    int32_t free_most;      // entries of the stack that may be read
    int32_t group, page_shift, target_few, target_many, rows_many;
    int32_t many_blocks;    // blocks that share out the requests of many rows
};

// a + b, 2^32 - 1 at most: sums of lengths that no batch can have stay above every bound they are compared with
__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_or_0(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}

__device__ __forceinline__ uint32_t wave_scan(uint32_t v)
{
    v = add_sat(v, dpp_or_0<0x111, 0xf>(v));    // row_shr 1, 2, 4, 8: sums within sixteen lanes
    v = add_sat(v, dpp_or_0<0x112, 0xf>(v));
    v = add_sat(v, dpp_or_0<0x114, 0xf>(v));
    v = add_sat(v, dpp_or_0<0x118, 0xf>(v));
    v = add_sat(v, dpp_or_0<0x142, 0xa>(v));    // row_bcast 15 into rows 1 and 3, 31 into rows 2 and 3
    v = add_sat(v, dpp_or_0<0x143, 0xc>(v));
    return v;
}

// Inclusive sum over the block's threads in their order; *total receives the whole sum.  `tmp`: a number a wave, in LDS.
template <int THREADS>
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t *tmp, uint32_t *total)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    v = wave_scan(v);
    if constexpr (THREADS == 64) {
        *total = (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
        return v;
    } else {
        __syncthreads();          // the last scan's readers are done with tmp
        if (lane == 63) tmp[wave] = v;
        __syncthreads();
        const uint32_t sums = wave_scan(lane < THREADS / 64 ? tmp[lane] : 0);
        *total = (uint32_t)__builtin_amdgcn_readlane((int)sums, 63);
        return add_sat(v, wave ? (uint32_t)__shfl((int)sums, wave - 1) : 0);
    }
}

// Sum of whole numbers below 2^53 in all, in every thread.
template <int THREADS>
__device__ __forceinline__ double block_sum(double v, double *tmp)
{
    v = wave_sum_f64(v);
    if constexpr (THREADS > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
        __syncthreads();
        const int lane = threadIdx.x & 63;
        v = wave_sum_f64(lane < THREADS / 64 ? tmp[lane] : 0.0);
    }
    return v;
}

template <int THREADS>
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t *tmp)
{
    for (int d = 32; d > 0; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
    if constexpr (THREADS > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
        __syncthreads();
        for (int w = 0; w < THREADS / 64; ++w) v = max(v, tmp[w]);
    }
    return v;
}

// first i with sums[i] > x, sums ascending; n if there is none
__device__ __forceinline__ int first_above(const int32_t *sums, int n, int x)
{
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid] > x) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// Steps [kt0, kt1) over the cached tokens that rows of a request see, tokens [tok_first, tok_last].
__host__ __device__ __forceinline__ void key_steps(const moe_kv_step_t &s, int ctx, int n_new, int tok_first, int tok_last, int &kt0, int &kt1)
{
    const int hi = s.causal ? ctx + tok_last + 1 : ctx + n_new, first = ctx + tok_first + 1 - s.window;
    const int lo = s.window > 0 && first > 0 ? first : 0;
    kt0 = lo / KT;
    kt1 = (hi + KT - 1) / KT;
}

// The steps of a block where `all` steps are shared out to `target` blocks of at least `least`.  A million rows of a thousand heads
// have up to 2^42 steps: no tile is split from 2^19 on, so what a block gets beyond an int is cut off.
__host__ __device__ __forceinline__ int share(double all, int target, int least)
{
    const int64_t even = ((int64_t)all + target - 1) / target;
    return even > least ? even < 0x7FFFFFFF ? (int)even : 0x7FFFFFFF : least;
}

// Tiles of few rows: the steps of a block.
__host__ __device__ __forceinline__ uint32_t first_chunk(uint32_t line, uint32_t tiles, uint32_t target)
{
    const uint32_t even = (line + target - 1) / target, least = tiles <= target ? MIN_KT_FEW : 1;
    return even > least ? even : least;
}

// Where there is a block for every tile (tiles <= target): the steps of a block if tiles begin with a block of their own, 0 if they had better
// not.  `blocks`: how many blocks first_chunk's steps would make that way, where the longest tile takes more than one.
// Costs are compared in steps: SPLIT_STEPS to join a tile's parts, LINE_STEPS for a block with the end of one tile and the beginning of another.
__host__ __device__ __forceinline__ uint32_t own_chunk(uint32_t line, uint32_t tiles, uint32_t target, uint32_t longest, uint32_t chunk, uint32_t blocks)
{
    if (longest <= chunk + SPLIT_STEPS) return longest > 1 ? longest : 1;      // a tile a block
    if (blocks <= target) return chunk;
    // of c steps there are no more than (line + tiles (c - 1)) / c blocks
    uint32_t own = tiles < target ? (line - tiles + target - tiles - 1) / (target - tiles) : longest;
    if (longest <= own + SPLIT_STEPS) own = longest;
    return own + (own < longest ? SPLIT_STEPS : 0) <= chunk + SPLIT_STEPS + LINE_STEPS ? own : 0;
}

// Writes the items of one tile, in as many parts as `n`.
__device__ __forceinline__ void put_items(Item *items, Item it, int n, int item0, int join, int part0)
{
    const int lo = it.kt0, len = it.kt1 - it.kt0;
    it.part0 = part0;
    it.parts = n;
    it.join = join;
    if (n == 1) {
        it.part = -1;
        items[item0] = it;
        return;
    }
    for (uint32_t p = 0; p < (uint32_t)n; ++p) {        // less than 2^19 steps, 2^11 parts
        it.kt0 = lo + (int)((uint32_t)len * p / (uint32_t)n);
        it.kt1 = lo + (int)((uint32_t)len * (p + 1) / (uint32_t)n);
        it.part = part0 + (int)p;
        items[item0 + p] = it;
    }
}

// THREADS: a thread has at most PER requests.  One wave's sums need no LDS and no barrier: 8 requests take 3.5 us with 64 threads and 5.0 with
// 256, 200 requests 5.1 with 256 and 6.9 with 1024.  2048 requests of 77 thousand rows take 12.6 us; with one block for the requests of
// many rows 14.8, with that block sharing out the others' too 17.
template <int THREADS, int PER>
__global__ void __launch_bounds__(THREADS) k_kv_plan(PlanArgs a)
{
    extern __shared__ int32_t lds[];
    __shared__ double tmp_d[THREADS / 64];
    uint32_t *tmp = reinterpret_cast<uint32_t *>(tmp_d);
    const moe_kv_step_t &s = a.s;
    const int R = s.n_requests, T = s.n_tokens, tid = threadIdx.x, page = s.page, shift = a.page_shift;
    int32_t *row_end = lds, *need_before = lds + R, *sums = lds + 2 * R;   // sums: what the block's own role needs
    const int per = PER == 1 ? 1 : div_up(R, THREADS), r0 = tid * per;
    const int free_n = min(max(0, a.io.free_count[0]), a.free_most);
    auto pages = [&](int n) { return (int)(((uint32_t)n + page - 1) >> shift); };      // n < 2^31

    // rows
    int ctx[PER], now[PER], st[PER], first[PER];
    uint32_t sum = 0, total;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        // no branch around the loads: they are on their way together
        const int r = r0 + i;
        ctx[i] = a.io.ctx_len[min(r, R - 1)];
        now[i] = a.io.new_len[min(r, R - 1)];
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int r = r0 + i;
        st[i] = 0;
        if (i >= per || r >= R) {
            ctx[i] = now[i] = 0;
        } else {
            if (ctx[i] < 0 || now[i] < 0 || now[i] > s.max_new) st[i] = MOE_KV_BAD_SIZE;
            ctx[i] = max(ctx[i], 0);
            now[i] = min(max(now[i], 0), T + 1);
        }
        sum = add_sat(sum, now[i]);
    }
    uint32_t at = block_scan<THREADS>(sum, tmp, &total) - sum;
    // pages needed
    uint32_t need_sum = 0;
    int need[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int r = r0 + i;
        first[i] = (int)min(at, (uint32_t)T);
        at = add_sat(at, now[i]);
        need[i] = 0;
        if (i < per && r < R) {
            if (at > (uint32_t)T) st[i] = MOE_KV_BAD_SIZE;
            const int blocks = (int)(((uint32_t)ctx[i] + (uint32_t)now[i] + page - 1) >> shift);    // below 2^31 + 2^20 tokens
            if (!st[i] && blocks > s.max_blocks) st[i] = MOE_KV_TOO_LONG;
            if (!st[i]) need[i] = blocks - pages(ctx[i]);
            const int end = (int)min(at, (uint32_t)T);
            row_end[r] = end;
            now[i] = end - first[i];                        // rows that exist
        }
        need_sum = add_sat(need_sum, need[i]);
    }
    uint32_t before = block_scan<THREADS>(need_sum, tmp, &total) - need_sum;
    uint32_t used = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int r = r0 + i;
        if (i < per && r < R) {
            if (need[i] > 0 && add_sat(before, need[i]) > (uint32_t)free_n) st[i] = MOE_KV_NO_PAGES;
            if (!st[i]) used += need[i];
            // pages: at most free_n where it is used; the block that shares out tiles looks up the cached tokens instead
            need_before[r] = st[i] ? -1 : (int)blockIdx.x <= a.many_blocks ? ctx[i] : (int)min(before, 0x7FFFFFFFu);
        }
        before = add_sat(before, need[i]);
    }

    const int role = blockIdx.x;
    if (role == 0) {
        // what is per request, and the requests of few rows
        block_scan<THREADS>(used, tmp, &total);
        // Tiles of 32 rows, one after the other on a line of steps (a tile that sees nothing takes one step of it), cut into blocks of
        // `chunk` steps.  Either every block gets a piece of the line of the same length, whatever tiles begin and end in it; or
        // each tile begins with a block of its own (its end is padded to a whole chunk), where there are blocks enough for that: see own_chunk.
        // Sums, and what is added to them to round up, stay below 2^32: 8192 tiles of less than 2^19 steps, or 512 blocks of as many.
        constexpr int TILES = FEW_MOST / ROWS_FEW;
        int tiles[PER], kt0[PER][TILES], kt1[PER][TILES];
        uint32_t steps = 0, line, longest = 0, n_tiles = 0, all_tiles;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int r = r0 + i, rows = now[i] * a.group;
            tiles[i] = rows > FEW_MOST || st[i] == MOE_KV_BAD_SIZE ? 0 : div_up(rows, ROWS_FEW);
            if (i < per && r < R) {
                a.io.row_start[r + 1] = first[i] + now[i];
                a.io.kv_len[r] = st[i] ? ctx[i] : ctx[i] + now[i];
                a.io.status[r] = st[i];
            }
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                kt0[i][t] = kt1[i][t] = 0;
                if (t < tiles[i]) {
                    if (!st[i]) key_steps(s, ctx[i], now[i], t * ROWS_FEW / a.group, (min((t + 1) * ROWS_FEW, rows) - 1) / a.group, kt0[i][t], kt1[i][t]);
                    steps += max(1, kt1[i][t] - kt0[i][t]);
                    longest = max(longest, (uint32_t)(kt1[i][t] - kt0[i][t]));
                    ++n_tiles;
                }
            }
        }
        if (tid == 0) {
            a.io.row_start[0] = 0;
            a.io.free_left[0] = free_n - (int)total;
        }
        const uint32_t start = block_scan<THREADS>(steps, tmp, &line) - steps;
        block_scan<THREADS>(n_tiles, tmp, &all_tiles);
        longest = block_max<THREADS>(longest, tmp);
        const uint32_t target = (uint32_t)a.target_few;
        bool apart = false;
        uint32_t chunk = first_chunk(line, all_tiles, target), pos = start;
        if (all_tiles <= target) {
            uint32_t at = 0, all = 0;
            auto blocks_of_chunk = [&] {
                uint32_t n = 0;
#pragma unroll
                for (int i = 0; i < PER; ++i)
#pragma unroll
                    for (int t = 0; t < TILES; ++t)
                        if (t < tiles[i]) n += (max(1, kt1[i][t] - kt0[i][t]) + chunk - 1) / chunk;
                at = block_scan<THREADS>(n, tmp, &all) - n;
            };
            if (longest > chunk + SPLIT_STEPS) blocks_of_chunk();
            const uint32_t own = own_chunk(line, all_tiles, target, longest, chunk, all);
            if (own) {
                apart = true;
                chunk = own;
                blocks_of_chunk();
                pos = at * chunk;
                line = all * chunk;
            }
        }
        const uint32_t begin = pos;
        uint32_t items = 0, split = 0;      // split: joins << 16 | parts
        auto next_at = [&](uint32_t end) { return apart ? (end + chunk - 1) / chunk * chunk : end; };
        uint32_t b0[PER][TILES], parts[PER][TILES];
#pragma unroll
        for (int i = 0; i < PER; ++i)
#pragma unroll
            for (int t = 0; t < TILES; ++t)
                if (t < tiles[i]) {
                    const uint32_t len = max(1, kt1[i][t] - kt0[i][t]);
                    b0[i][t] = pos / chunk;
                    const uint32_t n = parts[i][t] = (pos + len - 1) / chunk - b0[i][t] + 1;
                    items += n;
                    split += n > 1 ? (1u << 16) + n : 0;
                    pos = next_at(pos + len);
                }
        uint32_t all_items, all_split;
        uint32_t item0 = block_scan<THREADS>(items, tmp, &all_items) - items, split0 = block_scan<THREADS>(split, tmp, &all_split) - split;
        pos = begin;
#pragma unroll
        for (int i = 0; i < PER; ++i)
#pragma unroll
            for (int t = 0; t < TILES; ++t)
                if (t < tiles[i]) {
                    const int len = kt1[i][t] - kt0[i][t];
                    const uint32_t n = parts[i][t];
                    Item it{r0 + i, first[i], now[i], ctx[i], t, 0, 0, -1, (int)(split0 & 0xFFFF), (int)n, (int)(split0 >> 16), 0};
                    for (uint32_t p = 0; p < n; ++p) {
                        const int at = (int)((b0[i][t] + p) * chunk - pos);      // where the block's piece begins, from the tile's first step
                        it.kt0 = kt0[i][t] + max(0, at);
                        it.kt1 = kt0[i][t] + min(len, at + (int)chunk);
                        it.part = n > 1 ? it.part0 + (int)p : -1;
                        a.p.few[item0 + p] = it;
                        if (at >= 0) a.p.few_first[b0[i][t] + p] = item0 + p;    // the block's first item
                    }
                    item0 += n;
                    split0 += n > 1 ? (1u << 16) + n : 0;
                    pos = next_at(pos + max(1, len));
                }
        if (tid == 0) {
            const uint32_t blocks = (line + chunk - 1) / chunk;
            a.p.head->few_blocks = (int)blocks;
            a.p.few_first[blocks] = (int)all_items;
        }
        return;
    }
    if (role <= a.many_blocks) {
        // Tiles of the other requests.  A request of a bad size has none: it may have more rows than the lists
        // are made for.
        auto tiles_of = [&](int i) {
            const int rows = now[i] * a.group;
            return rows <= FEW_MOST || st[i] == MOE_KV_BAD_SIZE ? 0 : div_up(rows, a.rows_many);
        };
        uint32_t units = 0, n_units;
#pragma unroll
        for (int i = 0; i < PER; ++i) units += tiles_of(i);
        uint32_t unit_at = block_scan<THREADS>(units, tmp, &n_units) - units;
        if (n_units == 0) {
            if (tid == 0 && role == 1) a.p.head->many = 0;
            return;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            unit_at += tiles_of(i);
            if (i < per && r0 + i < R) sums[r0 + i] = (int)unit_at;
        }
        __syncthreads();
        auto unit = [&](int u, Item &it) {
            const int r = first_above(sums, R, u);
            const int begin = r ? row_end[r - 1] : 0, n = row_end[r] - begin;
            it.req = r;
            it.row0 = begin;
            it.n_new = n;
            it.ctx = max(need_before[r], 0);
            it.tile = sums[r] - 1 - u;                   // the last rows see most: they go first
            it.kt0 = it.kt1 = 0;                         // turned down: nothing to attend to
            if (need_before[r] >= 0)
                key_steps(s, it.ctx, n, it.tile * a.rows_many / a.group, (min((it.tile + 1) * a.rows_many, n * a.group) - 1) / a.group, it.kt0, it.kt1);
        };
        double steps = 0.0;
        uint32_t longest = 0;
        for (int u = tid; u < (int)n_units; u += THREADS) {
            Item it{};
            unit(u, it);
            steps += it.kt1 - it.kt0;
            longest = max(longest, (uint32_t)(it.kt1 - it.kt0));
        }
        const int chunk = share(block_sum<THREADS>(steps, tmp_d), a.target_many, MIN_KT_MANY);
        if (block_max<THREADS>(longest, tmp) <= (uint32_t)chunk) {
            // no tile is split: items are tiles, and the blocks of this role write them together
            for (int u = (role - 1) * THREADS + tid; u < (int)n_units; u += a.many_blocks * THREADS) {
                Item it{};
                unit(u, it);
                put_items(a.p.many, it, 1, u, 0, 0);
            }
            if (tid == 0 && role == 1) a.p.head->many = (int)n_units;
            return;
        }
        if (role > 1) return;
        uint32_t items = 0, split = 0;
        for (int base = 0; base < (int)n_units; base += THREADS) {
            Item it{};
            int n = 0;
            if (base + tid < (int)n_units) {
                unit(base + tid, it);
                n = max(1, div_up(it.kt1 - it.kt0, chunk));
            }
            const uint32_t mine = n > 1 ? (1u << 16) + n : 0;
            uint32_t all_items, all_split;
            const uint32_t item0 = items + block_scan<THREADS>(n, tmp, &all_items) - n, split0 = split + block_scan<THREADS>(mine, tmp, &all_split) - mine;
            items += all_items;
            split += all_split;
            put_items(a.p.many, it, n, item0, split0 >> 16, split0 & 0xFFFF);
        }
        if (tid == 0) a.p.head->many = (int)items;
        return;
    }

    // pages touched
    uint32_t touched = 0, n_seg;
    int seg[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        seg[i] = st[i] || !now[i] ? 0 : pages(ctx[i] + now[i]) - (ctx[i] >> shift);
        touched += seg[i];
    }
    uint32_t seg_at = block_scan<THREADS>(touched, tmp, &n_seg) - touched;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        seg_at += seg[i];
        if (i < per && r0 + i < R) sums[r0 + i] = (int)seg_at;
    }
    __syncthreads();
    // A page of a request: an old one from the table, a new one from the stack.
    auto page_of = [&](int r, int c, int blk) {
        const int held = pages(c);
        if (blk < held) return a.io.block_table[(int64_t)r * s.max_blocks + blk];
        return a.io.free_pages[free_n - 1 - (need_before[r] + blk - held)];
    };
    const int worker = role - 1 - a.many_blocks, workers = gridDim.x - 1 - a.many_blocks;
    for (int i = worker * THREADS + tid; i < (a.p.max_joins_few + a.p.max_joins_many) * s.kv_heads; i += workers * THREADS) a.p.joins_few[i] = 0;
    for (int t = worker * THREADS + tid; t < T; t += workers * THREADS) {
        const int r = first_above(row_end, R, t);
        int pos = -1, slot = -1;
        if (r < R && need_before[r] >= 0) {
            const int c = max(a.io.ctx_len[r], 0);
            pos = c + t - (r ? row_end[r - 1] : 0);
            const int id = page_of(r, c, pos >> shift);
            if ((unsigned)id < (unsigned)s.n_pages) slot = id * page + (pos & (page - 1));
        }
        a.io.positions[t] = pos;
        a.p.positions[t] = pos;
        a.io.slots[t] = slot;
    }
    for (int g = worker * THREADS + tid; g < (int)n_seg; g += workers * THREADS) {
        const int r = first_above(sums, R, g);
        const int c = max(a.io.ctx_len[r], 0), begin = r ? row_end[r - 1] : 0, n = row_end[r] - begin;
        const int blk = (c >> shift) + g - (r ? sums[r - 1] : 0);
        const int lo = max(c, blk << shift), hi = min(c + n, (blk + 1) << shift);
        const int id = page_of(r, c, blk);
        if (blk << shift >= c) a.io.block_table[(int64_t)r * s.max_blocks + blk] = id;
        a.p.segments[g] = Segment{begin + lo - c, hi - lo, (unsigned)id < (unsigned)s.n_pages ? id : -1, lo & (page - 1), lo, {0, 0, 0}};
    }
    if (worker == 0 && tid == 0) a.p.head->segments = (int)n_seg;
}

// One block; requests one after the other, so that the stack's order is the order of the call.
__global__ void __launch_bounds__(256) k_kv_release(const int32_t *requests, int n, int n_requests, int n_pages, int page, int max_blocks,
                                                     int32_t *ctx_len, const int32_t *block_table, int32_t *free_pages, int capacity, int32_t *free_count)
{
    __shared__ int count[5];
    int top = min(max(free_count[0], 0), capacity);
    __syncthreads();
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int i = 0; i < n; ++i) {
        const int r = requests[i];
        if (r < 0 || r >= n_requests) continue;
        const int c = ctx_len[r];
        const int held = c <= 0 ? 0 : min((int)(((int64_t)c + page - 1) / page), max_blocks);
        for (int b0 = 0; b0 < held; b0 += 256) {
            const int b = b0 + threadIdx.x;
            const int id = b < held ? block_table[(int64_t)r * max_blocks + b] : -1;
            const bool good = (unsigned)id < (unsigned)n_pages;
            const uint64_t vote = __ballot(good);
            if (lane == 0) count[wave] = __popcll(vote);
            __syncthreads();
            int at = top, all = 0;
            for (int w = 0; w < 4; ++w) {
                if (w < wave) at += count[w];
                all += count[w];
            }
            at += __popcll(vote & (((uint64_t)1 << lane) - 1));
            if (good && at < capacity) free_pages[at] = id;
            top = min(top + all, capacity);
            __syncthreads();
        }
        if (threadIdx.x == 0) ctx_len[r] = 0;
        __syncthreads();      // the same request again finds nothing
    }
    if (threadIdx.x == 0) free_count[0] = top;
}

}  // namespace kv
}  // namespace moe
