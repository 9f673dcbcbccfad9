// The pages of a step and how its attention is shared out, from the requests' lengths.
//
// Everything follows from prefix sums over the requests: rows (where a request's rows lie), pages needed (which free pages
// it gets), pages touched (the segments that the store works on), tiles of rows and steps over cached tokens (the attention's
// blocks).  Up to 4096 requests are 16 KB of lengths, so every block of the launch makes the sums it needs by
// itself, in LDS, and there is no exchange between blocks: block 0 writes what is per request and shares out the requests of
// few rows, block 1 those of many, the others look up rows and pages with a binary search in the sums.  Latency is all there is
// to it: 2048 requests with 77 thousand rows move 0.7 MB.
#pragma once
#include "kernels_kv_common.h"

namespace moe {
namespace kv {

constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_PER = MOE_KV_MAX_REQUESTS / PLAN_THREADS;   // requests of a thread at most

struct PlanArgs {
    moe_kv_step_t s;
    moe_kv_lists_t io;
    Plan p;
    int32_t group, page_shift, target_few, target_many;
};

__device__ __forceinline__ int64_t wave_scan(int64_t v)
{
    const int lane = threadIdx.x & 63;
    for (int d = 1; d < 64; d *= 2) {
        const int64_t o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// Inclusive sum over the block's threads in their order; *total receives the whole sum.  `tmp`: 17 numbers in LDS.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t *tmp, int64_t *total)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    v = wave_scan(v);
    __syncthreads();          // the last scan's readers are done with tmp
    if (lane == 63) tmp[wave] = v;
    __syncthreads();
    int64_t before = 0, all = 0;
    for (int w = 0; w < PLAN_THREADS / 64; ++w) {
        if (w < wave) before += tmp[w];
        all += tmp[w];
    }
    *total = all;
    return v + before;
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

// Steps [kt0, kt1) over the cached tokens that rows [first, last] of a request see.
__device__ __forceinline__ void key_steps(const moe_kv_step_t &s, int ctx, int n_new, int tok_first, int tok_last, int &kt0, int &kt1)
{
    const int hi = s.causal ? ctx + tok_last + 1 : ctx + n_new;
    const int lo = s.window > 0 ? max(0, ctx + tok_first + 1 - s.window) : 0;
    kt0 = lo / KT;
    kt1 = (hi + KT - 1) / KT;
}

__global__ void __launch_bounds__(PLAN_THREADS) k_kv_plan(PlanArgs a)
{
    extern __shared__ int32_t lds[];
    __shared__ int64_t tmp[PLAN_THREADS / 64];
    const moe_kv_step_t &s = a.s;
    const int R = s.n_requests, T = s.n_tokens, tid = threadIdx.x, page = s.page;
    int32_t *row_end = lds, *need_before = lds + R, *sums = lds + 2 * R;   // sums: what the block's own role needs
    const int per = div_up(R, PLAN_THREADS), r0 = tid * per;
    const int free_n = min(max(0, a.io.free_count[0]), s.n_pages);

    // rows
    int ctx[PLAN_PER], now[PLAN_PER], st[PLAN_PER];
    int64_t sum = 0, total;
#pragma unroll
    for (int i = 0; i < PLAN_PER; ++i) {
        const int r = r0 + i;
        ctx[i] = now[i] = st[i] = 0;
        if (i < per && r < R) {
            ctx[i] = a.io.ctx_len[r];
            now[i] = a.io.new_len[r];
            if (ctx[i] < 0 || now[i] < 0 || now[i] > s.max_new) st[i] = MOE_KV_BAD_SIZE;
            ctx[i] = max(ctx[i], 0);
            now[i] = min(max(now[i], 0), T + 1);
        }
        sum += now[i];
    }
    int64_t at = block_scan(sum, tmp, &total) - sum;
    // pages needed
    int64_t need_sum = 0;
    int need[PLAN_PER];
#pragma unroll
    for (int i = 0; i < PLAN_PER; ++i) {
        const int r = r0 + i;
        const int64_t first = at;
        at += now[i];
        need[i] = 0;
        if (i < per && r < R) {
            if (at > T) st[i] = MOE_KV_BAD_SIZE;
            const int64_t blocks = ((int64_t)ctx[i] + now[i] + page - 1) >> a.page_shift;
            if (!st[i] && blocks > s.max_blocks) st[i] = MOE_KV_TOO_LONG;
            if (!st[i]) need[i] = (int)(blocks - (((int64_t)ctx[i] + page - 1) >> a.page_shift));
            row_end[r] = (int)min(at, (int64_t)T);
            now[i] = (int)(min(at, (int64_t)T) - min(first, (int64_t)T));     // rows that exist
        }
        need_sum += need[i];
    }
    int64_t before = block_scan(need_sum, tmp, &total) - need_sum;
    int64_t used = 0;
#pragma unroll
    for (int i = 0; i < PLAN_PER; ++i) {
        const int r = r0 + i;
        if (i < per && r < R) {
            if (need[i] > 0 && before + need[i] > free_n) st[i] = MOE_KV_NO_PAGES;
            if (!st[i]) used += need[i];
            need_before[r] = st[i] ? -1 : (int)before;      // at most free_n where it is used
        }
        before += need[i];
    }

    const int role = blockIdx.x;
    if (role == 0) {
        block_scan(used, tmp, &total);
#pragma unroll
        for (int i = 0; i < PLAN_PER; ++i) {
            const int r = r0 + i;
            if (i < per && r < R) {
                a.io.row_start[r + 1] = row_end[r];
                a.io.kv_len[r] = st[i] ? ctx[i] : ctx[i] + now[i];
                a.io.status[r] = st[i];
            }
        }
        if (tid == 0) {
            a.io.row_start[0] = 0;
            a.io.free_left[0] = (int)(free_n - total);
        }
    }
    if (role <= 1) {
        // Units: requests of few rows (block 0), tiles of 128 rows of the others (block 1).  A request of a bad size
        // has none: it may have more rows than the lists are made for.
        const bool many = role == 1;
        auto units_of = [&](int i) {
            const int rows = st[i] == MOE_KV_BAD_SIZE ? 0 : now[i] * a.group;
            return rows == 0 || (rows > ROWS_FEW) != many ? 0 : many ? div_up(rows, ROWS_MANY) : 1;
        };
        int64_t units = 0;
#pragma unroll
        for (int i = 0; i < PLAN_PER; ++i) {
            units += units_of(i);
        }
        int64_t n_units;
        int64_t unit_at = block_scan(units, tmp, &n_units) - units;
#pragma unroll
        for (int i = 0; i < PLAN_PER; ++i) {
            const int r = r0 + i;
            unit_at += units_of(i);
            if (i < per && r < R) sums[r] = (int)unit_at;
        }
        __syncthreads();
        const int tile_rows = many ? ROWS_MANY : ROWS_FEW;
        auto unit = [&](int u, Item &it) {
            const int r = first_above(sums, R, u);
            const int begin = r ? row_end[r - 1] : 0, n = row_end[r] - begin;
            const int local = u - (r ? sums[r - 1] : 0), tiles = sums[r] - (r ? sums[r - 1] : 0);
            it.req = r;
            it.row0 = begin;
            it.n_new = n;
            it.ctx = max(a.io.ctx_len[r], 0);
            it.tile = tiles - 1 - local;                 // the last rows see most: they go first
            it.kt0 = it.kt1 = 0;                         // turned down: nothing to attend to
            if (need_before[r] >= 0)
                key_steps(s, it.ctx, n, it.tile * tile_rows / a.group, (min((it.tile + 1) * tile_rows, n * a.group) - 1) / a.group, it.kt0, it.kt1);
        };
        int64_t steps = 0, all_steps;
        for (int u = tid; u < n_units; u += PLAN_THREADS) {
            Item it{};
            unit(u, it);
            steps += it.kt1 - it.kt0;
        }
        block_scan(steps, tmp, &all_steps);
        const int target = many ? a.target_many : a.target_few;
        const int chunk = (int)max((int64_t)(many ? MIN_KT_MANY : MIN_KT_FEW), (all_steps + target - 1) / target);
        int64_t done = 0;                                // items | joins << 24 | parts << 44, so far
        for (int base = 0; base < n_units; base += PLAN_THREADS) {
            Item it{};
            int n = 0;
            if (base + tid < n_units) {
                unit(base + tid, it);
                n = max(1, div_up(it.kt1 - it.kt0, chunk));
            }
            const int64_t mine = n | (n > 1 ? ((int64_t)1 << 24) | ((int64_t)n << 44) : 0);
            int64_t all;
            const int64_t upto = done + block_scan(mine, tmp, &all) - mine;
            done += all;
            const int item0 = (int)(upto & 0xFFFFFF), join0 = (int)((upto >> 24) & 0xFFFFF), part0 = (int)(upto >> 44);
            const int lo = it.kt0, len = it.kt1 - it.kt0;
            for (int p = 0; p < n; ++p) {
                it.kt0 = lo + (int)((int64_t)len * p / n);
                it.kt1 = lo + (int)((int64_t)len * (p + 1) / n);
                it.part = n > 1 ? part0 + p : -1;
                (many ? a.p.many : a.p.few)[item0 + p] = it;
            }
            if (n > 1) (many ? a.p.joins_many : a.p.joins_few)[join0] = Join{it.row0, it.n_new, it.tile, part0, n, {0, 0, 0}};
        }
        if (tid == 0) {
            (many ? a.p.head->many : a.p.head->few) = (int)(done & 0xFFFFFF);
            (many ? a.p.head->joins_many : a.p.head->joins_few) = (int)((done >> 24) & 0xFFFFF);
        }
        return;
    }

    // pages touched
    int64_t touched = 0, n_seg;
    int seg[PLAN_PER];
#pragma unroll
    for (int i = 0; i < PLAN_PER; ++i) {
        seg[i] = st[i] || !now[i] ? 0 : (int)((((int64_t)ctx[i] + now[i] + page - 1) >> a.page_shift) - (ctx[i] >> a.page_shift));
        touched += seg[i];
    }
    int64_t seg_at = block_scan(touched, tmp, &n_seg) - touched;
#pragma unroll
    for (int i = 0; i < PLAN_PER; ++i) {
        seg_at += seg[i];
        if (i < per && r0 + i < R) sums[r0 + i] = (int)seg_at;
    }
    __syncthreads();
    // A page of a request: an old one from the table, a new one from the stack.
    auto page_of = [&](int r, int c, int blk) {
        const int held = (int)(((int64_t)c + page - 1) >> a.page_shift);
        if (blk < held) return a.io.block_table[(int64_t)r * s.max_blocks + blk];
        return a.io.free_pages[free_n - 1 - (need_before[r] + blk - held)];
    };
    const int worker = role - 2, workers = gridDim.x - 2;
    for (int t = worker * PLAN_THREADS + tid; t < T; t += workers * PLAN_THREADS) {
        const int r = first_above(row_end, R, t);
        int pos = -1, slot = -1;
        if (r < R && need_before[r] >= 0) {
            const int c = max(a.io.ctx_len[r], 0);
            pos = c + t - (r ? row_end[r - 1] : 0);
            const int id = page_of(r, c, pos >> a.page_shift);
            if ((unsigned)id < (unsigned)s.n_pages) slot = id * page + (pos & (page - 1));
        }
        a.io.positions[t] = pos;
        a.p.positions[t] = pos;
        a.io.slots[t] = slot;
    }
    for (int g = worker * PLAN_THREADS + tid; g < n_seg; g += workers * PLAN_THREADS) {
        const int r = first_above(sums, R, g);
        const int c = max(a.io.ctx_len[r], 0), begin = r ? row_end[r - 1] : 0, n = row_end[r] - begin;
        const int blk = (c >> a.page_shift) + g - (r ? sums[r - 1] : 0);
        const int lo = max(c, blk << a.page_shift), hi = min(c + n, (blk + 1) << a.page_shift);
        const int id = page_of(r, c, blk);
        if ((int64_t)blk << a.page_shift >= c) a.io.block_table[(int64_t)r * s.max_blocks + blk] = id;
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
