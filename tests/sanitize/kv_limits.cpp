// What the host and k_kv_plan work out for a step's lists where a step is as large as it may be: the largest table that is accepted
// for each page, and the shares of the most steps that requests of many rows can have.
#include "../../paper_2312_17238_amd/csrc/kv.hip"

// no device code: nothing to register
extern "C" {
void **__hipRegisterFatBinary(const void *) { static void *handle; return &handle; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *, char *, const char *, unsigned, uint3 *, uint3 *, dim3 *, dim3 *, int *) {}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
const char __hip_fatbin[8] = {0};
}

int32_t moe::report_error(int32_t code, int32_t, const char *) { return code; }

static int failures = 0;

static void need(bool ok, const char *what, long long a, long long b)
{
    if (!ok) {
        printf("%s: %lld, %lld\n", what, a, b);
        ++failures;
    }
}

static moe_kv_step_t large_step(int page, int max_blocks)
{
    moe_kv_step_t s{};
    s.n_requests = MOE_KV_MAX_REQUESTS;
    s.n_tokens = MOE_KV_MAX_TOKENS;
    s.max_new = MOE_KV_MAX_TOKENS;
    s.max_blocks = max_blocks;
    s.n_pages = 1 << 20;
    s.page = page;
    s.kv_heads = 1;
    s.head_dim = 64;
    s.q_heads = 1024;
    s.causal = 1;
    return s;
}

int main()
{
    for (int page = 16; page <= 128; page *= 2) {
        int lo = 1, hi = 1 << 28;               // the widest table that is accepted
        while (lo + 1 < hi) {
            const int mid = lo + (hi - lo) / 2;
            const moe_kv_step_t s = large_step(page, mid);
            (step_ok(&s) ? lo : hi) = mid;
        }
        const moe_kv_step_t s = large_step(page, lo);
        need((int64_t)lo * page >= (1 << 24) - 128, "a table narrower than it has to be", page, lo);
        // requests of few rows, all with every token that the table can name
        const int64_t steps = ((int64_t)lo * page + KT - 1) / KT;
        const int64_t tiles = (int64_t)MOE_KV_MAX_REQUESTS * (FEW_MOST / ROWS_FEW), target = 2 * COMPUTE_UNITS;
        need(steps * tiles + target <= 1ll << 32, "the line of steps leaves 32 bits", page, steps * tiles + target);
        const uint32_t chunk = first_chunk((uint32_t)std::min<int64_t>(steps * tiles, 0xFFFFFFFF), (uint32_t)tiles, (uint32_t)target);
        need(steps * tiles <= (int64_t)chunk * target, "more blocks than there is room for", page, chunk);
        // requests of many rows, likewise
        const Sizes z = sizes_of(&s);
        const int64_t most = ((int64_t)s.n_tokens * z.group / z.rows_many + s.n_requests) * steps;
        for (int64_t all = most; all > 0; all /= 2) {
            const int many = target_blocks(BLOCKS_MANY, s.kv_heads), of_block = share((double)all, many, MIN_KT_MANY);
            need(of_block >= MIN_KT_MANY && ((int64_t)of_block * many >= all || of_block >= steps), "share", all, of_block);
        }
    }
    // grids: every block in one piece, no piece of 2^32 threads
    for (int64_t blocks : {(int64_t)0, (int64_t)1, MOST_BLOCKS, MOST_BLOCKS + 1, 3 * MOST_BLOCKS - 1, (int64_t)(1 << 30) + 5}) {
        int64_t next = 0;
        in_pieces(blocks, [&](uint32_t first, unsigned n) {
            need(first == next && n >= 1 && (uint64_t)n * 256 < (1ull << 32), "pieces", first, n);
            next = (int64_t)first + n;
        });
        need(next == blocks, "all pieces", blocks, next);
    }
    // attention is one launch: its largest steps
    for (int heads = 1; heads <= 256; heads *= 2) {
        moe_kv_step_t s = large_step(16, 1 << 19);
        s.kv_heads = heads;
        const Sizes z = sizes_of(&s);
        const int64_t blocks = ((int64_t)z.p.max_many + z.p.blocks_few) * heads;
        need(step_ok(&s) && blocks <= MOST_BLOCKS, "blocks of the attention", heads, blocks);
    }
    if (failures == 0) printf("ok\n");
    return failures != 0;
}
