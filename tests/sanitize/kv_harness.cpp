// The bounds that the host works out for a step's lists and partial results, against what sharing out the attention of random lengths
// takes: the rules of k_kv_plan's first two roles, one request after the other, with the kernel's own constants and helpers.
#include "../../paper_2312_17238_amd/csrc/kv.hip"

#include <cstdlib>
#include <random>
#include <vector>

// no device code: nothing to register
extern "C" {
void **__hipRegisterFatBinary(const void *) { static void *handle; return &handle; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *, char *, const char *, unsigned, uint3 *, uint3 *, dim3 *, dim3 *, int *) {}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
const char __hip_fatbin[8] = {0};
}

int32_t moe::report_error(int32_t code, int32_t, const char *) { return code; }

static void need(bool ok, const char *what, int run)
{
    if (!ok) {
        printf("run %d: %s\n", run, what);
        exit(1);
    }
}

int main()
{
    std::mt19937 rng(7);
    auto pick = [&](int lo, int hi) { return (int)(lo + rng() % (uint32_t)(hi - lo + 1)); };
    long long items_most = 0, split_runs = 0;
    for (int run = 0; run < 4000; ++run) {
        moe_kv_step_t s{};
        s.page = 16 << pick(0, 3);
        s.head_dim = 64 << pick(0, 2);
        s.kv_heads = 1 << pick(0, 8);
        s.q_heads = s.kv_heads * pick(1, std::max(1, std::min(70, 1024 / s.kv_heads)));
        s.n_requests = pick(0, 3) ? pick(1, 40) : pick(1, 3000);
        s.max_new = pick(0, 1) ? pick(1, 9) : pick(1, s.n_requests > 40 ? 300 : 900);
        s.causal = pick(0, 1);
        s.window = pick(0, 2) ? 0 : pick(1, 500);
        const int ctx_most = pick(0, 2) ? pick(0, 400) : pick(0, 60000);
        std::vector<int> ctx, now;
        std::vector<bool> served;
        int rows = 0, blocks = 1;
        for (int r = 0; r < s.n_requests; ++r) {
            ctx.push_back(pick(0, ctx_most));
            now.push_back(pick(0, s.max_new));
            served.push_back(pick(0, 9) > 0);
            rows += now[r];
            if (served[r]) blocks = std::max(blocks, div_up(ctx[r] + now[r], s.page));
        }
        s.n_tokens = std::max(1, rows);
        s.max_blocks = blocks;
        s.n_pages = 100;
        need(step_ok(&s), "step", run);
        const Sizes z = sizes_of(&s);
        const Plan &p = z.p;
        long long segments = 0;
        for (int r = 0; r < s.n_requests; ++r)
            if (now[r] && served[r]) segments += div_up(ctx[r] + now[r], s.page) - ctx[r] / s.page;
        need(segments <= p.max_segments, "segments", run);
        for (int many = 0; many < 2; ++many) {
            const int tile = many ? z.rows_many : ROWS_FEW;
            std::vector<int> len;
            for (int r = 0; r < s.n_requests; ++r) {
                const int n = now[r] * z.group;
                if (n == 0 || (n > FEW_MOST) != (many == 1)) continue;
                for (int t = 0; t < div_up(n, tile); ++t) {
                    int a = 0, b = 0;
                    if (served[r]) key_steps(s, ctx[r], now[r], t * tile / z.group, (std::min((t + 1) * tile, n) - 1) / z.group, a, b);
                    need(b >= a && a >= 0, "steps", run);
                    len.push_back(b - a);
                }
            }
            long long items = 0, parts = 0, joins = 0, total = 0, line = 0, longest = 0;
            for (int l : len) {
                total += l;
                line += std::max(1, l);
                longest = std::max<long long>(longest, l);
            }
            if (many) {
                need(len.empty() || z.many, "requests of many rows that the host does not expect", run);
                const long long chunk = share((double)total, target_blocks(BLOCKS_MANY, s.kv_heads), MIN_KT_MANY);
                for (int l : len) {
                    const long long n = std::max<long long>(1, (l + chunk - 1) / chunk);
                    items += n;
                    if (n > 1) { parts += n; ++joins; }
                }
                need(items <= p.max_many && parts <= p.parts_many && joins <= p.max_joins_many, "lists of many rows", run);
            } else {
                const long long target = p.blocks_few, tiles = (long long)len.size();
                uint32_t chunk = first_chunk((uint32_t)line, (uint32_t)tiles, (uint32_t)target), own = 0;
                if (tiles <= target) {
                    long long blocks = 0;
                    for (int l : len) blocks += (std::max(1, l) + chunk - 1) / chunk;
                    own = own_chunk((uint32_t)line, (uint32_t)tiles, (uint32_t)target, (uint32_t)longest, chunk, (uint32_t)blocks);
                    if (own) chunk = own;
                }
                long long pos = 0;
                for (int l : len) {
                    const long long w = std::max(1, l), n = (pos + w - 1) / chunk - pos / chunk + 1;
                    items += n;
                    if (n > 1) { parts += n; ++joins; }
                    pos += w;
                    if (own) pos = (pos + chunk - 1) / chunk * chunk;
                    need(pos < (1ll << 32), "32-bit line", run);
                }
                need((pos + chunk - 1) / chunk <= p.blocks_few, "blocks", run);
                need(items <= p.max_few && parts <= p.parts_few && joins <= p.max_joins_few, "lists of few rows", run);
            }
            need(parts < 65536 && joins < 65536, "packed sums", run);
            items_most = std::max(items_most, items);
            split_runs += parts > 0;
        }
        need((long long)p.parts_few * s.kv_heads * ROWS_FEW * s.head_dim * 4 < (1ll << 32) && (long long)p.parts_many * s.kv_heads * z.rows_many * s.head_dim * 4 < (1ll << 32),
             "32-bit offsets of parts", run);
    }
    printf("ok: 4000 steps, %lld lists with parts, %lld items at most\n", split_runs, items_most);
    return 0;
}
