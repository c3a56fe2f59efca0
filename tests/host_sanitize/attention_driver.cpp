// The host half of the attention entry points (csrc/cf_attn_api.cpp) with launchers that check what they are handed: random calls, most of them
// valid, none of which may launch anything that reaches outside the buffers it was given.  Runs under sanitizers, without a device.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>

#include "cf_attn.h"
#include "compactfusion.h"

namespace {
int g_failures, g_prompts, g_paged, g_joins, g_appends, g_split, g_many;
bool g_refuse;
char *g_ws;
size_t g_ws_bytes;
int64_t g_longest;
const void *g_parts_expected;

void expect(bool ok, const char *what, int line)
{
    if (!ok) {
        std::printf("line %d: %s\n", line, what);
        ++g_failures;
    }
}
#define EXPECT(x) expect((x), #x, __LINE__)
}  // namespace

namespace cf {
namespace attn {
static void check_parts(const Parts &p, int n, int dim, int64_t rows)
{
    const char *o = reinterpret_cast<const char *>(p.o), *end = reinterpret_cast<const char *>(p.lse + (int64_t)n * rows);
    EXPECT(p.n_rows == rows);
    EXPECT(o >= g_ws + CF_ATTN_COUNTER_BYTES && end <= g_ws + g_ws_bytes);
    EXPECT(reinterpret_cast<const char *>(p.lse) == o + (int64_t)n * rows * dim * 4);
    EXPECT(reinterpret_cast<uintptr_t>(o) % 16 == 0);
    EXPECT((int64_t)n * rows * dim * 4 < (int64_t)1 << 31);         // the device addresses the parts with 32 bits
}
hipError_t launch_prompt(const PromptArgs &a, hipStream_t)
{
    ++g_prompts;
    EXPECT(a.h.group * a.h.kv_heads == a.h.q_heads && a.h.scale_log2 > 0.0f);
    EXPECT(a.n_splits >= 1 && a.n_splits <= kMaxParts);
    EXPECT((int64_t)a.n_q * a.h.q_heads <= (1 << 30) && a.n_k <= (1 << 30));
    if (a.n_splits > 1) {
        ++g_split;
        EXPECT(a.split_keys % 64 == 0 && (int64_t)a.n_splits * a.split_keys >= g_longest && (int64_t)(a.n_splits - 1) * a.split_keys < g_longest);
        check_parts(a.parts, a.n_splits, a.h.head_dim, (int64_t)a.n_q * a.h.q_heads);
    }
    EXPECT(a.n_k == 0 || (a.k.token >= a.h.head_dim * 2 && a.v.token >= a.h.head_dim * 2));
    return g_refuse ? hipErrorLaunchFailure : hipSuccess;
}
hipError_t launch_paged(const PagedArgs &a, hipStream_t)
{
    ++g_paged;
    const int64_t units = (int64_t)a.h.kv_heads * ((a.h.group + kPagedHeads - 1) / kPagedHeads);
    EXPECT(a.n_splits >= 1 && a.n_splits <= kMaxParts);
    EXPECT(a.table_stride >= a.max_pages && (1 << a.cache.page_shift) == a.cache.page_size);
    EXPECT(a.cache.page_bytes >= (int64_t)a.h.kv_heads * a.cache.page_size * a.h.head_dim * 2);
    if (a.n_splits > 1) {
        ++g_split;
        g_many += a.many;
        EXPECT(a.split_keys % 128 == 0 && (int64_t)a.n_splits * a.split_keys >= g_longest);
        EXPECT(reinterpret_cast<char *>(a.counters) == g_ws && a.n_seqs * units * 4 <= (int64_t)CF_ATTN_COUNTER_BYTES && a.n_seqs <= kMostListed);
        check_parts(a.parts, a.n_splits, a.h.head_dim, (int64_t)a.n_seqs * a.h.q_heads);
    } else {
        EXPECT(!a.many);
    }
    return g_refuse ? hipErrorLaunchFailure : hipSuccess;
}
hipError_t launch_join(const JoinArgs &a, hipStream_t)
{
    ++g_joins;
    EXPECT(!g_refuse);              // nothing is joined after a launch that was refused
    for (int i = 0; i < a.n_parts; ++i) EXPECT(a.parts[i] && a.lses[i]);
    return hipSuccess;
}
hipError_t launch_append(const AppendArgs &a, hipStream_t)
{
    ++g_appends;
    EXPECT(a.rotary_dim % 16 == 0 && a.rotary_dim <= a.h.head_dim);
    EXPECT(a.rotary_dim == 0 || (a.cos && a.sin && a.positions && a.n_positions > 0));
    return g_refuse ? hipErrorLaunchFailure : hipSuccess;
}
}  // namespace attn
}  // namespace cf

int main()
{
    std::mt19937 rng(7);
    auto up_to = [&](int64_t n) { return (int64_t)(rng() % (uint64_t)(n + 1)); };
    auto spread = [&](int64_t n) { return up_to((int64_t)1 << up_to(63 - __builtin_clzll((uint64_t)n))) % (n + 1); };      // small ones as often as large ones
    const uintptr_t at = (uintptr_t)1 << 44;
    const uintptr_t step = (uintptr_t)1 << 42;              // between operands: no valid one is as long
    for (int i = 0; i < 60000; ++i) {
        const int dims[3] = {64, 128, 256};
        cf_attn_desc d = {CF_BF16 + (int)up_to(1), 0, 1 + (int)up_to(9), dims[up_to(2)], 0.0f};
        d.q_heads = d.kv_heads * (1 + (int)up_to(40));
        const size_t sizes[4] = {CF_ATTN_WORKSPACE_BYTES, 0, (size_t)spread(CF_ATTN_WORKSPACE_BYTES), (size_t)1 << 33};
        g_ws_bytes = sizes[up_to(3)];
        g_ws = g_ws_bytes ? reinterpret_cast<char *>(at) : nullptr;
        if (g_ws_bytes > CF_ATTN_WORKSPACE_BYTES && up_to(1)) g_ws_bytes = CF_ATTN_WORKSPACE_BYTES;
        g_refuse = up_to(19) == 0;
        auto rows = [&](int n, int64_t heads) {
            cf_rows r = {reinterpret_cast<void *>(at + step * (uintptr_t)n), heads * d.head_dim + 8 * up_to(3), d.head_dim};
            if (up_to(30) == 0) r.token = (int64_t)rng() - 2000000000;
            if (up_to(40) == 0) r.head = (int64_t)rng() - 2000000000;
            if (up_to(60) == 0) r.data = reinterpret_cast<void *>(at + step * (uintptr_t)n + 2);
            return r;
        };
        auto words = [&](int n) { return reinterpret_cast<int32_t *>(at + step * (uintptr_t)n); };
        cf_status st;
        if (i % 3 == 0) {
            cf_prompt p = {(int32_t)spread(3000), (int32_t)up_to(1), spread(200000), spread(2000000), 0, words(1), words(2), rows(3, d.q_heads), rows(4, d.kv_heads),
                           rows(5, d.kv_heads), rows(6, d.q_heads), up_to(1) ? reinterpret_cast<float *>(words(7)) : nullptr};
            p.max_k = up_to(1) ? spread(p.n_k + 1000) : 0;
            g_longest = p.max_k > 0 && p.max_k < p.n_k ? p.max_k : p.n_k;
            st = cf_attn_prompt(&d, &p, g_ws, g_ws_bytes, nullptr);
        } else {
            const int pages[4] = {16, 32, 64, 32768};
            cf_kv_cache c = {words(8), words(9), 1 + spread(100000), 0, pages[up_to(3)]};
            if (i % 3 == 1) {
                cf_paged p = {(int32_t)spread(20000), 1 + (int32_t)spread(60000), 0, 0, words(1), words(2), rows(3, d.q_heads), rows(6, d.q_heads), nullptr};
                const int64_t capacity = (int64_t)p.max_pages * c.page_size;
                p.max_len = up_to(1) ? spread(2000000) : 0;
                g_longest = p.max_len > 0 && p.max_len < capacity ? p.max_len : capacity < (1 << 30) ? capacity : 1 << 30;
                st = cf_attn_paged(&d, &c, &p, g_ws, g_ws_bytes, nullptr);
            } else {
                cf_append p;
                std::memset(&p, 0, sizeof p);
                p.n_tokens = spread(300000);
                p.k = rows(1, d.kv_heads), p.v = rows(2, d.kv_heads), p.slots = reinterpret_cast<int64_t *>(words(3));
                if (up_to(1)) p.q = rows(4, d.q_heads), p.q_out = up_to(1) ? p.q : rows(5, d.q_heads);
                if (up_to(1)) p.rotary_dim = 16 * (int32_t)up_to(d.head_dim / 16), p.positions = words(6), p.cos = reinterpret_cast<float *>(words(7)), p.sin = p.cos, p.n_positions = 1 + up_to(10000);
                st = cf_kv_append(&d, &c, &p, nullptr);
            }
        }
        EXPECT(st == CF_OK || st == CF_ERR_INVALID_ARG || st == CF_ERR_SHAPE || st == CF_ERR_WORKSPACE || (st == CF_ERR_DEVICE && g_refuse));
    }
    std::printf("%d prompts, %d paged, %d appends, %d split, %d of them by many, %d joins\n", g_prompts, g_paged, g_appends, g_split, g_many, g_joins);
    EXPECT(g_prompts > 5000 && g_paged > 5000 && g_appends > 5000 && g_split > 1000 && g_many > 100 && g_joins > 300);
    if (g_failures) return 1;
    std::printf("all calls hold\n");
    return 0;
}
