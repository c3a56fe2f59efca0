// The host half of the attention entry points (csrc/cf_attn_api.cpp) at the ends of what its arguments can hold: strides and pages up to the largest
// numbers, as many sequences, tokens and parts as are taken.  Nothing may overflow, no launch may have more work-items than the device counts
// (32 bits), and caches that overlap are refused however far they reach.  Runs under sanitizers, without a device.
#include <cstdio>
#include <cstring>
#include <random>

#include "cf_attn.h"
#include "compactfusion.h"

namespace {
int g_failures, g_launches, g_shape;
int64_t g_sequences;            // that the last paged call's launches took, one after another
const int32_t *g_first_len;
int g_least_splits;

void expect(bool ok, const char *what, int line)
{
    if (!ok && ++g_failures < 20) std::printf("line %d: %s\n", line, what);
}
#define EXPECT(x) expect((x), #x, __LINE__)
}  // namespace

namespace cf {
namespace attn {
static hipError_t check_grid(int64_t workgroups)
{
    ++g_launches;
    EXPECT(workgroups >= 1 && workgroups * 256 < (int64_t)1 << 32);
    return hipSuccess;
}
hipError_t launch_prompt(const PromptArgs &a, hipStream_t) { return check_grid(prompt_workgroups(a)); }
hipError_t launch_paged(const PagedArgs &a, hipStream_t)
{
    if (g_sequences == 0) g_first_len = a.lens, g_least_splits = a.n_splits;
    EXPECT(a.lens == g_first_len + g_sequences);
    EXPECT(a.n_splits == 1 || (a.n_seqs <= kMostListed && paged_units(a) * (int64_t)sizeof(uint32_t) <= (int64_t)CF_ATTN_COUNTER_BYTES));      // what the device has places for
    g_sequences += a.n_seqs;
    if (a.n_splits < g_least_splits) g_least_splits = a.n_splits;
    return check_grid(paged_workgroups(a));
}
hipError_t launch_join(const JoinArgs &a, hipStream_t) { return check_grid(join_workgroups(a)); }
hipError_t launch_append(const AppendArgs &a, hipStream_t) { return check_grid(append_workgroups(a)); }
}  // namespace attn
}  // namespace cf

int main()
{
    std::mt19937_64 rng(11);
    auto up_to = [&](int64_t n) { return (int64_t)(rng() % ((uint64_t)n + 1)); };
    auto any = [&](int64_t n) { return n >> up_to(62 - __builtin_clzll((uint64_t)n)); };        // as many bits as n has, or fewer
    auto wide = [&]() -> int64_t {
        const int64_t x = (int64_t)(rng() >> up_to(63));
        return up_to(2) ? x & ~(int64_t)7 : x;
    };
    const uintptr_t at = (uintptr_t)1 << 20;
    float *const f = reinterpret_cast<float *>(at);
    for (int i = 0; i < 400000; ++i) {
        const int dims[3] = {64, 128, 256};
        cf_attn_desc d = {CF_BF16, 0, 1 + (int)any(4000), dims[up_to(2)], 0.0f};
        d.q_heads = d.kv_heads * (1 + (int)up_to(3));
        auto rows = [&](int n, bool dense) {
            cf_rows r = {reinterpret_cast<void *>(at + ((uintptr_t)n << 59)), (int64_t)d.q_heads * d.head_dim, d.head_dim};
            if (!dense && up_to(2) == 0) r.token = wide();
            if (!dense && up_to(2) == 0) r.head = wide();
            return r;
        };
        void *ws = up_to(1) ? reinterpret_cast<void *>((uintptr_t)1 << 40) : nullptr;
        cf_kv_cache c = {reinterpret_cast<void *>(at), reinterpret_cast<void *>(at + (up_to(1) ? (uintptr_t)1 << 61 : up_to(((int64_t)1 << 61) / 16) * 16)), 1 + any(INT32_MAX), 0,
                         16 << up_to(5)};
        if (up_to(1)) c.page_stride = wide();
        cf_status st;
        if (i % 4 == 0) {
            cf_prompt p = {(int32_t)any(1 << 30), (int32_t)up_to(1), any((int64_t)1 << 30), any((int64_t)1 << 30), any((int64_t)1 << 40), (int32_t *)f, (int32_t *)f,
                           rows(1, false), rows(2, false), rows(2, false), rows(3, true), nullptr};
            st = cf_attn_prompt(&d, &p, ws, ws ? CF_ATTN_WORKSPACE_BYTES : 0, nullptr);
        } else if (i % 4 == 1) {
            cf_paged p = {(int32_t)any(1 << 30), 1 + (int32_t)any(INT32_MAX - 1), up_to(1) ? wide() : 0, any(INT64_MAX), (int32_t *)f, (int32_t *)f, rows(8, false), rows(9, true), nullptr};
            g_sequences = 0;
            st = cf_attn_paged(&d, &c, &p, ws, ws ? CF_ATTN_WORKSPACE_BYTES : 0, nullptr);
            EXPECT(g_sequences == (st == CF_OK ? p.n_seqs : 0));
        } else if (i % 4 == 2) {
            cf_append p;
            std::memset(&p, 0, sizeof p);
            p.n_tokens = any((int64_t)1 << 30), p.k = rows(8, false), p.v = rows(8, false), p.slots = reinterpret_cast<int64_t *>(f);
            if (up_to(1)) p.q = rows(8, false), p.q_out = rows(9, true);
            if (up_to(1)) p.rotary_dim = 64, p.positions = (int32_t *)f, p.cos = p.sin = f, p.n_positions = any(INT64_MAX);
            st = cf_kv_append(&d, &c, &p, nullptr);
        } else {
            const void *parts[CF_JOIN_MAX_PARTS];
            const float *lses[CF_JOIN_MAX_PARTS];
            for (int n = 0; n < CF_JOIN_MAX_PARTS; ++n) parts[n] = f, lses[n] = f;
            cf_join j = {1 + (int32_t)up_to(CF_JOIN_MAX_PARTS - 1), up_to(1) ? CF_F32 : CF_BF16, any((int64_t)1 << 30), parts, lses, rows(9, up_to(1)), nullptr};
            st = cf_attn_join(&d, &j, nullptr);
        }
        EXPECT(st == CF_OK || st == CF_ERR_INVALID_ARG || st == CF_ERR_SHAPE);
        g_shape += st == CF_ERR_SHAPE;
    }
    std::printf("%d launches, %d refused for their sizes\n", g_launches, g_shape);
    EXPECT(g_launches > 20000 && g_shape > 20000);

    // Values in the middle of the keys' pages, which reach further than 64 bits of bytes can say.
    const cf_attn_desc d = {CF_BF16, 1, 1, 64, 0.0f};
    const cf_kv_cache c = {reinterpret_cast<void *>(at), reinterpret_cast<void *>(at + ((uintptr_t)1 << 41)), (int64_t)1 << 30, (int64_t)1 << 40, 16};
    cf_paged p = {1, 1, 0, 0, (int32_t *)f, (int32_t *)f, {f, 64, 64}, {f + 64, 64, 64}, nullptr};
    EXPECT(cf_attn_paged(&d, &c, &p, nullptr, 0, nullptr) == CF_ERR_SHAPE);

    // More sequences than a workgroup lists are split as fewer are, whatever their number; without a workspace they stay whole, in one launch.
    const cf_attn_desc g = {CF_BF16, 8, 1, 128, 0.0f};
    const cf_kv_cache k = {reinterpret_cast<void *>(at), reinterpret_cast<void *>(at + ((uintptr_t)1 << 41)), 100000, 0, 16};
    for (int i = 0; i < 5 * 16; ++i) {
        const int n = i % 5 == 0 ? 2048 : i % 5 == 1 ? 2049 : i % 5 == 2 ? 2100 : i % 5 == 3 ? 4096 : 30000, pages = 1 << (i / 5);
        cf_paged q = {n, pages, 0, 0, (int32_t *)f, (int32_t *)f, {(void *)((uintptr_t)1 << 50), 1024, 128}, {(void *)((uintptr_t)1 << 51), 1024, 128}, nullptr};
        g_sequences = 0;
        EXPECT(cf_attn_paged(&g, &k, &q, reinterpret_cast<void *>((uintptr_t)1 << 40), CF_ATTN_WORKSPACE_BYTES, nullptr) == CF_OK && g_sequences == n && (g_least_splits > 3 || pages < 2048));
        const int before = g_launches;
        g_sequences = 0;
        EXPECT(cf_attn_paged(&g, &k, &q, nullptr, 0, nullptr) == CF_OK && g_sequences == n && g_launches == before + 1);
    }
    if (g_failures) return 1;
    std::printf("all calls hold\n");
    return 0;
}
