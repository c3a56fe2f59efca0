// The host half of the entry points for the cache in 8 bits (csrc/cf_attn8_api.cpp) with launchers that check what they are handed: random calls, many of them
// valid, none of which may launch anything that reaches outside the buffers it was given.  Runs under sanitizers, without a device.
#include <cstdio>
#include <cstdlib>
#include <random>

#include "cf_attn8.h"
#include "compactfusion.h"

namespace {
int g_failures, g_appends, g_paged, g_shared, g_split, g_listed, g_selects, g_plans, g_seqs_left;
int64_t g_rows_left;
bool g_refuse;
char *g_ws;
size_t g_ws_bytes;

void expect(bool ok, const char *what, int line)
{
    if (!ok) {
        std::printf("line %d: %s\n", line, what);
        ++g_failures;
    }
}
#define EXPECT(x) expect((x), #x, __LINE__)
constexpr int64_t kMost = (((int64_t)1 << 32) - 1) / 256;
}  // namespace

namespace cf {
namespace attn {
static void check_cache(const Cache8 &c, const Heads &h)
{
    EXPECT((1 << c.page_shift) == c.page_size && c.page_size >= 16 && c.page_size <= 128 && c.n_pages >= 1);
    EXPECT(c.page_bytes >= (int64_t)h.kv_heads * c.page_size * h.head_dim && c.page_bytes % 16 == 0 && c.k && c.v && c.k_scale && c.v_scale);
}
hipError_t launch_paged8(const Paged8Args &a, hipStream_t)
{
    ++g_paged;
    const PagedArgs &p = a.p;
    check_cache(a.cache, p.h);
    const int64_t n = paged8_workgroups(a), rows = (int64_t)p.n_seqs * p.h.q_heads;
    EXPECT(n >= 1 && n <= kMost && p.n_seqs >= 1 && p.n_seqs <= g_seqs_left);
    g_seqs_left -= p.n_seqs;
    EXPECT(p.n_splits >= 1 && p.n_splits <= kMaxParts && p.table_stride >= p.max_pages);
    EXPECT((a.blocks != nullptr) == (a.count > 0));
    if (a.blocks) ++g_listed;
    if (p.n_splits > 1) {
        ++g_split;
        const char *o = reinterpret_cast<const char *>(p.parts.o), *end = reinterpret_cast<const char *>(p.parts.lse + (int64_t)p.n_splits * rows);
        EXPECT(p.parts.n_rows == rows && o >= g_ws + CF_ATTN_COUNTER_BYTES && end <= g_ws + g_ws_bytes && end - o <= (int64_t)CF_ATTN_WORKSPACE_BYTES);
        EXPECT(reinterpret_cast<const char *>(p.parts.lse) == o + (int64_t)p.n_splits * rows * p.h.head_dim * 4);
        EXPECT(reinterpret_cast<const char *>(p.counters) == g_ws && paged_units(p) * 4 <= (int64_t)CF_ATTN_COUNTER_BYTES);
        EXPECT(p.many || p.split_keys % 128 == 0);
    } else EXPECT(!p.many && p.split_keys >= (1 << 30));
    if (p.many) {
        ++g_shared;
        EXPECT(p.n_seqs <= kMostListed && p.n_splits > 1);
        EXPECT((int64_t)p.n_seqs * (((int64_t)p.max_pages << a.cache.page_shift) / 256 + 2) <= INT32_MAX);
    }
    return g_refuse ? hipErrorLaunchFailure : hipSuccess;
}
hipError_t launch_append8(const Append8Args &a, hipStream_t)
{
    ++g_appends;
    check_cache(a.cache, a.h);
    EXPECT(a.chunk >= 8 && a.chunk <= 64 && a.page_groups % kXcds == 0);
    EXPECT((int64_t)a.chunks_each * kXcds * a.chunk >= a.n_tokens && (int64_t)a.chunks_each * kXcds * 2 * a.h.kv_heads == a.page_groups);
    EXPECT(append8_workgroups(a) <= kMost / (kAppendThreads / 256));
    EXPECT(!a.q.data || (append8_workgroups(a) - a.page_groups) * kAppendThreads * kAppendTurns >= a.n_tokens * a.h.q_heads * (a.h.head_dim / 16));
    EXPECT(a.rotary_dim % 16 == 0 && a.rotary_dim <= a.h.head_dim && (a.rotary_dim == 0 || (a.positions && a.cos && a.sin && a.n_positions > 0)));
    return g_refuse ? hipErrorLaunchFailure : hipSuccess;
}
hipError_t launch_select(const SelectArgs &a, hipStream_t)
{
    ++g_selects;
    check_cache(a.cache, a.h);
    EXPECT(a.cache.bounds && a.columns == a.max_pages && a.n_rows >= 1 && a.n_rows <= g_rows_left && a.groups >= 1 && a.n_rows * a.groups <= kMost);
    g_rows_left -= a.n_rows;
    const char *s = reinterpret_cast<const char *>(a.scores);
    EXPECT(s >= g_ws + CF_ATTN_COUNTER_BYTES && s + a.n_rows * a.columns * 8 <= g_ws + g_ws_bytes && reinterpret_cast<uintptr_t>(s) % 8 == 0);
    EXPECT(a.count >= 1 && a.first >= 0 && a.recent >= 0 && a.first + a.recent <= a.count);
    return g_refuse ? hipErrorLaunchFailure : hipSuccess;
}
hipError_t launch_plan(const PlanArgs &a, hipStream_t)
{
    ++g_plans;
    EXPECT(a.workgroups >= 1 && a.workgroups <= 64 && (a.workgroups == 1 || a.counter) && a.n_ring >= 1 && a.max_pages >= 1 && a.table_stride >= a.max_pages);
    return g_refuse ? hipErrorLaunchFailure : hipSuccess;
}
}  // namespace attn
}  // namespace cf

int main()
{
    std::mt19937_64 r(5);
    auto pick = [&](int64_t lo, int64_t hi) { return (int64_t)(lo + r() % (uint64_t)(hi - lo + 1)); };
    auto wide = [&](int64_t hi) { return pick(0, 3) ? pick(0, 1 + pick(0, hi) / 1000) : pick(0, hi); };
    g_ws = static_cast<char *>(aligned_alloc(256, CF_ATTN_WORKSPACE_BYTES));
    char *const far = reinterpret_cast<char *>((uintptr_t)1 << 50);
    int done[4] = {}, refused[4] = {};
    for (int i = 0; i < 200000; ++i) {
        const int kv = (int)pick(1, pick(0, 9) ? 12 : pick(0, 5) ? 300 : 65536), dims[] = {64, 128, 256, 96};
        cf_attn_desc d = {(int32_t)pick(pick(0, 19) ? 1 : 0, 2), (int32_t)(kv * (kv > 300 ? 1 : pick(1, 20))), kv, dims[pick(0, 20) ? pick(0, 2) : 3], pick(0, 3) ? 0.0f : 0.3f};
        const int pages[] = {16, 32, 64, 128, 48};
        cf_kv_cache8 c = {};
        c.page_size = pages[pick(0, 20) ? pick(0, 3) : 4];
        c.n_pages = 1 + wide(100000);
        c.page_stride = pick(0, 2) ? 0 : (int64_t)kv * c.page_size * d.head_dim * pick(1, 3) + 16 * pick(0, 2) + (pick(0, 20) ? 0 : 8);
        c.k = far, c.v = far + ((int64_t)1 << 46), c.k_scale = reinterpret_cast<float *>(far + ((int64_t)2 << 46)), c.v_scale = reinterpret_cast<float *>(far + ((int64_t)3 << 46));
        if (pick(0, 3)) c.bounds = far + ((int64_t)4 << 46);
        if (!pick(0, 30)) c.v = far + pick(0, 1) * 16;
        if (!pick(0, 30)) c.v_scale = c.k_scale;
        g_ws_bytes = pick(0, 2) ? CF_ATTN_WORKSPACE_BYTES : pick(0, 1) ? 0 : (size_t)pick(1, CF_ATTN_WORKSPACE_BYTES / 256) * 256;
        void *ws = g_ws_bytes || pick(0, 1) ? g_ws : nullptr;
        g_refuse = !pick(0, 50);
        char *const near = far + ((int64_t)5 << 46);
        auto rows = [&](int at, int heads) { return cf_rows{near + ((int64_t)at << 42), (int64_t)heads * d.head_dim + 8 * pick(0, 2), d.head_dim}; };
        auto list = [&](int at) { return near + ((int64_t)at << 42); };
        cf_status st = CF_OK;
        const int call = (int)pick(0, 3);
        int before = 0, after = 0;
        if (call == 0) {
            cf_append a = {};
            a.n_tokens = wide((int64_t)1 << 30);
            a.k = rows(1, kv), a.v = rows(2, kv), a.slots = reinterpret_cast<int64_t *>(list(3));
            if (pick(0, 1)) a.q = rows(4, d.q_heads), a.q_out = pick(0, 1) ? a.q : rows(5, d.q_heads);
            a.rotary_dim = (int32_t)pick(0, d.head_dim / 16) * 16;
            a.positions = reinterpret_cast<int32_t *>(list(6)), a.cos = reinterpret_cast<float *>(list(7)), a.sin = reinterpret_cast<float *>(list(8));
            a.n_positions = pick(1, 1000), a.interleaved = (int32_t)pick(0, 1);
            before = g_appends;
            st = cf_kv_append8(&d, &c, &a, nullptr);
            after = g_appends;
            EXPECT(st == CF_OK || st == CF_ERR_DEVICE ? after == before + (a.n_tokens > 0) : after == before);
        } else if (call == 1 || call == 2) {
            const int32_t n = (int32_t)wide(pick(0, 1) ? 5000 : 1 << 24), most = (int32_t)(1 + wide(pick(0, 20) ? 20000 : INT32_MAX - 1));
            const int64_t stride = pick(0, 1) ? 0 : most + pick(0, 5), longest = pick(0, 1) ? 0 : wide((int64_t)1 << 40);
            const int32_t count = (int32_t)(1 + wide(1 << 20));
            g_seqs_left = n, g_rows_left = (int64_t)n * kv;
            if (call == 1) {
                cf_paged a = {n, most, stride, longest, reinterpret_cast<int32_t *>(list(1)), reinterpret_cast<int32_t *>(list(2)), rows(3, d.q_heads), rows(4, d.q_heads),
                              pick(0, 1) ? reinterpret_cast<float *>(list(5)) : nullptr};
                cf_blocks b = {reinterpret_cast<int32_t *>(list(6)), count};
                before = g_paged;
                st = cf_attn_paged8(&d, &c, &a, pick(0, 1) ? &b : nullptr, ws, g_ws_bytes, nullptr);
                after = g_paged;
                if (st == CF_OK) EXPECT(g_seqs_left == 0);
            } else {
                cf_select a = {n, most, stride, longest, reinterpret_cast<int32_t *>(list(1)), reinterpret_cast<int32_t *>(list(2)), rows(3, d.q_heads), count,
                               (int32_t)pick(0, 3), (int32_t)pick(0, 3), reinterpret_cast<int32_t *>(list(6))};
                before = g_selects;
                st = cf_attn_select(&d, &c, &a, ws, g_ws_bytes, nullptr);
                after = g_selects;
                if (st == CF_OK) EXPECT(g_rows_left == 0);
            }
        } else {
            cf_plan a = {};
            a.n_seqs = (int32_t)wide(1 << 30), a.page_size = 16 << pick(0, 11), a.max_pages = (int32_t)(1 + wide(INT32_MAX - 1)), a.n_ring = (int32_t)(1 + wide(INT32_MAX - 1));
            if (!pick(0, 20)) a.page_size += 1;
            a.n_tokens = wide((int64_t)1 << 30);
            a.lens = reinterpret_cast<int32_t *>(list(1)), a.news = reinterpret_cast<int32_t *>(list(2)), a.ring = reinterpret_cast<int32_t *>(list(3));
            a.state = reinterpret_cast<int64_t *>(list(4)), a.state_out = pick(0, 1) ? reinterpret_cast<int64_t *>(list(4)) : reinterpret_cast<int64_t *>(list(5));
            a.lens_out = pick(0, 1) ? reinterpret_cast<int32_t *>(list(1)) : reinterpret_cast<int32_t *>(list(6)), a.cu = reinterpret_cast<int32_t *>(list(7));
            a.slots = reinterpret_cast<int64_t *>(list(8)), a.positions = reinterpret_cast<int32_t *>(list(9)), a.refused = reinterpret_cast<int32_t *>(list(10));
            a.table = reinterpret_cast<int32_t *>(reinterpret_cast<char *>((uintptr_t)1 << 60));
            if (!pick(0, 20)) a.positions = reinterpret_cast<int32_t *>(list(7));
            before = g_plans;
            st = cf_kv_plan(&a, ws, g_ws_bytes, nullptr);
            after = g_plans;
        }
        EXPECT(st == CF_OK || st == CF_ERR_DEVICE || after == before);
        EXPECT(!g_refuse || st != CF_OK || after == before);
        (st == CF_OK || st == CF_ERR_DEVICE ? done : refused)[call]++;
    }
    for (int k = 0; k < 4; ++k) EXPECT(done[k] > 3000 && refused[k] > 300);
    EXPECT(g_shared > 500 && g_split > g_shared && g_listed > 1000);
    std::printf("%d %d %d %d done, %d %d %d %d refused, %d split, %d shared\n", done[0], done[1], done[2], done[3], refused[0], refused[1], refused[2], refused[3], g_split, g_shared);
    std::free(g_ws);
    if (g_failures) return 1;
    std::printf("all calls hold\n");
    return 0;
}
