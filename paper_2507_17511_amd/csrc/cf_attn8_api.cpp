// Host half of the entry points for the cache in 8 bits: arguments are checked here, and the work is split, before anything is enqueued.
#include "cf_attn8.h"
#include "cf_attn_checks.h"

using namespace cf::attn;

namespace {

constexpr int32_t kMostListedPages = 1 << 20;       // of a head
constexpr int64_t kPlanWorkgroups = 64;
constexpr int64_t kMostGroups = 65536;             // that score the pages of a head

Span bytes_at(const void *p, int64_t bytes) { return {reinterpret_cast<uintptr_t>(p), 1, 0, 1, 0, bytes}; }

// What a cache consists of.
struct Spans8 {
    Span s[5];
    int n;
    bool meets(const Span &x) const
    {
        for (int i = 0; i < n; ++i)
            if (meet(s[i], x)) return true;
        return false;
    }
};

cf_status check_cache8(const cf_kv_cache8 *c, const Heads &h, Cache8 &out, Spans8 &spans)
{
    if (!c) return CF_ERR_INVALID_ARG;
    if (!c->k || !c->v || !aligned(c->k, 16) || !aligned(c->v, 16)) return CF_ERR_INVALID_ARG;
    if (!c->k_scale || !c->v_scale || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4) || !aligned(c->bounds, 16)) return CF_ERR_INVALID_ARG;
    if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128) return CF_ERR_SHAPE;
    if (c->n_pages < 1 || c->n_pages > INT32_MAX) return CF_ERR_SHAPE;
    const int64_t dense = (int64_t)h.kv_heads * c->page_size * h.head_dim;
    const int64_t stride = c->page_stride ? c->page_stride : dense;
    if (stride < dense || stride % 16 != 0 || stride > ((int64_t)1 << 40) || c->n_pages > kMostSpan / stride) return CF_ERR_SHAPE;
    out.k = static_cast<char *>(c->k);
    out.v = static_cast<char *>(c->v);
    out.k_scale = c->k_scale;
    out.v_scale = c->v_scale;
    out.bounds = static_cast<uint16_t *>(c->bounds);
    out.page_bytes = stride;
    out.n_pages = (int32_t)c->n_pages;
    out.page_size = c->page_size;
    out.page_shift = __builtin_ctz((unsigned)c->page_size);
    spans.n = c->bounds ? 5 : 4;
    spans.s[0] = spans.s[1] = {reinterpret_cast<uintptr_t>(c->k), c->n_pages, stride, 1, 0, dense};
    spans.s[1].at = reinterpret_cast<uintptr_t>(c->v);
    spans.s[2] = bytes_at(c->k_scale, c->n_pages * h.kv_heads * 4);
    spans.s[3] = bytes_at(c->v_scale, c->n_pages * h.kv_heads * 4);
    spans.s[4] = bytes_at(c->bounds, c->n_pages * h.kv_heads * h.head_dim * 4);
    for (int i = 0; i < spans.n; ++i)
        for (int j = 0; j < i; ++j)
            if (meet(spans.s[i], spans.s[j])) return CF_ERR_INVALID_ARG;
    return CF_OK;
}

// Rows of a table, and lengths.
cf_status check_table(int32_t n_seqs, int32_t max_pages, int64_t stride, int64_t max_len, const void *table, const void *lens)
{
    if (n_seqs < 0 || max_pages < 1 || stride < max_pages || stride > ((int64_t)1 << 40) || max_len < 0) return CF_ERR_SHAPE;
    if (n_seqs == 0) return CF_OK;
    if (stride > kMostSpan / (int64_t)sizeof(int32_t) / n_seqs) return CF_ERR_SHAPE;
    return table && lens && aligned(table, 4) && aligned(lens, 4) ? CF_OK : CF_ERR_INVALID_ARG;
}

constexpr int64_t kMostPartKeys8 = 2048;

// A workgroup for each part of a context, two a CU: of 256 to 2048 keys each, or 128 where a context is 1024 at most.  us in a graph, parts of 128 / 256 keys, 2 and 8 heads: 1 x 901 of
// 128 8.2 / 8.9 and 8.7 / 9.0, of 256 8.6 / 10.0 and 9.0 / 10.1; 1 x 1500 of 128 8.3 / 9.0 and 9.1 / 9.3, of 64 7.5 / 7.6 and 8.5 / 8.0; 1 x 2048 of 128 8.5 / 9.0 and 9.6 / 9.4; 1 x 4000 9.1 / 9.1
// and 11.4 / 10.1, of 256 10.4 / 10.5 and 12.6 / 11.4: between 1024 and 3000 keys the better one goes by heads and their width, by a tenth.  Where 32 parts of each already give a workgroup a CU
// there are no more of them, as each adds to the join: 8 heads of 128, 1 x 16384 13.5 for 15.9, 1 x 32768 18.1 for 20.9, 1 x 60000 26.0 for 26.4.
//
// Past four workgroups a CU, and where contexts that may differ could fill 64 MB, equal shares of all keys for as many workgroups as the device holds.  The host does not know the lengths: contexts
// that differ gain, a few that are alike may lose.  us in a graph, a workgroup for each part / shares, heads of 128: 96 x 160 to 16000 keys, 8 heads, 157 / 139; 150 x 90 to 9000, 1 head, 37 / 23;
// 64 x 8192, 8 heads, 203 / 187; 2 x 131100 104 / 104; 8 x 8192 27 / 30; lists of 64 pages of 64 (with their selection) for 64 contexts of 320 to 32000
// 95 / 91, for 8 of 131072 40 / 43; 2 x 131100, 24 heads of 64, 157 / 150.
// Heads of 256: 48 x 160 to 16000, 2 heads, 51 / 36, 8 heads 167 / 136; 16 x 600 to 60000, 2 heads, 89 / 53; 24 x 8192 44 / 51; 4 x 60000 45 / 59.
hipError_t paged8_at_once(Paged8Args &b, int64_t longest, void *workspace, size_t workspace_bytes, hipStream_t s)
{
    PagedArgs &a = b.p;
    const int64_t units = paged_units(a);
    const int64_t rows = (int64_t)a.n_seqs * a.h.q_heads;
    const int64_t grain = longest <= 1024 ? 128 : 256;
    int64_t keys = round_up((longest * units + 2 * kCUs - 1) / (2 * kCUs), grain);
    if (units * 32 >= kCUs && keys < longest / 32) keys = round_up(longest / 32, grain);
    if (keys > kMostPartKeys8) keys = kMostPartKeys8;
    int64_t splits = (longest + keys - 1) / keys;
    const int64_t fit = parts_that_fit(workspace_bytes, rows, a.h.head_dim);
    if (splits > fit) splits = fit;
    if (splits > kMaxParts) splits = kMaxParts;
    if (a.n_seqs > kMostListed || units > kCounters) splits = 1;        // no places for more in the kernel's list, or for more counters
    a.n_splits = 1;
    a.split_keys = (int32_t)kMostRows;
    if (splits > 1) {
        a.split_keys = (int32_t)round_up((longest + splits - 1) / splits, 128);
        a.n_splits = (int32_t)((longest + a.split_keys - 1) / a.split_keys);
    }
    const bool counted = (int64_t)a.n_seqs * (((int64_t)a.max_pages << b.cache.page_shift) / 256 + 2) <= INT32_MAX;      // shares are in 32 bits
    a.many = counted && a.n_splits > 1 && (units * a.n_splits > 4 * kCUs || (a.n_seqs > 1 && units * longest * a.h.head_dim * 2 >= (int64_t)64 << 20));
    if (a.many) a.n_splits = (int32_t)(fit < kMaxParts ? fit : kMaxParts);       // at most, of shares that the lengths decide
    if (a.n_splits > 1) place_parts(a.parts, workspace, rows, a.n_splits, a.h.head_dim);
    a.counters = static_cast<uint32_t *>(workspace);
    return launch_paged8(b, s);
}

}  // namespace

extern "C" {

cf_status cf_kv_append8(const cf_attn_desc *desc, const cf_kv_cache8 *cache, const cf_append *args, void *stream)
{
    Append8Args a = {};
    Spans8 held;
    Span sk, sv, sq, so;
    cf_status st = check_desc(desc, a.h);
    if (st != CF_OK) return st;
    if (!args) return CF_ERR_INVALID_ARG;
    if ((st = check_cache8(cache, a.h, a.cache, held)) != CF_OK) return st;
    if (args->n_tokens < 0 || args->n_tokens > kMostRows) return CF_ERR_SHAPE;
    if (args->rotary_dim < 0 || args->rotary_dim > desc->head_dim || args->rotary_dim % 16 != 0) return CF_ERR_SHAPE;
    if (args->n_tokens == 0) return CF_OK;
    const int64_t n = args->n_tokens, d = desc->head_dim;
    if ((st = check_rows(args->k, n, desc->kv_heads, d, false, 0, a.k, sk)) != CF_OK) return st;
    if ((st = check_rows(args->v, n, desc->kv_heads, d, false, 0, a.v, sv)) != CF_OK) return st;
    if (!args->slots || !aligned(args->slots, 8)) return CF_ERR_INVALID_ARG;
    if (held.meets(sk) || held.meets(sv)) return CF_ERR_INVALID_ARG;
    if (args->q.data || args->q_out.data) {
        if ((st = check_rows(args->q, n, desc->q_heads, d, false, 0, a.q, sq)) != CF_OK) return st;
        if ((st = check_rows(args->q_out, n, desc->q_heads, d, true, 0, a.q_out, so)) != CF_OK) return st;
        const bool in_place = a.q.data == a.q_out.data && a.q.token == a.q_out.token && a.q.head == a.q_out.head;
        if ((!in_place && meet(sq, so)) || meet(so, sk) || meet(so, sv) || held.meets(so) || held.meets(sq)) return CF_ERR_INVALID_ARG;
    }
    if (args->rotary_dim > 0) {
        if (!args->positions || !aligned(args->positions, 4) || !args->cos || !args->sin || !aligned(args->cos, 16) || !aligned(args->sin, 16)) return CF_ERR_INVALID_ARG;
        if (args->n_positions < 1 || args->n_positions > INT32_MAX) return CF_ERR_SHAPE;
        a.positions = args->positions;
        a.cos = args->cos;
        a.sin = args->sin;
        a.n_positions = (int32_t)args->n_positions;
    }
    a.slots = args->slots;
    a.n_tokens = n;
    a.rotary_dim = args->rotary_dim;
    a.interleaved = args->interleaved ? 1 : 0;
    // Some 2048 workgroups, or what 64 tokens each give: those that find no page's begin, or leave lone tokens to a neighbour, cost their launch.
    const int64_t chunk = round_up((n * 2 * a.h.kv_heads + 2047) / 2048, 8);
    a.chunk = (int32_t)(chunk < 64 ? chunk : 64);
    const int64_t each = ((n + a.chunk - 1) / a.chunk + kXcds - 1) / kXcds, groups = each * kXcds * 2 * a.h.kv_heads;
    if (groups > kMostWorkgroups) return CF_ERR_SHAPE;
    a.chunks_each = (int32_t)each;
    a.page_groups = (int32_t)groups;
    if (append8_workgroups(a) > kMostWorkgroups / (kAppendThreads / 256)) return CF_ERR_SHAPE;
    return status_of(launch_append8(a, static_cast<hipStream_t>(stream)));
}

cf_status cf_attn_paged8(const cf_attn_desc *desc, const cf_kv_cache8 *cache, const cf_paged *args, const cf_blocks *blocks, void *workspace, size_t workspace_bytes,
                         void *stream)
{
    Paged8Args b = {};
    PagedArgs &a = b.p;
    Spans8 held;
    Span sq, so;
    cf_status st = check_desc(desc, a.h);
    if (st != CF_OK) return st;
    if (!args) return CF_ERR_INVALID_ARG;
    if ((st = check_cache8(cache, a.h, b.cache, held)) != CF_OK) return st;
    if ((st = check_workspace(workspace, workspace_bytes)) != CF_OK) return st;
    const int64_t stride = args->table_stride ? args->table_stride : args->max_pages;
    if (args->n_seqs > kMostRows / desc->q_heads) return CF_ERR_SHAPE;
    if (blocks && (blocks->count < 1 || blocks->count > kMostListedPages)) return CF_ERR_SHAPE;
    if ((st = check_table(args->n_seqs, args->max_pages, stride, args->max_len, args->table, args->lens)) != CF_OK) return st;
    if (args->n_seqs == 0) return CF_OK;
    if (blocks && (!blocks->blocks || !aligned(blocks->blocks, 4))) return CF_ERR_INVALID_ARG;
    if ((st = check_rows(args->q, args->n_seqs, desc->q_heads, desc->head_dim, false, 0, a.q, sq)) != CF_OK) return st;
    if ((st = check_rows(args->out, args->n_seqs, desc->q_heads, desc->head_dim, true, 0, a.out, so)) != CF_OK) return st;
    if (meet(so, sq) || held.meets(so)) return CF_ERR_INVALID_ARG;
    if (!aligned(args->lse, 4)) return CF_ERR_INVALID_ARG;
    a.lse = args->lse;
    a.table = args->table;
    a.lens = args->lens;
    a.table_stride = stride;
    a.n_seqs = args->n_seqs;
    a.max_pages = args->max_pages;
    b.blocks = blocks ? blocks->blocks : nullptr;
    b.count = blocks ? blocks->count : 0;

    const int64_t capacity = (int64_t)args->max_pages * b.cache.page_size;
    int64_t longest = args->max_len > 0 && args->max_len < capacity ? args->max_len : capacity;
    if (blocks && longest > (int64_t)b.count * b.cache.page_size) longest = (int64_t)b.count * b.cache.page_size;
    if (longest > kMostRows) longest = kMostRows;
    // Of many sequences some at a time: as many as a workgroup lists and counters go round, or, where their contexts are not split, as a launch has workgroups for.
    const int64_t units = paged_units(a) / a.n_seqs, listed = kCounters / units < kMostListed ? kCounters / units : kMostListed;
    int64_t most = a.n_seqs;
    if (a.n_seqs > listed) most = listed > 0 && longest > 4 * kMostPartKeys8 && parts_that_fit(workspace_bytes, listed * a.h.q_heads, a.h.head_dim) > 1 ? listed : kMostWorkgroups / units;
    most = (a.n_seqs + (a.n_seqs + most - 1) / most - 1) / ((a.n_seqs + most - 1) / most);
    hipError_t e = hipSuccess;
    for (int64_t first = 0; e == hipSuccess && first < args->n_seqs; first += most) {
        Paged8Args some = b;
        some.p.n_seqs = (int32_t)(args->n_seqs - first < most ? args->n_seqs - first : most);
        some.p.q.data += first * a.q.token;
        some.p.out.data += first * a.out.token;
        if (a.lse) some.p.lse += first * a.h.q_heads;
        some.p.table += first * a.table_stride;
        some.p.lens += first;
        if (b.blocks) some.blocks += first * a.h.kv_heads * b.count;
        e = paged8_at_once(some, longest, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
    }
    return status_of(e);
}

cf_status cf_attn_select(const cf_attn_desc *desc, const cf_kv_cache8 *cache, const cf_select *args, void *workspace, size_t workspace_bytes, void *stream)
{
    SelectArgs a = {};
    Spans8 held;
    Span sq;
    cf_status st = check_desc(desc, a.h);
    if (st != CF_OK) return st;
    if (!args) return CF_ERR_INVALID_ARG;
    if ((st = check_cache8(cache, a.h, a.cache, held)) != CF_OK) return st;
    if (!a.cache.bounds) return CF_ERR_INVALID_ARG;
    if ((st = check_workspace(workspace, workspace_bytes)) != CF_OK) return st;
    const int64_t stride = args->table_stride ? args->table_stride : args->max_pages;
    if (args->n_seqs > kMostRows / desc->q_heads) return CF_ERR_SHAPE;
    if (args->count < 1 || args->count > kMostListedPages || args->first < 0 || args->recent < 0 || args->first > args->count || args->recent > args->count - args->first) return CF_ERR_SHAPE;
    if ((st = check_table(args->n_seqs, args->max_pages, stride, args->max_len, args->table, args->lens)) != CF_OK) return st;
    if (args->n_seqs == 0) return CF_OK;
    if ((st = check_rows(args->q, args->n_seqs, desc->q_heads, desc->head_dim, false, 0, a.q, sq)) != CF_OK) return st;
    if (!args->blocks || !aligned(args->blocks, 4)) return CF_ERR_INVALID_ARG;
    const int64_t rows = (int64_t)args->n_seqs * a.h.kv_heads;
    const Span so = bytes_at(args->blocks, rows * args->count * 4);
    if (meet(so, sq) || held.meets(so) || meet(so, {reinterpret_cast<uintptr_t>(args->table), args->n_seqs, stride * 4, 1, 0, (int64_t)args->max_pages * 4}) ||
        meet(so, bytes_at(args->lens, (int64_t)args->n_seqs * 4)))
        return CF_ERR_INVALID_ARG;
    a.table = args->table;
    a.lens = args->lens;
    a.table_stride = stride;
    a.n_seqs = args->n_seqs;
    a.max_pages = args->max_pages;
    a.count = args->count;
    a.first = args->first;
    a.recent = args->recent;
    a.blocks = args->blocks;
    // scores of every page that there may be, of as many rows at a time as the workspace holds; workgroups by the longest context as it is said to be
    a.columns = args->max_pages;
    if (workspace_bytes > CF_ATTN_WORKSPACE_BYTES) workspace_bytes = CF_ATTN_WORKSPACE_BYTES;
    const int64_t fit = workspace_bytes > CF_ATTN_COUNTER_BYTES ? (int64_t)(workspace_bytes - CF_ATTN_COUNTER_BYTES) / 8 / a.columns : 0;
    if (fit < 1) return CF_ERR_WORKSPACE;
    a.scores = reinterpret_cast<uint64_t *>(static_cast<char *>(workspace) + CF_ATTN_COUNTER_BYTES);
    int64_t pages = args->max_pages;
    if (args->max_len > 0 && (args->max_len + a.cache.page_size - 1) / a.cache.page_size < pages) pages = (args->max_len + a.cache.page_size - 1) / a.cache.page_size;
    a.groups = (int32_t)((pages + kSelectPages - 1) / kSelectPages < kMostGroups ? (pages + kSelectPages - 1) / kSelectPages : kMostGroups);      // they go round
    int64_t most = fit < rows ? fit : rows;
    if (most > kMostWorkgroups / 4 / a.groups) most = kMostWorkgroups / 4 / a.groups;
    hipError_t e = hipSuccess;
    for (a.first_row = 0; e == hipSuccess && a.first_row < rows; a.first_row += most) {
        a.n_rows = rows - a.first_row < most ? rows - a.first_row : most;
        e = launch_select(a, static_cast<hipStream_t>(stream));
    }
    return status_of(e);
}

cf_status cf_kv_plan(const cf_plan *args, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!args) return CF_ERR_INVALID_ARG;
    cf_status st = check_workspace(workspace, workspace_bytes);
    if (st != CF_OK) return st;
    if (args->page_size < 16 || args->page_size > 32768 || (args->page_size & (args->page_size - 1)) != 0) return CF_ERR_SHAPE;
    if (args->n_ring < 1 || args->n_tokens < 0 || args->n_tokens > kMostRows || args->n_seqs > kMostRows) return CF_ERR_SHAPE;
    const int64_t stride = args->table_stride ? args->table_stride : args->max_pages, n = args->n_seqs;
    if ((st = check_table(args->n_seqs, args->max_pages, stride, 0, args->table, args->lens)) != CF_OK) return st;
    const void *words[] = {args->ring, args->cu, args->refused};
    for (const void *p : words)
        if (!p || !aligned(p, 4)) return CF_ERR_INVALID_ARG;
    if (!args->state || !args->state_out || !aligned(args->state, 8) || !aligned(args->state_out, 8)) return CF_ERR_INVALID_ARG;
    if (n > 0 && (!args->news || !args->lens_out || !aligned(args->news, 4) || !aligned(args->lens_out, 4))) return CF_ERR_INVALID_ARG;
    if (args->n_tokens > 0 && (!args->slots || !args->positions || !aligned(args->slots, 8) || !aligned(args->positions, 4))) return CF_ERR_INVALID_ARG;
    // what is written, and then what is read alone; lengths and state may be updated in place
    const Span none = {0, 0, 0, 0, 0, 0};
    const Span spans[] = {n > 0 ? Span{reinterpret_cast<uintptr_t>(args->table), n, stride * 4, 1, 0, (int64_t)args->max_pages * 4} : none,
                          bytes_at(args->ring, (int64_t)args->n_ring * 4),
                          bytes_at(args->state_out, 16),
                          n > 0 ? bytes_at(args->lens_out, n * 4) : none,
                          bytes_at(args->cu, (n + 1) * 4),
                          bytes_at(args->refused, 4),
                          args->n_tokens > 0 ? bytes_at(args->slots, args->n_tokens * 8) : none,
                          args->n_tokens > 0 ? bytes_at(args->positions, args->n_tokens * 4) : none,
                          n > 0 ? bytes_at(args->news, n * 4) : none,
                          args->state != args->state_out ? bytes_at(args->state, 16) : none,
                          n > 0 && args->lens != args->lens_out ? bytes_at(args->lens, n * 4) : none};
    constexpr int kWritten = 8, kAll = sizeof(spans) / sizeof(spans[0]);
    for (int i = 0; i < kWritten; ++i)
        for (int j = i + 1; j < kAll; ++j)
            if (meet(spans[i], spans[j])) return CF_ERR_INVALID_ARG;
    PlanArgs a = {};
    a.lens = args->lens;
    a.news = args->news;
    a.table = args->table;
    a.ring = args->ring;
    a.state = args->state;
    a.state_out = args->state_out;
    a.lens_out = args->lens_out;
    a.cu = args->cu;
    a.positions = args->positions;
    a.refused = args->refused;
    a.slots = args->slots;
    a.counter = static_cast<uint32_t *>(workspace);
    a.table_stride = stride;
    a.n_seqs = args->n_seqs;
    a.page_shift = __builtin_ctz((unsigned)args->page_size);
    a.max_pages = args->max_pages;
    a.n_ring = args->n_ring;
    a.n_tokens = (int32_t)args->n_tokens;
    // Few threads where there is little to do: what all of them compute is most of the time.  A token for each of many: us, 1500 sequences that bring 36579 tokens, one / two / four at a
    // time for a thread 11.8 / 13.1 / 16.3, 14 prompts of 2768 5.5 / 6.3 / 6.3.
    a.wide = args->n_seqs > kPlanThreads / 4 || args->n_tokens > kPlanThreads;
    int64_t groups = (args->n_tokens + kPlanThreads - 1) / kPlanThreads;
    if (groups > kPlanWorkgroups) groups = kPlanWorkgroups;
    if (groups < 1 || workspace_bytes < sizeof(uint32_t)) groups = 1;
    a.workgroups = (int32_t)groups;
    return status_of(launch_plan(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
