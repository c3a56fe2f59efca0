// Host half of the attention entry points: arguments are checked here, and the work is split, before anything is enqueued.
#include "cf_attn_checks.h"

using namespace cf::attn;

namespace {

// How many workgroups of the prompt kernel a CU holds, what they take over 64 keys, us, and which share of that fewer of them take: one CU's worth of
// whole tiles for each, 1 to 4 a CU (128 tiles of 64 keys 120 / 173 / 250 / 307 us at head_dim 64; 64 of them 82 / 133 at 128, 237 / 258 at 256).
struct Pace {
    int64_t per_cu;
    double step_us, share[4];
};
Pace prompt_pace(int dim)
{
    if (dim == 64) return {4, 2.4, {0.39, 0.56, 0.81, 1.0}};
    if (dim == 128) return {2, 1.95, {0.62, 1.0}};
    return {2, 3.9, {0.92, 1.0}};
}

// Into how many parts the keys of `busy` workgroups are split: what takes the least time, where the join moves the parts twice at 5 TB/s, 4 us at least.
// 2 x 333 tokens over 20333 keys, 84 workgroups: 6 parts, 235 us.
int64_t prompt_splits(int64_t busy, int64_t longest, int64_t rows, int dim, int64_t most)
{
    const Pace pace = prompt_pace(dim);
    const int64_t slots = pace.per_cu * kCUs, steps = (longest + 63) / 64;
    const double part_us = (double)rows * (dim + 1) * 4 * 2 / 5.0e6;
    int64_t best = 1;
    double least = 0.0;
    for (int64_t n = 1; n <= (most > 1 ? most : 1); ++n) {
        const int64_t rest = busy * n % slots;
        const double rounds = (double)(busy * n / slots) + (rest == 0 ? 0.0 : pace.share[(rest - 1) / kCUs]);
        const double us = rounds * (double)((steps + n - 1) / n) * pace.step_us + (n > 1 ? 4.0 + part_us * (double)n : 0.0);
        if (n == 1 || us < least) {
            best = n;
            least = us;
        }
    }
    return best;
}

constexpr int64_t kMostPartKeys = 1024, kMostPartKeysOfMany = 4096, kLongOfMany = 16384;

// One launch, and another one that joins parts of more than the device holds at a time.
hipError_t paged_at_once(PagedArgs &a, int64_t longest, int64_t most_keys, void *workspace, size_t workspace_bytes, hipStream_t s)
{
    const int64_t units = paged_units(a);
    const int64_t rows = (int64_t)a.n_seqs * a.h.q_heads;
    // Two workgroups a CU, of 128 to 1024 keys each (4096 where there are many sequences, more where 64 parts or the workspace's do not reach), and 32 parts at most
    // where that gives every CU one: a part costs its join about 0.1 us, 128
    // keys a workgroup 1.2 us.  us, on one card: 1 x 901 keys, 2 heads of keys: parts of 128 / 256 / 512 keys 8.2 / 9.6 / 11.4; 1 x 8192, 8 heads: 128 / 256
    // / 512 16.7 / 13.0 / 13.6; 8 x 8192, 8 heads: two / three / six workgroups a CU 45 / 49 / 53; 64 x 7 to 700: 14.5 / 18.1 / 16.1.  Parts of 512 / 1024 /
    // 2048 keys, 8 heads of 128: 96 x 160 to 16000 275 / 273 / 271, 96 x 3540 264 / 251 / 243; of 256: 48 x 160 to 16000 282 / 279 / 300; of 64: 200 x 50
    // to 5000 93 / 95 / 102; one of 128: 150 x 90 to 9000 33 / 35 / 57.
    int64_t keys = round_up((longest * units + 2 * kCUs - 1) / (2 * kCUs), 128);
    if (units * 32 >= kCUs && keys < longest / 32) keys = round_up(longest / 32, 128);
    if (keys > most_keys) keys = most_keys;
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
    if (a.n_splits > 1) place_parts(a.parts, workspace, rows, a.n_splits, a.h.head_dim);
    a.counters = static_cast<uint32_t *>(workspace);
    // Listed parts where there are more than the device holds, and where contexts that may differ could fill 128 MB: a workgroup for every part that there may
    // be leaves those of the long contexts on a few XCDs.  us, one for each / listed: 8 x 270 to 27465 keys, 4 heads of 256, 85 / 39; 4 x 1270 to 126712, 4 of
    // 128, 126 / 89; 16 x 40 to 4000, 8 of 128, 26 / 19, but 16 x 4000 43.1 / 44.2, 8 x 8192 43.6 / 45.8, 3 x 120 to 12000, 8 of 64, 11.6 / 12.8.
    a.many = a.n_splits > 1 && (units * a.n_splits > 4 * kCUs || (a.n_seqs > 1 && units * longest * a.h.head_dim * 4 >= (int64_t)128 << 20));
    hipError_t e = launch_paged(a, s);
    if (e == hipSuccess && a.many) {
        JoinArgs j = parts_to_join(a.h, a.parts, a.n_splits, a.out, a.lse);
        j.lens = a.lens;
        j.split_keys = a.split_keys;
        e = launch_join(j, s);
    }
    return e;
}

}  // namespace

extern "C" {

cf_status cf_kv_append(const cf_attn_desc *desc, const cf_kv_cache *cache, const cf_append *args, void *stream)
{
    AppendArgs a = {};
    Span ck, cv, sk, sv, sq, so;
    cf_status st = check_desc(desc, a.h);
    if (st != CF_OK) return st;
    if (!args) return CF_ERR_INVALID_ARG;
    if ((st = check_cache(cache, a.h, a.cache, ck, cv)) != CF_OK) return st;
    if (args->n_tokens < 0 || args->n_tokens > kMostRows) return CF_ERR_SHAPE;
    if (args->rotary_dim < 0 || args->rotary_dim > desc->head_dim || args->rotary_dim % 16 != 0) return CF_ERR_SHAPE;
    if (args->n_tokens == 0) return CF_OK;
    const int64_t n = args->n_tokens, d = desc->head_dim;
    if ((st = check_rows(args->k, n, desc->kv_heads, d, false, 0, a.k, sk)) != CF_OK) return st;
    if ((st = check_rows(args->v, n, desc->kv_heads, d, false, 0, a.v, sv)) != CF_OK) return st;
    if (!args->slots || !aligned(args->slots, 8)) return CF_ERR_INVALID_ARG;
    if (meet(sk, ck) || meet(sk, cv) || meet(sv, ck) || meet(sv, cv)) return CF_ERR_INVALID_ARG;
    if (args->q.data || args->q_out.data) {
        if ((st = check_rows(args->q, n, desc->q_heads, d, false, 0, a.q, sq)) != CF_OK) return st;
        if ((st = check_rows(args->q_out, n, desc->q_heads, d, true, 0, a.q_out, so)) != CF_OK) return st;
        const bool in_place = a.q.data == a.q_out.data && a.q.token == a.q_out.token && a.q.head == a.q_out.head;
        if ((!in_place && meet(sq, so)) || meet(so, sk) || meet(so, sv) || meet(so, ck) || meet(so, cv) || meet(sq, ck) || meet(sq, cv)) return CF_ERR_INVALID_ARG;
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
    if (append_workgroups(a) > kMostWorkgroups) return CF_ERR_SHAPE;
    return status_of(launch_append(a, static_cast<hipStream_t>(stream)));
}

cf_status cf_attn_prompt(const cf_attn_desc *desc, const cf_prompt *args, void *workspace, size_t workspace_bytes, void *stream)
{
    PromptArgs a = {};
    Span sq, sk, sv, so;
    cf_status st = check_desc(desc, a.h);
    if (st != CF_OK) return st;
    if (!args) return CF_ERR_INVALID_ARG;
    if ((st = check_workspace(workspace, workspace_bytes)) != CF_OK) return st;
    if (args->n_seqs < 0 || args->n_q < 0 || args->n_k < 0 || args->max_k < 0 || args->n_k > kMostRows || args->n_q > kMostRows / desc->q_heads || args->n_seqs > kMostRows) return CF_ERR_SHAPE;
    if (args->n_seqs == 0 || args->n_q == 0) return CF_OK;
    const int64_t d = desc->head_dim;
    if ((st = check_rows(args->q, args->n_q, desc->q_heads, d, false, 0, a.q, sq)) != CF_OK) return st;
    if ((st = check_rows(args->out, args->n_q, desc->q_heads, d, true, 0, a.out, so)) != CF_OK) return st;
    if (meet(so, sq)) return CF_ERR_INVALID_ARG;
    if (args->n_k > 0) {
        if ((st = check_rows(args->k, args->n_k, desc->kv_heads, d, false, d, a.k, sk)) != CF_OK) return st;
        if ((st = check_rows(args->v, args->n_k, desc->kv_heads, d, false, d, a.v, sv)) != CF_OK) return st;
        if (meet(so, sk) || meet(so, sv)) return CF_ERR_INVALID_ARG;
    }
    if (!args->cu_q || !args->cu_k || !aligned(args->cu_q, 4) || !aligned(args->cu_k, 4) || !aligned(args->lse, 4)) return CF_ERR_INVALID_ARG;
    a.lse = args->lse;
    a.cu_q = args->cu_q;
    a.cu_k = args->cu_k;
    a.n_seqs = args->n_seqs;
    a.n_q = (int32_t)args->n_q;
    a.n_k = (int32_t)args->n_k;
    a.causal = args->causal ? 1 : 0;

    const int64_t longest = args->max_k > 0 && args->max_k < args->n_k ? args->max_k : args->n_k;
    const int64_t rows = args->n_q * a.h.q_heads;
    const int64_t busy = (args->n_q * a.h.group + kPromptRows - 1) / kPromptRows * a.h.kv_heads;
    int64_t most = parts_that_fit(workspace_bytes, rows, a.h.head_dim);
    if (most > longest / 256) most = longest / 256;
    if (most > kMaxParts) most = kMaxParts;
    a.n_splits = 1;
    a.split_keys = (int32_t)kMostRows;
    if (prompt_workgroups(a) > kMostWorkgroups) return CF_ERR_SHAPE;
    if (most > kMostWorkgroups / prompt_workgroups(a)) most = kMostWorkgroups / prompt_workgroups(a);
    const int64_t splits = prompt_splits(busy, longest, rows, a.h.head_dim, most);
    if (splits > 1) {
        a.split_keys = (int32_t)round_up((longest + splits - 1) / splits, 64);
        a.n_splits = (int32_t)((longest + a.split_keys - 1) / a.split_keys);
    }
    if (a.n_splits > 1) place_parts(a.parts, workspace, rows, a.n_splits, a.h.head_dim);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = launch_prompt(a, s);
    if (e == hipSuccess && a.n_splits > 1) {
        JoinArgs j = parts_to_join(a.h, a.parts, a.n_splits, a.out, a.lse);
        j.cover = a.cu_q;
        j.n_cover = a.n_seqs;
        e = launch_join(j, s);
    }
    return status_of(e);
}

cf_status cf_attn_paged(const cf_attn_desc *desc, const cf_kv_cache *cache, const cf_paged *args, void *workspace, size_t workspace_bytes,
                        void *stream)
{
    PagedArgs a = {};
    Span ck, cv, sq, so;
    cf_status st = check_desc(desc, a.h);
    if (st != CF_OK) return st;
    if (!args) return CF_ERR_INVALID_ARG;
    if ((st = check_cache(cache, a.h, a.cache, ck, cv)) != CF_OK) return st;
    if ((st = check_workspace(workspace, workspace_bytes)) != CF_OK) return st;
    const int64_t stride = args->table_stride ? args->table_stride : args->max_pages;
    if (args->n_seqs < 0 || args->max_pages < 1 || stride < args->max_pages || stride > ((int64_t)1 << 40) || args->max_len < 0 || args->n_seqs > kMostRows / desc->q_heads) return CF_ERR_SHAPE;
    if (args->n_seqs == 0) return CF_OK;
    if (stride > kMostSpan / (int64_t)sizeof(int32_t) / args->n_seqs) return CF_ERR_SHAPE;
    if ((st = check_rows(args->q, args->n_seqs, desc->q_heads, desc->head_dim, false, 0, a.q, sq)) != CF_OK) return st;
    if ((st = check_rows(args->out, args->n_seqs, desc->q_heads, desc->head_dim, true, 0, a.out, so)) != CF_OK) return st;
    if (meet(so, sq) || meet(so, ck) || meet(so, cv)) return CF_ERR_INVALID_ARG;
    if (!args->table || !args->lens || !aligned(args->table, 4) || !aligned(args->lens, 4) || !aligned(args->lse, 4)) return CF_ERR_INVALID_ARG;
    a.lse = args->lse;
    a.table = args->table;
    a.lens = args->lens;
    a.table_stride = stride;
    a.n_seqs = args->n_seqs;
    a.max_pages = args->max_pages;

    const int64_t capacity = (int64_t)args->max_pages * a.cache.page_size;
    int64_t longest = args->max_len > 0 && args->max_len < capacity ? args->max_len : capacity;
    if (longest > kMostRows) longest = kMostRows;
    // Of many sequences some at a time: as many as a launch has workgroups for, or, where their contexts are split, as a workgroup lists.  us, a workgroup for each of 2100
    // contexts, 8 heads over one of 128 / parts of 4096 keys: up to 32768 keys, ragged 1410 / 1278, all as long 5035 / 4930, one long one among 1 to 500 keys 335 /
    // 125; up to 16384 694 / 725, 2518 / 2525, 179 / 120; 32 over 8 heads of 64, 4096 keys each (up to 32768, it was said) 2710 / 2775.  Parts of 1024 keys: up to 16384 668 / 641,
    // 2522 / 2707, up to 4096 182 / 226, 638 / 706.
    const int64_t units = paged_units(a) / a.n_seqs, listed = kCounters / units < kMostListed ? kCounters / units : kMostListed;
    const bool many = a.n_seqs > listed;
    int64_t most = many ? kMostWorkgroups / units : a.n_seqs;
    if (many && longest > kLongOfMany && parts_that_fit(workspace_bytes, listed * a.h.q_heads, a.h.head_dim) > 1) most = listed;
    most = (a.n_seqs + (a.n_seqs + most - 1) / most - 1) / ((a.n_seqs + most - 1) / most);
    hipError_t e = hipSuccess;
    for (int64_t first = 0; e == hipSuccess && first < args->n_seqs; first += most) {
        PagedArgs some = a;
        some.n_seqs = (int32_t)(args->n_seqs - first < most ? args->n_seqs - first : most);
        some.q.data += first * a.q.token;
        some.out.data += first * a.out.token;
        if (a.lse) some.lse += first * a.h.q_heads;
        some.table += first * a.table_stride;
        some.lens += first;
        e = paged_at_once(some, longest, many ? kMostPartKeysOfMany : kMostPartKeys, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
    }
    return status_of(e);
}

cf_status cf_attn_join(const cf_attn_desc *desc, const cf_join *args, void *stream)
{
    JoinArgs a = {};
    Span so;
    cf_status st = check_desc(desc, a.h);
    if (st != CF_OK) return st;
    if (!args || !args->parts || !args->lses) return CF_ERR_INVALID_ARG;
    if (args->part_dtype != CF_F32 && args->part_dtype != desc->dtype) return CF_ERR_UNSUPPORTED;
    if (args->n_parts < 1 || args->n_parts > CF_JOIN_MAX_PARTS || args->n_tokens < 0 || args->n_tokens > kMostRows / desc->q_heads) return CF_ERR_SHAPE;
    if (args->n_tokens == 0) return CF_OK;
    if ((st = check_rows(args->out, args->n_tokens, desc->q_heads, desc->head_dim, true, 0, a.out, so)) != CF_OK) return st;
    if (!aligned(args->lse, 4)) return CF_ERR_INVALID_ARG;
    a.n_rows = args->n_tokens * desc->q_heads;
    const int64_t width = (int64_t)desc->q_heads * desc->head_dim * (args->part_dtype == CF_F32 ? 4 : 2);
    for (int i = 0; i < args->n_parts; ++i) {
        if (!args->parts[i] || !aligned(args->parts[i], 16) || !args->lses[i] || !aligned(args->lses[i], 4)) return CF_ERR_INVALID_ARG;
        if (meet(so, {reinterpret_cast<uintptr_t>(args->parts[i]), 1, 0, 1, 0, args->n_tokens * width})) return CF_ERR_INVALID_ARG;
        if (args->lse && meet({reinterpret_cast<uintptr_t>(args->lse), 1, 0, 1, 0, a.n_rows * 4}, {reinterpret_cast<uintptr_t>(args->lses[i]), 1, 0, 1, 0, a.n_rows * 4})) return CF_ERR_INVALID_ARG;
        a.parts[i] = args->parts[i];
        a.lses[i] = args->lses[i];
    }
    a.lse = args->lse;
    a.n_parts = args->n_parts;
    a.part_dtype = args->part_dtype;
    if (join_workgroups(a) > kMostWorkgroups) return CF_ERR_SHAPE;
    return status_of(launch_join(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
