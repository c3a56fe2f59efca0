// Internal interface between the host half of the attention entry points (cf_attn_api.cpp) and their
// kernels (cf_attn_prompt.hip, cf_attn_paged.hip, cf_attn_rows.hip).  Not installed; not part of the ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cf {
namespace attn {

// Strides in bytes from here on.
struct Rows {
    char *data;
    int64_t token, head;
};

struct Heads {
    int32_t dtype;                  // cf_dtype
    int32_t q_heads, kv_heads, group, head_dim;
    float scale_log2;               // scale * log2(e): the kernels' exponentials are powers of two
};

struct Cache {
    char *k, *v;
    int64_t page_bytes;             // from page to page
    int32_t n_pages, page_size, page_shift;
};

// Parts of the keys that were attended apart: part s of row (t, h) is o[(s * n_rows + t * q_heads + h) * head_dim],
// fp32 and normalised, with its natural log-sum-exp in lse[s * n_rows + ...].
struct Parts {
    float *o, *lse;
    int64_t n_rows;                 // tokens * q_heads
};

constexpr int kPromptRows = 128;    // query rows (token, head of the group) of a workgroup
constexpr int kPagedHeads = 16;     // query heads of a workgroup: the columns of a 16 x 16 product
constexpr int kMostListed = 2048;   // sequences whose parts a workgroup lists
constexpr int kMaxParts = 64;       // CF_JOIN_MAX_PARTS

struct PromptArgs {
    Heads h;
    Rows q, k, v, out;
    float *lse;
    const int32_t *cu_q, *cu_k;
    int32_t n_seqs, n_q, n_k, causal;
    int32_t n_splits, split_keys;   // split s has the keys [s * split_keys, (s + 1) * split_keys) of a sequence, the last one all the rest
    Parts parts;                    // of n_splits > 1
};

struct PagedArgs {
    Heads h;
    Cache cache;
    Rows q, out;
    float *lse;
    const int32_t *table, *lens;
    int64_t table_stride;
    int32_t n_seqs, max_pages;      // of one launch: some of a call's sequences where there are many
    int32_t n_splits, split_keys;
    int32_t many;                   // parts are listed and taken in turn, and joined by a kernel of its own: where there are more than four a CU, or contexts that may differ
                                    // could fill 128 MB
    uint32_t *counters;             // one for every (sequence, unit of heads): parts that have landed; zero between calls
    Parts parts;                    // its log-sum-exps are of powers of two unless `many`
};

struct JoinArgs {
    Heads h;
    Rows out;
    float *lse;
    int64_t n_rows;                 // tokens * q_heads
    int32_t n_parts;
    int32_t part_dtype;             // cf_dtype
    const int32_t *cover;           // if set, only the tokens from cover[0] to cover[n_cover] are joined
    int32_t n_cover;
    const int32_t *lens;            // if set, token t has max(1, min(ceil(lens[t] / split_keys), n_parts)) parts, and one of one part is done already
    int32_t split_keys;
    const void *parts[kMaxParts];
    const float *lses[kMaxParts];
};

struct AppendArgs {
    Heads h;
    Cache cache;
    Rows k, v, q, q_out;            // q.data null: none
    const int64_t *slots;
    const int32_t *positions;
    const float *cos, *sin;
    int64_t n_tokens;
    int32_t n_positions, rotary_dim, interleaved;
};

// Workgroups of 256 threads that a call launches.  A launch counts its work-items with 32 bits.
constexpr int64_t kMostWorkgroups = (((int64_t)1 << 32) - 1) / 256;

inline int64_t prompt_tiles(const PromptArgs &a) { return ((int64_t)a.n_q * a.h.group + kPromptRows - 1) / kPromptRows + a.n_seqs; }      // at most: a part of one for every sequence
inline int64_t prompt_workgroups(const PromptArgs &a) { return prompt_tiles(a) * a.h.kv_heads * a.n_splits; }

inline int64_t paged_units(const PagedArgs &a) { return a.n_seqs * (int64_t)a.h.kv_heads * ((a.h.group + kPagedHeads - 1) / kPagedHeads); }
inline int64_t paged_workgroups(const PagedArgs &a)
{
    const int64_t items = paged_units(a) * a.n_splits, held = 256 * (a.h.head_dim == 64 ? 4 : a.h.head_dim == 128 ? 3 : 2);
    return a.many && held < items ? held : items;
}

// Lanes that share 8 elements of a row.  Up to 8 parts a lane each alone: lanes that meet cost a row more than loads in a row do (us: 12 parts of 98304 rows of 128 bf16,
// spread over 4 / 16 lanes 76 / 141; 6 of 10656 rows of 256 floats, over 1 / 8 lanes 12.7 / 24.8).  Past that a lane's loads are too many (48 parts, over 4 / 16 lanes
// 118 / 76), and many parts are of few rows: the lanes of a whole workgroup fill the device.
constexpr int join_spread(int n_parts, int dim) { return n_parts <= 8 ? 1 : n_parts <= 16 ? 4 : 256 / (dim / 8); }
inline int64_t join_workgroups(const JoinArgs &a)
{
    const int rows = 256 / (a.h.head_dim / 8 * join_spread(a.n_parts, a.h.head_dim));
    return (a.n_rows + rows - 1) / rows;
}

inline int64_t append_workgroups(const AppendArgs &a)
{
    const int64_t rows = (a.q.data ? a.h.q_heads : 0) + 2 * (int64_t)a.h.kv_heads;
    return (a.n_tokens * rows * (a.h.head_dim / 16) + 255) / 256;
}

hipError_t launch_prompt(const PromptArgs &a, hipStream_t s);
hipError_t launch_paged(const PagedArgs &a, hipStream_t s);
hipError_t launch_join(const JoinArgs &a, hipStream_t s);
hipError_t launch_append(const AppendArgs &a, hipStream_t s);

}  // namespace attn
}  // namespace cf
