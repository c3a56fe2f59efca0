// Internal interface between the host half of the entry points for the cache in 8 bits (cf_attn8_api.cpp) and their
// kernels (cf_attn8_paged.hip, cf_attn8_append.hip, cf_attn8_select.hip, cf_attn8_plan.hip).  Not installed; not part of the ABI.
#pragma once

#include "cf_attn.h"

namespace cf {
namespace attn {

struct Cache8 {
    char *k, *v;
    float *k_scale, *v_scale;       // [n_pages][kv_heads]
    uint16_t *bounds;               // [n_pages][kv_heads][2][head_dim] or null
    int64_t page_bytes;             // from page to page
    int32_t n_pages, page_size, page_shift;
};

struct Paged8Args {
    PagedArgs p;                    // its cache is not used
    Cache8 cache;
    const int32_t *blocks;          // [n_seqs][kv_heads][count], or null: all pages of a context, in order
    int32_t count;
};

struct Append8Args {
    Heads h;
    Cache8 cache;
    Rows k, v, q, q_out;            // q.data null: none
    const int64_t *slots;
    const int32_t *positions;
    const float *cos, *sin;
    int64_t n_tokens;
    int32_t n_positions, rotary_dim, interleaved;
    int32_t chunk;                  // tokens whose pages a workgroup takes, 64 at most
    int32_t chunks_each;            // that an XCD has
    int32_t page_groups;            // workgroups that store keys and values, a multiple of kXcds; those behind them rotate queries
};

struct SelectArgs {
    Heads h;
    Cache8 cache;
    Rows q;
    const int32_t *table, *lens;
    int64_t table_stride;
    int32_t n_seqs, max_pages;
    int32_t count, first, recent;
    int32_t *blocks;
    uint64_t *scores;               // [rows of a launch][columns]
    int64_t first_row, n_rows;      // (sequence, head of keys) rows of a launch
    int32_t columns;                // pages of the longest context that there may be
    int32_t groups;                 // workgroups that score a row's pages
};

struct PlanArgs {
    const int32_t *lens, *news;
    int32_t *table, *ring;
    const int64_t *state;
    int64_t *state_out;
    int32_t *lens_out, *cu, *positions, *refused;
    int64_t *slots;
    uint32_t *counter;              // zero between calls; of more than one workgroup
    int64_t table_stride;
    int32_t n_seqs, page_shift, max_pages, n_ring, n_tokens;
    int32_t workgroups;
    int32_t wide;                   // of kPlanThreads, else of a quarter
};

constexpr int kHeldWorkgroups = 2;  // of the attention's, a CU
constexpr int kXcds = 8;             // which take the workgroups in turn
constexpr int kSelectPages = 64;    // that a workgroup of the scores takes
constexpr int kAppendThreads = 256, kAppendTurns = 4;    // a lane rotates its part of so many heads' queries
constexpr int kPlanThreads = 1024;

// Scores as whole numbers in the same order; NaN is the least.
__host__ __device__ inline uint64_t ordered_score(double x)
{
    if (x != x) return 0;
    const uint64_t w = __builtin_bit_cast(uint64_t, x + 0.0);       // -0 is 0
    return w >> 63 ? ~w : w | (uint64_t)1 << 63;
}

// The scores from `from` to `end`, both among them, among which the least one that is taken is looked for, in kScoreBins bins of 2^shift.
constexpr int kScoreBits = 11, kScoreBins = 1 << kScoreBits;
struct ScoreRange {
    uint64_t from, end;
    __host__ __device__ int shift() const { return (end - from) >> kScoreBits ? 64 - kScoreBits - __builtin_clzll(end - from) : 0; }
    __host__ __device__ bool holds(uint64_t x) const { return x >= from && x <= end; }
    // One of the bins that hold scores.  The last one is cut off at `end`: it may reach past the largest number there is (infinity lies 2^52 below that, bins are up to 2^53 wide).
    __host__ __device__ ScoreRange bin(uint32_t i, int shift) const
    {
        const uint64_t at = from + ((uint64_t)i << shift), behind = ((uint64_t)1 << shift) - 1;
        return {at, end - at < behind ? end : at + behind};
    }
};

// Where workgroups have shares of all contexts (p.many): as many as the device holds at a time.
inline int64_t paged8_workgroups(const Paged8Args &a)
{
    if (!a.p.many) return paged_units(a.p) * a.p.n_splits;
    const int64_t units = paged_units(a.p) / a.p.n_seqs, held = 256 * kHeldWorkgroups;
    return units * (held > units ? held / units : 1);
}

inline int64_t append8_workgroups(const Append8Args &a)
{
    const int64_t lanes = a.q.data ? a.n_tokens * ((a.h.q_heads + kAppendTurns - 1) / kAppendTurns) * (a.h.head_dim / 16) : 0;
    return a.page_groups + (lanes + kAppendThreads - 1) / kAppendThreads;
}

hipError_t launch_paged8(const Paged8Args &a, hipStream_t s);
hipError_t launch_append8(const Append8Args &a, hipStream_t s);
hipError_t launch_select(const SelectArgs &a, hipStream_t s);
hipError_t launch_plan(const PlanArgs &a, hipStream_t s);

}  // namespace attn
}  // namespace cf
