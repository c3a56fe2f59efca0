// Which pages of a context a head attends to: every page has a bound on what its keys may score, and the largest bounds win.
//
// sum over heads h and elements i of max(q_hi least_i, q_hi largest_i) = sum_i largest_i P_i + least_i N_i, where P sums the positive q_hi of the heads that share
// the keys and N the others: one product of 2 D numbers a page, whatever the number of heads.  Sums are of 64 bits, and exact but for numbers that
// lie more than 2^36 apart, so that ties are ties, whatever the order.  k_select_scores reads every bound once and is bound by HBM, or by its launch;
// k_select_pages finds the least score that is taken by its bits, 11 at a time, a workgroup a row, and writes the pages in order.
#include "cf_attn8_device.h"

namespace cf {
namespace attn {
namespace {

// Scores as whole numbers in the same order; NaN is the least.
__device__ __forceinline__ uint64_t ordered(double x)
{
    if (x != x) return 0;
    const uint64_t w = __builtin_bit_cast(uint64_t, x + 0.0);       // -0 is 0
    return w >> 63 ? ~w : w | (uint64_t)1 << 63;
}

__device__ __forceinline__ int pages_of(const SelectArgs &a, int64_t seq)
{
    const int64_t held = ((int64_t)max(gconst<int32_t>(a.lens)[seq], 0) + a.cache.page_size - 1) >> a.cache.page_shift;
    return (int)min(held, (int64_t)a.max_pages);
}

template <int DT, int D> __global__ __launch_bounds__(256) void k_select_scores(SelectArgs a)
{
    constexpr int kLanes = D / 4;               // of a page: 8 elements each, of the least ones, then of the largest
    constexpr int kPages = 64 / kLanes;         // of a wave's load
    constexpr int kRounds = kSelectPages / 4 / kPages;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = blockIdx.x / a.groups, group = blockIdx.x % a.groups;
    const int64_t seq = (a.first_row + row) / a.h.kv_heads;
    const int head = (int)((a.first_row + row) % a.h.kv_heads), held = pages_of(a, seq);
    if (held <= a.count || group * kSelectPages >= held) return;        // all of them are taken; none is left

    const int element = lane % (kLanes / 2) * 8;
    const bool largest = lane / (kLanes / 2) % 2;
    double q[8] = {};
    for (int h = 0; h < a.h.group; ++h) {
        const u32x4 x = *gconst<u32x4>(a.q.data + seq * a.q.token + (int64_t)(head * a.h.group + h) * a.q.head + element * 2);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float lo = Elem<DT>::lo(x[k]), hi = Elem<DT>::hi(x[k]);
            q[2 * k] += lo > 0.0f == largest || lo != lo ? (double)lo : 0.0;
            q[2 * k + 1] += hi > 0.0f == largest || hi != hi ? (double)hi : 0.0;
        }
    }
    for (int64_t first = group * kSelectPages + wave * (kSelectPages / 4); first < held; first += (int64_t)a.groups * kSelectPages) {
        const int entry = gconst<int32_t>(a.table)[seq * a.table_stride + min(first + lane % (kSelectPages / 4), (int64_t)held - 1)];
        const int page = min(max(entry, 0), a.cache.n_pages - 1);
        u32x4 x[kRounds];
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            const int64_t here = __shfl(page, i * kPages + lane / kLanes);
            x[i] = gconst<u32x4>(a.cache.bounds + (here * a.h.kv_heads + head) * 2 * D)[lane % kLanes];
        }
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            double sum = 0.0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                sum = __builtin_fma((double)Elem<BF16>::lo(x[i][k]), q[2 * k], sum);
                sum = __builtin_fma((double)Elem<BF16>::hi(x[i][k]), q[2 * k + 1], sum);
            }
#pragma unroll
            for (int d = 1; d < kLanes; d <<= 1) sum += __shfl_xor(sum, d);
            const int64_t j = first + i * kPages + lane / kLanes;
            if (lane % kLanes == 0 && j < held) gmut<uint64_t>(a.scores)[row * a.columns + j] = ordered(sum);
        }
    }
}

constexpr int kPickThreads = 1024, kPickWaves = kPickThreads / 64, kBins = 2048;

__global__ __launch_bounds__(kPickThreads) void k_select_pages(SelectArgs a)
{
    __shared__ uint32_t lds_bins[kBins];
    __shared__ uint64_t lds_least[kPickWaves], lds_largest[kPickWaves];
    __shared__ uint32_t lds_sums[kPickWaves], lds_ties[kPickWaves], lds_found[3];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = blockIdx.x, seq = (a.first_row + row) / a.h.kv_heads;
    const int held = pages_of(a, seq);
    CF_GLOBAL int32_t *out = gmut<int32_t>(a.blocks) + (a.first_row + row) * a.count;
    if (held <= a.count) {
        for (int j = threadIdx.x; j < a.count; j += kPickThreads) out[j] = j < held ? j : -1;
        return;
    }
    const CF_GLOBAL uint64_t *scores = gconst<uint64_t>(a.scores + row * a.columns);
    const int behind = held - a.recent;         // pages from `first` to here compete
    uint32_t rest = (uint32_t)(a.count - a.first - a.recent);
    uint64_t least = ~(uint64_t)0, largest = 0;
    if (rest > 0) {
        for (int j = a.first + threadIdx.x; j < behind; j += kPickThreads) {
            least = min(least, (uint64_t)scores[j]);
            largest = max(largest, (uint64_t)scores[j]);
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            least = min(least, (uint64_t)__shfl_xor((unsigned long long)least, d));
            largest = max(largest, (uint64_t)__shfl_xor((unsigned long long)largest, d));
        }
        if (lane == 0) lds_least[wave] = least, lds_largest[wave] = largest;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kPickWaves; ++w) {
            least = min(least, lds_least[w]);
            largest = max(largest, lds_largest[w]);
        }
    }

    // Scores past `least` are taken, and of those that equal it the first `rest`: all, if so many are.  The range that holds the one that decides is narrowed by 2^11 a time.
    uint64_t from = least;
    bool all = false;
    while (rest > 0) {
        const uint64_t range = largest - from;
        const int shift = range >> 11 ? 64 - 11 - __builtin_clzll(range) : 0;
        for (int i = threadIdx.x; i < kBins; i += kPickThreads) lds_bins[i] = 0;
        __syncthreads();
        for (int j = a.first + threadIdx.x; j < behind; j += kPickThreads) {
            const uint64_t x = scores[j];
            if (x >= from && x <= largest) atomicAdd(&lds_bins[(x - from) >> shift], 1u);
        }
        __syncthreads();
        // scores in this thread's two bins, and in all bins from there on
        const uint32_t low = lds_bins[2 * threadIdx.x], high = lds_bins[2 * threadIdx.x + 1];
        uint32_t upto = low + high;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t above = __shfl_down(upto, d);
            if (lane + d < 64) upto += above;
        }
        if (lane == 0) lds_sums[wave] = upto;
        __syncthreads();
        for (int w = wave + 1; w < kPickWaves; ++w) upto += lds_sums[w];
        const uint32_t from_high = upto - low, past = from_high - high;     // scores from the upper bin on, and past it
        if (past < rest && rest <= from_high) lds_found[0] = 2 * threadIdx.x + 1, lds_found[1] = past, lds_found[2] = high;
        if (from_high < rest && rest <= upto) lds_found[0] = 2 * threadIdx.x, lds_found[1] = from_high, lds_found[2] = low;
        __syncthreads();
        const uint64_t bin = lds_found[0];
        rest -= lds_found[1];
        all = lds_found[2] == rest;
        from += bin << shift;
        if (all || shift == 0) break;
        largest = min(largest, from + (((uint64_t)1 << shift) - 1));
        __syncthreads();
    }
    // -> a score is taken if it is past `from`, or if it equals it and is one of the first `rest`, or (all) if it is not less; nothing competes if rest was 0
    const bool some = a.count > a.first + a.recent;
    uint32_t taken = 0, ties = 0;
    for (int base = 0; base < held; base += kPickThreads) {
        const int j = base + threadIdx.x;
        const bool there = j < held, always = there && (j < a.first || j >= behind), competes = there && !always && some;
        const uint64_t x = competes ? (uint64_t)scores[j] : 0;
        const bool tie = competes && !all && x == from;
        const uint64_t tie_mask = __ballot(tie), before = ((uint64_t)1 << lane) - 1;
        __syncthreads();
        if (lane == 0) lds_ties[wave] = __builtin_popcountll(tie_mask);
        __syncthreads();
        uint32_t rank = ties + __builtin_popcountll(tie_mask & before);
        for (int w = 0; w < kPickWaves; ++w) {
            if (w < wave) rank += lds_ties[w];
            ties += lds_ties[w];
        }
        const bool take = always || (competes && (all ? x >= from : x > from || (tie && rank < rest)));
        const uint64_t mask = __ballot(take);
        if (lane == 0) lds_sums[wave] = __builtin_popcountll(mask);
        __syncthreads();
        uint32_t at = taken + __builtin_popcountll(mask & before);
        for (int w = 0; w < kPickWaves; ++w) {
            if (w < wave) at += lds_sums[w];
            taken += lds_sums[w];
        }
        if (take) out[at] = j;
    }
}

template <int DT> hipError_t scores_typed(const SelectArgs &a, hipStream_t s)
{
    const int64_t n = a.n_rows * a.groups;
    switch (a.h.head_dim) {
    case 64: return enqueue(k_select_scores<DT, 64>, n, s, a);
    case 128: return enqueue(k_select_scores<DT, 128>, n, s, a);
    default: return enqueue(k_select_scores<DT, 256>, n, s, a);
    }
}

}  // namespace

hipError_t launch_select(const SelectArgs &a, hipStream_t s)
{
    hipError_t e = hipSuccess;
    if (a.max_pages > a.count && a.count > a.first + a.recent) e = a.h.dtype == BF16 ? scores_typed<BF16>(a, s) : scores_typed<F16>(a, s);
    return e == hipSuccess ? enqueue_of<kPickThreads>(k_select_pages, a.n_rows, s, a) : e;
}

}  // namespace attn
}  // namespace cf
