// Which pages of a context a head attends to: every page has a bound on what its keys may score, and the largest bounds win.
//
// sum over heads h and elements i of max(q_hi least_i, q_hi largest_i) = sum_i largest_i P_i + least_i N_i, where P sums the positive q_hi of the heads that share
// the keys and N the others: one product of 2 D numbers a page, whatever the number of heads.  Sums are of 64 bits, and every page's in the same order, so that
// equal bounds have equal scores.  They are exact, and equal whatever the order, where what is summed spans 53 bits at most: 9 of 512 terms, 8 of a bound, 8 (fp16: 11) of a
// query and log2 of the heads that share keys leave 28 (25) powers of two, less that logarithm, between the largest and the least number of the queries and of the bounds together.  k_select_scores reads every bound once and is bound by HBM, or by its launch;
// k_select_pages finds the least score that is taken by its bits, 11 at a time, a workgroup a row, and writes the pages in order.  A thread has 8 neighbouring pages, whose
// scores stay in registers, and whose places follow from a sum over the threads.  us in a graph, both and the attention over what they select: 2048 pages for each of 8 heads 4.7 + 5.2 + 9.9,
// 24 contexts of 1 to 1875 pages 12.0 (3.6 TB/s) + 6.5 + 31.
#include "cf_attn8_device.h"

namespace cf {
namespace attn {
namespace {

__device__ __forceinline__ int pages_of(const SelectArgs &a, int64_t seq)
{
    const int64_t held = ((int64_t)max(gconst<int32_t>(a.lens)[seq], 0) + a.cache.page_size - 1) >> a.cache.page_shift;
    return (int)min(held, (int64_t)a.max_pages);
}

// Sums with the lane 32 (16) away: of x in the lower half (the even sixteens), of y in the other.
__device__ __forceinline__ double of_halves(double x, double y)
{
    const u32x2 a = __builtin_bit_cast(u32x2, x), b = __builtin_bit_cast(u32x2, y);
    const u32x2 low = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(a[0], b[0], false, false)), high = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(a[1], b[1], false, false));
    return __builtin_bit_cast(double, (u32x2){low[0], high[0]}) + __builtin_bit_cast(double, (u32x2){low[1], high[1]});
}
__device__ __forceinline__ double of_quarters(double x, double y)
{
    const u32x2 a = __builtin_bit_cast(u32x2, x), b = __builtin_bit_cast(u32x2, y);
    const u32x2 low = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false)), high = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false));
    return __builtin_bit_cast(double, (u32x2){low[0], high[0]}) + __builtin_bit_cast(double, (u32x2){low[1], high[1]});
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
    for (int h0 = 0; h0 < a.h.group; h0 += 4) {
        u32x4 x[4];
#pragma unroll
        for (int h = 0; h < 4; ++h)
            if (h0 + h < a.h.group) x[h] = *gconst<u32x4>(a.q.data + seq * a.q.token + (int64_t)(head * a.h.group + h0 + h) * a.q.head + element * 2);
#pragma unroll
        for (int h = 0; h < 4; ++h)
            if (h0 + h < a.h.group)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float lo = Elem<DT>::lo(x[h][k]), hi = Elem<DT>::hi(x[h][k]);
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
        double sum[kRounds];
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            sum[i] = 0.0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                sum[i] = __builtin_fma((double)Elem<BF16>::lo(x[i][k]), q[2 * k], sum[i]);
                sum[i] = __builtin_fma((double)Elem<BF16>::hi(x[i][k]), q[2 * k + 1], sum[i]);
            }
        }
        // Every exchange halves what a lane has, down to 4 sums of sixteen lanes: of rounds r, r + 4 in the odd sixteens, and r + 8, r + 12 in the upper half.
        if constexpr (kRounds == 16)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] = of_halves(sum[i], sum[i + 8]);
        if constexpr (kRounds >= 8)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = of_quarters(sum[i], sum[i + 4]);
        double mine = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            double t = sum[i];
            t += moved<0xb1>(t);
            t += moved<0x4e>(t);
            t += moved<0x141>(t);
            t += moved<0x140>(t);
            if ((lane & 3) == i) mine = t;
        }
        const int sixteen = lane >> 4, r = lane & 3;
        const int64_t j = first + (kRounds == 4 ? r * 4 + sixteen : kRounds == 8 ? (r + 4 * (sixteen & 1)) * 2 + (sixteen >> 1) : r + 4 * (sixteen & 1) + 8 * (sixteen >> 1));
        if ((lane & 15) < 4 && j < held) gmut<uint64_t>(a.scores)[row * a.columns + j] = ordered_score(mine);
    }
}

constexpr int kBins = kScoreBins, kEach = 8;      // pages of a thread

template <int THREADS> __global__ __launch_bounds__(THREADS) void k_select_pages(SelectArgs a)
{
    constexpr int kWavesHere = THREADS / 64, kOwnBins = kBins / THREADS;
    __shared__ uint32_t lds_bins[kBins];
    __shared__ uint32_t lds_least[kWavesHere], lds_largest[kWavesHere], lds_sums[2][kWavesHere], lds_found[3];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = blockIdx.x, seq = (a.first_row + row) / a.h.kv_heads;
    const int held = pages_of(a, seq);
    CF_GLOBAL int32_t *out = gmut<int32_t>(a.blocks) + (a.first_row + row) * a.count;
    if (held <= a.count) {
        for (int j = threadIdx.x; j < a.count; j += THREADS) out[j] = j < held ? j : -1;
        return;
    }
    const CF_GLOBAL uint64_t *scores = gconst<uint64_t>(a.scores + row * a.columns);
    const int behind = held - a.recent;         // pages from `first` to here compete
    const bool some = a.count > a.first + a.recent;
    uint64_t x[kEach];                          // scores of pages base + kEach * threadIdx.x .., 0 where they do not compete
    auto read = [&](int base) {
        const int j = base + kEach * threadIdx.x;
#pragma unroll
        for (int k = 0; k < kEach; ++k) x[k] = some && j + k >= a.first && j + k < behind ? scores[j + k] : 0;
    };
    auto competes = [&](int base, int k) {
        const int j = base + kEach * (int)threadIdx.x + k;
        return some && j >= a.first && j < behind;
    };
    constexpr int kTurn = THREADS * kEach;
    const bool once = held <= kTurn;            // they stay in registers
    read(0);

    // -> how many of the threads before this one, and in all
    int turn = 0;
    auto upto = [&](uint32_t mine, uint32_t &all) {
        const uint32_t s = sums(mine);
        if (lane == 63) lds_sums[turn & 1][wave] = s;
        __syncthreads();
        const uint32_t w = sums_of_sixteen((lane & 15) < kWavesHere ? lds_sums[turn & 1][min(lane & 15, kWavesHere - 1)] : 0);
        all = __builtin_amdgcn_readlane(w, 15);
        ++turn;
        return s - mine + (wave > 0 ? __builtin_amdgcn_readlane(w, wave - 1) : 0);
    };

    // Scores past `from` are taken, and of those that equal it the first `rest`: all, if so many are.  The range that holds the one that decides is narrowed by 2^11 a time; there are
    // `rest` scores in it at least, and one at least to be taken.
    ScoreRange range = {};
    uint32_t rest = (uint32_t)(a.count - a.first - a.recent);
    bool all = false;
    if (some) {
        uint32_t least = ~0u, largest = 0;      // by their upper halves
        for (int base = 0; base < behind; base += kTurn) {
            if (base > 0) read(base);
#pragma unroll
            for (int k = 0; k < kEach; ++k) {
                const uint32_t high = (uint32_t)(x[k] >> 32);
                if (competes(base, k)) least = min(least, high);
                largest = max(largest, high);
            }
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) least = min(least, __shfl_xor(least, d)), largest = max(largest, __shfl_xor(largest, d));
        if (lane == 0) lds_least[wave] = least, lds_largest[wave] = largest;
        for (int i = threadIdx.x; i < kBins; i += THREADS) lds_bins[i] = 0;
        __syncthreads();
        for (int w = 0; w < kWavesHere; ++w) least = min(least, lds_least[w]), largest = max(largest, lds_largest[w]);
        range = {(uint64_t)least << 32, (uint64_t)largest << 32 | ~0u};
        for (;;) {
            const int shift = range.shift();
            for (int base = 0; base < behind; base += kTurn) {
                if (!once) read(base);
#pragma unroll
                for (int k = 0; k < kEach; ++k)
                    if (competes(base, k) && range.holds(x[k])) atomicAdd(&lds_bins[(x[k] - range.from) >> shift], 1u);
            }
            __syncthreads();
            // scores in this thread's bins, and in all bins past them
            uint32_t bin[kOwnBins], mine = 0, total;
#pragma unroll
            for (int k = 0; k < kOwnBins; ++k) {
                bin[k] = lds_bins[kOwnBins * threadIdx.x + k];
                lds_bins[kOwnBins * threadIdx.x + k] = 0;
                mine += bin[k];
            }
            const uint32_t below = upto(mine, total);
            uint32_t past = total - below - mine;
#pragma unroll
            for (int k = kOwnBins - 1; k >= 0; --k) {
                if (past < rest && rest <= past + bin[k]) lds_found[0] = kOwnBins * threadIdx.x + k, lds_found[1] = past, lds_found[2] = bin[k];
                past += bin[k];
            }
            __syncthreads();
            rest -= lds_found[1];
            all = lds_found[2] == rest;
            range = range.bin(lds_found[0], shift);
            if (all || shift == 0) break;
            __syncthreads();
        }
    }
    const uint64_t from = range.from;
    // -> a page is taken if its score is past `from`, or if it equals it and is one of the first `rest`, or (all) if it is not less; and if it does not compete
    uint32_t taken = 0, ties = 0;
    for (int base = 0; base < held; base += kTurn) {
        if (!once) read(base);
        const int j = base + kEach * threadIdx.x;
        uint32_t tie = 0, take = 0;
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            if (competes(base, k)) {
                if (all ? x[k] >= from : x[k] > from) take |= 1u << k;
                else if (!all && x[k] == from) tie |= 1u << k;
            } else if (j + k < held && (j + k < a.first || j + k >= behind)) take |= 1u << k;
        }
        if (some && !all) {
            uint32_t in_all;
            uint32_t rank = ties + upto(__builtin_popcount(tie), in_all);
            for (; tie != 0; tie &= tie - 1, ++rank)
                if (rank < rest) take |= tie & -tie;
            ties += in_all;
        }
        uint32_t in_all;
        uint32_t at = taken + upto(__builtin_popcount(take), in_all);
        taken += in_all;
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            if (take >> k & 1) {
                if (at < (uint32_t)a.count) out[at] = j + k;      // as many as are taken; whatever the scores, nothing goes into another row
                ++at;
            }
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
    if (e != hipSuccess) return e;
    // By what the scores of a row may be, for which the table's width speaks (the hint of the longest context may be wrong): 256 threads that have all of them in registers, or four times as
    // many, which read them less often.  us of both kernels in a graph, 8 heads of 128, 256 / 1024 threads: 2048 pages 16.8 / 18.9, 24 contexts of 900 28 / 30, of 200 in a table of 8192
    // 46 / 48; 4096 pages 29 / 20, 8192 49 / 26.
    return a.max_pages <= 256 * kEach ? enqueue_of<256>(k_select_pages<256>, a.n_rows, s, a) : enqueue_of<1024>(k_select_pages<1024>, a.n_rows, s, a);
}

}  // namespace attn
}  // namespace cf
