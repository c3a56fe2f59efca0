// A step's positions and slots from the sequences' lengths, and the pages that they take and give back.
//
// Three running sums over the sequences (tokens, pages needed, pages given back) say where everything goes.  They are short: every workgroup computes them
// all, 1024 sequences at a time, and then looks up its share of the tokens in them.  Lengths and the ring's state may be updated in place: the workgroup that
// is done last writes them, when all others have read them.  Bound by its launch and a chain of latencies: what it reads and writes is some 100 kB.
#include "cf_attn8.h"
#include "cf_attn_device.h"

namespace cf {
namespace attn {
namespace {

constexpr int kWavesHere = kPlanThreads / 64;

__global__ __launch_bounds__(kPlanThreads) void k_kv_plan(PlanArgs a)
{
    __shared__ int64_t lds_waves[kWavesHere][4];
    __shared__ int32_t lds_upto[kPlanThreads];          // tokens of the sequences up to each, of all; past n_tokens: n_tokens
    __shared__ int32_t lds_back[kPlanThreads];          // pages that those up to each give back, of these 1024
    __shared__ int32_t lds_len[kPlanThreads];           // tokens held, -1: not served
    __shared__ int32_t lds_fresh[kPlanThreads];         // where in the ring the new pages begin
    __shared__ uint32_t lds_count;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int page_size = 1 << a.page_shift;
    const int64_t capacity = min((int64_t)a.max_pages << a.page_shift, (int64_t)INT32_MAX);
    const int64_t taken = max((int64_t)gconst<int64_t>(a.state)[0], (int64_t)0), put = max((int64_t)gconst<int64_t>(a.state)[1], taken);
    const int64_t free_pages = min(put - taken, (int64_t)a.n_ring);
    auto pages_in = [&](int64_t tokens) { return (tokens + page_size - 1) >> a.page_shift; };

    struct Totals {
        int64_t tokens, needed, used, back;
        int32_t refused;
    };
    // One more chunk of sequences.  -> this thread's one, and the totals with it; the tables in LDS are of this chunk.
    struct Mine {
        int32_t len, now;               // as given, and after the call
        int64_t begin;
    };
    auto scan = [&](int base, Totals &t, bool tables) {
        const int b = base + threadIdx.x;
        Mine mine = {0, 0, 0};
        int32_t news = 0;
        if (b < a.n_seqs) mine.len = gconst<int32_t>(a.lens)[b], news = gconst<int32_t>(a.news)[b];
        const bool ended = news < 0, sane = mine.len >= 0 && mine.len <= capacity;
        const int64_t len = sane ? mine.len : 0, n = max(news, 0), held = pages_in(len);
        const int64_t need = !ended && sane && len + n <= capacity ? pages_in(len + n) - held : 0, back = ended ? held : 0;
        int64_t sums[3] = {n, need, back};
#pragma unroll
        for (int d = 1; d < 64; d <<= 1)
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                const int64_t below = __shfl_up((long long)sums[k], d);
                if (lane >= d) sums[k] += below;
            }
        __syncthreads();
        if (lane == 63)
#pragma unroll
            for (int k = 0; k < 3; ++k) lds_waves[wave][k] = sums[k];
        __syncthreads();
        int64_t all[3] = {t.tokens, t.needed, 0}, own[3] = {sums[0] + t.tokens, sums[1] + t.needed, sums[2]};
        for (int w = 0; w < kWavesHere; ++w)
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                const int64_t x = lds_waves[w][k];
                all[k] += x;
                if (w < wave) own[k] += x;
            }
        const bool fits = !ended && sane && len + n <= capacity && own[0] <= a.n_tokens;
        const bool served = fits && (need == 0 || own[1] <= free_pages);
        int64_t used = served ? need : 0;
        int32_t refused = !ended && !served && n > 0;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            used += __shfl_xor((long long)used, d);
            refused += __shfl_xor(refused, d);
        }
        if (lane == 0) lds_waves[wave][3] = used << 11 | refused;       // 64 of them at most
        if (tables) {
            lds_upto[threadIdx.x] = (int32_t)min(own[0], (int64_t)a.n_tokens);
            lds_back[threadIdx.x] = (int32_t)min(own[2], (int64_t)INT32_MAX);
            lds_len[threadIdx.x] = served ? (int32_t)len : -1;
            lds_fresh[threadIdx.x] = served && need > 0 ? (int32_t)((taken + own[1] - need) % a.n_ring) : 0;
        }
        mine.begin = own[0] - n;
        mine.now = ended ? 0 : served ? (int32_t)(len + n) : mine.len;
        __syncthreads();
        for (int w = 0; w < kWavesHere; ++w) {
            t.used += lds_waves[w][3] >> 11;
            t.refused += (int32_t)(lds_waves[w][3] & 2047);
        }
        t.tokens = all[0], t.needed = all[1], t.back = all[2];
        return mine;
    };
    // the first of this chunk's sequences with more up to it than x
    auto find = [&](const int32_t *upto, int x) {
        int first = 0, last = kPlanThreads - 1;
        while (first < last) {
            const int middle = (first + last) >> 1;
            if (upto[middle] > x) last = middle;
            else first = middle + 1;
        }
        return first;
    };
    auto write_totals = [&](const Totals &t, int64_t back) {
        if (threadIdx.x > 0) return;
        gmut<int64_t>(a.state_out)[0] = taken + t.used;
        gmut<int64_t>(a.state_out)[1] = put + back;
        gmut<int32_t>(a.refused)[0] = t.refused;
    };

    const bool alone = a.workgroups == 1;
    Totals t = {};
    int64_t back = 0;
    for (int base = 0; base < a.n_seqs; base += kPlanThreads) {
        const int64_t before = min(t.tokens, (int64_t)a.n_tokens);
        const Mine mine = scan(base, t, true);
        const int b = base + threadIdx.x;
        if (b < a.n_seqs) {
            if (base / kPlanThreads % a.workgroups == (int)blockIdx.x) gmut<int32_t>(a.cu)[b] = (int32_t)min(mine.begin, (int64_t)a.n_tokens);
            if (alone) gmut<int32_t>(a.lens_out)[b] = mine.now;
        }
        // tokens, 1024 at a time in turn
        const int64_t end = min(t.tokens, (int64_t)a.n_tokens);
        int64_t stripe = before / kPlanThreads;
        stripe += ((int64_t)blockIdx.x - stripe % a.workgroups + a.workgroups) % a.workgroups;
        for (; stripe * kPlanThreads < end; stripe += a.workgroups) {
            const int64_t row = stripe * kPlanThreads + threadIdx.x;
            if (row < before || row >= end) continue;
            const int i = find(lds_upto, (int)row), len = lds_len[i];
            int64_t slot = -1;
            int32_t pos = -1;
            if (len >= 0) {
                pos = len + (int32_t)(row - (i > 0 ? lds_upto[i - 1] : before));
                const int index = pos >> a.page_shift, held = (int)pages_in(len);
                CF_GLOBAL int32_t *entry = gmut<int32_t>(a.table) + (base + i) * a.table_stride + index;
                int32_t page;
                if (index < held) page = *entry;
                else {
                    int64_t at = (int64_t)lds_fresh[i] + (index - held);        // fewer than n_ring of them
                    if (at >= a.n_ring) at -= a.n_ring;
                    page = gconst<int32_t>(a.ring)[at];
                    if ((pos & (page_size - 1)) == 0) *entry = page;
                }
                slot = ((int64_t)page << a.page_shift) + (pos & (page_size - 1));
            }
            gmut<int64_t>(a.slots)[row] = slot;
            gmut<int32_t>(a.positions)[row] = pos;
        }
        // pages that come back
        const int64_t room = a.n_ring - (put - taken) - back, here = min(t.back, (int64_t)INT32_MAX);
        const int64_t behind = (put + back) % a.n_ring;
        for (int64_t i = (int64_t)blockIdx.x * kPlanThreads + threadIdx.x; i < min(here, room); i += (int64_t)a.workgroups * kPlanThreads) {
            const int s = find(lds_back, (int)i);
            const int32_t page = gconst<int32_t>(a.table)[(base + s) * a.table_stride + (i - (s > 0 ? lds_back[s - 1] : 0))];
            gmut<int32_t>(a.ring)[(behind + i) % a.n_ring] = page;
        }
        back += min(here, max(room, (int64_t)0));
        __syncthreads();
    }
    // rows behind the last token
    const int64_t total = min(t.tokens, (int64_t)a.n_tokens);
    for (int64_t row = total + (int64_t)blockIdx.x * kPlanThreads + threadIdx.x; row < a.n_tokens; row += (int64_t)a.workgroups * kPlanThreads) {
        gmut<int64_t>(a.slots)[row] = -1;
        gmut<int32_t>(a.positions)[row] = -1;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) gmut<int32_t>(a.cu)[a.n_seqs] = (int32_t)total;
    __syncthreads();
    if (alone) return write_totals(t, back);

    // The last workgroup updates what the others read.  A workgroup's loads have returned when it is counted: their values were used.
    if (threadIdx.x == 0) lds_count = __hip_atomic_fetch_add((CF_GLOBAL uint32_t *)a.counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (lds_count != (uint32_t)a.workgroups - 1) return;
    if (threadIdx.x == 0) __hip_atomic_store((CF_GLOBAL uint32_t *)a.counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    Totals again = {};
    for (int base = 0; base < a.n_seqs; base += kPlanThreads) {
        const Mine mine = scan(base, again, false);
        if (base + (int)threadIdx.x < a.n_seqs) gmut<int32_t>(a.lens_out)[base + threadIdx.x] = mine.now;
    }
    write_totals(t, back);
}

}  // namespace

hipError_t launch_plan(const PlanArgs &a, hipStream_t s) { return enqueue_of<kPlanThreads>(k_kv_plan, a.workgroups, s, a); }

}  // namespace attn
}  // namespace cf
