// A step's positions and slots from the sequences' lengths, and the pages that they take and give back.
//
// Three running sums over the sequences (tokens, pages needed, pages given back) say where everything goes.  They are short: every workgroup computes them
// all, as many sequences at a time as it has threads, and then looks up its share of the tokens in them.  Sums are of 32 bits and stay at the largest number: what passes n_tokens or
// the free pages is not served, by how much it passes them does not matter.  Lengths and the ring's state may be updated in place: the workgroup that
// is done last writes them, when all others have read them.  Bound by its launch and a chain of latencies (what it reads and writes is some 100 kB), and by the number of
// instructions, on the few CUs that it runs on: sums by moves between lanes, no 64-bit division (us in a graph: 48 sequences of a token 4.1, 14 prompts of 2768 tokens 5.4, 1500 sequences
// of 36579 11.9; with sums of 64 bits through LDS 11.6, 18.4, 34.3).
#include "cf_attn8_device.h"

namespace cf {
namespace attn {
namespace {

// x % n for 0 <= x < 2^53; some number below n otherwise.
__device__ __forceinline__ uint32_t modulo(int64_t x, uint32_t n)
{
    int64_t r = x - (int64_t)__builtin_floor((double)x / (double)n) * n;
    r += r < 0 ? n : 0;
    return (uint32_t)min(max(r >= n ? r - n : r, (int64_t)0), (int64_t)n - 1);
}

template <int THREADS> __global__ __launch_bounds__(THREADS) void k_kv_plan(PlanArgs a)
{
    constexpr int kWavesHere = THREADS / 64;
    __shared__ uint32_t lds_waves[2][3][16];
    __shared__ uint32_t lds_upto[THREADS];              // tokens of the sequences up to each
    __shared__ uint32_t lds_back[THREADS];              // pages that those up to each give back, of these
    __shared__ int32_t lds_len[THREADS];                // tokens held, -1: not served
    __shared__ uint32_t lds_fresh[THREADS];             // where in the ring the new pages begin
    __shared__ uint32_t lds_used[kWavesHere], lds_refused[kWavesHere], lds_count;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int shift = a.page_shift, mask = (1 << shift) - 1;
    const uint32_t n_tokens = a.n_tokens, n_ring = a.n_ring;
    const int64_t capacity = min((int64_t)a.max_pages << shift, (int64_t)INT32_MAX);
    int32_t next_len = 0, next_news = 0;
    auto ask = [&](int64_t base) {
        const int64_t b = base + threadIdx.x;
        next_len = b < a.n_seqs ? gconst<int32_t>(a.lens)[b] : 0, next_news = b < a.n_seqs ? gconst<int32_t>(a.news)[b] : 0;
    };
    ask(0);
    const int64_t taken = max((int64_t)gconst<int64_t>(a.state)[0], (int64_t)0), put = max((int64_t)gconst<int64_t>(a.state)[1], taken);
    const uint32_t free_pages = (uint32_t)min(put - taken, (int64_t)n_ring);
    const uint32_t fresh0 = modulo(taken, n_ring);
    auto wrapped = [&](uint32_t at) { return at >= n_ring ? at - n_ring : at; };        // of what is below twice as much

    struct Totals {
        uint32_t tokens, needed, used, refused;     // the last two are this wave's
    };
    struct Mine {                                   // this thread's sequence: its length after the call, and where its tokens begin
        int32_t now;
        uint32_t begin;
    };
    // THREADS more sequences.  -> pages that they give back; the tables in LDS are of these.
    auto scan = [&](int64_t base, Totals &t, Mine &mine, int turn) {
        const int32_t len_given = next_len, news = next_news;
        if (base + THREADS < a.n_seqs) ask(base + THREADS);
        const bool ended = news < 0, sane = len_given >= 0 && len_given <= capacity;
        const int32_t len = sane ? len_given : 0;
        const uint32_t n = ended ? 0 : news, held = ((uint32_t)len + mask) >> shift, total = (uint32_t)len + n;
        const bool room = !ended && sane && total <= (uint64_t)capacity;
        const uint32_t need = room ? ((total + mask) >> shift) - held : 0, back = ended ? held : 0;
        const uint32_t s0 = sums(n), s1 = sums(need), s2 = sums(back);
        if (lane == 63) lds_waves[turn & 1][0][wave] = s0, lds_waves[turn & 1][1][wave] = s1, lds_waves[turn & 1][2][wave] = s2;
        __syncthreads();
        const int w = min(lane & 15, kWavesHere - 1);       // every sixteen lanes sum up the waves
        uint32_t own[3] = {add(s0, t.tokens), add(s1, t.needed), s2}, all[3] = {t.tokens, t.needed, 0};
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const uint32_t x = sums_of_sixteen((lane & 15) < kWavesHere ? lds_waves[turn & 1][k][w] : 0);
            if (wave > 0) own[k] = add(own[k], __builtin_amdgcn_readlane(x, wave - 1));
            all[k] = add(all[k], __builtin_amdgcn_readlane(x, 15));
        }
        const bool served = room && own[0] <= n_tokens && (need == 0 || own[1] <= free_pages);
        // pages are used by those up to the last one that is served and needs some
        const uint64_t users = __ballot(served && need > 0);
        if (users) t.used = __builtin_amdgcn_readlane(own[1], 63 - __builtin_clzll(users));
        t.refused += __builtin_popcountll(__ballot(!ended && !served && n > 0));
        lds_upto[threadIdx.x] = min(own[0], n_tokens);
        lds_back[threadIdx.x] = own[2];
        lds_len[threadIdx.x] = served ? len : -1;
        lds_fresh[threadIdx.x] = served && need > 0 ? wrapped(fresh0 + (own[1] - need)) : 0;
        t.tokens = all[0], t.needed = all[1];
        mine.now = ended ? 0 : served ? (int32_t)total : len_given;
        mine.begin = own[0] - n;                    // of no use where the sum has stayed at the largest number: that is past n_tokens
        if (own[0] > n_tokens) mine.begin = min(mine.begin, n_tokens);
        __syncthreads();
        return all[2];
    };

    const bool alone = a.workgroups == 1;
    Totals t = {};
    Mine mine = {};
    uint32_t back = 0;
    const uint32_t room = n_ring - free_pages;          // for pages that come back
    int turn = 0;
    for (int64_t base = 0; base < a.n_seqs; base += THREADS, ++turn) {
        const uint32_t before = min(t.tokens, n_tokens);
        const uint32_t here = scan(base, t, mine, turn);
        const int64_t b = base + threadIdx.x;
        const int some = (int)min((int64_t)THREADS, a.n_seqs - base);
        if (b < a.n_seqs) {
            if (turn % a.workgroups == (int)blockIdx.x) gmut<int32_t>(a.cu)[b] = (int32_t)min(mine.begin, n_tokens);
            if (alone) gmut<int32_t>(a.lens_out)[b] = mine.now;
        }
        // the first of these sequences with more up to it than x
        auto find = [&](const uint32_t *upto, uint32_t x) {
            int first = 0, last = some - 1;
            while (first < last) {
                const int middle = (first + last) >> 1;
                if (upto[middle] > x) last = middle;
                else first = middle + 1;
            }
            return first;
        };
        // tokens, THREADS at a time in turn
        const uint32_t end = min(t.tokens, n_tokens);
        uint32_t stripe = before / THREADS;
        stripe += (blockIdx.x + a.workgroups - stripe % a.workgroups) % a.workgroups;
        for (; stripe * THREADS < end; stripe += a.workgroups) {
            const uint32_t row = stripe * THREADS + threadIdx.x;
            if (row < before || row >= end) continue;
            const int i = find(lds_upto, row), len = lds_len[i];
            int64_t slot = -1;
            int32_t pos = -1;
            if (len >= 0) {
                pos = len + (int32_t)(row - (i > 0 ? lds_upto[i - 1] : before));
                const uint32_t index = pos >> shift, held = ((uint32_t)len + mask) >> shift;
                CF_GLOBAL int32_t *entry = gmut<int32_t>(a.table) + (base + i) * a.table_stride + index;
                const int64_t page = index < held ? *entry : gconst<int32_t>(a.ring)[wrapped(lds_fresh[i] + (index - held))];
                if (index >= held && (pos & mask) == 0) *entry = (int32_t)page;
                slot = (page << shift) + (pos & mask);
            }
            gmut<int64_t>(a.slots)[row] = slot;
            gmut<int32_t>(a.positions)[row] = pos;
        }
        // pages that come back
        const uint32_t coming = min(here, room - back), behind = wrapped(wrapped(fresh0 + free_pages) + back);
        for (uint32_t i = blockIdx.x * THREADS + threadIdx.x; i < coming; i += a.workgroups * THREADS) {
            const int s = find(lds_back, i);
            const int32_t page = gconst<int32_t>(a.table)[(base + s) * a.table_stride + (i - (s > 0 ? lds_back[s - 1] : 0))];
            gmut<int32_t>(a.ring)[wrapped(behind + i)] = page;
        }
        back += coming;
        __syncthreads();
    }
    // rows behind the last token
    const uint32_t total = min(t.tokens, n_tokens);
    for (uint32_t row = total + blockIdx.x * THREADS + threadIdx.x; row < n_tokens; row += a.workgroups * THREADS) {
        gmut<int64_t>(a.slots)[row] = -1;
        gmut<int32_t>(a.positions)[row] = -1;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) gmut<int32_t>(a.cu)[a.n_seqs] = (int32_t)total;

    if (!alone) {       // The last workgroup updates what the others read.  A workgroup's loads have returned when it is counted: their values were used.
        if (threadIdx.x == 0) lds_count = __hip_atomic_fetch_add((CF_GLOBAL uint32_t *)a.counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (lds_count != (uint32_t)a.workgroups - 1) return;
        if (threadIdx.x == 0) __hip_atomic_store((CF_GLOBAL uint32_t *)a.counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (a.n_seqs > THREADS) {       // lengths once more; those of the only turn are at hand
            t = {};
            turn = 0;
            ask(0);
            for (int64_t base = 0; base < a.n_seqs; base += THREADS, ++turn) {
                scan(base, t, mine, turn);
                if (base + threadIdx.x < a.n_seqs) gmut<int32_t>(a.lens_out)[base + threadIdx.x] = mine.now;
            }
        } else if ((int)threadIdx.x < a.n_seqs) gmut<int32_t>(a.lens_out)[threadIdx.x] = mine.now;
    }
    if (lane == 0) lds_used[wave] = t.used, lds_refused[wave] = t.refused;
    __syncthreads();
    if (threadIdx.x > 0) return;
    uint32_t used = 0, refused = 0;
    for (int w = 0; w < kWavesHere; ++w) used = max(used, lds_used[w]), refused += lds_refused[w];
    gmut<int64_t>(a.state_out)[0] = taken + used;
    gmut<int64_t>(a.state_out)[1] = put + back;
    gmut<int32_t>(a.refused)[0] = (int32_t)refused;
}

}  // namespace

hipError_t launch_plan(const PlanArgs &a, hipStream_t s)
{
    return a.wide ? enqueue_of<kPlanThreads>(k_kv_plan<kPlanThreads>, a.workgroups, s, a) : enqueue_of<kPlanThreads / 4>(k_kv_plan<kPlanThreads / 4>, a.workgroups, s, a);
}

}  // namespace attn
}  // namespace cf
