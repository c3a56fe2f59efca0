// The search for the least score that is taken (ScoreRange in csrc/cf_attn8.h), round by round as the kernel makes it, against a sort: random scores with infinities, NaN, ties,
// spreads of all sizes.  Runs under sanitizers, without a device.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <limits>
#include <random>
#include <vector>

#include "cf_attn8.h"

using namespace cf::attn;

// -> how many of the scores are taken, or -1: a bin that is none, a search that finds nothing or does not end.
static int taken_of(const std::vector<uint64_t> &x, uint32_t rest, std::vector<bool> &take)
{
    uint32_t least = ~0u, largest = 0;
    for (const uint64_t s : x) least = std::min(least, (uint32_t)(s >> 32)), largest = std::max(largest, (uint32_t)(s >> 32));
    ScoreRange range = {(uint64_t)least << 32, (uint64_t)largest << 32 | ~0u};
    bool all = false;
    for (int round = 0;; ++round) {
        if (round > 6 || range.from > range.end) return -1;
        std::vector<uint32_t> bins(kScoreBins);
        const int shift = range.shift();
        for (const uint64_t s : x)
            if (range.holds(s)) {
                if ((s - range.from) >> shift >= (uint64_t)kScoreBins) return -1;
                ++bins[(s - range.from) >> shift];
            }
        uint32_t past = 0;
        int found = kScoreBins - 1;
        for (; found >= 0 && past + bins[found] < rest; --found) past += bins[found];
        if (found < 0) return -1;
        rest -= past;
        all = bins[found] == rest;
        range = range.bin((uint32_t)found, shift);
        if (all || shift == 0) break;
    }
    int n = 0;
    uint32_t ties = 0;
    take.assign(x.size(), false);
    for (size_t i = 0; i < x.size(); ++i) {
        take[i] = all ? x[i] >= range.from : x[i] > range.from || (x[i] == range.from && ties++ < rest);
        n += take[i];
    }
    return n;
}

int main()
{
    std::mt19937_64 r(7);
    std::normal_distribution<double> normal;
    const double inf = std::numeric_limits<double>::infinity(), nan = std::numeric_limits<double>::quiet_NaN();
    const double odd[] = {inf, -inf, nan, 0.0, -0.0, 1.7976931348623157e308, -1.7976931348623157e308, 5e-324, -5e-324};
    int wrong = 0, cases[2] = {};
    for (int i = 0; i < 60000; ++i) {
        const int n = 2 + (int)(r() % 300), kind = (int)(r() % 6), some = (int)(r() % 9);
        std::vector<uint64_t> x(n);
        bool infinite = false;
        for (uint64_t &s : x) {
            double v = normal(r) * std::exp2((double)((int)(r() % 41) - 20) * (kind < 2 ? 1.0 : 40.0));
            if (kind == 0) v = std::round(v);
            if (kind == 1) v = r() % 2 ? inf : -inf;
            if (kind == 3 && r() % 4 == 0) v = odd[some];
            if (kind >= 4) v = r() % (kind - 2) ? odd[r() % 9] : v;
            infinite |= std::isinf(v);
            s = ordered_score(v);
        }
        const uint32_t rest = 1 + (uint32_t)(r() % (n - 1));
        std::vector<int> order(n);
        for (int k = 0; k < n; ++k) order[k] = k;
        std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return x[a] > x[b]; });
        std::vector<bool> take, want(n, false);
        for (uint32_t k = 0; k < rest; ++k) want[order[k]] = true;
        const int got = taken_of(x, rest, take);
        ++cases[infinite];
        if (got != (int)rest || take != want) {
            if (++wrong < 10) std::printf("%d scores of kind %d, %u to be taken: %d\n", n, kind, rest, got);
        }
    }
    std::printf("%d of %d and %d cases are wrong\n", wrong, cases[0], cases[1]);
    if (wrong) return 1;
    std::printf("all selections hold\n");
    return 0;
}
