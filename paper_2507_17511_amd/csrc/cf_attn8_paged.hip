// Attention of one new token per sequence over a paged cache of 8-bit codes: as over the one in 16 bits, every key and value is read once
// for 16 query heads that share it, straight into registers, and the same matrix instructions of 16-bit numbers take them.  In between a
// conversion brings two codes, times the scale of their page, into the type of the queries; codes times scales are exact there.
//
// Bound by HBM: 96 contexts of 160 to 16000 keys, 32 / 8 heads of 128, 137 us (5.1 TB/s), 64 of 8192 187 us (5.7; sums over rows of 2 GiB, read once, reach 5.9), 2 of 131100, 24 heads of
// 64, 144 us (5.6); one of 901 keys, 8 / 2 heads, by latency: 8.3 us.  Two workgroups a CU with 64 keys a wave in flight read faster than three, whose registers spill, or
// four with 32 keys (96 contexts: 149 us for 164 and 157).
//
// A wave takes 64 keys at a time (32 where head_dim is 256), so that as many bytes are on their way to a CU as with 16 bits.  Of K a lane reads 16
// neighbouring elements, the left operands of two instructions over the head dimension (the queries' lanes lie alike).  Of V it reads 4 (8, 16) elements
// of 8 neighbouring keys; a byte permute brings the codes of two keys together before they are converted.
#include "cf_attn_parts.h"
#include "cf_attn8_device.h"

namespace cf {
namespace attn {
namespace {

// SHARED: as many workgroups as the device holds have an equal share of all contexts' keys each, which they find in the lengths: a share may be the end of one context,
// some short ones and the beginning of another.  Otherwise a workgroup for each part that there may be.  Either way the last workgroup that is done with a context's head
// joins its parts.  LISTED: heads attend to the listed pages of their contexts alone; keys are counted along the list.  TOGETHER: as many of a step's keys
// as lie on one page for sure, 16 at least.
template <int DT, int D, bool SHARED, bool LISTED, int TOGETHER> __global__ __launch_bounds__(kWaves * 64, kHeldWorkgroups) void k_attn_paged8(Paged8Args b)
{
    using E = Elem<DT>;
    using C = Code<DT>;
    constexpr int kTiles = D == 256 ? 1 : 2;    // of 32 keys: a wave's step
    constexpr int kKeys = 32 * kTiles;
    constexpr int kLoads = D / 64;              // of 16 elements of a key
    constexpr int kSteps = D / 32;              // matrix instructions over the head dimension
    constexpr int kPer = D / 16;                // elements of a value row that a lane reads
    constexpr int kWords = kPer / 4;
    constexpr int kGroups = kKeys / TOGETHER;
    constexpr int kGroupKeys = TOGETHER;
    static_assert(TOGETHER >= 16 && TOGETHER <= kKeys, "groups of a step");
    constexpr int kGrain = kWaves * 64;         // keys: a step of the workgroup's
    const PagedArgs &a = b.p;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quarter = lane >> 4;
    const int head_tiles = (a.h.group + kPagedHeads - 1) / kPagedHeads;
    const int units = a.h.kv_heads * head_tiles;
    const int shift = b.cache.page_shift, mask = b.cache.page_size - 1;
    const int64_t capacity = min((int64_t)a.max_pages << shift, (int64_t)1 << 30);
    auto context_of = [&](int seq) { return (int)min((int64_t)max(((const CF_CONST int32_t *)a.lens)[seq], 0), capacity); };
    auto keys_of = [&](int len) { return LISTED ? (int)min((int64_t)((len + mask) >> shift), (int64_t)b.count) << shift : len; };
    const int unit = (int)(blockIdx.x % units), kv_head = unit / head_tiles, head0 = (unit % head_tiles) * kPagedHeads;
    int seq = (int)(blockIdx.x / units), split = 0, parts = 1, begin = 0, end = 0;

    // A context counts as its keys, kGrain at a time, and one more for its beginning and its end.
    __shared__ uint32_t lds_upto[SHARED ? kMostListed : 1];     // of the sequences up to each
    __shared__ uint32_t lds_longest;
    uint32_t share = 0, at_work = 0, stop = 0;
    const uint32_t group = blockIdx.x / units;
    if constexpr (SHARED) {
        if (wave == 0) {
            uint32_t upto = 0, longest = 0;
            for (int base = 0; base < a.n_seqs; base += 64) {
                uint32_t here = base + lane < a.n_seqs ? (keys_of(context_of(base + lane)) + kGrain - 1) / kGrain + 1 : 0;
                longest = max(longest, here);
                here = sums(here);
                if (base + lane < a.n_seqs) lds_upto[base + lane] = upto + here;
                upto += __builtin_amdgcn_readlane(here, 63);
            }
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) longest = max(longest, __shfl_xor(longest, d));
            if (lane == 0) lds_longest = longest;
        }
        __syncthreads();
        const uint32_t total = __builtin_amdgcn_readfirstlane(lds_upto[a.n_seqs - 1]), groups = gridDim.x / units;
        // 256-wide heads: six grains at least, as a part's output is what two keys are.  us for one grain at least / six: 48 contexts of 160 to 16000, 2 heads, 40 / 36, 8 heads 136 / 136;
        // 200 of 20 to 2000, 2 heads, 29 / 29; but 96 of 40 to 4096, 4 heads, 41 / 47, 16 of 600 to 60000, 2 heads, 50 / 53, 24 of 8192 each 41 / 51.
        share = max(max((total + groups - 1) / groups, (__builtin_amdgcn_readfirstlane(lds_longest) + a.n_splits - 2) / (a.n_splits - 1)), D == 256 ? 6u : 1u);       // a context is in n_splits shares at most
        at_work = (uint32_t)min((uint64_t)group * share, (uint64_t)total), stop = min(total, at_work + share);
        for (seq = 0; seq < a.n_seqs; seq += 64) {      // the first sequence with more up to it than this share begins with
            const uint64_t past = __ballot(seq + lane < a.n_seqs && lds_upto[min(seq + lane, a.n_seqs - 1)] > at_work);
            if (past) {
                seq += __builtin_ctzll(past);
                break;
            }
        }
    } else {
        split = seq / a.n_seqs;
        seq %= a.n_seqs;
    }
    for (; !SHARED || at_work < stop; ++seq) {
        const int len = context_of(seq), keys = keys_of(len);
        if constexpr (SHARED) {
            const uint32_t base = seq > 0 ? __builtin_amdgcn_readfirstlane(lds_upto[seq - 1]) : 0, top = __builtin_amdgcn_readfirstlane(lds_upto[seq]), from = at_work;
            at_work = min(stop, top);
            begin = from > base ? (int)(from - base - 1) * kGrain : 0, end = min((int)(at_work - base - 1) * kGrain, keys);
            if (keys > 0 && begin >= end) continue;             // its beginning alone
            split = keys > 0 ? (int)(group - (base + 1) / share) : 0;
            parts = keys > 0 ? (int)((top - 1) / share - (base + 1) / share) + 1 : 1;
            __syncthreads();                // LDS of the part before is free
        } else {
            parts = max(min((keys + a.split_keys - 1) / a.split_keys, a.n_splits), 1);      // a context of no keys has an empty one
            if (split >= parts) return;
            begin = (int)min((int64_t)split * a.split_keys, (int64_t)keys);
            end = split == a.n_splits - 1 ? keys : min(keys, begin + a.split_keys);
        }
        const int heads = min(a.h.group - head0, kPagedHeads);

        float m = kNoMax, l = 0.0f;
        f32x4 o[kPer];
#pragma unroll
        for (int d = 0; d < kPer; ++d) o[d] = (f32x4){0, 0, 0, 0};

        if (begin < end) {
            u32x4 q[kSteps];        // in the order of a lane's elements of K: 16 of them for two instructions
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    q[2 * i + t] = *gconst<u32x4>(a.q.data + (int64_t)seq * a.q.token + (kv_head * a.h.group + head0 + min(col, heads - 1)) * a.q.head + i * 128 + quarter * 32 + t * 16);

            const float c = a.h.scale_log2;
            // all of these are read by scalar loads
            const CF_CONST int32_t *table = (const CF_CONST int32_t *)a.table + seq * a.table_stride;
            const CF_CONST int32_t *list = LISTED ? (const CF_CONST int32_t *)b.blocks + ((int64_t)seq * a.h.kv_heads + kv_head) * b.count : nullptr;
            const CF_CONST float *k_scale = (const CF_CONST float *)b.cache.k_scale + kv_head, *v_scale = (const CF_CONST float *)b.cache.v_scale + kv_head;
            const int64_t head_bytes = (int64_t)kv_head * b.cache.page_size * D;
            const char *k_head = b.cache.k + head_bytes, *v_head = b.cache.v + head_bytes;
            const int last = end - 1, held = (len + mask) >> shift;

            // Where a step's groups of keys are, their scales, and how many of the keys are there.  Groups past the end are read on its last page, and not used.
            struct Step {
                int64_t at[kGroups];
                float k[kGroups], v[kGroups];
                int there[kGroups];
            };
            auto find = [&](int key0) {
                Step s;
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    const int key = key0 + g * kGroupKeys, off = key & mask;
                    int block = min(key, last) >> shift;
                    s.there[g] = end - key;
                    if constexpr (LISTED) {
                        const int listed = list[block];
                        block = min(max(listed, 0), held - 1);
                        s.there[g] = listed == block && key < end ? len - (block << shift) - off : 0;
                    }
                    const int64_t page = min(max(table[block], 0), b.cache.n_pages - 1);
                    s.at[g] = page * b.cache.page_bytes + off * D;
                    s.k[g] = k_scale[page * a.h.kv_heads];
                    s.v[g] = v_scale[page * a.h.kv_heads];
                    if (LISTED && s.there[g] <= 0) s.v[g] = 1.0f;       // an infinite scale of a page that is not attended to would make NaN of the zeros that stand for its values
                }
                return s;
            };
            // what is said of a tile's group of keys: of its second one, where it has two
            auto group_at = [](const auto &x, int g, bool second) {
                const auto low = x[32 * g / kGroupKeys], high = x[(32 * g + 16) / kGroupKeys];
                return second ? high : low;
            };
            auto key_of = [](int g, int x) { return (32 * g + x) % kGroupKeys; };      // of its group: key x of tile g
            u32x4 k[kTiles][2][kLoads];
            auto load_k = [&](const Step &s) {
#pragma unroll
                for (int g = 0; g < kTiles; ++g)
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const int x = 8 * (col >> 2) + 4 * t + (col & 3);
                        const char *src = k_head + group_at(s.at, g, x >= 16) + key_of(g, x) * D + quarter * 16;
#pragma unroll
                        for (int i = 0; i < kLoads; ++i) k[g][t][i] = *gconst<u32x4>(src + i * 64);
                    }
            };
            uint32_t v[kTiles][8][kWords];
            auto load_v = [&](const Step &s) {
#pragma unroll
                for (int g = 0; g < kTiles; ++g)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int x = 8 * quarter + j;
                        const char *src = v_head + group_at(s.at, g, x >= 16) + key_of(g, x) * D + col * kPer;
                        if constexpr (kWords == 1) v[g][j][0] = *gconst<uint32_t>(src);
                        else if constexpr (kWords == 2) {
                            const u32x2 y = *gconst<u32x2>(src);
                            v[g][j][0] = y[0], v[g][j][1] = y[1];
                        } else {
                            const u32x4 y = *gconst<u32x4>(src);
#pragma unroll
                            for (int w = 0; w < 4; ++w) v[g][j][w] = y[w];
                        }
                    }
            };
            auto most_of = [&](const Step &s, int g) { return group_at(s.there, g, quarter >= 2) - key_of(g, 8 * quarter); };    // of a lane's 8 keys

            // K of the next step is asked for as soon as this one's is used up, V of this one before that.
            int key0 = begin + wave * kKeys;
            Step at = find(key0);
            if (key0 < end) load_k(at);
            while (key0 < end) {
                const int next0 = key0 + kWaves * kKeys;
                const Step next = find(next0);
                load_v(at);
                __builtin_amdgcn_sched_barrier(0);
                f32x4 s[kTiles][2];
#pragma unroll
                for (int g = 0; g < kTiles; ++g) {
                    const float scale = group_at(at.k, g, col >= 8);
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        s[g][t] = (f32x4){0, 0, 0, 0};
#pragma unroll
                        for (int i = 0; i < kLoads; ++i) {
                            const u32x4 x = k[g][t][i];
                            s[g][t] = E::mfma16((u32x4){C::template pair<false>(x[0], scale), C::template pair<true>(x[0], scale), C::template pair<false>(x[1], scale), C::template pair<true>(x[1], scale)}, q[2 * i], s[g][t]);
                            s[g][t] = E::mfma16((u32x4){C::template pair<false>(x[2], scale), C::template pair<true>(x[2], scale), C::template pair<false>(x[3], scale), C::template pair<true>(x[3], scale)}, q[2 * i + 1], s[g][t]);
                        }
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                if (next0 < end) load_k(next);
                __builtin_amdgcn_sched_barrier(0);
                float top = -__builtin_inff();
                bool whole = true;          // whether all of the step's keys are there
#pragma unroll
                for (int g = 0; g < kGroups; ++g) whole &= at.there[g] >= kGroupKeys;
#pragma unroll
                for (int g = 0; g < kTiles; ++g) {
                    const int most = most_of(at, g);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if (!whole && j >= most) s[g][j >> 2][j & 3] = -__builtin_inff();
                        top = fmaxf(top, s[g][j >> 2][j & 3]);
                    }
                }
                top *= c;
                bool moves = __any(top > m + E::kMostOver);
                if constexpr (E::kFollow) {     // a row's four lanes: has one of them a key that is near enough?
                    uint64_t near = __ballot(!(top < m + kLeastOver));
                    near |= near >> 32;
                    near |= near >> 16;
                    if ((near & 0xffff) != 0xffff) {
                        const float row_top = max_quarters(max_halves(top));
                        moves |= __any(row_top < m + kLeastOver && row_top > -__builtin_inff() && max_quarters(max_halves(l)) < kFullTotal);
                    }
                }
                if (moves) {
                    const float fresh = reference<DT>(m, max_quarters(max_halves(top)), true, E::kFollow ? max_quarters(max_halves(l)) : 0.0f), scale = exp2_fast(m - fresh);
#pragma unroll
                    for (int d = 0; d < kPer; ++d)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[d][i] *= scale;
                    l *= scale;
                    m = fresh;
                }
#pragma unroll
                for (int g = 0; g < kTiles; ++g) {
                    if (!whole) {           // what lies in places that are not there may be NaN: 0 times it is not 0
                        const int most = most_of(at, g);
#pragma unroll
                        for (int j = 0; j < 8; ++j)
#pragma unroll
                            for (int w = 0; w < kWords; ++w) v[g][j][w] = j < most ? v[g][j][w] : 0u;
                    }
                    // Scaled scores are rounded as their maximum was: of scores of any size the largest has the weight 1.  Weights are rounded once, to the type that the matrix instructions
                    // take; their sum is of those that were not.  An output's error is that of its own rounding and up to 7 % more (96 contexts, bf16: 1.59e-3 of it, 1.56e-3 with fp32 weights).
                    u32x4 p;
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        const float p0 = exp2_fast(s[g][j >> 2][j & 3] * c - m), p1 = exp2_fast(s[g][j >> 2][(j & 3) + 1] * c - m);
                        l += p0 + p1;
                        p[j >> 1] = E::pack(p0, p1);
                    }
                    const float scale = group_at(at.v, g, quarter >= 2);
#pragma unroll
                    for (int w = 0; w < kWords; ++w) {
                        u32x4 x[4];         // elements 4w .. 4w + 3 of this lane's 8 keys
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t low = __builtin_amdgcn_perm(v[g][2 * j + 1][w], v[g][2 * j][w], 0x05010400), high = __builtin_amdgcn_perm(v[g][2 * j + 1][w], v[g][2 * j][w], 0x07030602);
                            x[0][j] = C::template pair<false>(low, scale);
                            x[1][j] = C::template pair<true>(low, scale);
                            x[2][j] = C::template pair<false>(high, scale);
                            x[3][j] = C::template pair<true>(high, scale);
                        }
#pragma unroll
                        for (int d = 0; d < 4; ++d) o[4 * w + d] = E::mfma16(x[d], p, o[4 * w + d]);
                    }
                }
                key0 = next0;
                at = next;
            }
            l = sum_quarters(sum_halves(l));
        }

        join_waves<D>(m, l, o, lane, wave);
        finish_part<DT, D, false>(a, seq, unit, units, kv_head, head0, split, parts, lane, wave, m, l, o);
        if constexpr (!SHARED) return;
    }
}

template <int DT, int D, bool SHARED, int TOGETHER> hipError_t paged8_pages(const Paged8Args &a, int64_t n, hipStream_t s)
{
    return a.blocks ? enqueue(k_attn_paged8<DT, D, SHARED, true, TOGETHER>, n, s, a) : enqueue(k_attn_paged8<DT, D, SHARED, false, TOGETHER>, n, s, a);
}

template <int DT, int D, bool SHARED> hipError_t paged8_over(const Paged8Args &a, hipStream_t s)
{
    const int64_t n = paged8_workgroups(a);
    constexpr int kStep = D == 256 ? 32 : 64;       // keys of a wave's
    const int together = a.cache.page_size < kStep ? a.cache.page_size : kStep;
    if (together == 64) return paged8_pages<DT, D, SHARED, kStep>(a, n, s);
    if (together == 32) return paged8_pages<DT, D, SHARED, 32>(a, n, s);
    return paged8_pages<DT, D, SHARED, 16>(a, n, s);
}

template <int DT, int D> hipError_t paged8_dim(const Paged8Args &a, hipStream_t s) { return a.p.many ? paged8_over<DT, D, true>(a, s) : paged8_over<DT, D, false>(a, s); }

template <int DT> hipError_t paged8_typed(const Paged8Args &a, hipStream_t s)
{
    switch (a.p.h.head_dim) {
    case 64: return paged8_dim<DT, 64>(a, s);
    case 128: return paged8_dim<DT, 128>(a, s);
    default: return paged8_dim<DT, 256>(a, s);
    }
}

}  // namespace

hipError_t launch_paged8(const Paged8Args &a, hipStream_t s) { return a.p.h.dtype == BF16 ? paged8_typed<BF16>(a, s) : paged8_typed<F16>(a, s); }

}  // namespace attn
}  // namespace cf
