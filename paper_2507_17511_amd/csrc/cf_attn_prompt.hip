// Attention over whole prompts: out = softmax(scale q k^T) v per sequence, one pass over the keys with a running
// maximum and sum.
//
// The rows of a workgroup are (token, head) pairs of the query heads that share one head of keys, token-major, so that
// grouped heads fill a tile of few tokens and the tile's causal edge is short.  A wave has 32 rows.  Both products are
// taken transposed: S^T = K Q^T gives a lane the scores of ONE row (its column) and 16 of 32 keys; in that layout the weights are
// the right operand of O^T = V^T P^T, up to an order of the keys that the reads of V follow, so weights
// never leave their lane, and the row's maximum, sum and scale are scalars of the lane.
//
// Bound by the matrix cores and what feeds them: 16384 tokens of 24 heads of 128 over as many keys 2.84 to 3.04 ms on three cards, 1085 to 1160 TFLOP/s.  The matrix cores
// are busy in 63 % of the cycles, with 4.5 vector instructions each beside them, and the clock falls with the power that this takes: 2.06 ms where all operands are zeros.  Two workgroups a CU, 256 registers a lane: a wave of 64 rows reads half of the LDS per product
// but is alone on its SIMD (3.01 ms, zeros 2.57).  2 x 8191 tokens of 32 / 8 heads, causal, 0.97 to 1.05 ms (1045 to 1130 TFLOP/s); ragged batches are bound by
// what a workgroup does before its first and after its last product: 14 x 1 to 2003 tokens 79 to 83 us (700 to 730 TFLOP/s).
#include <type_traits>

#include "cf_attn_device.h"

namespace cf {
namespace attn {
namespace {

constexpr int kWaves = 4;           // enqueue() launches as many
// How often the reference of a wave's rows falls.  For a first token that all rows attend to, and for one in a sequence's middle, once; where scores differ widely everywhere rows
// would have it fall and rise in turn, a tile done again for each (us, queries 3 and 10 times as large, without a limit / two falls / none and no lift: 8192 tokens of 24 heads of
// 128 over as many keys 929 / 887 / 871 and 1318 / 893 / 863; of 64 587 / 526 / 507 and 953 / 566 / 540).
constexpr int kMostFalls = 2;
static_assert(kPromptRows == kWaves * 32, "a wave has 32 rows");

// Where the 16-byte vectors of a staged tile's row lie: XORed so that neither the reads of K (16 rows, one vector each) nor the
// transposing reads of V (4 rows, 4 neighbouring vectors each) meet in a bank.
template <int D> __device__ __forceinline__ constexpr int k_turn(int row) { return D == 64 ? (row >> 1) & 7 : D == 128 ? row & 15 : row & 7; }
template <int D> __device__ __forceinline__ constexpr int v_turn(int row) { return D == 64 ? ((row >> 1) & 1) << 2 : (row & 3) << 2; }

struct Tile {
    int seq_q, len_q;           // the sequence's first row of q, and how many
    int seq_k, len_k;
    int index;                  // which row tile of the sequence; -1: none
};

__device__ __forceinline__ int clamped(int x, int most) { return min(max(x, 0), most); }

// Over the wave: the sum, or the largest of numbers that are not negative.
template <bool MAX> __device__ __forceinline__ int over_wave(int x)
{
    auto with = [&](int y) { x = MAX ? max(x, y) : x + y; };
    with(__builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));    // from the lane 1, 2, 4, 8 before it, of 16
    with(__builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
    with(__builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
    with(__builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
    with(__builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));    // the 16th lane's to the next 16, then the 32nd's to the other half
    with(__builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
    return __builtin_amdgcn_readlane(x, 63);
}

// The n-th row tile of 64 sequences, then of the 64 before them: by falling index, so that with a causal edge the tiles of most keys come
// first and short ones fill the end.  A lane has a sequence; how many tiles lie above an index is a sum over the wave.  Starts are clamped to the rows there
// are.  20 sequences of 814 tokens 57.5 -> 52.5 us, 14 of 1 to 2003 96 -> 91, 25 of 256 54.8 -> 56.5, against sequence by sequence.
__device__ __forceinline__ Tile find_tile(const PromptArgs &a, int n)
{
    Tile t = {0, 0, 0, 0, -1};
    const int lane = threadIdx.x & 63;
    for (int end = a.n_seqs; end > 0; end -= 64) {
        const int b = end - 1 - lane;
        int q0 = 0, len = 0, k0 = 0, len_k = 0, tiles = 0;
        if (b >= 0) {
            q0 = clamped(gconst<int32_t>(a.cu_q)[b], a.n_q);
            len = max(clamped(gconst<int32_t>(a.cu_q)[b + 1], a.n_q) - q0, 0);
            k0 = clamped(gconst<int32_t>(a.cu_k)[b], a.n_k);
            len_k = max(clamped(gconst<int32_t>(a.cu_k)[b + 1], a.n_k) - k0, 0);
            tiles = (int)(((int64_t)len * a.h.group + kPromptRows - 1) / kPromptRows);
        }
        const int total = over_wave<false>(tiles);
        if (n < total) {
            int least = 0, most = over_wave<true>(tiles) - 1;       // the index: the least one that n tiles at most lie above
            while (least < most) {
                const int middle = (least + most) >> 1;
                if (over_wave<false>(max(tiles - 1 - middle, 0)) <= n) most = middle;
                else least = middle + 1;
            }
            const uint64_t have = __ballot(tiles > least);
            const int nth = n - over_wave<false>(max(tiles - 1 - least, 0));
            const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(have >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)have, 0));
            const int who = __builtin_ctzll(__ballot(tiles > least && before == nth));
            t.seq_q = __builtin_amdgcn_readlane(q0, who);
            t.len_q = __builtin_amdgcn_readlane(len, who);
            t.seq_k = __builtin_amdgcn_readlane(k0, who);
            t.len_k = __builtin_amdgcn_readlane(len_k, who);
            t.index = least;
            return t;
        }
        n -= total;
    }
    return t;
}

// Brings 16 bytes from `base` + `from_all` + `from` to `to` + 16 * lane in LDS; those of which `from` is past `bytes` are zeros.
__device__ __forceinline__ void stage(const char *base, uint32_t bytes, uint32_t from, uint32_t from_all, char *to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc((void *)base, 0, (int)bytes, 0x00020000), (CF_LDS void *)to, 16, from, from_all, 0, 0);
}

template <int DT, int D> __global__ __launch_bounds__(kWaves * 64, D == 64 ? 4 : 2) void k_attn_prompt(PromptArgs a)
{
    using E = Elem<DT>;
    constexpr int kKeys = D == 256 ? 32 : 64;               // keys of a staged tile
    // Whether the next tile's scores are taken while this one's weights are computed.  Narrow heads do better with four workgroups a CU, of 128 registers a
    // lane, that do this for one another (8192 tokens of 24 heads of 64 over as many keys: 476 us, three that take scores ahead 485, two 492; 14 of 1 to 2003
    // tokens 49.7 / 49.4 / 54.4); wide ones lack the registers.
    constexpr bool kAhead = D == 128;
    constexpr int kSteps = D / 16;                          // matrix instructions over the head dimension
    constexpr int kBlocks = D / 32;                         // 32-row blocks of O^T
    constexpr int kSub = kKeys / 32;
    constexpr int kVecs = D / 8;                            // 16-byte vectors of a row
    constexpr int kStepRows = kWaves * 64 / kVecs;          // rows that the workgroup brings with one load a lane
    static_assert(k_turn<D>(kStepRows) == 0 && v_turn<D>(kStepRows) == 0, "every kStepRows rows are turned alike");
    constexpr int kLoads = kKeys * kVecs / (kWaves * 64);   // vectors of a tile that a lane brings
    constexpr int kTile = kKeys * D * 2;
    __shared__ __align__(256) char lds[4 * kTile];          // two tiles of K, two of V
    char *const lds_k = lds, *const lds_v = lds + 2 * kTile;
    __shared__ int64_t lds_at[kWaves][32], lds_dst[kWaves][32];      // where a wave's rows go, -1: nowhere; kept here while registers are short

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    const int unit = blockIdx.x % (a.h.kv_heads * a.n_splits);
    const int kv_head = unit % a.h.kv_heads, split = unit / a.h.kv_heads;
    const Tile t = find_tile(a, blockIdx.x / (a.h.kv_heads * a.n_splits));
    if (t.index < 0) return;

    // this lane's row
    const int row0 = t.index * kPromptRows + wave * 32, rows = t.len_q * a.h.group;
    const int shift = a.causal ? t.len_k - t.len_q + 1 : t.len_k;
    const int split_begin = split * a.split_keys;
    const int split_end = split == a.n_splits - 1 ? t.len_k : min(split_begin + a.split_keys, t.len_k);
    auto seen_by = [&](int token) { return min(max(a.causal ? token + shift : t.len_k, 0), t.len_k); };      // keys that a token's rows see
    const int row = min(row0 + col, rows - 1), token = row / a.h.group, head = kv_head * a.h.group + row - token * a.h.group;
    const int seen = min(seen_by(token), split_end);
    u32x4 q[kSteps];
    {
        const char *src = a.q.data + (t.seq_q + (int64_t)token) * a.q.token + head * a.q.head + half * 16;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) q[i] = *gconst<u32x4>(src + i * 32);
    }
    if (half == 0) {
        const int64_t at = row0 + col < rows ? (t.seq_q + (int64_t)token) * a.h.q_heads + head : -1;
        lds_at[wave][col] = at;
        lds_dst[wave][col] = at < 0 ? -1 : a.n_splits > 1 ? ((int64_t)split * a.parts.n_rows + at) * (D * 4) : (t.seq_q + (int64_t)token) * a.out.token + head * a.out.head;
    }
    // keys that no row of the workgroup sees begin at `end`, those that no row of the wave sees at `limit`, and those that not all of its rows see at `edge`
    const int end = min(split_end, seen_by((min((t.index + 1) * kPromptRows, rows) - 1) / a.h.group));
    const int limit = row0 < rows ? min(split_end, seen_by((min(row0 + 32, rows) - 1) / a.h.group)) : 0;
    const int edge = min(limit, seen_by(min(row0, rows - 1) / a.h.group));

    // Wide queries are there before the first tile is asked for: while the compiler holds them to be under way, it waits for all loads at the top of the loops, where the
    // next tile's have just been sent (2 x 333 tokens of 16 / 2 heads over 20333 keys that no cache holds, bf16, 231 us for 266).
    if constexpr (D == 256) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) asm("" : "+v"(q[i]));
    }

    f32x16 o[kBlocks];
#pragma unroll
    for (int d = 0; d < kBlocks; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    float m = kNoMax, l = 0.0f;
    const float c = a.h.scale_log2;

    // where this lane's vectors of a tile come from: the n-th is n * kStepRows rows further on, and turned alike
    const int from_row = (wave * 64 + lane) / kVecs, place = lane % kVecs;
    const uint32_t k_from = (uint32_t)from_row * (uint32_t)a.k.token + (place ^ k_turn<D>(from_row)) * 16;
    const uint32_t v_from = (uint32_t)from_row * (uint32_t)a.v.token + (place ^ v_turn<D>(from_row)) * 16;
    const char *k_base = a.k.data + t.seq_k * a.k.token + kv_head * a.k.head;
    const char *v_base = a.v.data + t.seq_k * a.v.token + kv_head * a.v.head;
    auto bring = [&](const char *base, int64_t stride, uint32_t from, char *to, int at) {
        base += at * stride;
        if (at + kKeys <= t.len_k) {
#pragma unroll
            for (int n = 0; n < kLoads; ++n) stage(base, 0xffffffffu, from, n * (uint32_t)(kStepRows * stride), to + (n * kWaves + wave) * 1024);
        } else {            // rows past the sequence come as zeros
#pragma unroll 1
            for (int n = 0; n < kLoads; ++n) {
                const int rows_here = min(t.len_k - at - n * kStepRows, kStepRows);
                stage(base + n * kStepRows * stride, rows_here > 0 ? (uint32_t)(rows_here - 1) * (uint32_t)stride + D * 2 : 0, from, 0, to + (n * kWaves + wave) * 1024);
            }
        }
    };
    auto bring_k = [&](int at, int buffer) { bring(k_base, a.k.token, k_from, lds_k + buffer, at); };
    auto bring_v = [&](int at, int buffer) { bring(v_base, a.v.token, v_from, lds_v + buffer, at); };

    const CF_LDS char *k_read = (const CF_LDS char *)lds_k + col * (D * 2) + ((half ^ k_turn<D>(col)) << 4);
    const int v_row = 4 * half + ((lane & 15) >> 2);
    const int v_vec = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    const CF_LDS char *v_read = (const CF_LDS char *)lds_v + v_row * (D * 2) + ((v_vec ^ v_turn<D>(v_row)) << 4) + (lane & 1) * 8;
    // elements d * 32 + col of keys 16 g + 4 half + {0 .. 3, 8 .. 11} of the tile
    auto values = [&](int buffer, int g, int d) {
        const CF_LDS char *at = (const CF_LDS char *)((uintptr_t)v_read ^ (d << 6)) + buffer + g * 16 * D * 2;
        const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((CF_LDS s16x4 *)at));
        const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((CF_LDS s16x4 *)(at + 8 * D * 2)));
        return (u32x4){x[0], x[1], y[0], y[1]};
    };

    // A tile's scores are taken while the weights of the tile before are computed.  While V of tile n and K of tile n + 1 are read, V of tile
    // n + 1 and K of tile n + 2 come, into the other buffers.  The waves of a workgroup meet here once a tile, wherever in the
    // loops below they are.
    int key0 = split_begin, buffer = 0;         // the tile in work, and where its V is; K of the next one is in the other buffer
    auto send = [&]() {
        if (key0 + kKeys < end) bring_v(key0 + kKeys, buffer ^ kTile);
        if constexpr (kAhead) {
            if (key0 + 2 * kKeys < end) bring_k(key0 + 2 * kKeys, buffer);
        } else {
            if (key0 + kKeys < end) bring_k(key0 + kKeys, buffer ^ kTile);
        }
    };
    auto advance = [&]() {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        key0 += kKeys;
        buffer ^= kTile;
        send();
    };
    f32x16 s[kSub];
    u32x4 p[kSub * 2];
    auto scores = [&](f32x16 (&s)[kSub], int buffer) {
#pragma unroll
        for (int b = 0; b < kSub; ++b) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[b][i] = 0.0f;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const u32x4 k = *(const CF_LDS u32x4 *)((const CF_LDS char *)((uintptr_t)k_read ^ (i << 5)) + buffer + b * 32 * D * 2);
                s[b] = E::mfma32(k, q[i], s[b]);
            }
        }
    };
    auto largest = [&](const f32x16 (&s)[kSub]) {
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < kSub; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
        return max_halves(top) * c;
    };
    auto rescale = [&](float top, bool fall) {
        const float fresh = reference<DT>(m, top, fall, E::kFollow ? max_halves(l) : 0.0f), scale = exp2_fast(m - fresh);
#pragma unroll
        for (int d = 0; d < kBlocks; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] *= scale;
        l *= scale;
        m = fresh;
    };
    // -> their sum.  Of scores of any size the largest has the weight 1 if scaled scores are rounded before the maximum, rounded alike, is taken off: `any`.
    // Without that rounding it is off by a factor of 2^(half a unit in the last place of m).
    auto weights = [&](auto any) {
        float sum = 0.0f;
        auto less = [&](float x) { return decltype(any)::value ? x * c - m : __builtin_fmaf(x, c, -m); };
#pragma unroll
        for (int b = 0; b < kSub; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float p0 = exp2_fast(less(s[b][i])), p1 = exp2_fast(less(s[b][i + 1]));
                sum += p0 + p1;
                p[b * 2 + (i >> 3)][(i & 7) >> 1] = E::pack(p0, p1);
            }
        return sum;
    };
    auto products = [&]() {
#pragma unroll
        for (int g = 0; g < kSub * 2; ++g)
#pragma unroll
            for (int d = 0; d < kBlocks; ++d) o[d] = E::mfma32(values(buffer, g, d), p[g], o[d]);
    };

    if (key0 < end) {
        bring_k(key0, 0);
        __builtin_amdgcn_sched_barrier(0);          // loads arrive in order: those of K are not waited for with those sent after them
        bring_v(key0, 0);
        if constexpr (kAhead) {
            if (key0 + kKeys < end) {
                bring_k(key0 + kKeys, kTile);
                asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"(2 * kLoads) : "memory");
            } else {
                asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"(kLoads) : "memory");
            }
            scores(s, 0);
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");      // V is there, and K's first buffer free again
        send();
    }
    // Tiles that all rows of the wave see, up to the last but one.  Their maximum is not looked for: weights are positive, so
    // that none is larger than their sum.  Where that passes kMostSum, in any lane, the tile is done again after its maximum has been taken and the
    // accumulators scaled; most often that is the first tile alone.  That happens outside of the inner loop, where the compiler keeps them in place.
    // A tile is done again once, for a lane's weights sum up to less than 2^kLift * 2 * 32 then, and falls are counted: either scores are rounded as the maximum is, or that is
    // kMostExact at most, and the wave of a row beyond it, whose scores are of no use, infinite or none, takes the loop after this one.  The rounding costs
    // 16384 rows of 24 heads of 128 3022 us for 2937; with the way out instead of it, wide heads' accumulators would leave the registers (325 us for
    // 245: 2 x 333 tokens over 20333 keys).
    int settled = 0;            // the tile that the reference was set for
    int falls = kMostFalls;
    bool fall = false;
    // Whether a tile has to be done again: its weights sum up to too much, or in fp16 to too little.
    auto unfit = [&](float sum) -> bool {
        if constexpr (!E::kFollow) return __any(sum > kMostSum);
        if (__builtin_expect(!__any(sum > kMostSum || sum < kLeastSum), 1)) return false;
        fall = falls > 0 && key0 != settled && __any(sum_halves(sum) < kLeastSum && max_halves(l) < kFullTotal);
        falls -= fall;
        return fall || __any(sum > kMostSum);
    };
    if constexpr (kAhead) {
        while (key0 + 2 * kKeys <= edge) {
            rescale(largest(s), fall);
            settled = key0;
            if (__any(fabsf(m) > kMostExact)) break;
            do {
                f32x16 next[kSub];
                scores(next, buffer ^ kTile);
                const float sum = weights(std::false_type{});
                if (unfit(sum)) break;
                l += sum;
                products();
#pragma unroll
                for (int b = 0; b < kSub; ++b) s[b] = next[b];
                advance();
            } while (key0 + 2 * kKeys <= edge);
        }
    } else {
        while (key0 + kKeys <= edge) {
            scores(s, buffer);
            rescale(largest(s), fall);
            settled = key0;
            do {
                scores(s, buffer);
                const float sum = weights(std::true_type{});
                if (unfit(sum)) break;
                l += sum;
                products();
                advance();
            } while (key0 + kKeys <= edge);
        }
    }
    // The last of them, and tiles of which some rows see a part.
    auto mask = [&](int key0) {
#pragma unroll
        for (int b = 0; b < kSub; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (b * 32 + 8 * (i >> 2) + (i & 3) >= seen - key0 - 4 * half) s[b][i] = -__builtin_inff();
    };
    // Takes s in.
    auto weigh = [&]() {
        const float top = largest(s);
        fall = E::kFollow && falls > 0 && __any(top < m + kLeastOver && top > -__builtin_inff() && max_halves(l) < kFullTotal);
        falls -= fall;
        if (fall || __any(top > m + E::kMostOver)) rescale(top, fall);
        l += weights(std::true_type{});
    };
    int odd_from = limit;       // the tiles from here on are done at the end
    while (key0 < limit) {
        if constexpr (!kAhead) scores(s, buffer);
        if (key0 + kKeys > edge) {
            mask(key0);
            // A weight of zero does not keep an infinity or NaN out of a sum.  Is there one among the values that not all rows see, this tile and the one after it,
            // if there is one, wait for the end.
            uint32_t odd = 0;
#pragma unroll 1
            for (int g = max(edge - key0, 0) >> 4; g < kSub * 2; ++g)
#pragma unroll
                for (int d = 0; d < kBlocks; ++d) {
                    const u32x4 v = values(buffer, g, d);
#pragma unroll
                    for (int w = 0; w < 4; ++w) odd |= E::Odd::carry(v[w]);
                }
            if (__builtin_expect(__any(E::Odd::any(odd)) != 0, 0)) {
                odd_from = key0;
                break;
            }
        }
        weigh();
        products();
        if (kAhead && key0 + kKeys < limit) scores(s, buffer ^ kTile);
        advance();
    }
    // Tiles that only other waves see.
    while (key0 < end) advance();

    if (row0 >= rows) return;
    // The tiles with infinities or NaN among values that not all rows see, as above, but from memory, and with zeros in the place of these: that leaves all sums
    // that they are no part of as they are, to the last bit.  Then they are added, key by key, to the rows that see them.  Here, where the loops above are over, this costs
    // them no registers: done within them, it cost 14 prompts of 1 to 2003 tokens 101 us for 89, 50 of 128 54 for 42.  16384 tokens of 4 heads of 64 / 128 / 256, causal,
    // with a NaN in the last value: 272 / 490 / 1060 us, without it 278 / 337 / 904.
    if (__builtin_expect(odd_from < limit, 0)) {
#pragma unroll 1
        for (int first = odd_from; first < limit; first += kKeys) {
#pragma unroll
            for (int b = 0; b < kSub; ++b) {
                const char *from = k_base + min(first + b * 32 + col, t.len_k - 1) * (int64_t)a.k.token + half * 16;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = 0.0f;
#pragma unroll
                for (int i = 0; i < kSteps; ++i) s[b] = E::mfma32(*gconst<u32x4>(from + i * 32), q[i], s[b]);
            }
            mask(first);
            weigh();
#pragma unroll
            for (int g = 0; g < kSub * 2; ++g)
#pragma unroll
                for (int d = 0; d < kBlocks; ++d) {
                    u32x4 v;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        uint32_t x[2];
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const int key = first + g * 16 + half * 4 + (w >> 1) * 8 + (w & 1) * 2 + j;
                            x[j] = *gconst<uint16_t>(v_base + min(key, t.len_k - 1) * (int64_t)a.v.token + d * 64 + col * 2);
                            if (key >= t.len_k || E::Odd::any(E::Odd::carry(x[j]))) x[j] = 0;
                        }
                        v[w] = x[0] | x[1] << 16;
                    }
                    o[d] = E::mfma32(v, p[g], o[d]);
                }
        }
#pragma unroll 1
        for (int key = odd_from; key < limit; ++key) {
            const char *k_from = k_base + key * (int64_t)a.k.token + half * 16, *v_from = v_base + key * (int64_t)a.v.token + half * 8;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const u32x4 k = *gconst<u32x4>(k_from + i * 32);
#pragma unroll
                for (int w = 0; w < 4; ++w) sum = __builtin_fmaf(E::lo(k[w]), E::lo(q[i][w]), __builtin_fmaf(E::hi(k[w]), E::hi(q[i][w]), sum));
            }
            const float weight = exp2_fast(sum_halves(sum) * c - m);
#pragma unroll
            for (int d = 0; d < kBlocks; ++d)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const u32x2 v = *gconst<u32x2>(v_from + d * 64 + i * 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float x = j & 1 ? E::hi(v[j >> 1]) : E::lo(v[j >> 1]);
                        if (key < seen && !(fabsf(x) < __builtin_inff())) o[d][i + j] = __builtin_fmaf(weight, x, o[d][i + j]);
                    }
                }
        }
    }
    // All waves have left the tiles behind.  A wave turns its rows in LDS, 128 columns at a time, so that it stores whole lines.
    l = sum_halves(l);
    const float inv = inverse_of(l);
    if (l == 0.0f)              // no key, or none with a score above -infinity: 0 times an infinite value is none of the row's
#pragma unroll
        for (int d = 0; d < kBlocks; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    const int64_t at = lds_at[wave][col];
    float *lse = a.n_splits > 1 ? a.parts.lse + (int64_t)split * a.parts.n_rows : a.lse;
    if (lse && at >= 0 && half == 0) gmut<float>(lse)[at] = lse_of(m, l);
    constexpr int kPass = D < 128 ? D / 32 : 4;             // blocks of 32 columns of a pass
    CF_LDS char *const mine = (CF_LDS char *)lds + wave * (kTile * 4 / kWaves);
    auto store = [&](char *base, auto wide) {
        constexpr int kSize = decltype(wide)::value ? 4 : 2, kRow = kPass * 32 * kSize, kLine = kRow / 16;
        static_assert(32 * kRow <= kTile * 4 / kWaves, "a wave's rows fit its share of LDS");
#pragma unroll
        for (int d0 = 0; d0 < kBlocks; d0 += kPass) {
#pragma unroll
            for (int d = 0; d < kPass; ++d)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const f32x16 &x = o[d0 + d];
                    if constexpr (kSize == 4) *(CF_LDS f32x4 *)(mine + col * kRow + (((d * 8 + i / 2 + half) ^ (col & (kLine - 1))) << 4)) = (f32x4){x[i] * inv, x[i + 1] * inv, x[i + 2] * inv, x[i + 3] * inv};
                    else *(CF_LDS u32x2 *)(mine + col * kRow + (((d * 4 + i / 4) ^ (col & (kLine - 1))) << 4) + half * 8) = (u32x2){E::pack(x[i] * inv, x[i + 1] * inv), E::pack(x[i + 2] * inv, x[i + 3] * inv)};
                }
#pragma unroll
            for (int n = 0; n < kLine / 2; ++n) {
                const int r = n * (64 / kLine) + lane / kLine, place = lane % kLine;
                const int64_t dst = lds_dst[wave][r];
                const u32x4 x = *(const CF_LDS u32x4 *)(mine + r * kRow + ((place ^ (r & (kLine - 1))) << 4));
                if (dst >= 0) *gmut<u32x4>(base + dst + d0 * 32 * kSize + place * 16) = x;
            }
        }
    };
    if (a.n_splits > 1) {
        if (!__any(l != 0.0f)) return;                      // the join does not read outputs of parts without keys
        store(reinterpret_cast<char *>(a.parts.o), std::true_type{});
    } else {
        store(a.out.data, std::false_type{});
    }
}

}  // namespace

hipError_t launch_prompt(const PromptArgs &a, hipStream_t s)
{
    const bool bf16 = a.h.dtype == BF16;
    const int64_t n = prompt_workgroups(a);
    switch (a.h.head_dim) {
    case 64: return bf16 ? enqueue(k_attn_prompt<BF16, 64>, n, s, a) : enqueue(k_attn_prompt<F16, 64>, n, s, a);
    case 128: return bf16 ? enqueue(k_attn_prompt<BF16, 128>, n, s, a) : enqueue(k_attn_prompt<F16, 128>, n, s, a);
    default: return bf16 ? enqueue(k_attn_prompt<BF16, 256>, n, s, a) : enqueue(k_attn_prompt<F16, 256>, n, s, a);
    }
}

}  // namespace attn
}  // namespace cf
