// Keys and values into the paged cache of 8-bit codes, rotated on the way, and the queries' rotation.
//
// What a call's tokens bring to one page is one piece of work for each head of keys and of values: their largest magnitude decides the scale.  Such
// tokens are neighbours in the call, so that a workgroup finds where they begin by looking at the slots alone.  It takes the pages that begin among `chunk`
// tokens: lone tokens, one of a page, as a step of generation brings them, for four heads, a wave each, as many at a time as a wave has room for their rows;
// neighbours on a page for one head, or as many as its four waves have room for.  They read the rows twice, once for the scale and once for the codes, the
// second time from the caches.  To keep them in registers instead took so many that few waves were there to wait for memory (16384 tokens, 8 heads of 128,
// no queries: 83 us; as it is 35).
//
// 16384 tokens of 24 + 2 x 8 heads of 128 in 68 us (4.5 TB/s): bound by HBM for the queries, by instructions (60 % of the time) and latencies for the pages;
// 6331 of 16 + 2 x 2 heads of 256 in 25 (5.0 TB/s); 48 in 4.7, by its launch.  Fewer waves for a row leave instructions out and time in (no queries,
// two rows a workgroup 50 us, four 78); eight waves, which read rows once, 55.
#include "cf_attn8_device.h"

namespace cf {
namespace attn {
namespace {

constexpr int kWaves = kAppendThreads / 64;

// 16 elements of a row: two vectors of 8, which hold the two halves of 8 pairs where pairs lie rotary_dim / 2 apart (or, PAIRS, side by side).
struct Place {
    int first, second;
    bool rotated;
};
template <bool PAIRS> __device__ __forceinline__ Place place_of(int lane, int half)
{
    Place p;
    const int lanes = half >> 3;
    p.rotated = lane < lanes;
    p.first = !PAIRS && p.rotated ? lane : 2 * lane;
    p.second = !PAIRS && p.rotated ? lane + lanes : p.first + 1;
    return p;
}

struct Elements {
    float x[16];
};
struct Angles {
    f32x4 c[2], s[2];
};
struct Raw {
    u32x4 x, y;
};

// A lane's part of a position's row of cosines and sines.
__device__ __forceinline__ Angles angles_of(const Append8Args &a, int pos, int half, int lane)
{
    const CF_GLOBAL f32x4 *c = gconst<f32x4>(a.cos + (int64_t)pos * half + lane * 8), *s = gconst<f32x4>(a.sin + (int64_t)pos * half + lane * 8);
    return {{c[0], c[1]}, {s[0], s[1]}};
}

template <int DT, bool PAIRS> __device__ __forceinline__ Elements turn(const Raw &in, const Angles &g, bool rotated)
{
    Elements r;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        r.x[2 * k] = Elem<DT>::lo(in.x[k]), r.x[2 * k + 1] = Elem<DT>::hi(in.x[k]);
        r.x[8 + 2 * k] = Elem<DT>::lo(in.y[k]), r.x[8 + 2 * k + 1] = Elem<DT>::hi(in.y[k]);
    }
    if (rotated) {
        if constexpr (!PAIRS) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float a = r.x[k], b = r.x[8 + k], co = g.c[k >> 2][k & 3], si = g.s[k >> 2][k & 3];
                r.x[k] = a * co - b * si;
                r.x[8 + k] = b * co + a * si;
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float a = r.x[2 * k], b = r.x[2 * k + 1], co = g.c[k >> 2][k & 3], si = g.s[k >> 2][k & 3];
                r.x[2 * k] = a * co - b * si;
                r.x[2 * k + 1] = b * co + a * si;
            }
        }
    }
    return r;
}

constexpr int kTurns = kAppendTurns;

// A lane has its part of the rows of kTurns heads of a token, which turn by the same angles (16384 tokens of 24 heads of 128: 35 us for 42 with angles for each).
template <int DT, int D, bool PAIRS> __device__ __forceinline__ void rotate_queries(const Append8Args &a, uint32_t group)
{
    constexpr int kLanes = D / 16;
    const uint32_t of_token = (a.h.q_heads + kTurns - 1) / kTurns * kLanes;
    const uint32_t id = group * (kWaves * 64) + threadIdx.x;        // a launch counts fewer than 2^32 work-items
    const int64_t token = id / of_token;
    const uint32_t rest = id % of_token, lane = rest % kLanes;
    const int head0 = rest / kLanes * kTurns, heads = min(a.h.q_heads - head0, kTurns), half = a.rotary_dim >> 1;
    if (token >= a.n_tokens) return;
    const Place place = place_of<PAIRS>(lane, half);
    const char *src = a.q.data + token * a.q.token + head0 * a.q.head;
    char *dst = a.q_out.data + token * a.q_out.token + head0 * a.q_out.head;
    Raw raw[kTurns];
#pragma unroll
    for (int i = 0; i < kTurns; ++i)
        if (i < heads) {
            const CF_GLOBAL u32x4 *at = gconst<u32x4>(src + i * a.q.head);
            raw[i] = {at[place.first], at[place.second]};
        }
    Angles angles;
    if (half) {
        const int pos = gconst<int32_t>(a.positions)[token];
        if (pos < 0 || pos >= a.n_positions) return;
        if (place.rotated) angles = angles_of(a, pos, half, lane);
    }
#pragma unroll
    for (int i = 0; i < kTurns; ++i)
        if (i < heads) {
            const Elements r = turn<DT, PAIRS>(raw[i], angles, place.rotated);
            u32x4 u, w;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                u[k] = Elem<DT>::pack(r.x[2 * k], r.x[2 * k + 1]);
                w[k] = Elem<DT>::pack(r.x[8 + 2 * k], r.x[8 + 2 * k + 1]);
            }
            CF_GLOBAL u32x4 *at = gmut<u32x4>(dst + i * a.q_out.head);
            at[place.first] = u;
            at[place.second] = w;
        }
}

// Of two fp16 numbers each.  NaN yields to a number.
template <bool LARGEST> __device__ __forceinline__ uint32_t extreme(uint32_t a, uint32_t b)
{
    const f16x2 x = __builtin_bit_cast(f16x2, a), y = __builtin_bit_cast(f16x2, b);
    return __builtin_bit_cast(uint32_t, LARGEST ? __builtin_elementwise_max(x, y) : __builtin_elementwise_min(x, y));
}
// Over the lanes of sixteen that hold the same elements, every LANES-th one.
template <bool LARGEST, int LANES> __device__ __forceinline__ uint32_t over_sixteen(uint32_t x)
{
    if constexpr (LANES <= 4) x = extreme<LARGEST>(x, moved<0x124>(x));     // 4 lanes on
    if constexpr (LANES <= 8) x = extreme<LARGEST>(x, moved<0x128>(x));     // 8
    return x;
}
// Of x and the lane 32 (16) away in the lower half (the even sixteens), of y in the other.
template <bool LARGEST> __device__ __forceinline__ uint32_t of_halves(uint32_t x, uint32_t y)
{
    const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(x, y, false, false));
    return extreme<LARGEST>(r[0], r[1]);
}
template <bool LARGEST> __device__ __forceinline__ uint32_t of_quarters(uint32_t x, uint32_t y)
{
    const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(x, y, false, false));
    return extreme<LARGEST>(r[0], r[1]);
}
// The largest of LANES neighbouring lanes.
template <int LANES> __device__ __forceinline__ float over_lanes(float x)
{
    x = fmaxf(x, moved<0xb1>(x));                                 // of pairs
    x = fmaxf(x, moved<0x4e>(x));                                 // of fours
    if constexpr (LANES >= 8) x = fmaxf(x, moved<0x141>(x));      // eight lanes turned round
    if constexpr (LANES >= 16) x = fmaxf(x, moved<0x140>(x));     // sixteen
    return x;
}

template <int DT> __device__ __forceinline__ float within(float x) { return x > Code<DT>::kMost ? Code<DT>::kMost : x < -Code<DT>::kMost ? -Code<DT>::kMost : x; }      // NaN stays

// Codes of 8 neighbouring elements.
__device__ __forceinline__ u32x2 encode8(const float *x, float by)
{
    return {encode4(x[0] * by, x[1] * by, x[2] * by, x[3] * by), encode4(x[4] * by, x[5] * by, x[6] * by, x[7] * by)};
}

// Codes of a head's page go by a new scale, 2^by times as large.  `step` lanes share them; places of this call are written behind them.
__device__ __forceinline__ void rescale(char *codes, int bytes, int by, int lane, int step)
{
    const float f = power_of_two(max(by, -126));
    for (int i = lane * 16; i < bytes; i += step * 16) {
        u32x4 w = *gconst<u32x4>(codes + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const auto low = __builtin_amdgcn_cvt_pk_f32_fp8(w[k], false), high = __builtin_amdgcn_cvt_pk_f32_fp8(w[k], true);
            w[k] = encode4(low[0] * f, low[1] * f, high[0] * f, high[1] * f);
        }
        *gmut<u32x4>(codes + i) = w;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

struct Where {
    int off, pos;               // off < 0: not there, or left out
};
__device__ __forceinline__ Where where_is(const Append8Args &a, int64_t token)
{
    Where w = {-1, 0};
    if (a.rotary_dim) w.pos = gconst<int32_t>(a.positions)[token];
    const int off = (int)(gconst<int64_t>(a.slots)[token] & (a.cache.page_size - 1));
    if (!a.rotary_dim || (w.pos >= 0 && w.pos < a.n_positions)) w.off = off;
    else w.pos = 0;
    return w;
}

// What a row of work is about: one head of keys or of values.
struct Row {
    const char *data;           // of token 0
    int64_t token;
    char *codes;                // of page 0
    float *scale;               // of page 0
    uint16_t *bounds;           // of page 0, or null
    bool rotated;
};
template <int D> __device__ __forceinline__ Row row_of(const Append8Args &a, int row)
{
    const bool value = row >= a.h.kv_heads;
    const int head = value ? row - a.h.kv_heads : row;
    const Rows &in = value ? a.v : a.k;
    return {in.data + head * in.head, in.token, (value ? a.cache.v : a.cache.k) + (int64_t)head * a.cache.page_size * D, (value ? a.cache.v_scale : a.cache.k_scale) + head,
            value || !a.cache.bounds ? nullptr : a.cache.bounds + (int64_t)head * 2 * D, !value && a.rotary_dim > 0};
}

// A token that is the only one of its page, for every LANES lanes: `there` says so.
template <int DT, int D, bool PAIRS> __device__ __forceinline__ void store_lone(const Append8Args &a, const Row &row, int64_t token, int page, bool there, int lane)
{
    constexpr int kLanes = D / 16;
    const int row_lane = lane % kLanes;
    if (!there) return;
    const Where where = where_is(a, token);
    if (where.off < 0) return;
    const Place place = place_of<PAIRS>(row_lane, row.rotated ? a.rotary_dim >> 1 : 0);
    const CF_GLOBAL u32x4 *src = gconst<u32x4>(row.data + token * row.token);
    const Raw raw = {src[place.first], src[place.second]};
    Angles angles;
    if (place.rotated) angles = angles_of(a, where.pos, a.rotary_dim >> 1, row_lane);
    float *scale_at = row.scale + (int64_t)page * a.h.kv_heads;
    const float scale_was = *gconst<float>(scale_at);
    uint16_t *bounds = row.bounds ? row.bounds + (int64_t)page * a.h.kv_heads * 2 * D : nullptr;
    const bool begins = where.off == 0;
    u32x4 was[2][2] = {};
    if (bounds && !begins) {
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
            for (int high = 0; high < 2; ++high) was[v][high] = gconst<u32x4>(bounds + high * D)[v ? place.second : place.first];
    }
    Elements r = turn<DT, PAIRS>(raw, angles, place.rotated);
    float most = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; ++k) most = fmaxf(most, fabsf(r.x[k]));
    most = over_lanes<kLanes>(most);
    if (most > Code<DT>::kMost) {
        most = Code<DT>::kMost;
#pragma unroll
        for (int k = 0; k < 16; ++k) r.x[k] = within<DT>(r.x[k]);
    }
    const int before = begins ? kLeastExponent : exponent_of(scale_was), e = max(exponent_for(most), before);
    char *codes = row.codes + page * a.cache.page_bytes;
    if (!begins && e > before) rescale(codes, a.cache.page_size * D, before - e, row_lane, kLanes);
    const float by = power_of_two(-e), scale = power_of_two(e);
    if (row_lane == 0) *gmut<float>(scale_at) = scale;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        const int at = v ? place.second : place.first;
        const u32x2 c = encode8(r.x + 8 * v, by);
        *gmut<u32x2>(codes + where.off * D + at * 8) = c;
        if (!bounds) continue;
        u32x4 least, largest;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const auto y = k & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(c[k >> 1], true) : __builtin_amdgcn_cvt_pk_f32_fp8(c[k >> 1], false);
            float low[2], high[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                low[j] = high[j] = y[j] == y[j] ? y[j] * scale : 0.0f;
                if (begins) continue;
                const float old_low = j ? Elem<BF16>::hi(was[v][0][k]) : Elem<BF16>::lo(was[v][0][k]), old_high = j ? Elem<BF16>::hi(was[v][1][k]) : Elem<BF16>::lo(was[v][1][k]);
                low[j] = y[j] == y[j] ? fminf(low[j], old_low) : old_low;
                high[j] = y[j] == y[j] ? fmaxf(high[j], old_high) : old_high;
            }
            least[k] = Elem<BF16>::pack(low[0], low[1]);
            largest[k] = Elem<BF16>::pack(high[0], high[1]);
        }
        gmut<u32x4>(bounds)[at] = least;
        gmut<u32x4>(bounds + D)[at] = largest;
    }
}

struct Shared {
    float most[kWaves];
    bool begins[kWaves];
    _Float16 bounds[kWaves][512];   // [least, largest][D], codes' values
};

// Tokens first .. first + n - 1, two at least, go to one page: a row of them, by `waves` of the workgroup's from wave0 on.  A wave without a row has no tokens.
template <int DT, int D, bool PAIRS>
__device__ __forceinline__ void store_neighbours(const Append8Args &a, Shared &lds, const Row &row, int64_t first, int n, int page, int lane, int wave, int wave0, int waves)
{
    constexpr int kLanes = D / 16;              // of a row
    constexpr int kTokens = 64 / kLanes;        // of a wave's round
    const int round = kTokens * waves;
    const int row_lane = lane % kLanes, half = a.rotary_dim >> 1;
    const int mine = (wave - wave0) * kTokens + lane / kLanes;        // a lane's row of a round
    const Place place = place_of<PAIRS>(row_lane, row.rotated ? half : 0);
    auto elements = [&](int i, const Where &w) {
        const CF_GLOBAL u32x4 *src = gconst<u32x4>(row.data + (first + i) * row.token);
        const Raw raw = {src[place.first], src[place.second]};
        Angles angles;
        if (place.rotated) angles = angles_of(a, w.pos, half, row_lane);
        return turn<DT, PAIRS>(raw, angles, place.rotated);
    };
    float *scale_at = row.scale + (int64_t)page * a.h.kv_heads;
    const float scale_was = *gconst<float>(scale_at);
    float most = -1.0f;                         // of no token
    bool begins = false;
#pragma unroll 2
    for (int i = mine; i < n; i += round) {
        const Where w = where_is(a, first + i);
        if (w.off < 0) continue;
        const Elements r = elements(i, w);
        most = fmaxf(most, 0.0f);
#pragma unroll
        for (int k = 0; k < 16; ++k) most = fmaxf(most, fabsf(r.x[k]));
        begins |= w.off == 0;
    }
    most = max_quarters(max_halves(over_lanes<16>(most)));
    begins = __any(begins);
    if (lane == 0) lds.most[wave] = most, lds.begins[wave] = begins;
    __syncthreads();                            // and every wave has read the scale
    for (int w = wave0; w < wave0 + waves; ++w) most = fmaxf(most, lds.most[w]), begins |= lds.begins[w];

    const bool some = most >= 0.0f;             // not all of the page's tokens are left out
    const bool limited = most > Code<DT>::kMost;
    const int before = begins ? kLeastExponent : exponent_of(scale_was), e = max(exponent_for(fminf(most, Code<DT>::kMost)), before);
    char *codes = row.codes + page * a.cache.page_bytes;
    if (some && !begins && e > before) rescale(codes, a.cache.page_size * D, before - e, (wave - wave0) * 64 + lane, waves * 64);
    __syncthreads();

    const float by = power_of_two(-e), scale = power_of_two(e);
    uint32_t least[8], largest[8];              // of codes' values, in pairs: fp16 holds them
#pragma unroll
    for (int k = 0; k < 8; ++k) least[k] = 0x7c007c00u, largest[k] = 0xfc00fc00u;
    for (int i = mine; i < n; i += round) {
        const Where w = where_is(a, first + i);
        if (w.off < 0) continue;
        Elements r = elements(i, w);
        if (limited)
#pragma unroll
            for (int k = 0; k < 16; ++k) r.x[k] = within<DT>(r.x[k]);
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            const u32x2 c = encode8(r.x + 8 * v, by);
            *gmut<u32x2>(codes + w.off * D + (v ? place.second : place.first) * 8) = c;
            if (!row.bounds) continue;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t pair = k & 1 ? Code<F16>::pair<true>(c[k >> 1], 1.0f) : Code<F16>::pair<false>(c[k >> 1], 1.0f);
                least[4 * v + k] = extreme<false>(least[4 * v + k], pair);
                largest[4 * v + k] = extreme<true>(largest[4 * v + k], pair);
            }
        }
    }
    if (some && wave == wave0 && lane == 0) *gmut<float>(scale_at) = scale;

    if (row.bounds) {           // every exchange halves what a lane has: 4 of the 16 pairs, 2 of the least and 2 of the largest ones
#pragma unroll
        for (int k = 0; k < 4; ++k) least[k] = of_halves<false>(least[k], least[k + 4]), largest[k] = of_halves<true>(largest[k], largest[k + 4]);
        u32x2 low, high;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            low[k] = over_sixteen<false, kLanes>(of_quarters<false>(least[k], least[k + 2]));
            high[k] = over_sixteen<true, kLanes>(of_quarters<true>(largest[k], largest[k + 2]));
        }
        const int at = (lane < 32 ? place.first : place.second) * 8 + (lane & 16) / 4;
        if (lane % 16 < kLanes) *(u32x2 *)&lds.bounds[wave][at] = low, *(u32x2 *)&lds.bounds[wave][D + at] = high;
    }
    __syncthreads();
    if (row.bounds && some) {
        uint16_t *bounds = row.bounds + (int64_t)page * a.h.kv_heads * 2 * D;
        for (int i = (wave - wave0) * 64 + lane; i < D; i += waves * 64) {      // two neighbours of the 2 D numbers
            const bool high = 2 * i >= D;
            uint32_t x = *(const uint32_t *)&lds.bounds[wave0][2 * i];
            for (int w = wave0 + 1; w < wave0 + waves; ++w) {
                const uint32_t other = *(const uint32_t *)&lds.bounds[w][2 * i];
                x = high ? extreme<true>(x, other) : extreme<false>(x, other);
            }
            const float y[2] = {Elem<F16>::lo(x), Elem<F16>::hi(x)};
            const bool any[2] = {fabsf(y[0]) < __builtin_inff(), fabsf(y[1]) < __builtin_inff()};       // a channel may be all NaN
            float z[2] = {any[0] ? y[0] * scale : 0.0f, any[1] ? y[1] * scale : 0.0f};
            CF_GLOBAL uint32_t *to = gmut<uint32_t>(bounds) + i;
            if (!begins) {
                const uint32_t was = *to;
                const float old[2] = {Elem<BF16>::lo(was), Elem<BF16>::hi(was)};
#pragma unroll
                for (int k = 0; k < 2; ++k) z[k] = !any[k] ? old[k] : high ? fmaxf(z[k], old[k]) : fminf(z[k], old[k]);
            }
            *to = Elem<BF16>::pack(z[0], z[1]);
        }
    }
    __syncthreads();                            // LDS is free
}

template <int DT, int D, bool PAIRS> __global__ __launch_bounds__(kWaves * 64, 5) void k_kv_append8(Append8Args a)
{
    constexpr int kLanes = D / 16, kTokens = 64 / kLanes;
    if (blockIdx.x >= (unsigned)a.page_groups) return rotate_queries<DT, D, PAIRS>(a, blockIdx.x - a.page_groups);
    __shared__ Shared lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // an XCD has neighbouring tokens: where pages begin every so many of them, each XCD has its share
    const uint32_t xcd = blockIdx.x % kXcds, mine = blockIdx.x / kXcds;
    const int rows = 2 * a.h.kv_heads, row_here = (int)(mine % (uint32_t)rows);
    const int64_t begin = ((int64_t)xcd * a.chunks_each + mine / (uint32_t)rows) * a.chunk;

    const int64_t slots_end = (int64_t)a.cache.n_pages << a.cache.page_shift;
    auto page_of = [&](int64_t token) {         // -1: none
        const int64_t slot = token >= 0 && token < a.n_tokens ? gconst<int64_t>(a.slots)[token] : -1;
        return slot < 0 || slot >= slots_end ? -1 : (int)(slot >> a.cache.page_shift);
    };
    uint64_t lone, starts;      // of tokens whose page no neighbour shares; of those that begin neighbours on one page
    int page;
    {
        const bool there = lane < a.chunk;
        page = there ? page_of(begin + lane) : -1;
        const int before = there ? page_of(begin + lane - 1) : -1, behind = there ? page_of(begin + lane + 1) : -1;
        lone = __ballot(page >= 0 && before != page && behind != page);
        starts = __ballot(page >= 0 && before != page && behind == page);
    }
    if (lone && row_here % kWaves == 0 && row_here + wave < rows) {
        const Row row = row_of<D>(a, row_here + wave);
        for (int i = 0; i < a.chunk; i += kTokens) {
            const int at = i + lane / kLanes;
            const int mine = __shfl(page, at & 63);
            store_lone<DT, D, PAIRS>(a, row, begin + at, mine, at < a.chunk && (lone >> at & 1), lane);
        }
    }
    for (; starts != 0; starts &= starts - 1) {
        const int at = __builtin_ctzll(starts);
        const int64_t first = begin + at;
        const int here = __builtin_amdgcn_readlane(page, at);
        int n = 1;                              // tokens that go to this page
        for (;; n += 64) {
            const uint64_t others = __ballot(page_of(first + n + lane) != here);
            if (others) {
                n += __builtin_ctzll(others);
                break;
            }
        }
        const int waves = n <= kTokens ? 1 : n <= 2 * kTokens ? 2 : kWaves;     // of a row
        if (row_here % (kWaves / waves) != 0) continue;                          // it is another workgroup's
        const int row = row_here + wave / waves;
        store_neighbours<DT, D, PAIRS>(a, lds, row_of<D>(a, min(row, rows - 1)), first, row < rows ? n : 0, here, lane, wave, wave / waves * waves, waves);
    }
}

template <int DT, int D> hipError_t append8_dim(const Append8Args &a, hipStream_t s)
{
    const int64_t n = append8_workgroups(a);
    return a.interleaved ? enqueue_of<kAppendThreads>(k_kv_append8<DT, D, true>, n, s, a) : enqueue_of<kAppendThreads>(k_kv_append8<DT, D, false>, n, s, a);
}

template <int DT> hipError_t append8_typed(const Append8Args &a, hipStream_t s)
{
    switch (a.h.head_dim) {
    case 64: return append8_dim<DT, 64>(a, s);
    case 128: return append8_dim<DT, 128>(a, s);
    default: return append8_dim<DT, 256>(a, s);
    }
}

}  // namespace

hipError_t launch_append8(const Append8Args &a, hipStream_t s) { return a.h.dtype == BF16 ? append8_typed<BF16>(a, s) : append8_typed<F16>(a, s); }

}  // namespace attn
}  // namespace cf
