// Keys and values into the paged cache of 8-bit codes, rotated on the way, and the queries' rotation.
//
// What a call's tokens bring to one page is one piece of work for each head of keys and of values: their largest magnitude decides the scale.  Such
// tokens are neighbours in the call, so that a wave finds where they begin by looking at the slots alone: WAVES waves take the pages that begin among
// `chunk` tokens, read their rows once (up to kKeep rounds of them stay in registers), agree on the scale, and store the codes.  Everything is read and
// written once, and the call is bound by HBM, or by its launch where it is small.
#include "cf_attn8_device.h"

namespace cf {
namespace attn {
namespace {

constexpr int kKeep = 4;        // rounds of rows that wait in registers for their scale

// 16 elements of a row: two vectors of 8, which hold the two halves of 8 pairs where pairs lie rotary_dim / 2 apart.
struct Place {
    int first, second;
    bool apart, rotated;
};
__device__ __forceinline__ Place place_of(int lane, int half, bool interleaved)
{
    Place p;
    const int lanes = half >> 3;
    p.rotated = lane < lanes;
    p.apart = p.rotated && !interleaved;
    p.first = p.apart ? lane : 2 * lane;
    p.second = p.apart ? lane + lanes : p.first + 1;
    return p;
}

template <int DT> __device__ __forceinline__ void turn(u32x4 x, u32x4 y, const Place &p, const float *cos, const float *sin, float (&r)[16])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        r[2 * k] = Elem<DT>::lo(x[k]), r[2 * k + 1] = Elem<DT>::hi(x[k]);
        r[8 + 2 * k] = Elem<DT>::lo(y[k]), r[8 + 2 * k + 1] = Elem<DT>::hi(y[k]);
    }
    if (!p.rotated) return;
    const CF_GLOBAL f32x4 *c = gconst<f32x4>(cos), *s = gconst<f32x4>(sin);
    const f32x4 cs[2] = {c[0], c[1]}, sn[2] = {s[0], s[1]};
    if (p.apart) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float a = r[k], b = r[8 + k], co = cs[k >> 2][k & 3], si = sn[k >> 2][k & 3];
            r[k] = a * co - b * si;
            r[8 + k] = b * co + a * si;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float a = r[2 * k], b = r[2 * k + 1], co = cs[k >> 2][k & 3], si = sn[k >> 2][k & 3];
            r[2 * k] = a * co - b * si;
            r[2 * k + 1] = b * co + a * si;
        }
    }
}

template <int DT, int D> __device__ __forceinline__ void rotate_queries(const Append8Args &a, int64_t id)
{
    constexpr int kLanes = D / 16;
    const int64_t token = id / (a.h.q_heads * kLanes);
    if (token >= a.n_tokens) return;
    const int rest = (int)(id - token * (a.h.q_heads * kLanes)), lane = rest % kLanes, head = rest / kLanes, half = a.rotary_dim >> 1;
    int pos = 0;
    if (half) {
        pos = gconst<int32_t>(a.positions)[token];
        if (pos < 0 || pos >= a.n_positions) return;
    }
    const Place p = place_of(lane, half, a.interleaved);
    const CF_GLOBAL u32x4 *src = gconst<u32x4>(a.q.data + token * a.q.token + head * a.q.head);
    float r[16];
    const int64_t at = (int64_t)pos * half + lane * 8;
    turn<DT>(src[p.first], src[p.second], p, a.cos + at, a.sin + at, r);
    CF_GLOBAL u32x4 *dst = gmut<u32x4>(a.q_out.data + token * a.q_out.token + head * a.q_out.head);
    u32x4 u, w;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        u[k] = Elem<DT>::pack(r[2 * k], r[2 * k + 1]);
        w[k] = Elem<DT>::pack(r[8 + 2 * k], r[8 + 2 * k + 1]);
    }
    dst[p.first] = u;
    dst[p.second] = w;
}

template <int DT, int D, int WAVES> __global__ __launch_bounds__(256) void k_kv_append8(Append8Args a)
{
    constexpr int kLanes = D / 16;              // of a row
    constexpr int kTokens = 64 / kLanes;        // of a wave's round
    constexpr int kRound = kTokens * WAVES;
    if (blockIdx.x >= (unsigned)a.page_groups) return rotate_queries<DT, D>(a, (int64_t)(blockIdx.x - a.page_groups) * 256 + threadIdx.x);
    __shared__ float lds_most[WAVES > 1 ? WAVES : 1];
    __shared__ bool lds_begins[WAVES > 1 ? WAVES : 1];
    __shared__ float lds_bounds[WAVES > 1 ? WAVES : 1][kLanes][32];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row_lane = lane % kLanes;
    const int share = WAVES > 1 ? wave : 0;     // of a page's rows
    const int64_t item = WAVES > 1 ? blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
    const int rows = 2 * a.h.kv_heads, head = (int)(item % rows) % a.h.kv_heads;
    const bool value = (int)(item % rows) >= a.h.kv_heads;
    const int64_t begin = item / rows * a.chunk;
    if (begin >= a.n_tokens) return;            // the whole workgroup, where its waves share pages

    const int half = a.rotary_dim >> 1;
    const Place place = place_of(row_lane, value ? 0 : half, a.interleaved);
    const Rows &in = value ? a.v : a.k;
    const int64_t slots_end = (int64_t)a.cache.n_pages << a.cache.page_shift;
    auto page_of = [&](int64_t token) {         // -1: none
        const int64_t slot = gconst<int64_t>(a.slots)[token];
        return slot < 0 || slot >= slots_end ? -1 : (int)(slot >> a.cache.page_shift);
    };
    uint64_t starts;
    {
        const int64_t token = begin + lane;
        const int page = lane < a.chunk && token < a.n_tokens ? page_of(token) : -1;
        starts = __ballot(page >= 0 && (token == 0 || page_of(token - 1) != page));
    }
    for (; starts != 0; starts &= starts - 1) {
        const int64_t first = begin + __builtin_ctzll(starts);
        const int page = __builtin_amdgcn_readfirstlane(page_of(first));
        int64_t n = 0;                          // tokens that go to this page
        for (;; n += 64) {
            const int64_t token = first + n + lane;
            const uint64_t others = __ballot(token >= a.n_tokens || page_of(token) != page);
            if (others) {
                n += __builtin_ctzll(others);
                break;
            }
        }

        // Rows are read as they are, then rotated: all of the kept ones are on their way together.
        u32x4 raw[kKeep][2];
        int off[kKeep], pos[kKeep];             // off < 0: not there, or left out
        auto locate = [&](int64_t i, int &off, int &pos) {
            const int64_t token = first + i;
            off = -1, pos = 0;
            if (i >= n) return;
            if (half) pos = gconst<int32_t>(a.positions)[token];
            if (half && (pos < 0 || pos >= a.n_positions)) return;
            off = (int)(gconst<int64_t>(a.slots)[token] & (a.cache.page_size - 1));
        };
        auto fetch_rows = [&](int64_t i, u32x4 (&x)[2]) {
            const CF_GLOBAL u32x4 *src = gconst<u32x4>(in.data + (first + i) * in.token + head * in.head);
            x[0] = src[place.first], x[1] = src[place.second];
        };
        auto finish_rows = [&](const u32x4 (&x)[2], int pos, float (&r)[16]) {
            const int64_t at = (int64_t)pos * half + row_lane * 8;
            turn<DT>(x[0], x[1], place, a.cos + at, a.sin + at, r);
#pragma unroll
            for (int k = 0; k < 16; ++k) r[k] = r[k] > Code<DT>::kMost ? Code<DT>::kMost : r[k] < -Code<DT>::kMost ? -Code<DT>::kMost : r[k];      // NaN stays
        };
        const int mine = share * kTokens + lane / kLanes;       // a lane's row of a round
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            off[i] = -1;
            if (i * kRound < n) locate(i * kRound + mine, off[i], pos[i]);
            if (off[i] >= 0) fetch_rows(i * kRound + mine, raw[i]);
        }
        float x[kKeep][16], most = -1.0f;
        bool begins = false;
#pragma unroll
        for (int i = 0; i < kKeep; ++i)
            if (off[i] >= 0) {
                finish_rows(raw[i], pos[i], x[i]);
                most = fmaxf(most, 0.0f);
#pragma unroll
                for (int k = 0; k < 16; ++k) most = fmaxf(most, fabsf(x[i][k]));
                begins |= off[i] == 0;
            }
        for (int64_t i = kKeep * kRound + mine; i - mine < n; i += kRound) {        // those that are read twice
            int off, pos;
            locate(i, off, pos);
            if (off < 0) continue;
            u32x4 y[2];
            float r[16];
            fetch_rows(i, y);
            finish_rows(y, pos, r);
            most = fmaxf(most, 0.0f);
#pragma unroll
            for (int k = 0; k < 16; ++k) most = fmaxf(most, fabsf(r[k]));
            begins |= off == 0;
        }
        most = max_quarters(max_halves(most));
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) most = fmaxf(most, __shfl_xor(most, d));
        begins = __any(begins);
        if constexpr (WAVES > 1) {
            __syncthreads();                    // what the page before left there has been read
            if (lane == 0) lds_most[wave] = most, lds_begins[wave] = begins;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WAVES; ++w) most = fmaxf(most, lds_most[w]), begins |= lds_begins[w];
        }
        if (most < 0.0f) continue;              // all of the page's tokens are left out

        float *scale_at = (value ? a.cache.v_scale : a.cache.k_scale) + (int64_t)page * a.h.kv_heads + head;
        const int before = begins ? kLeastExponent : exponent_of(*gconst<float>(scale_at));
        const int e = max(exponent_for(most), before);
        char *codes = (value ? a.cache.v : a.cache.k) + page * a.cache.page_bytes + (int64_t)head * a.cache.page_size * D;
        if (!begins && e > before) {            // the other places' codes go by the new scale; places of this call are written behind them
            const float by = power_of_two(max(before - e, -126));
            for (int i = (share * 64 + lane) * 16; i < a.cache.page_size * D; i += 64 * WAVES * 16) {
                u32x4 w = *gconst<u32x4>(codes + i);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const auto low = __builtin_amdgcn_cvt_pk_f32_fp8(w[k], false), high = __builtin_amdgcn_cvt_pk_f32_fp8(w[k], true);
                    w[k] = encode4(low[0] * by, low[1] * by, high[0] * by, high[1] * by);
                }
                *gmut<u32x4>(codes + i) = w;
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        if constexpr (WAVES > 1) __syncthreads();       // and every wave has read the scale

        const float by = power_of_two(-e), scale = power_of_two(e);
        const bool bounded = a.cache.bounds && !value;
        float low[16], high[16];                // of codes
#pragma unroll
        for (int k = 0; k < 16; ++k) low[k] = __builtin_inff(), high[k] = -__builtin_inff();
        auto store = [&](const float (&r)[16], int off) {
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                u32x2 w;
#pragma unroll
                for (int k = 0; k < 2; ++k) w[k] = encode4(r[8 * v + 4 * k] * by, r[8 * v + 4 * k + 1] * by, r[8 * v + 4 * k + 2] * by, r[8 * v + 4 * k + 3] * by);
                *gmut<u32x2>(codes + off * D + (v ? place.second : place.first) * 8) = w;
                if (bounded)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const auto y = k & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(w[k >> 1], true) : __builtin_amdgcn_cvt_pk_f32_fp8(w[k >> 1], false);
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const float z = y[j] == y[j] ? y[j] : 0.0f;
                            low[8 * v + 2 * k + j] = fminf(low[8 * v + 2 * k + j], z);
                            high[8 * v + 2 * k + j] = fmaxf(high[8 * v + 2 * k + j], z);
                        }
                    }
            }
        };
#pragma unroll
        for (int i = 0; i < kKeep; ++i)
            if (off[i] >= 0) store(x[i], off[i]);
        for (int64_t i = kKeep * kRound + mine; i - mine < n; i += kRound) {
            int off, pos;
            locate(i, off, pos);
            if (off < 0) continue;
            u32x4 y[2];
            float r[16];
            fetch_rows(i, y);
            finish_rows(y, pos, r);
            store(r, off);
        }
        if (share == 0 && lane == 0) *gmut<float>(scale_at) = scale;
        if (!bounded) continue;

        // the rows' bounds meet in the first row's lanes
        if (n > 1) {
#pragma unroll
            for (int d = kLanes; d < 64; d <<= 1)
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    low[k] = fminf(low[k], __shfl_xor(low[k], d));
                    high[k] = fmaxf(high[k], __shfl_xor(high[k], d));
                }
        }
        if constexpr (WAVES > 1) {
            if (lane < kLanes)
#pragma unroll
                for (int k = 0; k < 16; ++k) lds_bounds[wave][lane][k] = low[k], lds_bounds[wave][lane][16 + k] = high[k];
            __syncthreads();
            if (wave > 0) continue;             // to the barrier that the next page begins with
            if (lane < kLanes)
#pragma unroll
                for (int w = 1; w < WAVES; ++w)
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        low[k] = fminf(low[k], lds_bounds[w][lane][k]);
                        high[k] = fmaxf(high[k], lds_bounds[w][lane][16 + k]);
                    }
        }
        if (lane < kLanes) {
            uint16_t *least = a.cache.bounds + ((int64_t)page * a.h.kv_heads + head) * 2 * D;
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                const int at = v ? place.second : place.first;
                u32x4 lo, hi;
                const u32x4 lo_was = begins ? (u32x4){0, 0, 0, 0} : gconst<u32x4>(least)[at], hi_was = begins ? (u32x4){0, 0, 0, 0} : gconst<u32x4>(least + D)[at];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float l0 = low[8 * v + 2 * k] * scale, l1 = low[8 * v + 2 * k + 1] * scale, h0 = high[8 * v + 2 * k] * scale, h1 = high[8 * v + 2 * k + 1] * scale;
                    if (!begins) {
                        l0 = fminf(l0, Elem<BF16>::lo(lo_was[k])), l1 = fminf(l1, Elem<BF16>::hi(lo_was[k]));
                        h0 = fmaxf(h0, Elem<BF16>::lo(hi_was[k])), h1 = fmaxf(h1, Elem<BF16>::hi(hi_was[k]));
                    }
                    lo[k] = Elem<BF16>::pack(l0, l1);
                    hi[k] = Elem<BF16>::pack(h0, h1);
                }
                gmut<u32x4>(least)[at] = lo;
                gmut<u32x4>(least + D)[at] = hi;
            }
        }
    }
}

template <int DT, int D> hipError_t append8_dim(const Append8Args &a, hipStream_t s)
{
    const int64_t n = append8_workgroups(a);
    return a.chunk > 1 ? enqueue(k_kv_append8<DT, D, 4>, n, s, a) : enqueue(k_kv_append8<DT, D, 1>, n, s, a);
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
