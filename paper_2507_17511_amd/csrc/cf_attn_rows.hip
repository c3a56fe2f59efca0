// Row-wise kernels next to the attentions: appending to the paged cache with the rotation of positions, and the
// join of attentions over parts of the keys.  Both move each byte once and compute next to nothing: they are bound by
// HBM, and by their launch where they are small: 16384 tokens of 24 + 2 x 8 heads of 128 appended in 64 us (5.3 TB/s), 48 tokens of 32 + 2 x 8 in 3.5;
// 4 bf16 parts of 98304 rows of 128 joined in 22 us (5.8 TB/s, of which caches hold a part), 64 parts of 48 rows of 64 in 6.
#include "cf_attn_device.h"

namespace cf {
namespace attn {
namespace {

// ---------------------------------------------------------------- append
//
// A lane moves 16 elements of one head's row as two vectors of 16 bytes: vectors that hold the two halves of 8 pairs
// where pairs lie rotary_dim / 2 apart, neighbouring ones otherwise.  Rows of a token: the queries' heads, then the
// keys', then the values'; head_dim / 16 lanes each.
template <int DT, int D> __global__ __launch_bounds__(256) void k_kv_append(AppendArgs a)
{
    constexpr int kLanes = D / 16;
    const int q_heads = a.q.data ? a.h.q_heads : 0;
    const int rows = q_heads + 2 * a.h.kv_heads;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t token = id / (rows * kLanes);
    if (token >= a.n_tokens) return;
    const int rest = (int)(id - token * (rows * kLanes));
    const int lane = rest % kLanes;
    int head = rest / kLanes;

    const int half = a.rotary_dim >> 1;
    int pos = 0;
    if (half) {
        pos = gconst<int32_t>(a.positions)[token];
        if (pos < 0 || pos >= a.n_positions) return;
    }
    const char *src;
    char *dst;
    bool rotate = half != 0;
    if (head < q_heads) {
        src = a.q.data + token * a.q.token + head * a.q.head;
        dst = a.q_out.data + token * a.q_out.token + head * a.q_out.head;
    } else {
        head -= q_heads;
        const int64_t slot = gconst<int64_t>(a.slots)[token];
        if (slot < 0 || slot >= (int64_t)a.cache.n_pages << a.cache.page_shift) return;
        const bool value = head >= a.h.kv_heads;
        if (value) {
            head -= a.h.kv_heads;
            rotate = false;
        }
        const Rows &r = value ? a.v : a.k;
        src = r.data + token * r.token + head * r.head;
        dst = (value ? a.cache.v : a.cache.k) + (slot >> a.cache.page_shift) * a.cache.page_bytes +
              ((int64_t)head * a.cache.page_size + (slot & (a.cache.page_size - 1))) * (D * 2);
    }
    // which two vectors: lane n of the rotated ones has vectors n and n + half / 8 of a row whose pairs lie apart
    const int pair_lanes = half >> 3;
    const bool apart = rotate && !a.interleaved && lane < pair_lanes;
    const int first = apart ? lane : 2 * lane;
    const int second = apart ? lane + pair_lanes : first + 1;
    const u32x4 x = gconst<u32x4>(src)[first], y = gconst<u32x4>(src)[second];
    u32x4 u = x, w = y;
    if (apart) {
        const CF_GLOBAL f32x4 *c = gconst<f32x4>(a.cos + (int64_t)pos * half + lane * 8), *s = gconst<f32x4>(a.sin + (int64_t)pos * half + lane * 8);
        const f32x4 cs[2] = {c[0], c[1]}, sn[2] = {s[0], s[1]};
        for (int k = 0; k < 4; ++k) {
            const float c0 = cs[k >> 1][2 * (k & 1)], c1 = cs[k >> 1][2 * (k & 1) + 1], s0 = sn[k >> 1][2 * (k & 1)], s1 = sn[k >> 1][2 * (k & 1) + 1];
            const float a0 = Elem<DT>::lo(x[k]), a1 = Elem<DT>::hi(x[k]), b0 = Elem<DT>::lo(y[k]), b1 = Elem<DT>::hi(y[k]);
            u[k] = Elem<DT>::pack(a0 * c0 - b0 * s0, a1 * c1 - b1 * s1);
            w[k] = Elem<DT>::pack(b0 * c0 + a0 * s0, b1 * c1 + a1 * s1);
        }
    } else if (rotate && a.interleaved && lane < pair_lanes) {
        const CF_GLOBAL f32x4 *c = gconst<f32x4>(a.cos + (int64_t)pos * half + lane * 8), *s = gconst<f32x4>(a.sin + (int64_t)pos * half + lane * 8);
        const f32x4 cs[2] = {c[0], c[1]}, sn[2] = {s[0], s[1]};
        for (int k = 0; k < 4; ++k) {
            const float a0 = Elem<DT>::lo(x[k]), b0 = Elem<DT>::hi(x[k]), a1 = Elem<DT>::lo(y[k]), b1 = Elem<DT>::hi(y[k]);
            u[k] = Elem<DT>::pack(a0 * cs[0][k] - b0 * sn[0][k], b0 * cs[0][k] + a0 * sn[0][k]);
            w[k] = Elem<DT>::pack(a1 * cs[1][k] - b1 * sn[1][k], b1 * cs[1][k] + a1 * sn[1][k]);
        }
    }
    gmut<u32x4>(dst)[first] = u;
    gmut<u32x4>(dst)[second] = w;
}

// ---------------------------------------------------------------- join
//
// SPREAD lanes share 8 elements of a row; each has every SPREAD-th part, EACH at most, and asks for all of them at once, log-sum-exps and
// outputs.  The largest log-sum-exp and the sums meet in LDS, by a tree, so that the order is the same in every call.
template <int DT, int PT, int D, int SPREAD, int EACH> __global__ __launch_bounds__(256) void k_attn_join(JoinArgs a)
{
    constexpr int kLanes = D / 8;                       // of a row
    constexpr int kRows = 256 / (kLanes * SPREAD);      // of a workgroup
    static_assert(kRows >= 1, "a workgroup has a row at least");
    const int row_here = threadIdx.x / (kLanes * SPREAD), share = threadIdx.x / kLanes % SPREAD, lane = threadIdx.x % kLanes;
    const int64_t row = (int64_t)blockIdx.x * kRows + row_here;
    const int64_t token = (row < a.n_rows ? row : 0) / a.h.q_heads;
    const int n_parts = a.lens ? (int)max(min((gconst<int32_t>(a.lens)[token] + (int64_t)a.split_keys - 1) / a.split_keys, (int64_t)a.n_parts), (int64_t)1) : a.n_parts;
    const bool there = row < a.n_rows && !(a.lens && n_parts == 1);
    float lse[EACH], top = -__builtin_inff(), total = 0.0f, o[8] = {};
    f32x4 x[EACH][2];
    if (there) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int p = share + i * SPREAD;
            lse[i] = -__builtin_inff();
            if (p < n_parts) {
                lse[i] = gconst<float>(a.lses[p])[row];
                if constexpr (PT == 0) {
                    const CF_GLOBAL f32x4 *src = gconst<f32x4>(static_cast<const float *>(a.parts[p]) + row * D + lane * 8);
                    x[i][0] = src[0], x[i][1] = src[1];
                } else {
                    const u32x4 v = *gconst<u32x4>(static_cast<const uint16_t *>(a.parts[p]) + row * D + lane * 8);
                    x[i][0] = (f32x4){Elem<DT>::lo(v[0]), Elem<DT>::hi(v[0]), Elem<DT>::lo(v[1]), Elem<DT>::hi(v[1])};
                    x[i][1] = (f32x4){Elem<DT>::lo(v[2]), Elem<DT>::hi(v[2]), Elem<DT>::lo(v[3]), Elem<DT>::hi(v[3])};
                }
            }
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i) top = fmaxf(top, lse[i]);
    }
    __shared__ float sums[SPREAD > 1 ? 256 : 1][9];
    if constexpr (SPREAD > 1) {
        sums[threadIdx.x][8] = top;
        for (int w = SPREAD / 2; w > 0; w >>= 1) {
            __syncthreads();
            if (share < w) sums[threadIdx.x][8] = top = fmaxf(top, sums[threadIdx.x + w * kLanes][8]);
        }
        __syncthreads();
        top = sums[threadIdx.x - share * kLanes][8];
        __syncthreads();
    }
    const float base = top == -__builtin_inff() ? 0.0f : top;
    if (there) {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (lse[i] != -__builtin_inff()) {          // of other parts the output is not read
                const float w = exp2_fast((lse[i] - base) * 1.44269504088896341f);
                total += w;
#pragma unroll
                for (int k = 0; k < 8; ++k) o[k] = __builtin_fmaf(w, x[i][k >> 2][k & 3], o[k]);
            }
    }
    if constexpr (SPREAD > 1) {
        for (int k = 0; k < 8; ++k) sums[threadIdx.x][k] = o[k];
        sums[threadIdx.x][8] = total;
        for (int w = SPREAD / 2; w > 0; w >>= 1) {
            __syncthreads();
            if (share < w) {
                for (int k = 0; k < 8; ++k) sums[threadIdx.x][k] = o[k] += sums[threadIdx.x + w * kLanes][k];
                sums[threadIdx.x][8] = total += sums[threadIdx.x + w * kLanes][8];
            }
        }
        if (share > 0) return;
    }
    if (!there) return;
    if (a.cover && (token < gconst<int32_t>(a.cover)[0] || token >= gconst<int32_t>(a.cover)[a.n_cover])) return;
    const float inv = inverse_of(total);
    u32x4 r;
    for (int k = 0; k < 4; ++k) r[k] = Elem<DT>::pack(o[2 * k] * inv, o[2 * k + 1] * inv);
    const int head = (int)(row - token * a.h.q_heads);
    gmut<u32x4>(a.out.data + token * a.out.token + head * a.out.head)[lane] = r;
    if (a.lse && lane == 0) gmut<float>(a.lse)[row] = total > 0.0f || total != total ? base + __log2f(total) * kLn2 : -__builtin_inff();
}

template <int DT, int PT, int D, int SPREAD, int EACH> hipError_t join_over(const JoinArgs &a, hipStream_t s)
{
    return enqueue(k_attn_join<DT, PT, D, SPREAD, EACH>, join_workgroups(a), s, a);
}

template <int DT, int PT, int D> hipError_t join_dim(const JoinArgs &a, hipStream_t s)
{
    constexpr int kMost = join_spread(kMaxParts, D);
    static_assert(join_spread(8, D) == 1 && join_spread(16, D) == 4 && kMost * (kMaxParts / kMost) == kMaxParts, "the lanes have all parts");
    if (a.n_parts <= 4) return join_over<DT, PT, D, 1, 4>(a, s);
    if (a.n_parts <= 8) return join_over<DT, PT, D, 1, 8>(a, s);
    if (a.n_parts <= 16) return join_over<DT, PT, D, 4, 4>(a, s);
    return join_over<DT, PT, D, kMost, kMaxParts / kMost>(a, s);
}

template <int DT, int PT> hipError_t join_typed(const JoinArgs &a, hipStream_t s)
{
    switch (a.h.head_dim) {
    case 64: return join_dim<DT, PT, 64>(a, s);
    case 128: return join_dim<DT, PT, 128>(a, s);
    default: return join_dim<DT, PT, 256>(a, s);
    }
}

template <int DT> hipError_t append_typed(const AppendArgs &a, hipStream_t s)
{
    const int64_t n = append_workgroups(a);
    switch (a.h.head_dim) {
    case 64: return enqueue(k_kv_append<DT, 64>, n, s, a);
    case 128: return enqueue(k_kv_append<DT, 128>, n, s, a);
    default: return enqueue(k_kv_append<DT, 256>, n, s, a);
    }
}

}  // namespace

hipError_t launch_join(const JoinArgs &a, hipStream_t s)
{
    if (a.h.dtype == BF16) return a.part_dtype == BF16 ? join_typed<BF16, BF16>(a, s) : join_typed<BF16, 0>(a, s);
    return a.part_dtype == F16 ? join_typed<F16, F16>(a, s) : join_typed<F16, 0>(a, s);
}

hipError_t launch_append(const AppendArgs &a, hipStream_t s) { return a.h.dtype == BF16 ? append_typed<BF16>(a, s) : append_typed<F16>(a, s); }

}  // namespace attn
}  // namespace cf
