// Row-wise kernels next to the attentions: appending to the paged cache with the rotation of positions, and the
// join of attentions over parts of the keys.  Both move each byte once and compute next to nothing: they are bound by
// HBM, and by their launch where they are small.
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
// A lane has 8 elements of a row and computes that row's weights for itself: the log-sum-exps of a row are read by the
// lanes of that row together, and from the cache after the first.
template <int DT, int PT, int D> __global__ __launch_bounds__(256) void k_attn_join(JoinArgs a)
{
    constexpr int kLanes = D / 8;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = id / kLanes;
    if (row >= a.n_rows) return;
    const int lane = (int)(id % kLanes);
    const int64_t token = row / a.h.q_heads;
    if (a.cover && (token < gconst<int32_t>(a.cover)[0] || token >= gconst<int32_t>(a.cover)[a.n_cover])) return;
    float top = -__builtin_inff();
    for (int p = 0; p < a.n_parts; ++p) top = fmaxf(top, gconst<float>(a.lses[p])[row]);
    const float base = top == -__builtin_inff() ? 0.0f : top;
    float total = 0.0f, o[8] = {};
    for (int p = 0; p < a.n_parts; ++p) {
        const float lse = gconst<float>(a.lses[p])[row];
        if (lse == -__builtin_inff()) continue;
        const float w = exp2_fast((lse - base) * 1.44269504088896341f);
        total += w;
        if constexpr (PT == 0) {
            const CF_GLOBAL f32x4 *src = gconst<f32x4>(static_cast<const float *>(a.parts[p]) + row * D + lane * 8);
            const f32x4 x = src[0], y = src[1];
            for (int k = 0; k < 4; ++k) {
                o[k] = __builtin_fmaf(w, x[k], o[k]);
                o[4 + k] = __builtin_fmaf(w, y[k], o[4 + k]);
            }
        } else {
            const u32x4 x = *gconst<u32x4>(static_cast<const uint16_t *>(a.parts[p]) + row * D + lane * 8);
            for (int k = 0; k < 4; ++k) {
                o[2 * k] = __builtin_fmaf(w, Elem<DT>::lo(x[k]), o[2 * k]);
                o[2 * k + 1] = __builtin_fmaf(w, Elem<DT>::hi(x[k]), o[2 * k + 1]);
            }
        }
    }
    const float inv = inverse_of(total);
    u32x4 r;
    for (int k = 0; k < 4; ++k) r[k] = Elem<DT>::pack(o[2 * k] * inv, o[2 * k + 1] * inv);
    const int head = (int)(row - token * a.h.q_heads);
    gmut<u32x4>(a.out.data + token * a.out.token + head * a.out.head)[lane] = r;
    if (a.lse && lane == 0) gmut<float>(a.lse)[row] = total > 0.0f || total != total ? base + __log2f(total) * kLn2 : -__builtin_inff();
}

template <int DT, int PT> hipError_t join_typed(const JoinArgs &a, hipStream_t s)
{
    const unsigned grid = (unsigned)((a.n_rows * (a.h.head_dim / 8) + 255) / 256);
    switch (a.h.head_dim) {
    case 64: hipLaunchKernelGGL((k_attn_join<DT, PT, 64>), dim3(grid), dim3(256), 0, s, a); break;
    case 128: hipLaunchKernelGGL((k_attn_join<DT, PT, 128>), dim3(grid), dim3(256), 0, s, a); break;
    default: hipLaunchKernelGGL((k_attn_join<DT, PT, 256>), dim3(grid), dim3(256), 0, s, a); break;
    }
    return hipGetLastError();
}

template <int DT> hipError_t append_typed(const AppendArgs &a, hipStream_t s)
{
    const int64_t rows = (a.q.data ? a.h.q_heads : 0) + 2 * a.h.kv_heads;
    const unsigned grid = (unsigned)((a.n_tokens * rows * (a.h.head_dim / 16) + 255) / 256);
    switch (a.h.head_dim) {
    case 64: hipLaunchKernelGGL((k_kv_append<DT, 64>), dim3(grid), dim3(256), 0, s, a); break;
    case 128: hipLaunchKernelGGL((k_kv_append<DT, 128>), dim3(grid), dim3(256), 0, s, a); break;
    default: hipLaunchKernelGGL((k_kv_append<DT, 256>), dim3(grid), dim3(256), 0, s, a); break;
    }
    return hipGetLastError();
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
