// What the kernels that attend one token of every sequence share: the waves of a workgroup, and the parts of a context, are joined alike
// whatever their keys were held in.
#pragma once

#include "cf_attn_device.h"
#include "compactfusion.h"

namespace cf {
namespace attn {

constexpr int kWaves = 4;

// Parts of a context meet in memory that the L2s of the XCDs do not keep to themselves: words are published and fetched at the
// device's scope, a part's words have landed before it is counted, and the workgroup that counts the last part joins them.  Nobody waits for another.
constexpr int kDeviceScope = 17;        // of buffer instructions: sc0 and sc1, past the L2 of the XCD
__device__ __forceinline__ void publish(float *base, int64_t at, f32x4 x)
{
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), __builtin_amdgcn_make_buffer_rsrc(base, 0, (int)CF_ATTN_WORKSPACE_BYTES, 0x00020000), (int)(at * 4), 0, kDeviceScope);
}
__device__ __forceinline__ void publish(float *base, int64_t at, float x) { __hip_atomic_store((CF_GLOBAL float *)base + at, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void publish_landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ f32x4 fetch4(const float *base, int64_t at)
{
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(__builtin_amdgcn_make_buffer_rsrc((void *)base, 0, (int)CF_ATTN_WORKSPACE_BYTES, 0x00020000), (int)(at * 4), 0, kDeviceScope));
}
__device__ __forceinline__ float fetch(const float *p) { return __hip_atomic_load((const CF_GLOBAL float *)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// The waves' parts are joined by halves: the upper waves hand theirs to the lower ones, in the lanes that hold the same elements.
template <int D> __device__ __forceinline__ void join_waves(float &m, float &l, f32x4 (&o)[D / 16], int lane, int wave)
{
    constexpr int kPer = D / 16;
    __shared__ f32x4 lds_o[kWaves / 2][kPer][64];
    __shared__ f32x2 lds_ml[kWaves / 2][kPagedHeads];
    const int col = lane & 15, quarter = lane >> 4;
    for (int w = kWaves / 2; w > 0; w >>= 1) {
        if (wave >= w && wave < 2 * w) {
#pragma unroll
            for (int d = 0; d < kPer; ++d) lds_o[wave - w][d][lane] = o[d];
            if (quarter == 0) lds_ml[wave - w][col] = (f32x2){m, l};
        }
        __syncthreads();
        if (wave < w) {
            const f32x2 other = lds_ml[wave][col];
            const float top = fmaxf(m, other[0]), mine = exp2_fast(m - top), theirs = exp2_fast(other[0] - top);
            l = __builtin_fmaf(other[1], theirs, l * mine);
            m = top;
#pragma unroll
            for (int d = 0; d < kPer; ++d) {
                const f32x4 x = lds_o[wave][d][lane];
#pragma unroll
                for (int i = 0; i < 4; ++i) o[d][i] = __builtin_fmaf(x[i], theirs, o[d][i] * mine);
            }
        }
        if (w > 1) __syncthreads();
    }
    if (l == 0.0f)              // no key, or none with a score above -infinity: 0 times an infinite value is none of the row's
#pragma unroll
        for (int d = 0; d < kPer; ++d) o[d] = (f32x4){0, 0, 0, 0};
}

// A workgroup's part goes to the output, if it is all of the context; to the other parts in memory, for a kernel of its own (MANY); or there
// until the last one of them, which joins them.  -> whether the workgroup goes on to other parts.
template <int DT, int D, bool MANY>
__device__ __forceinline__ bool finish_part(const PagedArgs &a, int seq, int unit, int units, int kv_head, int head0, int split, int parts, int lane, int wave, float m, float l,
                                            const f32x4 (&o)[D / 16])
{
    using E = Elem<DT>;
    constexpr int kPer = D / 16;
    const int col = lane & 15, quarter = lane >> 4, heads = min(a.h.group - head0, kPagedHeads);
    // lane `col` of the first wave has elements kPer * (4 * quarter + i) + d of its head
    const int head_first = kv_head * a.h.group + head0;
    const int64_t row_first = (int64_t)seq * a.h.q_heads + head_first;
    if (parts <= 1) {
        if (wave != 0 || col >= heads) return true;
        const float inv = inverse_of(l);
        char *dst = a.out.data + (int64_t)seq * a.out.token + (head_first + col) * a.out.head + 8 * kPer * quarter;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int d = 0; d < kPer; d += 4) *gmut<u32x2>(dst + (i * kPer + d) * 2) = (u32x2){E::pack(o[d][i] * inv, o[d + 1][i] * inv), E::pack(o[d + 2][i] * inv, o[d + 3][i] * inv)};
        if (a.lse && quarter == 0) gmut<float>(a.lse)[row_first + col] = lse_of(m, l);
        return true;
    }

    if constexpr (MANY) {
        if (wave != 0 || col >= heads) return true;
        const float inv = inverse_of(l);
        const int64_t row = (int64_t)split * a.parts.n_rows + row_first + col;
        float *dst = a.parts.o + row * D + 4 * kPer * quarter;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int d = 0; d < kPer; d += 4) *gmut<f32x4>(dst + i * kPer + d) = (f32x4){o[d][i] * inv, o[d + 1][i] * inv, o[d + 2][i] * inv, o[d + 3][i] * inv};
        if (quarter == 0) gmut<float>(a.parts.lse)[row] = lse_of(m, l);
    } else {
        __shared__ uint32_t lds_count;
        if (wave == 0) {
            if (col < heads) {
                const float inv = inverse_of(l);
                const int64_t row = (int64_t)split * a.parts.n_rows + row_first + col;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int d = 0; d < kPer; d += 4) publish(a.parts.o, row * D + 4 * kPer * quarter + i * kPer + d, (f32x4){o[d][i] * inv, o[d + 1][i] * inv, o[d + 2][i] * inv, o[d + 3][i] * inv});
                if (quarter == 0) publish(a.parts.lse, row, l > 0.0f || l != l ? m + __log2f(l) : -__builtin_inff());
            }
            publish_landed();
            if (lane == 0) lds_count = __hip_atomic_fetch_add((CF_GLOBAL uint32_t *)a.counters + (int64_t)seq * units + unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (lds_count != (uint32_t)parts - 1) return false;
        if (threadIdx.x == 0) __hip_atomic_store((CF_GLOBAL uint32_t *)a.counters + (int64_t)seq * units + unit, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);

        // What each part weighs for each head: 16 lanes a head, four parts a lane.
        __shared__ float lds_w[kMaxParts][kPagedHeads];
        static_assert(kMaxParts == 64 && kPagedHeads * 16 == kWaves * 64, "a lane has four parts of one head");
        {
            const int head = threadIdx.x >> 4, first = threadIdx.x & 15;
            float lse[4], top = -__builtin_inff(), total = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                lse[i] = -__builtin_inff();
                if (head < heads && first + 16 * i < parts) lse[i] = fetch(a.parts.lse + (int64_t)(first + 16 * i) * a.parts.n_rows + row_first + head);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, lse[i]);
#pragma unroll
            for (int i = 1; i < 16; i <<= 1) top = fmaxf(top, __shfl_xor(top, i));
            const float base = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
            for (int i = 0; i < 4; ++i) total += exp2_fast(lse[i] - base);
#pragma unroll
            for (int i = 1; i < 16; i <<= 1) total += __shfl_xor(total, i);
            const float inv = inverse_of(total);
#pragma unroll
            for (int i = 0; i < 4; ++i) lds_w[first + 16 * i][head] = exp2_fast(lse[i] - base) * inv;
            if (a.lse && first == 0 && head < heads) gmut<float>(a.lse)[row_first + head] = lse_of(base, total);
        }
        __syncthreads();
        // Four elements a lane; where there are fewer than lanes, `shares` lanes have every shares-th part each and their sums meet in LDS, in order.
        __shared__ float lds_sum[kWaves * 64][4];
        const int columns = heads * (D / 4), shares = max(kWaves * 64 / columns, 1);
        for (int n = threadIdx.x; n < max(columns * shares, kWaves * 64); n += kWaves * 64) {
            const int column = n % columns, share = n / columns, head = column / (D / 4), e = column % (D / 4) * 4;
            f32x4 x = {0, 0, 0, 0};
            if (share < shares)
                for (int p0 = share; p0 < parts; p0 += 16 * shares) {
                    f32x4 v[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = p0 + i * shares < parts ? fetch4(a.parts.o, ((p0 + i * shares) * a.parts.n_rows + row_first + head) * D + e) : (f32x4){0, 0, 0, 0};
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float w = lds_w[min(p0 + i * shares, kMaxParts - 1)][head];
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[j] = __builtin_fmaf(w, v[i][j], x[j]);
                    }
                }
            if (shares > 1) {
                *(f32x4 *)lds_sum[threadIdx.x] = x;
                __syncthreads();
                for (int i = 1; i < shares && share == 0; ++i) x += *(const f32x4 *)lds_sum[column + i * columns];
            }
            if (share == 0) *gmut<u32x2>(a.out.data + (int64_t)seq * a.out.token + (head_first + head) * a.out.head + e * 2) = (u32x2){E::pack(x[0], x[1]), E::pack(x[2], x[3])};
        }
    }
    return true;
}

}  // namespace attn
}  // namespace cf
