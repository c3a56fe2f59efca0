// Attention of one new token per sequence over a paged cache: every cached key and value is read once, by one
// workgroup, straight into registers in the layouts that the matrix instructions take; nothing is staged.
//
// A wave takes 32 keys at a time.  S^T = K Q^T in two products of 16 keys by 16 heads; which key is which row
// of them is chosen so that a lane's 8 scores are those of 8 neighbouring keys, the right operand of O^T = V^T P^T.
// For the left one a lane reads 8 (4, 16) elements of the same 8 keys and turns that block with byte permutes.
#include "cf_attn_device.h"

namespace cf {
namespace attn {
namespace {

constexpr int kWaves = 4;
constexpr int kKeys = 32;           // of a wave's step

template <int DT, int D> __global__ __launch_bounds__(kWaves * 64) void k_attn_paged(PagedArgs a)
{
    using E = Elem<DT>;
    constexpr int kSteps = D / 32;      // matrix instructions over the head dimension
    constexpr int kPer = D / 16;        // elements of a value row that a lane reads
    constexpr int kRow = D * 2;         // bytes of a row
    constexpr int kWords = kPer / 2;
    __shared__ float lds_o[kWaves][kPagedHeads][D + 4];
    __shared__ float lds_m[kWaves][kPagedHeads], lds_l[kWaves][kPagedHeads];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quarter = lane >> 4;
    const int head_tiles = (a.h.group + kPagedHeads - 1) / kPagedHeads;
    const int units = a.h.kv_heads * head_tiles;
    const int unit = blockIdx.x % units, rest = blockIdx.x / units;
    const int kv_head = unit / head_tiles, head0 = (unit % head_tiles) * kPagedHeads;
    const int seq = rest / a.n_splits, split = rest % a.n_splits;
    const int heads = min(a.h.group - head0, kPagedHeads);

    const int64_t capacity = min((int64_t)a.max_pages << a.cache.page_shift, (int64_t)1 << 30);
    int len = max(gconst<int32_t>(a.lens)[seq], 0);
    if (len > capacity) len = (int)capacity;
    const int64_t begin64 = (int64_t)split * a.split_keys;
    const int begin = begin64 < len ? (int)begin64 : len;
    const int end = split == a.n_splits - 1 ? len : min(len, begin + a.split_keys);

    float m = kNoMax, l = 0.0f;
    f32x4 o[kPer];
    for (int d = 0; d < kPer; ++d) o[d] = (f32x4){0, 0, 0, 0};

    if (begin < end) {
        const int head = kv_head * a.h.group + head0 + min(col, heads - 1);
        u32x4 q[kSteps];
        for (int i = 0; i < kSteps; ++i) q[i] = *gconst<u32x4>(a.q.data + (int64_t)seq * a.q.token + head * a.q.head + i * 64 + quarter * 16);

        const float c = a.h.scale_log2;
        const CF_GLOBAL int32_t *table = gconst<int32_t>(a.table) + seq * a.table_stride;
        const int64_t head_bytes = (int64_t)kv_head * a.cache.page_size * kRow;
        const char *k_head = a.cache.k + head_bytes, *v_head = a.cache.v + head_bytes;
        const int mask = a.cache.page_size - 1, last = end - 1;

        for (int key0 = begin + wave * kKeys; key0 < end; key0 += kWaves * kKeys) {
            // a step's first and second 16 keys are on one page each; keys past the end read the last one again
            const int page_a = min(max(table[min(key0, last) >> a.cache.page_shift], 0), a.cache.n_pages - 1);
            const int page_b = min(max(table[min(key0 + 16, last) >> a.cache.page_shift], 0), a.cache.n_pages - 1);
            const int64_t at_a = page_a * a.cache.page_bytes, at_b = page_b * a.cache.page_bytes;

            u32x4 k[2][kSteps];
            for (int t = 0; t < 2; ++t) {
                const int off = min(key0 + 8 * (col >> 2) + 4 * t + (col & 3), last) & mask;
                const char *src = k_head + (col >= 8 ? at_b : at_a) + off * kRow + quarter * 16;
                for (int i = 0; i < kSteps; ++i) k[t][i] = *gconst<u32x4>(src + i * 64);
            }
            uint32_t v[8][kWords];
            for (int j = 0; j < 8; ++j) {
                const int off = min(key0 + 8 * quarter + j, last) & mask;
                const char *src = v_head + (quarter >= 2 ? at_b : at_a) + off * kRow + col * (kPer * 2);
                if constexpr (kPer == 4) {
                    const u32x2 x = *gconst<u32x2>(src);
                    v[j][0] = x[0], v[j][1] = x[1];
                } else {
                    for (int w = 0; w < kWords; w += 4) {
                        const u32x4 x = *gconst<u32x4>(src + w * 4);
                        v[j][w] = x[0], v[j][w + 1] = x[1], v[j][w + 2] = x[2], v[j][w + 3] = x[3];
                    }
                }
            }

            f32x4 s[2];
            for (int t = 0; t < 2; ++t) {
                s[t] = (f32x4){0, 0, 0, 0};
                for (int i = 0; i < kSteps; ++i) s[t] = E::mfma16(k[t][i], q[i], s[t]);
            }
            const int most = end - key0 - 8 * quarter;
            float top = -__builtin_inff();
            for (int j = 0; j < 8; ++j) {
                if (j >= most) s[j >> 2][j & 3] = -__builtin_inff();
                top = fmaxf(top, s[j >> 2][j & 3]);
            }
            top *= c;
            if (__any(top > m + kMaxSlack)) {
                const float fresh = fmaxf(m, max_quarters(max_halves(top))), scale = exp2_fast(m - fresh);
                for (int d = 0; d < kPer; ++d)
                    for (int i = 0; i < 4; ++i) o[d][i] *= scale;
                l *= scale;
                m = fresh;
            }
            u32x4 p;
            for (int j = 0; j < 8; j += 2) {
                const float p0 = exp2_fast(__builtin_fmaf(s[j >> 2][j & 3], c, -m)), p1 = exp2_fast(__builtin_fmaf(s[j >> 2][(j & 3) + 1], c, -m));
                l += p0 + p1;
                p[j >> 1] = E::pack(p0, p1);
            }
            for (int d = 0; d < kPer; ++d) {
                u32x4 x;        // element d of this lane's 8 keys
                for (int j = 0; j < 4; ++j) x[j] = __builtin_amdgcn_perm(v[2 * j + 1][d >> 1], v[2 * j][d >> 1], d & 1 ? 0x07060302 : 0x05040100);
                o[d] = E::mfma16(x, p, o[d]);
            }
        }
        l = sum_quarters(sum_halves(l));
    }

    // the waves' parts: element (head, kPer * (4 * quarter + i) + d) is o[d][i] of the lanes with col = head
    if (quarter == 0) lds_m[wave][col] = m, lds_l[wave][col] = l;
    for (int i = 0; i < 4; ++i)
        for (int d = 0; d < kPer; d += 4)
            *(f32x4 *)&lds_o[wave][col][kPer * (4 * quarter + i) + d] = (f32x4){o[d][i], o[d + 1][i], o[d + 2][i], o[d + 3][i]};
    __syncthreads();
    constexpr int kVecs = D / 8;
    for (int n = threadIdx.x; n < heads * kVecs; n += kWaves * 64) {
        const int h = n / kVecs, e = (n % kVecs) * 8;
        float top = kNoMax;
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, lds_m[w][h]);
        float total = 0.0f, x[8] = {};
        for (int w = 0; w < kWaves; ++w) {
            const float f = exp2_fast(lds_m[w][h] - top);
            total = __builtin_fmaf(lds_l[w][h], f, total);
            for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf(lds_o[w][h][e + i], f, x[i]);
        }
        const float inv = inverse_of(total);
        const int head = kv_head * a.h.group + head0 + h;
        const int64_t row = (int64_t)seq * a.h.q_heads + head;
        if (a.n_splits > 1) {
            CF_GLOBAL f32x4 *dst = gmut<f32x4>(a.parts.o + ((int64_t)split * a.parts.n_rows + row) * D + e);
            dst[0] = (f32x4){x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
            dst[1] = (f32x4){x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv};
            if (e == 0) gmut<float>(a.parts.lse)[(int64_t)split * a.parts.n_rows + row] = lse_of(top, total);
        } else {
            u32x4 r;
            for (int i = 0; i < 4; ++i) r[i] = E::pack(x[2 * i] * inv, x[2 * i + 1] * inv);
            *gmut<u32x4>(a.out.data + (int64_t)seq * a.out.token + head * a.out.head + e * 2) = r;
            if (a.lse && e == 0) gmut<float>(a.lse)[row] = lse_of(top, total);
        }
    }
}

template <int DT> hipError_t paged_typed(const PagedArgs &a, hipStream_t s)
{
    const unsigned grid = (unsigned)((int64_t)a.n_seqs * a.n_splits * a.h.kv_heads * ((a.h.group + kPagedHeads - 1) / kPagedHeads));
    switch (a.h.head_dim) {
    case 64: hipLaunchKernelGGL((k_attn_paged<DT, 64>), dim3(grid), dim3(kWaves * 64), 0, s, a); break;
    case 128: hipLaunchKernelGGL((k_attn_paged<DT, 128>), dim3(grid), dim3(kWaves * 64), 0, s, a); break;
    default: hipLaunchKernelGGL((k_attn_paged<DT, 256>), dim3(grid), dim3(kWaves * 64), 0, s, a); break;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged(const PagedArgs &a, hipStream_t s) { return a.h.dtype == BF16 ? paged_typed<BF16>(a, s) : paged_typed<F16>(a, s); }

}  // namespace attn
}  // namespace cf
