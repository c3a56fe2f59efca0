// Attention of one new token per sequence over a paged cache: every cached key and value is read once for 16 query heads
// that share it (a group of 17 reads it twice), by one workgroup, straight into registers in the layouts that the matrix
// instructions take; nothing is staged.
//
// A wave takes 32 keys at a time.  S^T = K Q^T in two products of 16 keys by 16 heads; which key is which row
// of them is chosen so that a lane's 8 scores are those of 8 neighbouring keys, the right operand of O^T = V^T P^T.
// For the left one a lane reads 8 (4, 16) elements of the same 8 keys and turns that block with byte permutes.
//
// Bound by HBM: 96 contexts of 160 to 16000 keys, 32 / 8 heads of 128, 275 us (5.1 TB/s; sums over rows of 2 GiB, read once, reach 5.9); 2 of 131100, 24 heads
// of 64, 285 us (5.7 TB/s); one of 901 keys, 8 / 2 heads, by latency: 7.6 us, of which the launch is a third.  Through LDS the same bytes would wait for a barrier a step, and the
// products need 16 columns for the one to 16 heads that share keys, whoever brings them.
#include "cf_attn_device.h"
#include "compactfusion.h"

namespace cf {
namespace attn {
namespace {

constexpr int kWaves = 4;
constexpr int kKeys = 32;           // of a wave's step

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

// MANY: as many workgroups as the device holds take the parts of all contexts in turn, which they list from the lengths; a kernel of its
// own joins them.  Otherwise a workgroup per (head unit, sequence, part that there may be), which joins them too.
template <int DT, int D, bool MANY> __global__ __launch_bounds__(kWaves * 64, D == 256 ? 2 : 3) void k_attn_paged(PagedArgs a)
{
    using E = Elem<DT>;
    constexpr int kSteps = D / 32;      // matrix instructions over the head dimension
    constexpr int kPer = D / 16;        // elements of a value row that a lane reads
    constexpr int kRow = D * 2;         // bytes of a row
    constexpr int kWords = kPer / 2;
    __shared__ f32x4 lds_o[kWaves / 2][kPer][64];
    __shared__ f32x2 lds_ml[kWaves / 2][kPagedHeads];
    // Wide queries wait in LDS, each lane's its own, where the listing of parts takes registers too: the loop's operands do not fit with them (40 contexts of
    // 10000 keys, 40 / 8 heads of 256: 595 us for 615).
    constexpr bool kKeepQ = D < 256 || !MANY;
    __shared__ u32x4 lds_q[kKeepQ ? 1 : kWaves][kKeepQ ? 1 : kSteps][64];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quarter = lane >> 4;
    const int head_tiles = (a.h.group + kPagedHeads - 1) / kPagedHeads;
    const int units = a.h.kv_heads * head_tiles;
    const int64_t capacity = min((int64_t)a.max_pages << a.cache.page_shift, (int64_t)1 << 30);
    auto len_of = [&](int seq) { return (int)min((int64_t)max(gconst<int32_t>(a.lens)[seq], 0), capacity); };
    auto parts_of = [&](int len) { return max(min((len + a.split_keys - 1) / a.split_keys, a.n_splits), 1); };    // a context of no keys has an empty one
    __shared__ int lds_upto[MANY ? kMostListed : 1];        // parts of the sequences up to each
    int64_t items = gridDim.x;
    if constexpr (MANY) {
        if (wave == 0) {
            int upto = 0;
            for (int base = 0; base < a.n_seqs; base += 64) {
                int here = base + lane < a.n_seqs ? parts_of(len_of(base + lane)) : 0;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const int below = __shfl_up(here, d);
                    if (lane >= d) here += below;
                }
                if (base + lane < a.n_seqs) lds_upto[base + lane] = upto + here;
                upto += __builtin_amdgcn_readlane(here, 63);
            }
        }
        __syncthreads();
        items = (int64_t)lds_upto[a.n_seqs - 1] * units;
    }
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int unit = (int)(item % units), rest = (int)(item / units);
        const int kv_head = unit / head_tiles, head0 = (unit % head_tiles) * kPagedHeads;
        int seq = rest % a.n_seqs, split = rest / a.n_seqs;
        if constexpr (MANY) {
            int most = a.n_seqs - 1;        // the first sequence with more parts up to it than `rest`
            for (seq = 0; seq < most;) {
                const int middle = (seq + most) >> 1;
                if (lds_upto[middle] > rest) most = middle;
                else seq = middle + 1;
            }
            seq = __builtin_amdgcn_readfirstlane(seq);
            split = __builtin_amdgcn_readfirstlane(rest - (seq > 0 ? lds_upto[seq - 1] : 0));
            __syncthreads();                // LDS of the part before is free
        }
        const int heads = min(a.h.group - head0, kPagedHeads);

        const int len = len_of(seq);
        const int begin = (int)min((int64_t)split * a.split_keys, (int64_t)len);
        const int end = split == a.n_splits - 1 ? len : min(len, begin + a.split_keys);
        const int parts = parts_of(len);
        if (!MANY && split >= parts) return;

        float m = kNoMax, l = 0.0f;
        f32x4 o[kPer];
#pragma unroll
        for (int d = 0; d < kPer; ++d) o[d] = (f32x4){0, 0, 0, 0};

        if (begin < end) {
            u32x4 q[kKeepQ ? kSteps : 1];
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const u32x4 x = *gconst<u32x4>(a.q.data + (int64_t)seq * a.q.token + (kv_head * a.h.group + head0 + min(col, heads - 1)) * a.q.head + i * 64 + quarter * 16);
                if constexpr (kKeepQ) q[i] = x;
                else lds_q[wave][i][lane] = x;
            }

            const float c = a.h.scale_log2;
            // read by scalar loads, though this kernel writes memory: page numbers and addresses in vector registers would push the loop's operands out (595 us
            // for 710, 96 contexts of 160 to 16000 keys, 32 / 8 heads of 128, 272 for 277)
            const CF_CONST int32_t *table = (const CF_CONST int32_t *)a.table + seq * a.table_stride;
            const int64_t head_bytes = (int64_t)kv_head * a.cache.page_size * kRow;
            const char *k_head = a.cache.k + head_bytes, *v_head = a.cache.v + head_bytes;
            const int mask = a.cache.page_size - 1, last = end - 1;

            // Where the first and the second 16 keys of a step begin: each lies on one page.  Numbers past the context are those of its last page.
            struct Step {
                const char *k[2], *v[2];
            };
            auto find = [&](int key0) {
                Step at;
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const int page = min(max(table[min(key0 + 16 * g, last) >> a.cache.page_shift], 0), a.cache.n_pages - 1);
                    const int64_t off = page * a.cache.page_bytes + ((key0 + 16 * g) & mask) * kRow;
                    at.k[g] = k_head + off;
                    at.v[g] = v_head + off;
                }
                return at;
            };
            u32x4 k[2][kSteps];
            auto load_k = [&](const Step &at, int key0) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int x = min(8 * (col >> 2) + 4 * t + (col & 3), last - key0);        // keys past the end: the last one again
                    const char *src = (x >= 16 ? at.k[1] : at.k[0]) + (x & 15) * kRow + quarter * 16;
#pragma unroll
                    for (int i = 0; i < kSteps; ++i) k[t][i] = *gconst<u32x4>(src + i * 64);
                }
            };
            uint32_t v[8][kWords];
            auto load_v = [&](const Step &at, int key0) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int x = min(8 * quarter + j, last - key0);
                    const char *src = (x >= 16 ? at.v[1] : at.v[0]) + (x & 15) * kRow + col * (kPer * 2);
                    if constexpr (kPer == 4) {
                        const u32x2 y = *gconst<u32x2>(src);
                        v[j][0] = y[0], v[j][1] = y[1];
                    } else {
#pragma unroll
                        for (int w = 0; w < kWords; w += 4) {
                            const u32x4 y = *gconst<u32x4>(src + w * 4);
                            v[j][w] = y[0], v[j][w + 1] = y[1], v[j][w + 2] = y[2], v[j][w + 3] = y[3];
                        }
                    }
                }
            };

            // K of the next step is asked for as soon as this one's is used up, V of this one before that.
            int key0 = begin + wave * kKeys;
            Step at = find(key0);
            if (key0 < end) load_k(at, key0);
            while (key0 < end) {
                if constexpr (!kKeepQ) asm volatile("" ::: "memory");     // read them again in every step
                const int next0 = key0 + kWaves * kKeys;
                const Step next = find(next0);
                load_v(at, key0);
                __builtin_amdgcn_sched_barrier(0);
                f32x4 s[2];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    s[t] = (f32x4){0, 0, 0, 0};
#pragma unroll
                    for (int i = 0; i < kSteps; ++i) {
                        if constexpr (kKeepQ) s[t] = E::mfma16(k[t][i], q[i], s[t]);
                        else s[t] = E::mfma16(k[t][i], lds_q[wave][i][lane], s[t]);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                if (next0 < end) load_k(next, next0);
                __builtin_amdgcn_sched_barrier(0);
                const int most = end - key0 - 8 * quarter;
                float top = -__builtin_inff();
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (j >= most) s[j >> 2][j & 3] = -__builtin_inff();
                    top = fmaxf(top, s[j >> 2][j & 3]);
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
                if (key0 + kKeys > end) {       // the last key's value, read again for keys past it, may be infinite: 0 times it is not 0
#pragma unroll
                    for (int j = 0; j < 8; ++j)
#pragma unroll
                        for (int w = 0; w < kWords; ++w) v[j][w] = j < most ? v[j][w] : 0u;
                }
                u32x4 p;        // scaled scores are rounded as their maximum was: of scores of any size the largest has the weight 1
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const float p0 = exp2_fast(s[j >> 2][j & 3] * c - m), p1 = exp2_fast(s[j >> 2][(j & 3) + 1] * c - m);
                    l += p0 + p1;
                    p[j >> 1] = E::pack(p0, p1);
                }
#pragma unroll
                for (int d = 0; d < kPer; ++d) {
                    u32x4 x;        // element d of this lane's 8 keys
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = __builtin_amdgcn_perm(v[2 * j + 1][d >> 1], v[2 * j][d >> 1], d & 1 ? 0x07060302 : 0x05040100);
                    o[d] = E::mfma16(x, p, o[d]);
                }
                key0 = next0;
                at = next;
            }
            l = sum_quarters(sum_halves(l));
        }

        // The waves' parts are joined by halves: the upper waves hand theirs to the lower ones, in the lanes that hold the same elements.
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

        // lane `col` of the first wave has elements kPer * (4 * quarter + i) + d of its head
        const int head_first = kv_head * a.h.group + head0;
        const int64_t row_first = (int64_t)seq * a.h.q_heads + head_first;
        if (parts <= 1) {
            if (wave != 0 || col >= heads) continue;
            const float inv = inverse_of(l);
            char *dst = a.out.data + (int64_t)seq * a.out.token + (head_first + col) * a.out.head + 8 * kPer * quarter;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int d = 0; d < kPer; d += 4) *gmut<u32x2>(dst + (i * kPer + d) * 2) = (u32x2){E::pack(o[d][i] * inv, o[d + 1][i] * inv), E::pack(o[d + 2][i] * inv, o[d + 3][i] * inv)};
            if (a.lse && quarter == 0) gmut<float>(a.lse)[row_first + col] = lse_of(m, l);
            continue;
        }

        if constexpr (MANY) {
            if (wave != 0 || col >= heads) continue;
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
            if (lds_count != (uint32_t)parts - 1) return;
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
    }
}

template <int DT, int D> hipError_t paged_dim(const PagedArgs &a, hipStream_t s)
{
    return a.many ? enqueue(k_attn_paged<DT, D, true>, paged_workgroups(a), s, a) : enqueue(k_attn_paged<DT, D, false>, paged_workgroups(a), s, a);
}

template <int DT> hipError_t paged_typed(const PagedArgs &a, hipStream_t s)
{
    switch (a.h.head_dim) {
    case 64: return paged_dim<DT, 64>(a, s);
    case 128: return paged_dim<DT, 128>(a, s);
    default: return paged_dim<DT, 256>(a, s);
    }
}

}  // namespace

hipError_t launch_paged(const PagedArgs &a, hipStream_t s) { return a.h.dtype == BF16 ? paged_typed<BF16>(a, s) : paged_typed<F16>(a, s); }

}  // namespace attn
}  // namespace cf
