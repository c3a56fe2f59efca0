// What the attention entry points check of their arguments, and how parts are laid out in a workspace.  Host code.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "cf_attn.h"
#include "compactfusion.h"

namespace cf {
namespace attn {

constexpr int64_t kMostStride = (int64_t)1 << 24;       // elements: a tile's rows are addressed with 32 bits
constexpr int64_t kMostRows = (int64_t)1 << 30;
constexpr int64_t kMostSpan = (int64_t)1 << 60;         // bytes that a cache or a table spans
constexpr int64_t kCUs = 256;
constexpr int64_t kCounters = CF_ATTN_COUNTER_BYTES / sizeof(uint32_t);

inline bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

inline cf_status check_desc(const cf_attn_desc *d, Heads &h)
{
    if (!d) return CF_ERR_INVALID_ARG;
    if (d->dtype != CF_BF16 && d->dtype != CF_F16) return CF_ERR_UNSUPPORTED;
    if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256) return CF_ERR_UNSUPPORTED;
    if (d->kv_heads < 1 || d->q_heads < 1 || d->q_heads > 65536 || d->q_heads % d->kv_heads != 0) return CF_ERR_SHAPE;
    if (!(d->scale >= 0.0f) || !(d->scale <= 2.0e38f)) return CF_ERR_INVALID_ARG;      // times log2 e it is finite
    h.dtype = d->dtype;
    h.q_heads = d->q_heads;
    h.kv_heads = d->kv_heads;
    h.group = d->q_heads / d->kv_heads;
    h.head_dim = d->head_dim;
    const double scale = d->scale > 0.0f ? (double)d->scale : 1.0 / sqrt((double)d->head_dim);
    h.scale_log2 = (float)(scale * 1.4426950408889634);
    return CF_OK;
}

// A span of memory: `width` bytes for each of `heads` heads of `tokens` tokens, which lie so many bytes apart.
struct Span {
    uintptr_t at;
    int64_t tokens, token, heads, head, width;
    uintptr_t end() const { return at + (uintptr_t)((tokens - 1) * token + (heads - 1) * head + width); }
    // All of it, seen modulo a step that its strides are multiples of or do not reach.
    int64_t modulo(int64_t step) const { return width + (token % step == 0 ? 0 : (tokens - 1) * token) + (head % step == 0 ? 0 : (heads - 1) * head); }
};

// Whether two spans may share a byte.  Spans that lie side by side within a stride of theirs, token by token or head by head, do not.
inline bool meet(const Span &a, const Span &b)
{
    if (a.tokens < 1 || b.tokens < 1 || a.end() <= b.at || b.end() <= a.at) return false;
    for (const int64_t step : {a.token, a.head, b.token, b.head}) {
        if (step < 1) continue;
        const int64_t behind = (int64_t)((b.at > a.at ? b.at - a.at : a.at - b.at) % (uintptr_t)step), off = b.at >= a.at ? behind : (step - behind) % step;
        if (off >= a.modulo(step) && off + b.modulo(step) <= step) return false;
    }
    return true;
}

// Rows of `heads` heads of `tokens` tokens.  `least`: the least stride from token to token that the kernels take.
inline cf_status check_rows(const cf_rows &in, int64_t tokens, int64_t heads, int64_t dim, bool output, int64_t least, Rows &out, Span &span)
{
    int64_t token = in.token, head = in.head;
    if (!in.data || !aligned(in.data, 16)) return CF_ERR_INVALID_ARG;
    if (heads == 1) head = dim;             // strides that no element goes by
    if (tokens == 1) token = dim;
    if (token < 0 || head < 0 || token % 8 != 0 || head % 8 != 0 || token >= kMostStride || head >= kMostStride) return CF_ERR_SHAPE;
    if (tokens > 1 && token < least) return CF_ERR_SHAPE;
    if (output) {
        const bool by_token = head >= dim && (tokens == 1 || token >= (heads - 1) * head + dim);
        const bool by_head = token >= dim && (heads == 1 || head >= (tokens - 1) * token + dim);
        if (!by_token && !by_head) return CF_ERR_INVALID_ARG;
    }
    out.data = static_cast<char *>(in.data);
    out.token = token * 2;
    out.head = head * 2;
    span = {reinterpret_cast<uintptr_t>(in.data), tokens, out.token, heads, out.head, dim * 2};
    return CF_OK;
}

inline cf_status check_cache(const cf_kv_cache *c, const Heads &h, Cache &out, Span &k, Span &v)
{
    if (!c) return CF_ERR_INVALID_ARG;
    if (!c->k || !c->v || !aligned(c->k, 16) || !aligned(c->v, 16)) return CF_ERR_INVALID_ARG;
    if (c->page_size < 16 || c->page_size > 32768 || (c->page_size & (c->page_size - 1)) != 0) return CF_ERR_SHAPE;
    if (c->n_pages < 1 || c->n_pages > INT32_MAX) return CF_ERR_SHAPE;
    const int64_t dense = (int64_t)h.kv_heads * c->page_size * h.head_dim;
    const int64_t stride = c->page_stride ? c->page_stride : dense;
    if (stride < dense || stride % 8 != 0 || stride > ((int64_t)1 << 40) || c->n_pages > kMostSpan / 2 / stride) return CF_ERR_SHAPE;
    out.k = static_cast<char *>(c->k);
    out.v = static_cast<char *>(c->v);
    out.page_bytes = stride * 2;
    out.n_pages = (int32_t)c->n_pages;
    out.page_size = c->page_size;
    out.page_shift = __builtin_ctz((unsigned)c->page_size);
    k = {reinterpret_cast<uintptr_t>(c->k), c->n_pages, stride * 2, 1, 0, dense * 2};
    v = k;
    v.at = reinterpret_cast<uintptr_t>(c->v);
    return meet(k, v) ? CF_ERR_INVALID_ARG : CF_OK;
}

inline cf_status check_workspace(const void *workspace, size_t bytes)
{
    if (bytes > 0 && !workspace) return CF_ERR_WORKSPACE;
    return aligned(workspace, 256) ? CF_OK : CF_ERR_WORKSPACE;
}

// How many parts of `rows` rows fit the workspace, behind the counters.
inline int64_t parts_that_fit(size_t bytes, int64_t rows, int dim)
{
    if (bytes > CF_ATTN_WORKSPACE_BYTES) bytes = CF_ATTN_WORKSPACE_BYTES;
    return bytes > CF_ATTN_COUNTER_BYTES ? (int64_t)(bytes - CF_ATTN_COUNTER_BYTES) / (rows * (dim + 1) * (int64_t)sizeof(float)) : 0;
}

inline void place_parts(Parts &p, void *workspace, int64_t rows, int64_t n, int dim)
{
    p.o = reinterpret_cast<float *>(static_cast<char *>(workspace) + CF_ATTN_COUNTER_BYTES);
    p.lse = p.o + n * rows * dim;
    p.n_rows = rows;
}

inline cf_status status_of(hipError_t e) { return e == hipSuccess ? CF_OK : CF_ERR_DEVICE; }

inline JoinArgs parts_to_join(const Heads &h, const Parts &p, int n, const Rows &out, float *lse)
{
    JoinArgs j = {};
    j.h = h;
    j.out = out;
    j.lse = lse;
    j.n_rows = p.n_rows;
    j.n_parts = n;
    j.part_dtype = CF_F32;
    for (int i = 0; i < n; ++i) {
        j.parts[i] = p.o + i * p.n_rows * h.head_dim;
        j.lses[i] = p.lse + i * p.n_rows;
    }
    return j;
}

inline int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

}  // namespace attn
}  // namespace cf
