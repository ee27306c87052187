// Host side of the paged cache (wkv_paged in include/wkv.h): argument checks, workspace layout, launches.
// Nothing here computes attention, sums or evictions: wkv_paged.hip and wkv_evict.hip do.
#include "../../include/wkv.h"
#include "wkv_internal.h"

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

namespace {

int fail(int code, const char* fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return wkv_set_error(code, buf);
}

int elem_bytes(int dtype) { return dtype == WKV_FP32 ? 4 : 2; }
bool aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Everything but the pointers.
int check_shape(const wkv_paged& c)
{
    if (c.batch <= 0 || c.heads <= 0 || c.kv_heads <= 0) return fail(WKV_EINVAL, "batch, heads and kv_heads must be positive");
    if (c.heads % c.kv_heads != 0) return fail(WKV_EINVAL, "heads %d is no multiple of kv_heads %d", c.heads, c.kv_heads);
    if ((int64_t)c.batch * c.heads > (1 << 24)) return fail(WKV_ESIZE, "batch*heads exceeds 2^24");
    if (c.dtype != WKV_FP32 && c.dtype != WKV_FP16 && c.dtype != WKV_BF16)
        return fail(WKV_EINVAL, "dtype must be WKV_FP32, WKV_FP16 or WKV_BF16");
    const bool d_ok = c.head_dim == 64 || c.head_dim == 128 || (c.head_dim == 256 && c.dtype != WKV_FP32);
    if (!d_ok) return fail(WKV_EINVAL, "head_dim %d unsupported for this dtype (64, 128; 256 for 16-bit)", c.head_dim);
    if (c.page_size < 16 || c.page_size > 4096 || (c.page_size & (c.page_size - 1)) != 0)
        return fail(WKV_EINVAL, "page_size %d is no power of two in 16..4096", c.page_size);
    if (c.n_pages < 1 || c.max_pages < 1) return fail(WKV_EINVAL, "n_pages and max_pages must be positive");
    if ((int64_t)c.max_pages * c.page_size > (1 << 24)) return fail(WKV_ESIZE, "max_pages*page_size exceeds 2^24 slots");
    if (c.window < 0 || c.n_sink < 0) return fail(WKV_EINVAL, "window and n_sink must be >= 0");
    for (int r : c.reserved) if (r != 0) return fail(WKV_EINVAL, "reserved fields must be zero");
    if (c.scores && (c.score_stride <= (int64_t)(c.max_pages - 1) * c.page_size || c.score_stride > (int64_t)c.max_pages * c.page_size))
        return fail(WKV_EINVAL, "score_stride %lld: a row of sums ends within the last of %d pages of %d slots", (long long)c.score_stride,
                    c.max_pages, c.page_size);
    return WKV_OK;
}

// A chunk's sizes: rows and their bytes are counted in 32 bits per unit.
int check_chunk(const wkv_paged& c, int n_tokens, int max_new)
{
    if (max_new > 1 << 24) return fail(WKV_ESIZE, "max_new %d exceeds 2^24, the most slots of a sequence", max_new);
    if ((int64_t)n_tokens * c.heads > 1 << 30) return fail(WKV_ESIZE, "n_tokens*heads exceeds 2^30");
    return WKV_OK;
}

int check(const wkv_paged* c)
{
    if (!c) return fail(WKV_EINVAL, "null argument");
    const int rc = check_shape(*c);
    if (rc != WKV_OK) return rc;
    if (!c->k || !c->v || !c->table || !c->lens) return fail(WKV_EINVAL, "null device pointer");
    if (!aligned(c->k) || !aligned(c->v)) return fail(WKV_EINVAL, "the pools must be 16-byte aligned");
    if (((uintptr_t)c->table | (uintptr_t)c->lens | (uintptr_t)c->scores) & 3) return fail(WKV_EINVAL, "table, lens and scores must be 4-byte aligned");
    const int64_t unit = 16 / elem_bytes(c->dtype);
    if (c->page_stride < 0 || c->slot_stride < 0 || c->head_stride < 0 || (c->page_stride | c->slot_stride | c->head_stride) % unit != 0)
        return fail(WKV_EINVAL, "strides of the pools must be multiples of 16 bytes and not negative");
    if (c->slot_stride * elem_bytes(c->dtype) > 1 << 26) return fail(WKV_ESIZE, "slot_stride exceeds 2^26 bytes");
    if (c->table_stride < c->max_pages) return fail(WKV_EINVAL, "table_stride %lld is below max_pages %d", (long long)c->table_stride, c->max_pages);
    return WKV_OK;
}

WkvPages pages_of(const wkv_paged& p)
{
    const int64_t eb = elem_bytes(p.dtype);
    WkvPages c;
    c.k = (char*)p.k; c.v = (char*)p.v;
    c.page_bytes = p.page_stride * eb; c.slot_bytes = p.slot_stride * eb; c.head_bytes = p.head_stride * eb;
    c.table = p.table; c.table_stride = p.table_stride; c.lens = p.lens;
    c.scores = p.scores; c.score_stride = p.score_stride;
    c.batch = p.batch; c.kv_heads = p.kv_heads; c.group = p.heads / p.kv_heads;
    c.page_shift = __builtin_ctz((unsigned)p.page_size);
    c.n_pages = p.n_pages; c.max_pages = p.max_pages;
    c.max_slots = p.max_pages * p.page_size;
    if (p.scores) c.max_slots = (int)std::min<int64_t>(c.max_slots, p.score_stride);
    c.window = std::min(p.window, 1 << 25);          // (twice the most slots: what a position before slot 0 is further back stays in 32 bits)
    c.n_sink = p.n_sink;
    return c;
}

// Workspace of an attention call: each piece at a multiple of 256 bytes.
struct Layout {
    WkvPagedCall shape = {};
    size_t part = 0, ml = 0, logits = 0, lse = 0, colsums = 0, total = 0;
};

Layout layout(const wkv_paged& p, bool scores, int n_tokens, int max_new, bool step)
{
    const WkvPages c = pages_of(p);
    const int64_t units = (int64_t)c.batch * c.kv_heads;
    Layout l;
    const int64_t rows = (int64_t)max_new * c.group;
    l.shape.c = c;
    l.shape.n_tokens = n_tokens;
    l.shape.max_new = max_new;
    wkv_paged_shape(l.shape, units, rows, wkv_paged_most_keys(c, std::min(max_new, 128 / c.group + 2)), p.dtype, p.head_dim, step);
    auto take = [&](size_t bytes) { const size_t at = l.total; l.total += (bytes + 255) / 256 * 256; return at; };
    const int splits = l.shape.splits;
    const size_t cells = (size_t)units * l.shape.tiles * splits;
    if (splits > 1) l.part = take(cells * 16 * p.head_dim * sizeof(float));
    if (splits > 1 || (scores && step)) l.ml = take(cells * 32 * sizeof(float));
    l.shape.logit_stride = (c.max_slots + 31) / 32 * 32;
    l.shape.row_parts = scores && !step && p.dtype != WKV_FP32 ? wkv_paged_row_parts(units, c.max_slots, rows) : 1;
    if (scores && step) l.logits = take((size_t)units * c.group * l.shape.logit_stride * sizeof(float));
    if (scores && !step) l.lse = take((size_t)n_tokens * p.heads * sizeof(float));
    if (l.shape.row_parts > 1) l.colsums = take((size_t)l.shape.row_parts * units * l.shape.logit_stride * sizeof(float));
    return l;
}

size_t evict_bytes(const wkv_paged& p, int budget)
{
    return ((size_t)p.batch * 8 + 255) / 256 * 256 + (size_t)p.batch * p.kv_heads * budget * sizeof(int32_t);
}

// A launch of 2^32 threads and more is not refused by the runtime: the count wraps.
int check_launch(const WkvPagedCall& a)
{
    // (room for tiles of chunks of different lengths: half of what a launch holds)
    const int64_t groups = wkv_paged_groups(a);
    if (groups >= (a.slots ? 1 << 23 : 1 << 24))
        return fail(WKV_ESIZE, "%lld workgroups of 256 threads: a launch holds fewer than 2^32 threads", (long long)groups);
    return WKV_OK;
}

int check_work(const void* workspace, size_t have, size_t need)
{
    if (need == 0) return WKV_OK;
    if (!workspace) return fail(WKV_EINVAL, "null workspace");
    if (!aligned(workspace)) return fail(WKV_EINVAL, "the workspace must be 16-byte aligned");
    if (have < need) return fail(WKV_ESIZE, "the workspace needs %zu bytes, got %zu", need, have);
    return WKV_OK;
}

// What step and prefill have in common, up to the launches.
int attend(const wkv_paged* p, const wkv_paged_rows* r, const int32_t* starts, int n_tokens, int max_new, void* workspace, size_t workspace_bytes, hipStream_t stream)
{
    int rc = check(p);
    if (rc != WKV_OK) return rc;
    if (!r) return fail(WKV_EINVAL, "null argument");
    if (!r->q || !r->out || (!r->k) != (!r->v)) return fail(WKV_EINVAL, "null device pointer");
    if (!aligned(r->q) || !aligned(r->k) || !aligned(r->v) || !aligned(r->out)) return fail(WKV_EINVAL, "q, k, v and out must be 16-byte aligned");
    const int64_t eb = elem_bytes(p->dtype), unit = 16 / eb;
    const int64_t strides[] = {r->q_stride, r->q_head_stride, r->out_stride, r->out_head_stride, r->k ? r->k_stride : 0, r->k ? r->k_head_stride : 0,
                               r->v ? r->v_stride : 0, r->v ? r->v_head_stride : 0};
    for (int64_t s : strides)
        if (s < 0 || s % unit != 0) return fail(WKV_EINVAL, "strides of rows must be multiples of 16 bytes and not negative");
    if (r->k && std::max(r->k_stride, r->v_stride) * eb > 1 << 26) return fail(WKV_ESIZE, "k_stride and v_stride must not exceed 2^26 bytes");
    if ((n_tokens > 1 && r->out_stride < p->head_dim) || (p->heads > 1 && r->out_head_stride < p->head_dim))
        return fail(WKV_EINVAL, "rows of out must not overlap");
    const bool step = starts == nullptr;
    rc = check_chunk(*p, n_tokens, max_new);
    if (rc != WKV_OK) return rc;
    const Layout l = layout(*p, p->scores != nullptr, n_tokens, max_new, step);
    rc = check_launch(l.shape);
    if (rc != WKV_OK) return rc;
    rc = check_work(workspace, workspace_bytes, l.total);
    if (rc != WKV_OK) return rc;
    WkvPagedCall a = l.shape;
    a.c = pages_of(*p);
    a.q = (const char*)r->q; a.k_new = (const char*)r->k; a.v_new = (const char*)r->v; a.out = (char*)r->out;
    a.q_bytes = r->q_stride * eb; a.k_bytes = r->k_stride * eb; a.v_bytes = r->v_stride * eb; a.out_bytes = r->out_stride * eb;
    a.q_head = r->q_head_stride * eb; a.k_head = r->k_head_stride * eb; a.v_head = r->v_head_stride * eb; a.out_head = r->out_head_stride * eb;
    a.starts = starts; a.n_tokens = n_tokens; a.max_new = max_new;
    a.scale = (float)(1.4426950408889634 / std::sqrt((double)p->head_dim));
    char* w = (char*)workspace;
    if (a.splits > 1) a.part = (float*)(w + l.part);
    if (a.splits > 1 || (p->scores && step)) a.ml = (float*)(w + l.ml);
    if (p->scores && step) a.logits = (float*)(w + l.logits);
    if (p->scores && !step) a.lse = (float*)(w + l.lse);
    if (a.row_parts > 1) a.colsums = (float*)(w + l.colsums);
    const int64_t units = (int64_t)p->batch * p->kv_heads;
    if (a.logits && units * ((a.c.max_slots + 1023) / 1024) >= (1 << 23) - (1 << 16))
        return fail(WKV_ESIZE, "%lld units of %d slots: a launch holds fewer than 2^32 threads", (long long)units, a.c.max_slots);
    hipError_t e = wkv_launch_paged_attend(a, p->dtype, p->head_dim, stream);
    if (e == hipSuccess && !step && p->scores) e = wkv_launch_paged_sums(a, p->dtype, p->head_dim, stream);
    return e == hipSuccess ? WKV_OK : fail(WKV_EHIP, "kernel launch: %s", hipGetErrorString(e));
}

}  // namespace

extern "C" {

size_t wkv_paged_workspace_bytes(const wkv_paged* c, int n_tokens, int max_new)
{
    if (!c || check_shape(*c) != WKV_OK || n_tokens < 0 || max_new < 0 || max_new > n_tokens || check_chunk(*c, n_tokens, max_new) != WKV_OK) return 0;
    const bool scores = c->scores != nullptr;
    size_t need = std::max(layout(*c, scores, c->batch, 1, true).total, (size_t)256);
    if (max_new > 0) {
        const Layout l = layout(*c, scores, n_tokens, max_new, false);
        if (check_launch(l.shape) != WKV_OK) return 0;
        need = std::max(need, l.total);
    }
    if (scores) need = std::max(need, evict_bytes(*c, pages_of(*c).max_slots));
    return need;
}

int wkv_paged_step(const wkv_paged* c, const wkv_paged_rows* rows, void* workspace, size_t workspace_bytes, void* stream)
{
    return attend(c, rows, nullptr, c ? c->batch : 0, 1, workspace, workspace_bytes, (hipStream_t)stream);
}

int wkv_paged_prefill(const wkv_paged* c, const wkv_paged_rows* rows, const int32_t* starts, int n_tokens, int max_new,
                      void* workspace, size_t workspace_bytes, void* stream)
{
    if (!starts) return fail(WKV_EINVAL, "null device pointer");
    if ((uintptr_t)starts & 3) return fail(WKV_EINVAL, "starts must be 4-byte aligned");
    if (n_tokens < 1 || max_new < 1 || max_new > n_tokens) return fail(WKV_EINVAL, "1 <= max_new <= n_tokens is wanted: %d, %d", max_new, n_tokens);
    return attend(c, rows, starts, n_tokens, max_new, workspace, workspace_bytes, (hipStream_t)stream);
}

int wkv_paged_evict(const wkv_paged* c, int budget, int recent_window, int32_t* new_lens, float* new_scores, int32_t* kept,
                    void* workspace, size_t workspace_bytes, void* stream)
{
    int rc = check(c);
    if (rc != WKV_OK) return rc;
    if (!c->scores) return fail(WKV_EINVAL, "eviction needs scores");
    if (c->window != 0) return fail(WKV_EINVAL, "a cache with a window is not evicted from");
    if (!new_lens || !new_scores) return fail(WKV_EINVAL, "null device pointer");
    if (((uintptr_t)new_lens | (uintptr_t)new_scores | (uintptr_t)kept) & 3) return fail(WKV_EINVAL, "new_lens, new_scores and kept must be 4-byte aligned");
    if (budget < 1 || recent_window < 1 || (int64_t)c->n_sink + recent_window > budget)
        return fail(WKV_EINVAL, "1 <= recent_window and n_sink + recent_window <= budget are wanted: %d, %d, %d", recent_window, c->n_sink, budget);
    const WkvPages p = pages_of(*c);
    if (wkv_evict_groups((int64_t)c->batch * c->kv_heads, c->head_dim * elem_bytes(c->dtype)) >= 1 << 22)
        return fail(WKV_ESIZE, "%d units: a launch holds fewer than 2^32 threads", c->batch * c->kv_heads);
    // (a budget that no sequence can exceed leaves all of them as they are)
    rc = check_work(workspace, workspace_bytes, evict_bytes(*c, std::min(budget, p.max_slots)));
    if (rc != WKV_OK) return rc;
    int32_t* plan = (int32_t*)workspace;
    int32_t* list = (int32_t*)((char*)workspace + ((size_t)c->batch * 8 + 255) / 256 * 256);
    const hipError_t e = wkv_launch_paged_evict(p, c->head_dim * elem_bytes(c->dtype), budget, recent_window, new_lens, new_scores, kept,
                                                plan, list, (hipStream_t)stream);
    return e == hipSuccess ? WKV_OK : fail(WKV_EHIP, "kernel launch: %s", hipGetErrorString(e));
}

}  // extern "C"
