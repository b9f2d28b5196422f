// cb_serve_api.cpp -- host side of the calls that serve a receiver from pages
// (include/cachebridge.h): arguments are checked here, before anything is
// enqueued.  No call allocates, reads the device or waits.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "cb_serve_internal.h"

namespace {

cb_status fail(cb_status s, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return cb::api_error(s, buf);
}

cb::Strides strides_of(const cb_cache &c) { return {c.s_layer, c.s_kv, c.s_seq, c.s_head, c.s_tok}; }

cb_status check_width(int d) {
    if (d < 16 || d > 256 || d % 16) return fail(CB_ERR_UNSUPPORTED, "head_dim must be a multiple of 16 up to 256 (got %d)", d);
    return CB_OK;
}

cb_status check_pages(const cb_pages *p) {
    if (!p) return fail(CB_ERR_INVALID_ARGUMENT, "pages is NULL");
    const cb_cache &c = p->cache;
    if (p->dtype != CB_PAGES_BF16 && p->dtype != CB_PAGES_E4M3)
        return fail(CB_ERR_INVALID_ARGUMENT, "pages: unknown dtype %d", p->dtype);
    if (c.n_layers <= 0 || c.n_heads <= 0 || c.n_seqs <= 0 || c.seq_len <= 0)
        return fail(CB_ERR_SHAPE, "pages needs positive layer, head, page and page size counts");
    if (cb_status s = cb::api_check_cache("pages", &c, c.n_layers, c.n_heads, c.head_dim)) return s;
    const int el = p->dtype == CB_PAGES_E4M3 ? 1 : 2;
    if (el == 1) {
        const int64_t st[5] = {c.s_layer, c.s_kv, c.s_seq, c.s_head, c.s_tok};
        for (int i = 0; i < 5; ++i)
            if (st[i] % 16) return fail(CB_ERR_MISALIGNED, "strides of 8-bit pages must be multiples of 16 elements (16 bytes)");
        if (!p->scales) return fail(CB_ERR_INVALID_ARGUMENT, "8-bit pages need scales");
        if (((uintptr_t)p->scales) % 4) return fail(CB_ERR_MISALIGNED, "scales must be 4-byte aligned");
    }
    if ((int64_t)c.n_seqs * c.seq_len > INT32_MAX) return fail(CB_ERR_UNSUPPORTED, "a pool has fewer than 2^31 slots");
    // a row's place within one (layer, kv) is a 32-bit number of 16-byte units
    if (c.s_seq > (1LL << 40) || c.s_tok > (1LL << 40) ||
        (double)(c.n_seqs - 1) * (double)c.s_seq * el + (double)(c.seq_len - 1) * (double)c.s_tok * el >= 68719476736.0)
        return fail(CB_ERR_UNSUPPORTED, "the pages of one (layer, kv) must span less than 64 GiB");
    return CB_OK;
}

cb_status check_rows(const char *name, const cb_rows *r, int d) {
    if (!r) return fail(CB_ERR_INVALID_ARGUMENT, "%s is NULL", name);
    if (r->n_tokens < 0 || r->n_heads <= 0) return fail(CB_ERR_SHAPE, "%s needs n_tokens >= 0 and positive n_heads", name);
    if (r->head_dim != d) return fail(CB_ERR_SHAPE, "%s has head_dim %d, the call %d", name, r->head_dim, d);
    if (r->s_tok < 0 || r->s_head < 0) return fail(CB_ERR_SHAPE, "%s has a negative stride", name);
    if (r->s_tok % 8 || r->s_head % 8 || ((uintptr_t)r->data) % 16)
        return fail(CB_ERR_MISALIGNED, "%s rows must be 16-byte aligned", name);
    if (r->n_tokens > 0 && !r->data) return fail(CB_ERR_INVALID_ARGUMENT, "%s->data is NULL", name);
    if ((int64_t)r->n_tokens * r->n_heads > INT32_MAX) return fail(CB_ERR_UNSUPPORTED, "%s has 2^31 rows or more", name);
    return CB_OK;
}

// Rows of d elements at every combination of n indexes (counts, strides): false if two could share an
// element.  The dimensions have to nest: each stride is at least what the smaller ones span together.
bool rows_apart(int d, int n, const int64_t *count, const int64_t *stride) {
    int order[5], m = 0;
    for (int i = 0; i < n; ++i) {
        if (count[i] <= 1) continue;
        int j = m++;
        for (; j > 0 && stride[order[j - 1]] > stride[i]; --j) order[j] = order[j - 1];
        order[j] = i;
    }
    __int128 span = d;
    for (int j = 0; j < m; ++j) {
        if (stride[order[j]] < span) return false;
        span += (__int128)(count[order[j]] - 1) * stride[order[j]];
    }
    return true;
}

// Rows that a call writes: no two may share an element.
cb_status check_rows_written(const char *name, const cb_rows *r, int d) {
    if (cb_status s = check_rows(name, r, d)) return s;
    const int64_t count[2] = {r->n_tokens, r->n_heads}, stride[2] = {r->s_tok, r->s_head};
    if (!rows_apart(d, 2, count, stride)) return fail(CB_ERR_SHAPE, "%s is written: its rows must not overlap", name);
    return CB_OK;
}

// A cache or pool that a call writes: the rows of all its dimensions, or without kv those of K.
cb_status check_cache_written(const char *name, const cb_cache &c, bool kv) {
    const int64_t count[5] = {c.n_layers, kv ? 2 : 1, c.n_seqs, c.n_heads, c.seq_len};
    const int64_t stride[5] = {c.s_layer, c.s_kv, c.s_seq, c.s_head, c.s_tok};
    if (!rows_apart(c.head_dim, 5, count, stride))
        return fail(CB_ERR_SHAPE, "%s is written: its rows must not overlap", name);
    return CB_OK;
}

cb_status check_rope_axes(const cb_rope_axes_spec *r, int d, int64_t n_tokens, cb::RopeAxes *out) {
    if (!r->table || !r->positions) return fail(CB_ERR_INVALID_ARGUMENT, "rope: table and positions must be non-NULL");
    if (r->style != CB_ROPE_HALF_SPLIT && r->style != CB_ROPE_INTERLEAVED)
        return fail(CB_ERR_INVALID_ARGUMENT, "rope: unknown style %d", r->style);
    if (r->head_dim != d) return fail(CB_ERR_SHAPE, "rope was built for head_dim %d, the rows have %d", r->head_dim, d);
    if (r->n_pos < 0) return fail(CB_ERR_INVALID_ARGUMENT, "rope: n_pos is negative");
    if (r->n_axes < 1 || r->n_axes > 4) return fail(CB_ERR_INVALID_ARGUMENT, "rope: n_axes must be in 1..4 (got %d)", r->n_axes);
    if (r->axis_stride != 0 && r->axis_stride < n_tokens && r->n_axes > 1)
        return fail(CB_ERR_SHAPE, "rope: axis_stride (%lld) < tokens of the call (%lld)", (long long)r->axis_stride,
                    (long long)n_tokens);
    if (((uintptr_t)r->table) % 16 || ((uintptr_t)r->positions) % 4)
        return fail(CB_ERR_MISALIGNED, "rope: table must be 16-byte and positions 4-byte aligned");
    *out = {};
    for (int i = 0; i < d / 2; ++i) {
        if (r->axis[i] >= r->n_axes) return fail(CB_ERR_INVALID_ARGUMENT, "rope: pair %d has axis %d of %d", i, r->axis[i], r->n_axes);
        out->axis[i / 16] |= (uint32_t)r->axis[i] << (2 * (i % 16));
    }
    out->table = (const float2 *)r->table;
    out->positions = r->positions;
    out->axis_stride = r->axis_stride;
    out->n_pos = r->n_pos;
    out->style = r->style;
    return CB_OK;
}

// Geometry shared by cb_rope_axes and cb_page_write.
cb_status prepare_rows(const char *name, const cb_cache *in, cb::RowsArgs &a) {
    if (!in) return fail(CB_ERR_INVALID_ARGUMENT, "%s is NULL", name);
    if (cb_status s = check_width(in->head_dim)) return s;
    if (in->n_layers <= 0 || in->n_heads <= 0) return fail(CB_ERR_SHAPE, "%s needs positive layer and head counts", name);
    if (cb_status s = cb::api_check_cache(name, in, in->n_layers, in->n_heads, in->head_dim)) return s;
    if ((int64_t)in->n_seqs * in->seq_len > INT32_MAX) return fail(CB_ERR_UNSUPPORTED, "too many tokens in one call");
    if ((int64_t)in->n_layers * in->n_heads > (1 << 24)) return fail(CB_ERR_UNSUPPORTED, "too many (layer, head) rows");
    a.in = (const uint16_t *)in->data;
    a.is = strides_of(*in);
    a.seq_len = cb::make_fastdiv((uint32_t)(in->seq_len > 0 ? in->seq_len : 1));
    a.n_heads = cb::make_fastdiv((uint32_t)in->n_heads);
    a.nc2 = cb::make_fastdiv((uint32_t)in->head_dim / 16);
    a.page_size = cb::make_fastdiv(1);
    a.n_tokens = (int64_t)in->n_seqs * in->seq_len;
    a.n_lh = in->n_layers * in->n_heads;
    return CB_OK;
}

}  // namespace

extern "C" {

cb_status cb_page_tables(int32_t n_reqs, const int32_t *ctx_lens, const int32_t *q_lens, const int32_t *free_pages,
                         int32_t n_free, int32_t page_size, int32_t *block_table, int64_t table_stride,
                         int32_t table_width, int32_t max_tokens, int32_t *q_starts, int32_t *kv_lens, int32_t *slots,
                         int32_t *positions, int32_t *info, int32_t *n_used, void *stream) {
    if (n_reqs < 0 || n_free < 0 || table_width < 0 || max_tokens < 0)
        return fail(CB_ERR_INVALID_ARGUMENT, "n_reqs, n_free, table_width and max_tokens must be >= 0");
    if (page_size < 1) return fail(CB_ERR_INVALID_ARGUMENT, "page_size must be >= 1 (got %d)", page_size);
    if (n_reqs > cb::kMaxPageReqs) return fail(CB_ERR_UNSUPPORTED, "at most %d requests (got %d)", cb::kMaxPageReqs, n_reqs);
    if ((int64_t)table_width * page_size > INT32_MAX)
        return fail(CB_ERR_UNSUPPORTED, "table_width * page_size must be below 2^31");
    if (n_reqs > 1 && table_stride < table_width)
        return fail(CB_ERR_SHAPE, "table_stride (%lld) < table_width (%d)", (long long)table_stride, table_width);
    if (!q_starts || !n_used) return fail(CB_ERR_INVALID_ARGUMENT, "q_starts and n_used must be non-NULL");
    if (n_reqs > 0 && (!ctx_lens || !q_lens || !kv_lens || !info))
        return fail(CB_ERR_INVALID_ARGUMENT, "ctx_lens, q_lens, kv_lens and info must be non-NULL");
    if (n_reqs > 0 && table_width > 0 && !block_table) return fail(CB_ERR_INVALID_ARGUMENT, "block_table is NULL");
    if (n_free > 0 && !free_pages) return fail(CB_ERR_INVALID_ARGUMENT, "free_pages is NULL");
    if (max_tokens > 0 && (!slots || !positions)) return fail(CB_ERR_INVALID_ARGUMENT, "slots and positions must be non-NULL");
    const void *ptrs[] = {ctx_lens, q_lens, free_pages, block_table, q_starts, kv_lens, slots, positions, info, n_used};
    for (const void *q : ptrs)
        if (((uintptr_t)q) % 4) return fail(CB_ERR_MISALIGNED, "every array must be 4-byte aligned");
    cb::PageTablesArgs a = {};
    a.n_reqs = n_reqs;
    a.n_free = n_free;
    a.table_width = table_width;
    a.max_tokens = max_tokens;
    a.ctx_lens = ctx_lens;
    a.q_lens = q_lens;
    a.free_pages = free_pages;
    a.page_size = cb::make_fastdiv((uint32_t)page_size);
    a.block_table = block_table;
    a.table_stride = table_stride;
    a.q_starts = q_starts;
    a.kv_lens = kv_lens;
    a.slots = slots;
    a.positions = positions;
    a.info = info;
    a.n_used = n_used;
    if (cb::launch_page_tables(a, (hipStream_t)stream) != hipSuccess) return fail(CB_ERR_DEVICE, "page tables launch failed");
    return cb::api_ok();
}

cb_status cb_rope_axes(const cb_cache *in, const cb_cache *out, const cb_rope_axes_spec *rope, int32_t inverse,
                       void *stream) {
    if (!in || !out || !rope) return fail(CB_ERR_INVALID_ARGUMENT, "in, out and rope must be non-NULL");
    cb::RowsArgs a = {};
    if (cb_status s = prepare_rows("in", in, a)) return s;
    if (cb_status s = cb::api_check_cache("out", out, in->n_layers, in->n_heads, in->head_dim)) return s;
    if (out->n_seqs != in->n_seqs || out->seq_len != in->seq_len)
        return fail(CB_ERR_SHAPE, "in and out disagree on n_seqs / seq_len");
    if (cb_status s = check_rope_axes(rope, in->head_dim, a.n_tokens, &a.rope)) return s;
    if (a.n_tokens == 0) return cb::api_ok();
    const bool same = in->data == out->data;
    if (same && (in->s_layer != out->s_layer || in->s_kv != out->s_kv || in->s_seq != out->s_seq ||
                 in->s_head != out->s_head || in->s_tok != out->s_tok))
        return fail(CB_ERR_INVALID_ARGUMENT, "an in-place transform needs out to have in's strides");
    if (cb_status s = check_cache_written("out", *out, !same)) return s;
    a.out = out->data;
    a.os = strides_of(*out);
    a.n_rows = (same ? 1 : 2) * a.n_lh;
    a.sign = inverse ? -1.f : 1.f;
    if (cb::launch_rows(a, true, false, (hipStream_t)stream) != hipSuccess) return fail(CB_ERR_DEVICE, "rope launch failed");
    return cb::api_ok();
}

cb_status cb_page_write(const cb_cache *rows, const cb_pages *pages, int32_t layer0, const int32_t *slots,
                        const cb_rope_axes_spec *rope, const cb_rows *q, const cb_rows *q_out, void *stream) {
    cb::RowsArgs a = {};
    if (cb_status s = prepare_rows("rows", rows, a)) return s;
    if (cb_status s = check_pages(pages)) return s;
    const cb_cache &c = pages->cache;
    if (c.n_heads != rows->n_heads || c.head_dim != rows->head_dim)
        return fail(CB_ERR_SHAPE, "rows are %d heads x %d, pages %d x %d", rows->n_heads, rows->head_dim, c.n_heads, c.head_dim);
    if (layer0 < 0 || (int64_t)layer0 + rows->n_layers > c.n_layers)
        return fail(CB_ERR_INVALID_ARGUMENT, "layers %d .. %lld are outside the pool's %d", layer0,
                    (long long)layer0 + rows->n_layers - 1, c.n_layers);
    if ((q != nullptr) != (q_out != nullptr)) return fail(CB_ERR_INVALID_ARGUMENT, "q and q_out go together");
    if (q && !rope) return fail(CB_ERR_INVALID_ARGUMENT, "q is turned by rope, which is NULL");
    if (rope)
        if (cb_status s = check_rope_axes(rope, rows->head_dim, a.n_tokens, &a.rope)) return s;
    if (q) {
        if (cb_status s = check_rows("q", q, rows->head_dim)) return s;
        if (cb_status s = check_rows_written("q_out", q_out, rows->head_dim)) return s;
        if (q->n_tokens != a.n_tokens || q_out->n_tokens != a.n_tokens || q->n_heads != q_out->n_heads)
            return fail(CB_ERR_SHAPE, "q and q_out must have the tokens of rows and equal heads");
        if (q->n_heads > (1 << 24)) return fail(CB_ERR_UNSUPPORTED, "too many query heads");
        if (q->data == q_out->data && (q->s_tok != q_out->s_tok || q->s_head != q_out->s_head))
            return fail(CB_ERR_INVALID_ARGUMENT, "an in-place turn needs q_out to have q's strides");
        a.q = (const uint16_t *)q->data;
        a.q_out = (uint16_t *)q_out->data;
        a.q_tok = q->s_tok;
        a.q_head = q->s_head;
        a.qo_tok = q_out->s_tok;
        a.qo_head = q_out->s_head;
        a.n_qh = q->n_heads;
    }
    if (a.n_tokens == 0) return cb::api_ok();
    if (!slots) return fail(CB_ERR_INVALID_ARGUMENT, "slots is NULL");
    if (((uintptr_t)slots) % 4) return fail(CB_ERR_MISALIGNED, "slots must be 4-byte aligned");
    if (cb_status s = check_cache_written("pages", c, true)) return s;
    a.out = (char *)c.data + (int64_t)layer0 * c.s_layer * (pages->dtype == CB_PAGES_E4M3 ? 1 : 2);
    a.os = strides_of(c);
    a.slots = slots;
    a.n_slots = c.n_seqs * c.seq_len;
    a.page_size = cb::make_fastdiv((uint32_t)c.seq_len);
    a.n_rows = 2 * a.n_lh + a.n_qh;
    a.layer0 = layer0;
    a.scales = pages->scales;
    a.sign = 1.f;
    if (cb::launch_rows(a, rope != nullptr, pages->dtype == CB_PAGES_E4M3, (hipStream_t)stream) != hipSuccess)
        return fail(CB_ERR_DEVICE, "page write launch failed");
    return cb::api_ok();
}

int64_t cb_attn_paged_workspace_bytes(int32_t n_tokens, int32_t n_reqs, int32_t n_qheads, int32_t n_heads,
                                      int32_t head_dim, int32_t max_q_len) {
    if (n_tokens <= 0 || n_reqs <= 0 || n_heads <= 0 || n_qheads <= 0 || n_qheads % n_heads || head_dim <= 0 || max_q_len <= 0)
        return 0;
    return cb::attn_paged_workspace_bytes(head_dim, n_qheads / n_heads, n_reqs, max_q_len);
}

cb_status cb_attn_paged(const cb_rows *q, const cb_pages *pages, int32_t layer, int32_t n_reqs, const int32_t *q_starts,
                        const int32_t *kv_lens, const int32_t *block_table, int64_t table_stride, int32_t table_width,
                        const cb_rows *out, int32_t max_q_len, float scale, int32_t window, int32_t n_sinks, float *lse,
                        void *workspace, int64_t workspace_bytes, void *stream) {
    if (cb_status s = check_pages(pages)) return s;
    const cb_cache &c = pages->cache;
    const int d = c.head_dim;
    if (d != 64 && d != 96 && d != 128) return fail(CB_ERR_UNSUPPORTED, "head_dim must be 64, 96 or 128 (got %d)", d);
    if (layer < 0 || layer >= c.n_layers) return fail(CB_ERR_INVALID_ARGUMENT, "layer %d is outside the pool's %d", layer, c.n_layers);
    if (cb_status s = check_rows("q", q, d)) return s;
    if (cb_status s = check_rows_written("out", out, d)) return s;
    if (out->n_tokens != q->n_tokens || out->n_heads != q->n_heads) return fail(CB_ERR_SHAPE, "q and out disagree on tokens or heads");
    if (q->n_heads % c.n_heads) return fail(CB_ERR_SHAPE, "%d query heads are no multiple of %d KV heads", q->n_heads, c.n_heads);
    if (n_reqs < 0) return fail(CB_ERR_INVALID_ARGUMENT, "n_reqs is negative");
    if (table_width < 0) return fail(CB_ERR_INVALID_ARGUMENT, "table_width is negative");
    if (n_reqs > 1 && table_stride < table_width)
        return fail(CB_ERR_SHAPE, "table_stride (%lld) < table_width (%d)", (long long)table_stride, table_width);
    if ((int64_t)table_width * c.seq_len > INT32_MAX)
        return fail(CB_ERR_UNSUPPORTED, "table_width * page size must be below 2^31");
    if (max_q_len < 0) return fail(CB_ERR_INVALID_ARGUMENT, "max_q_len is negative");
    const float scale_log2 = scale * 1.4426950408889634f;
    if (!std::isfinite(scale_log2)) return fail(CB_ERR_INVALID_ARGUMENT, "scale must be finite (and so scale * log2 e)");
    if (window < 0 || n_sinks < 0) return fail(CB_ERR_INVALID_ARGUMENT, "window and n_sinks must be >= 0");
    if (workspace_bytes < 0) return fail(CB_ERR_INVALID_ARGUMENT, "workspace_bytes is negative");
    if (((uintptr_t)workspace) % 16 || ((uintptr_t)lse) % 4 || ((uintptr_t)q_starts) % 4 || ((uintptr_t)kv_lens) % 4 ||
        ((uintptr_t)block_table) % 4)
        return fail(CB_ERR_MISALIGNED, "workspace must be 16-byte, the other arrays 4-byte aligned");
    if (q->n_tokens == 0 || n_reqs == 0) return cb::api_ok();
    if (!q_starts || !kv_lens || (table_width > 0 && !block_table))
        return fail(CB_ERR_INVALID_ARGUMENT, "q_starts, kv_lens and block_table must be non-NULL");
    if (q->data == out->data) return fail(CB_ERR_INVALID_ARGUMENT, "out must not be q");
    const int el = pages->dtype == CB_PAGES_E4M3 ? 1 : 2;
    cb::PagedArgs a = {};
    a.q = (const uint16_t *)q->data;
    a.out = (uint16_t *)out->data;
    a.q_tok = q->s_tok;
    a.q_head = q->s_head;
    a.o_tok = out->s_tok;
    a.o_head = out->s_head;
    a.n_tokens = q->n_tokens;
    a.k = (const char *)c.data + (int64_t)layer * c.s_layer * el;
    a.v = a.k + c.s_kv * el;
    a.s_page = (uint32_t)(c.s_seq * el / 16);
    a.s_tok = (uint32_t)(c.s_tok * el / 16);
    a.s_head = c.s_head * el;
    a.n_pages = c.n_seqs;
    a.page_size = cb::make_fastdiv((uint32_t)c.seq_len);
    a.q_starts = q_starts;
    a.kv_lens = kv_lens;
    a.table = block_table;
    a.table_stride = table_stride;
    a.table_width = table_width;
    a.n_reqs = n_reqs;
    a.n_heads = c.n_heads;
    a.G = cb::make_fastdiv((uint32_t)(q->n_heads / c.n_heads));
    a.scale_log2 = scale_log2;
    if (el == 1) {
        a.kscale = pages->scales + (int64_t)layer * 2 * c.n_heads;
        a.vscale = a.kscale + c.n_heads;
    }
    a.window = window;
    a.n_sinks = n_sinks;
    a.lse = lse;
    if (cb::launch_attn_paged(a, d, el == 1, max_q_len, workspace, workspace ? workspace_bytes : 0, (hipStream_t)stream) !=
        hipSuccess)
        return fail(CB_ERR_DEVICE, "paged attention launch failed");
    return cb::api_ok();
}

}  // extern "C"
