// cb_serve_internal.h -- structures shared by the host side and the kernels of
// the calls that serve a receiver from pages.
#pragma once

#include "cb_internal.h"

namespace cb {

// Errors of the calling thread and the check of a cache's geometry and alignment (cb_api.cpp).
cb_status api_error(cb_status s, const char *message);
cb_status api_ok();
cb_status api_check_cache(const char *name, const cb_cache *c, int L, int H, int d);

// Tables of a serving step (cb_page_tables).
struct PageTablesArgs {
    int32_t n_reqs, n_free, table_width, max_tokens;
    const int32_t *ctx_lens, *q_lens, *free_pages;
    FastDiv page_size;
    int32_t *block_table;
    int64_t table_stride;
    int32_t *q_starts, *kv_lens, *slots, *positions, *info, *n_used;
};
constexpr int kMaxPageReqs = 4096;      // sums of all requests in the LDS of every workgroup

// Rotary positions with several axes, as the kernels take them.
struct RopeAxes {
    const float2 *table;      // [n_pos][d/2] (cos, sin)
    const int32_t *positions; // [n_axes][axis_stride]
    int64_t axis_stride;
    int32_t n_pos, style;
    uint32_t axis[8];         // two bits per channel pair
};

// Rows of a cache turned into another cache, or written into pages (out with
// n_seqs = pages, seq_len = page size) by slots, beside the step's queries.
struct RowsArgs {
    const uint16_t *in;
    void *out;                // pool, or the other cache
    Strides is, os;
    const int32_t *slots;     // NULL: token t goes to the same place of out
    int32_t n_slots;          // slots of the pool
    FastDiv page_size;        // tokens of a page
    FastDiv seq_len;          // tokens of a sequence of in
    FastDiv n_heads;
    FastDiv nc2;              // pairs of 16-byte chunks in a row: head_dim / 16
    int64_t n_tokens;
    int32_t n_lh, n_qh;       // (layer, head) rows and query rows of a token
    int32_t n_rows;           // K, then query, then V rows that are worked on
    int32_t group;            // rows of a token that one thread takes
    int32_t tok_per_wave;
    int32_t lgc;              // block pages: 2^lgc >= nc2
    int32_t layer0;           // the scales' layer of in's first
    const float *scales;      // e4m3 pages
    RopeAxes rope;
    float sign;               // +1 turn, -1 turn back
    const uint16_t *q;
    uint16_t *q_out;
    int64_t q_tok, q_head, qo_tok, qo_head;
};

// The last q_lens[r] of kv_lens[r] tokens of every request, by pages; row_starts[r] is the first one's row (or NULL).
struct SpanArgs {
    int32_t n_reqs, n_pages;
    const int32_t *row_starts, *q_lens, *kv_lens, *table;
    int64_t table_stride;
    int32_t most;             // tokens that a row of the table has places for
    int64_t n_tokens;
    FastDiv page_size;
};

// Bounds of pages (cb_page_bounds).  Strides in bytes.
struct BoundsArgs {
    const char *k;            // the first layer's K pages
    int64_t s_layer, s_page, s_head, s_tok;
    char *bounds;             // [layer][page][head][2][head_dim]
    FastDiv n_heads;
    int32_t n_lh, layer0;
    int32_t chunks, lgc;      // 16-byte chunks of a row, 2^lgc >= chunks
};

// Attention over pages (cb_attn_paged).  Strides of the pool in units of 16
// bytes, so that a row's place is a 32-bit number.
struct PagedClass {           // requests that are worked on in one way, and how their keys are divided
    int64_t row_min, row_max; // requests with row_min < rows <= row_max
    int32_t target;           // workgroups to divide long rows into, 0: never divide
    float *ws;                // [2 target][M (d + 2)] partial results
    uint32_t blocks;          // workgroups of the attention and of the joining, 0: no such requests
    uint32_t join_blocks;
};
struct PagedArgs {
    const uint16_t *q;
    uint16_t *out;
    int64_t q_tok, q_head, o_tok, o_head;
    int32_t n_tokens;
    const char *k, *v;        // the layer's K and V pages
    uint32_t s_page, s_tok;   // 16-byte units
    int64_t s_head;           // bytes
    int32_t n_pages;
    FastDiv page_size;
    const int32_t *q_starts, *kv_lens, *table;
    int64_t table_stride;
    int32_t table_width;
    int32_t n_reqs, n_heads;
    FastDiv G;
    float scale_log2;         // scale * log2(e)
    const float *kscale, *vscale;   // e4m3: [n_heads]; block scales: kscale [n_pages][n_heads][2]
    int32_t window, n_sinks;
    float *lse;               // NULL or [n_tokens][n_heads * G]
    PagedClass rows, tile;
    const int32_t *selected;  // attention over selected pages: [n_tokens][n_heads][n_selected]
    int32_t n_selected;
    FastDiv sel_parts, sel_tiles;   // parts of a row tile, row tiles of a token,
    FastDiv sel_tokens;             // or tokens of a row tile
};

// The choice of pages (cb_page_select).
struct SelectArgs {
    PagedArgs a;              // queries, requests, table, scales
    const char *bounds;       // of the layer: [page][head][2][head_dim]
    int32_t n_first, n_last, n_selected;
    int32_t *selected;        // [n_tokens][n_heads][n_selected]
    uint32_t *keys;           // [tok1 - tok0][n_heads][table_width] scores of a round's tokens, as numbers of their order
    int32_t tok0, tok1;
    int32_t head_dim, dtype;
    float *sizes;             // [tok1 - tok0][n_heads][slots] largest sums of the estimates' magnitudes
    int32_t slots;
};

// Launchers (return hipError_t of the launch).
hipError_t launch_page_tables(const PageTablesArgs &a, hipStream_t s);
hipError_t launch_rows(RowsArgs a, bool rope, bool f8, hipStream_t s);
hipError_t launch_page_quant(RowsArgs a, const SpanArgs &span, bool rope, float *scales, hipStream_t s);
hipError_t launch_page_read(RowsArgs a, const SpanArgs &span, bool rope, int32_t dtype, const float *scales, hipStream_t s);
hipError_t launch_page_bounds(BoundsArgs a, const SpanArgs &span, bool f8, int32_t max_q_len, hipStream_t s);
hipError_t launch_attn_paged(const PagedArgs &a, int32_t d, int32_t dtype, int32_t max_q_len, void *ws, int64_t ws_bytes,
                             hipStream_t s);
hipError_t launch_page_select(const SelectArgs &s, int32_t d, int32_t dtype, void *ws, int64_t ws_bytes, hipStream_t stream);
hipError_t launch_attn_selected(const PagedArgs &a, int32_t d, int32_t dtype, void *ws, int64_t ws_bytes, hipStream_t s);
int64_t select_row_bytes(int32_t table_width);   // workspace of one (token, head)
int64_t attn_selected_workspace_bytes(int64_t n_tokens, int32_t n_heads, int32_t G, int32_t d, int32_t page_size, int32_t n_selected);
int64_t attn_paged_workspace_bytes(int32_t d, int32_t G, int32_t n_reqs, int32_t max_q_len);

}  // namespace cb
