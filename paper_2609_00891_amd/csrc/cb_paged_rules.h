// cb_paged_rules.h -- how the serving calls are cut into workgroups, free of the
// HIP runtime so that it can be checked on the CPU: attention over pages, by rules
// on lengths that every workgroup evaluates for itself from the requests' lengths
// on the device (so no plan has to be built or kept), shared with the host that
// sizes grids and workspaces; and, on the host alone, the rows that are turned,
// copied or written into pages.
#pragma once
#include <cstdint>

#ifdef __HIPCC__
#define CB_HD __host__ __device__ __forceinline__
#else
#define CB_HD inline
#endif

namespace cb {

// Rows of a request (new token i, query head of one KV head) are numbered
// i * G + head; a row tile holds M of them.  Keys are visited in tiles of KT.
// The keys that some row of a row tile sees: tiles 0 .. sink - 1 (the first
// tokens that stay visible) and first .. first + n - sink - 1, as one list v =
// 0 .. n - 1.
struct KeyTiles {
    int32_t n, sink, first;
    CB_HD int32_t tile(int32_t v) const { return v < sink ? v : v - sink + first; }
};

// p_lo, p_hi: positions of the first and last row of the tile (p_hi may be
// negative: nothing to see).
CB_HD KeyTiles key_tiles(int32_t p_lo, int32_t p_hi, int32_t window, int32_t n_sinks, int32_t KT) {
    KeyTiles k = {0, 0, 0};
    if (p_hi < 0) return k;
    const int32_t end = p_hi / KT + 1;
    if (window > 0 && p_lo >= window) {                        // (p_lo - window may be below the least number)
        const int32_t lo = p_lo - window + 1;
        k.first = lo / KT;
        const int32_t s = n_sinks < lo ? n_sinks : lo;
        k.sink = s > 0 ? (s - 1) / KT + 1 : 0;
        if (k.sink >= k.first) k.sink = k.first = 0;
    }
    k.n = k.sink + end - k.first;
    return k;
}

// Bound on the key tiles of any of a request's row tiles: the work that one of
// them stands for where work is divided (tokens: most tokens in a row tile).
CB_HD int64_t key_tiles_bound(int32_t kv_len, int32_t tokens, int32_t window, int32_t n_sinks, int32_t KT) {
    const int64_t all = ((int64_t)kv_len + KT - 1) / KT;
    if (window <= 0) return all;
    const int64_t w = ((int64_t)window + tokens + KT - 2) / KT + 1 + ((int64_t)n_sinks + KT - 1) / KT;
    return w < all ? w : all;
}

// Key tiles of one part when W = sum of (row tiles x bound) over the requests is
// to make about `target` workgroups with H heads, at least c_min.
CB_HD int64_t part_tiles(int64_t W, int32_t H, int32_t target, int32_t c_min) {
    if (target <= 0) return INT64_MAX;
    const int64_t c = (W * H + target - 1) / target;
    return c > c_min ? c : c_min;
}

// Parts of a row tile with `bound` key tiles: the nearest number to bound / c (a
// tile a little longer than c is not worth the joining).  A tile in two parts or
// more has bound >= 1.5 c, so parts <= 4/3 bound / c: over all requests the parts
// of divided tiles are no more than 4/3 target / H, the divided tiles no more
// than 2/3 target / H, and the parts beyond the first no more than target / H.
// (Workspace and grid are sized by these.)
CB_HD int32_t parts_of(int64_t bound, int64_t c) {
    return bound <= c ? 1 : (int32_t)(bound / c + (bound % c >= c - c / 2 ? 1 : 0));
}

// ... and with fewer than `least` key tiles always one.
CB_HD int32_t parts_of(int64_t bound, int64_t c, int32_t least) { return bound < least ? 1 : parts_of(bound, c); }

// Part s of `parts` of a list of n key tiles: v in [begin, end).
CB_HD int32_t part_begin(int32_t n, int32_t s, int32_t parts) { return (int32_t)((int64_t)n * s / parts); }

// What a request is to one of the two kernels: those with row_min < rows <= row_max.
struct RequestWork {
    int32_t tiles;   // row tiles, 0: not this kernel's
    int32_t tokens;  // most tokens in a row tile
    int64_t bound;   // key tiles of a row tile
    uint32_t rows;
};
CB_HD RequestWork request_work(int32_t q_len, int32_t kv_len, int32_t G, int32_t M, int32_t KT, int64_t row_min,
                               int64_t row_max, int32_t window, int32_t n_sinks) {
    RequestWork w = {0, 0, 0, 0};
    const int64_t rows = (int64_t)q_len * G;
    if (rows <= row_min || rows > row_max) return w;
    w.rows = (uint32_t)rows;
    w.tiles = (int32_t)((rows + M - 1) / M);
    const int32_t t = (M - 1) / G + 2;
    w.tokens = t < q_len ? t : q_len;
    w.bound = key_tiles_bound(kv_len, w.tokens, window, n_sinks, KT);
    return w;
}

// Host side: row tiles that requests of n_tokens tokens can have together, if
// none counts that has more than row_max rows.
inline int64_t row_tiles_bound(int64_t n_tokens, int64_t n_reqs, int64_t G, int64_t M, int64_t row_max) {
    const int64_t all = n_tokens * G / M + n_reqs;
    const int64_t each = row_max / M + (row_max % M != 0);
    return each <= all / n_reqs ? n_reqs * each : all;
}

// Host side: the launch that turns n_rows rows of head_dim channels of each of n_tokens tokens.
// PAIRS: where half a row is no whole number of 128-byte lines, the lanes of two neighbouring tokens read
// and write one row of the two at a time and exchange the halves in registers.  12,282 tokens of 40 layers
// of 4 heads turned back: 96 channels 394 -> 297 us, 64 channels 246 -> 200.  A short call it makes longer
// (2,048 tokens of 4 layers of 8 heads of 96: 14.3 -> 15.6 us, a group of 1; 4,096 of 8 layers of 64: 25.2
// -> 24.0, a group of 4), so only groups of 4 rows or more take it.  8-bit pages do not (128 channels: 514
// -> 520 us, 64: 284 -> 296, 96: 428 -> 420).
constexpr int kPairsGroup = 4;
struct RowsCut {
    int32_t tok_per_wave;    // even
    int32_t group;           // rows of a token that one thread takes
    int64_t blocks, groups;  // the grid: workgroups of four waves, groups of rows
    bool pairs;
};
inline RowsCut rows_cut(int64_t n_tokens, int32_t n_rows, int32_t head_dim, bool f8) {
    RowsCut c;
    const int nc2 = head_dim / 16;
    c.tok_per_wave = (64 / nc2) & ~1;
    const int64_t per = 4 * (int64_t)c.tok_per_wave;
    c.blocks = (n_tokens + per - 1) / per;
    // up to 16 rows share a token's slot and angles while the launch still fills the chip
    c.group = 16;
    while (c.group > 1 && c.blocks * ((n_rows + c.group - 1) / c.group) < 2048) c.group /= 2;
    while ((n_rows + c.group - 1) / c.group > 65535) c.group *= 2;
    c.groups = (n_rows + c.group - 1) / c.group;
    c.pairs = !f8 && nc2 % 8 != 0 && c.group >= kPairsGroup;
    return c;
}

// Host side: the least l with n <= 2^l.
inline int log2_up(int n) {
    int l = 0;
    while ((1 << l) < n) ++l;
    return l;
}

// Host side: the launch that writes n_rows rows of head_dim channels of each of n_tokens tokens of n_reqs requests into
// pages with scales of their own, or reads them from pages.  A page's token has 2^lgc places for its pairs of 16-byte
// chunks.  wide: pages get enough tokens on average for teams of whole waves (of a call of many single tokens and a chunk
// they do not: teams of the chunk's whole pages then outgrow a wave and take turns).  pairs: the pairs of chunks of a
// thread, as many as hold a page's row in registers, up to 4, 0 where they do not.  group: the rows of a page that one
// workgroup takes: up to 16, which share its search, places and angles, while the launch fills the chip, at least 4 (1,811
// tokens of three requests, 56 rows of 96 channels each: 23.0 us with 1, 20.6 with 2, 17.8 with 4, 22.7 with 8) and as many
// as it has teams.
struct SpanCut {
    int lgc;
    bool wide;
    int pairs;
    int32_t group;
    int64_t blocks, groups;  // the grid: pages (workgroups go round while there are more), groups of rows
};
inline SpanCut span_cut(int64_t n_tokens, int64_t n_reqs, int32_t page_size, int32_t head_dim, int32_t n_rows) {
    SpanCut c;
    // Pages that the tokens can lie in together, unless requests share rows: a page has at least one token, all but a
    // request's first and last a whole page.
    int64_t items = n_tokens / page_size + 2 * n_reqs;
    if (items > n_tokens) items = n_tokens;
    c.lgc = log2_up(head_dim / 16);
    int64_t tokens = (n_tokens + n_reqs - 1) / n_reqs;
    if (tokens > page_size) tokens = page_size;
    const int64_t units = (int64_t)page_size << c.lgc;
    c.wide = tokens << c.lgc >= 64;
    c.pairs = units <= 256 ? 1 : units <= 512 ? 2 : units <= 1024 ? 4 : 0;
    int teams = 256 >> c.lgc;
    while (teams > 1 && (256 / teams) < tokens << c.lgc) teams /= 2;
    c.group = 16;
    while (c.group > 4 && items * ((n_rows + c.group - 1) / c.group) < 2048) c.group /= 2;
    if (c.group < teams) c.group = teams;
    while ((n_rows + c.group - 1) / c.group > 65535) c.group *= 2;
    c.groups = (n_rows + c.group - 1) / c.group;
    // (a launch has fewer than 2^32 threads in one direction)
    c.blocks = items < 1 ? 1 : items < 1 << 22 ? items : 1 << 22;
    return c;
}

// Host side: attention over n_selected pages of every token: row tiles of 16 query heads of one KV head, the listed keys in
// tiles of 32, each row tile's in parts for about 2,048 workgroups, of 16 tiles or more, where it has 36 or more (the
// same division as of single tokens over all their pages).
struct SelectedCut { int32_t tiles, parts; };
inline SelectedCut selected_cut(int64_t n_tokens, int32_t H, int32_t G, int32_t page_size, int32_t n_selected) {
    const int32_t tiles = (G + 15) / 16;
    const int64_t keys = ((int64_t)n_selected * page_size + 31) / 32;
    return {tiles, parts_of(keys, part_tiles(n_tokens * tiles * keys, H, 2048, 16), 36)};
}

// Tokens of a request that share a row tile of 16 and the keys that it reads: as many as have their query heads in it and
// their lists in `entries` places, while 1,024 workgroups are left, and 1 where requests have fewer than three on average.
// 512 tokens, 64 of 512 pages of 64 e4m3 tokens each (8 heads of 128), apart and shared: 8 query heads a head 276 and 229 us
// where neighbouring tokens' lists are near, 274 / 168 where they are alike, 302 / 307 where they are chosen at random; 4
// query heads 270 / 162, 270 / 100, 293 / 289; 1 query head 263 / 157, 263 / 96, 286 / 280.  256 tokens (1,024
// workgroups) 143 / 130 near and 152 / 173 at random; 256 requests of 2 tokens 146 / 152 and 187 / 200.
inline int32_t shared_tokens(int64_t n_tokens, int64_t n_reqs, int64_t H, int32_t G, int32_t n_selected, int32_t entries) {
    if (n_tokens < 3 * n_reqs) return 1;
    int64_t t = G > 8 ? 1 : 16 / G;
    if (t * n_selected > entries) t = entries / n_selected;
    if (t > n_tokens * H / 1024) t = n_tokens * H / 1024;
    return t < 1 ? 1 : (int32_t)t;
}

}  // namespace cb
