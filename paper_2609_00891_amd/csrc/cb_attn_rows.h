// cb_attn_rows.h -- attention over pages for rows whose keys go from memory straight
// into matrix-core operands (rows_body, described in cb_attn_paged.hip), and the
// joining of their parts: shared by attention over all visible pages
// (cb_attn_paged.hip) and over selected ones (cb_attn_selected.hip).
#pragma once
#include "cb_serve_internal.h"
#include "cb_paged_rules.h"

namespace cb {
namespace {


typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;

constexpr int kKT = 32;                 // keys of a tile
constexpr int kTileKT = 64;             // keys of a tile of the tile kernel
// Key tiles from which a row tile may be divided and the least of a part, for rows_body (1,152 and 512
// keys) and tile_body (1,536 and 512): what dividing saves must be worth the joining, a launch of about
// 3 us where nothing is divided and 8 us where rows are, and every part costs it something.  24 single tokens
// and three chunks with windows of 1,024 keys, undivided: 49 us; with parts of 256 keys and more: 61 us.
// Single tokens (8 heads of 128, 8 query heads each) with windows of 1,056, 1,500 and 4,000 keys, divided
// and not: one 18.9 / 16.4, 17.5 / 21.3 and 16.4 / 43.5 us, 8 of them 23.7 / 19.0, 20.7 / 24.7 and 34.3 /
// 51.2.  Where the rows fill the chip undivided and are alike, dividing them only costs: 24 of them 27.0 /
// 21.6, 41.6 / 27.9 and 84.4 / 74.9, 64 of them 56.4 / 45.9, 91.0 / 71.4 and 200.6 / 180.2 (such a caller
// passes no workspace).  One single token (8 heads of 128) over 8,192 and 131,072 keys: 18.5 and 113 us;
// with parts of at least 256 keys 18.0 and 113, of 768 21.3 and 111; over 131,072 keys of one head: 26.5,
// 33.9 and 25.4.
constexpr int part_min(int KT) { return KT == kKT ? 16 : 8; }
constexpr int split_min(int KT) { return KT == kKT ? 36 : 24; }
// Parts above which a row is joined by a workgroup instead of a wave: one single token over 131,072 keys
// (256 parts) 113 us, 121 by a wave.
constexpr int kWideParts = 16;
// Blocks of one kind in turn, one for every compute unit, where a launch has both.
constexpr uint32_t kRun = 256;
// Workgroups that long rows are divided into: four for each of the 512 that are resident, so that
// requests of different lengths end together (64 requests of 512 .. 16,384 keys: 262 us with 1,024,
// 268 with 4,096, 259 with 2,048).
constexpr int kTarget = 2048;
// Listed pages of the tokens of a row tile together, where they share it.
constexpr int kSharedEntries = 1024;

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    f32x2_t v = {lo, hi};
    bf16x2_t p = __builtin_convertvector(v, bf16x2_t);
    return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ float bf_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ bf16x8_t frag(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_bit_cast(bf16x8_t, make_uint4(a, b, c, d));
}
// Whether one of the two bf16 values is an infinity or a NaN.
__device__ __forceinline__ bool not_finite(uint32_t u) {
    return (u & 0x7f80u) == 0x7f80u || (u & 0x7f800000u) == 0x7f800000u;
}
// The bits of the bf16 values, and of the e4m3 ones, that are infinities or NaNs: an exponent (e4m3:
// a magnitude) of all ones carries into the sign's place when one is added to it.
__device__ __forceinline__ uint32_t not_finite_halves(uint32_t u) {
    const uint32_t t = ((u & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
    return t | (t - (t >> 15));
}
__device__ __forceinline__ uint32_t nan_bytes(uint32_t u) {
    const uint32_t t = ((u & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    return t | (t - (t >> 7));
}
// Two e4m3 values times a power of two (exact in bf16; of another number only the exponent counts).
template <bool HI> __device__ __forceinline__ uint32_t e4m3_pair(uint32_t u, float scale = 1.0f) {
    const bf16x2_t v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, scale, HI);
    return __builtin_bit_cast(uint32_t, v);
}
// Bits 0 .. k.
__device__ __forceinline__ uint32_t bits_to(int32_t k) { return k < 0 ? 0u : 0xffffffffu >> (31 - min(k, 31)); }
// Bit c: the key c places from the first is there and seen from the place p (c <= p, and c > p - window
// or c < sink).
__device__ __forceinline__ uint32_t visible(int32_t p, uint32_t there, int32_t window, int32_t sink) {
    uint32_t v = bits_to(p);
    if (window > 0 && p >= window) v &= ~bits_to(p - window) | bits_to(sink - 1);
    return v & there;
}
// x if bit c is set, else -infinity; no condition register.
__device__ __forceinline__ float keep_if(uint32_t bits, int c, float x) {
    const uint32_t k = (uint32_t)((int32_t)(bits << (31 - c)) >> 31);
    return __uint_as_float((__float_as_uint(x) & k) | (~k & 0xff800000u));
}
__device__ __forceinline__ uint32_t fast_div(uint32_t n, const FastDiv &f) {
    const uint32_t t = __umulhi(f.m, n);
    return (t + ((n - t) >> f.sh1)) >> f.sh2;
}

// ------------------------------------------------------------------ who does what

struct Request { int32_t row0, q_len, kv_len; };   // first token row, new tokens, keys

__device__ __forceinline__ Request request(const PagedArgs &a, int r) {
    const int32_t b = min(max(a.q_starts[r], 0), a.n_tokens), e = min(max(a.q_starts[r + 1], 0), a.n_tokens);
    const int64_t most = min((int64_t)a.table_width * a.page_size.d, (int64_t)INT32_MAX);
    return {b, max(e - b, 0), (int32_t)min((int64_t)max(a.kv_lens[r], 0), most)};
}

struct Item { int32_t req, tile, part, parts, slot; };   // slot: of the first part's partial result
template <int NW> struct SchedLds { double work[NW]; uint32_t items[NW], slots[NW]; Item item; int32_t found; };

// Inclusive sums over a wave by data-parallel moves: within rows of 16 lanes, then across them.
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t moved(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS> __device__ __forceinline__ double moved(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint64_t r = (uint64_t)moved<CTRL, ROWS>((uint32_t)(u >> 32)) << 32 | moved<CTRL, ROWS>((uint32_t)u);
    return __builtin_bit_cast(double, r);
}
template <typename T> __device__ __forceinline__ T wave_sums(T x) {
    x += moved<0x111, 0xf>(x);   // row_shr:1, 2, 4, 8
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    x += moved<0x118, 0xf>(x);
    x += moved<0x142, 0xa>(x);   // row_bcast:15, 31
    x += moved<0x143, 0xc>(x);
    return x;
}

// The row tile and part of index `idx`, or false behind the last.  JOIN: of the rows of all tiles in
// more than one part, four at a time (in more than kWideParts: one), the idx-th (it.part: which of the
// tile).  The work of all requests is summed in fp64: whole numbers, exact below 2^53, and the same in
// every workgroup.
template <int M, int KT, bool JOIN, int NW>
__device__ __forceinline__ bool find_item(const PagedArgs &a, const PagedClass &cl, uint32_t idx, SchedLds<NW> &sh, Item &out) {
    constexpr int NT = 64 * NW;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    auto work_of = [&](int r) __attribute__((always_inline)) {
        RequestWork w = {0, 0, 0, 0};
        if (r < a.n_reqs) {
            const Request q = request(a, r);
            w = request_work(q.q_len, q.kv_len, (int32_t)a.G.d, M, KT, cl.row_min, cl.row_max, a.window, a.n_sinks);
        }
        return w;
    };
    if (tid == 0) sh.found = 0;
    const RequestWork w0 = work_of(tid);
    double W = (double)w0.tiles * (double)w0.bound;
    for (int r = tid + NT; r < a.n_reqs; r += NT) {
        const RequestWork w = work_of(r);
        W += (double)w.tiles * (double)w.bound;
    }
    W = wave_sums(W);
    if (lane == 63) sh.work[wave] = W;
    __syncthreads();
    W = 0.0;
#pragma unroll
    for (int v = 0; v < NW; ++v) W += sh.work[v];
    // (only starts that decrease, each request claiming the same rows, could reach the limit)
    const int64_t c = W * a.n_heads < 4e18 ? part_tiles((int64_t)W, a.n_heads, cl.target, part_min(KT)) : INT64_MAX;
    uint32_t n_before = 0, s_before = 0;
    for (int r0 = 0; r0 < a.n_reqs; r0 += NT) {
        const RequestWork w = r0 == 0 ? w0 : work_of(r0 + tid);
        const int32_t parts = parts_of(w.bound, c, split_min(KT));
        const bool wide = JOIN && parts > kWideParts;
        const uint32_t n = JOIN ? (parts > 1 ? (wide ? w.rows : (w.rows + 3) / 4) : 0) : (uint32_t)w.tiles * parts;
        const uint32_t s = parts > 1 ? (uint32_t)w.tiles * parts : 0;
        uint32_t ni = wave_sums(n), si = wave_sums(s);
        if (r0 > 0) __syncthreads();                          // the last round's sums have been read
        if (lane == 63) {
            sh.items[wave] = ni;
            sh.slots[wave] = si;
        }
        __syncthreads();
        uint32_t total = 0, s_total = 0;
#pragma unroll
        for (int v = 0; v < NW; ++v) {
            if (v < wave) { ni += sh.items[v]; si += sh.slots[v]; }
            total += sh.items[v];
            s_total += sh.slots[v];
        }
        const uint32_t first = n_before + ni - n;
        if (idx - first < n) {
            // the last row tile, with the most keys, first: 2,048 tokens over themselves (8 heads of 128,
            // 8 query heads each) 97 us, 115 with the first one first
            const uint32_t k = idx - first, per = JOIN ? (wide ? M : M / 4) : (uint32_t)parts;
            const uint32_t tile = JOIN ? k / per : w.tiles - 1 - k / per;
            sh.item = {r0 + tid, (int32_t)tile, (int32_t)(k % per), parts, (int32_t)(s_before + si - s + tile * parts)};
            sh.found = 1;
        }
        n_before += total;
        s_before += s_total;
        __syncthreads();
        if (sh.found) break;
    }
    out = sh.item;
    return sh.found != 0;
}

// ------------------------------------------------------------------ rows kernel

// What pages hold: bf16, e4m3 with a scale for a head's K or V, e4m3 with one for every page and head.
enum { kBf16, kE4m3, kBlocks };

template <int D, bool F8> struct Geo {
    static constexpr int NS = D / 32;                          // 32-channel steps of Q . K
    static constexpr int E = D == 64 ? 4 : 8;                  // channels of V that a lane takes
    static constexpr int NC = D / E;                           // lanes (of 16) that take any: 16 or, for 96, 12
    static constexpr bool PAIR = F8 && NS % 2 == 0;            // two steps' bytes in one 16-byte piece
    static constexpr int KW = F8 ? 2 * NS : 4 * NS;            // dwords of K of a lane and subtile
    static constexpr int VW = F8 ? E / 4 : E / 2;              // dwords of V of a lane and key
    // channel of step s, lane group g, place 0 of Q . K's products
    static __device__ __forceinline__ int chan(int s, int g) {
        return PAIR ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
    }
};

template <int D, int NW> struct RowsLds {
    float o[NW][16][D + 4];                                    // each wave's results
    float ml[NW][16][2];
};

// The request that has token row `tok`, every wave for itself; false if none has.
__device__ __forceinline__ bool request_of(const PagedArgs &a, int32_t tok, int &req, Request &rq) {
    const int lane = threadIdx.x & 63;
    for (int r0 = 0; r0 < a.n_reqs; r0 += 64) {
        const Request r = request(a, min(r0 + lane, a.n_reqs - 1));
        const uint64_t has = __ballot(r0 + lane < a.n_reqs && tok >= r.row0 && tok < r.row0 + r.q_len);
        if (!has) continue;
        const int from = __builtin_ctzll(has);
        req = r0 + from;
        rq = {__builtin_amdgcn_readlane(r.row0, from), __builtin_amdgcn_readlane(r.q_len, from),
              __builtin_amdgcn_readlane(r.kv_len, from)};
        return true;
    }
    return false;
}

// Tile `idx` of all requests' tiles of tokens, tiles_of(q_len) for each, and its request, every wave for itself.
template <typename F>
__device__ __forceinline__ bool find_tile(const PagedArgs &a, uint32_t idx, F tiles_of, Request &rq, int32_t &req, int32_t &tile) {
    const int lane = threadIdx.x & 63;
    uint32_t before = 0;
    for (int r0 = 0; r0 < a.n_reqs; r0 += 64) {
        const Request r = request(a, min(r0 + lane, a.n_reqs - 1));
        const uint32_t n = r0 + lane < a.n_reqs ? tiles_of(r.q_len) : 0;
        const uint32_t sum = wave_sums(n), total = (uint32_t)__builtin_amdgcn_readlane((int)sum, 63);
        if (idx - before < total) {
            const uint32_t k = idx - before - (sum - n);
            const int from = __builtin_ctzll(__ballot(k < n));
            req = r0 + from;
            tile = __builtin_amdgcn_readlane((int)k, from);
            rq = {__builtin_amdgcn_readlane(r.row0, from), __builtin_amdgcn_readlane(r.q_len, from),
                  __builtin_amdgcn_readlane(r.kv_len, from)};
            return true;
        }
        before += total;
    }
    return false;
}

// The row tile and part of index `idx` of a call on selected pages, and its token as the one new token of a request that
// ends there; false for a token of no request.
__device__ __forceinline__ bool selected_item(const PagedArgs &a, uint32_t idx, Item &it, Request &rq) {
    const uint32_t unit = fast_div(idx, a.sel_parts), tok = fast_div(unit, a.sel_tiles);
    it.part = (int32_t)(idx - unit * a.sel_parts.d);
    it.parts = (int32_t)a.sel_parts.d;
    it.tile = (int32_t)(unit - tok * a.sel_tiles.d);
    it.slot = (int32_t)(unit * a.sel_parts.d);
    Request r;
    if (!request_of(a, (int32_t)tok, it.req, r)) return false;
    rq = {(int32_t)tok, 1, r.kv_len - r.q_len + ((int32_t)tok - r.row0) + 1};
    return true;
}

// The entries of a list of pages up to the last that is a page's number (not negative).
__device__ __forceinline__ int32_t list_length(const int32_t *list, int32_t n) {
    const int lane = threadIdx.x & 63;
    for (int32_t i0 = (n - 1) & ~63; i0 >= 0; i0 -= 64) {
        const uint64_t is = __ballot(i0 + lane < n && list[min(i0 + lane, n - 1)] >= 0);
        if (is) return i0 + 64 - __builtin_clzll(is);
    }
    return 0;
}

// The idx-th tile of a call on selected pages whose tiles have sel_tokens tokens of a request, as its new tokens.
__device__ __forceinline__ bool shared_item(const PagedArgs &a, uint32_t idx, Item &it, Request &rq) {
    Request r;
    int32_t tile;
    const auto tiles_of = [&](int32_t q) { return fast_div((uint32_t)(q + (int32_t)a.sel_tokens.d - 1), a.sel_tokens); };
    if (!find_tile(a, idx, tiles_of, r, it.req, tile)) return false;
    it.tile = it.part = it.slot = 0;
    it.parts = 1;
    const int32_t t0 = tile * (int32_t)a.sel_tokens.d, n = min(r.q_len - t0, (int32_t)a.sel_tokens.d);
    rq = {r.row0 + t0, n, r.kv_len - r.q_len + t0 + n};
    return true;
}

// The pages of several tokens' lists as one list, ascending, and whose they are (bit t: token t's).  A page that a token
// has twice stands in two places, each of them once that token's.
struct SharedList {
    uint32_t sorted[kSharedEntries], masks[kSharedEntries];
    int32_t pages[kSharedEntries];
};
__device__ __forceinline__ int32_t share_lists(const PagedArgs &a, const Request &rq, int head, SharedList &l) {
    constexpr int NT = 256;
    const int tid = threadIdx.x, lane = tid & 63, k = a.n_selected;
    for (int t = 0; t < rq.q_len; ++t) {
        const int32_t *list = a.selected + ((int64_t)(rq.row0 + t) * a.n_heads + head) * k;
        for (int i = tid; i < k; i += NT) {
            const int32_t page = list[i];
            l.sorted[t * k + i] = (uint32_t)page < (uint32_t)a.table_width ? (uint32_t)page << 4 | (uint32_t)t : ~0u;
        }
    }
    int n = 64;
    while (n < rq.q_len * k) n *= 2;
    for (int i = rq.q_len * k + tid; i < n; i += NT) l.sorted[i] = ~0u;
    for (int i = tid; i < n; i += NT) l.masks[i] = 0;
    __syncthreads();
    // bitonic: a pair (i, i + stride) is one thread's; with strides up to 64 a wave's pairs stay its own
    for (int size = 2, last = 1; size <= n; size *= 2)
        for (int stride = size / 2; stride > 0; stride /= 2) {
            if (max(last, stride) > 64) __syncthreads();
            else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            last = stride;
            for (int i = tid; i < n / 2; i += NT) {
                const int lo = 2 * i - (i & (stride - 1)), hi = lo + stride;
                const uint32_t x = l.sorted[lo], y = l.sorted[hi];
                if ((x > y) == ((lo & size) == 0)) {
                    l.sorted[lo] = y;
                    l.sorted[hi] = x;
                }
            }
        }
    __syncthreads();
    // every wave counts, one writes
    int32_t count = 0;
    for (int i0 = 0; i0 < n; i0 += 64) {
        const uint32_t x = l.sorted[i0 + lane], before = i0 + lane > 0 ? l.sorted[i0 + lane - 1] : ~0u;
        const uint64_t first = __ballot(x != ~0u && ((x ^ before) > 15u || x == before));
        if (tid < 64 && x != ~0u) {
            const int at = count + __builtin_popcountll(first & ((2ull << lane) - 1)) - 1;
            if ((first >> lane) & 1) l.pages[at] = (int32_t)(x >> 4);
            atomicOr(&l.masks[at], 1u << (x & 15));
        }
        count += __builtin_popcountll(first);
    }
    __syncthreads();
    return count;
}

// Which keys a row tile has: those that it sees of all pages, or those of the pages selected for its token, one list of keys
// (place i of the list: key i mod page_size of its page i / page_size; the row is the one new token of a request as
// long as its position).  kSelectedWhole: a key tile lies in one page, so that its place, scales and visible keys are one
// number each for the wave: no lane asks another, and the loads' addresses are a scalar and a constant of the lane.
// kSelectedShared: and the row tile has several tokens of a request, whose lists are joined; a row sees the keys of its own
// token's pages.
enum { kAll, kSelected, kSelectedWhole, kSelectedShared };
template <int D, int EL, int NW, int KEYS>
__device__ __forceinline__ void rows_body(const PagedArgs &a, const PagedClass &cl, uint32_t block, SchedLds<NW> &sched,
                                          RowsLds<D, NW> &lds) {
    constexpr bool F8 = EL != kBf16, BLK = EL == kBlocks, SEL = KEYS != kAll;
    constexpr bool SHARED = KEYS == kSelectedShared, WHOLE = KEYS == kSelectedWhole || SHARED;
    using Ge = Geo<D, F8>;
    constexpr int M = 16, E = Ge::E;
    auto &ol = lds.o;
    auto &ml = lds.ml;
    const int head = (int)(block % (uint32_t)a.n_heads);
    Item it;
    Request rq;
    if constexpr (SHARED) {
        if (!shared_item(a, block / (uint32_t)a.n_heads, it, rq)) return;
    } else if constexpr (SEL) {
        if (!selected_item(a, block / (uint32_t)a.n_heads, it, rq)) return;
    } else {
        if (!find_item<M, kKT, false, NW>(a, cl, block / (uint32_t)a.n_heads, sched, it)) return;
        rq = request(a, it.req);
    }

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, g = lane >> 4;
    const int32_t G = (int32_t)a.G.d;
    const int64_t rows = (int64_t)rq.q_len * G;                // at most M tiles of them exist: fits 32 bits below
    const int32_t row0 = it.tile * M;
    const int32_t n_rows = (int32_t)min(rows - row0, (int64_t)M);
    const int32_t tok0 = (int32_t)fast_div((uint32_t)row0, a.G), tok1 = (int32_t)fast_div((uint32_t)(row0 + n_rows - 1), a.G);
    const int32_t p_lo = rq.kv_len - rq.q_len + tok0, p_hi = rq.kv_len - rq.q_len + tok1;
    const int32_t *list = nullptr;                             // SEL: the row's pages
    int32_t listed = 0;
    KeyTiles kt = {0, 0, 0};
    SharedList &joint = *(SharedList *)&ol;                    // (read before the results are written)
    static_assert(!SHARED || sizeof(SharedList) <= sizeof(ol), "");
    if constexpr (SHARED) {
        listed = p_hi < 0 ? 0 : share_lists(a, rq, head, joint);
        kt.n = listed * (int32_t)(a.page_size.d / kKT);
    } else if constexpr (SEL) {
        list = a.selected + ((int64_t)rq.row0 * a.n_heads + head) * a.n_selected;
        listed = p_lo < 0 ? 0 : list_length(list, a.n_selected);
        kt.n = (listed * (int32_t)a.page_size.d + kKT - 1) / kKT;
    } else {
        kt = key_tiles(p_lo, p_hi, a.window, a.n_sinks, kKT);
    }
    const int32_t v1 = part_begin(kt.n, it.part + 1, it.parts);
    const int32_t *table = a.table + it.req * a.table_stride;
    const char *kp = a.k + head * a.s_head, *vp = a.v + head * a.s_head;

    // queries: row n (rows behind the last repeat it)
    bf16x8_t qf[Ge::NS];
    int32_t pos, own = 0;                                      // SHARED: the row's token among the tile's
    {
        const int32_t row = row0 + min(n, n_rows - 1);
        const int32_t tok = (int32_t)fast_div((uint32_t)row, a.G), u = row - tok * G;
        pos = rq.kv_len - rq.q_len + tok;
        own = tok;
        const uint16_t *q = a.q + (int64_t)(rq.row0 + tok) * a.q_tok + (int64_t)(head * G + u) * a.q_head;
#pragma unroll
        for (int s = 0; s < Ge::NS; ++s) qf[s] = *(const bf16x8_t *)(q + Ge::chan(s, g));
    }
    const float c2 = EL == kE4m3 ? a.scale_log2 * a.kscale[head] : a.scale_log2;

    // where the rows of a tile's keys are: lane's key 32 tile + (lane & 31), a tile ahead of the loads
    int32_t page = 0;
    uint32_t in_page = 0, off = 0;
    bool in_kv = false;
    int32_t entry = 0, entry_page = 0;                         // SEL: the place in the list and what stands there, a tile earlier still
    uint32_t entry_mask = 0, mask_l = 0, mask_n = 0, mask = 0; // SHARED: whose the page is,
    int32_t key_l = 0, key_n = 0, key = 0;                     // and the tile's first key: as looked up, requested, worked on
    auto peek = [&](int32_t tile) __attribute__((always_inline)) {
        entry = tile * kKT + (WHOLE ? 0 : lane & 31);
        const int32_t i = min((int32_t)fast_div((uint32_t)entry, a.page_size), listed - 1);
        entry_page = SHARED ? joint.pages[i] : list[i];
        if constexpr (SHARED) entry_mask = joint.masks[i];
    };
    int32_t seen = 0;                                          // WHOLE: keys of the tile up to the row's position, from its first
    auto look_up = [&](int32_t tile) __attribute__((always_inline)) {
        if constexpr (WHOLE) {
            const int32_t at = __builtin_amdgcn_readfirstlane(entry_page);
            const uint32_t idx = fast_div((uint32_t)entry, a.page_size);
            in_page = (uint32_t)entry - idx * a.page_size.d;
            in_kv = (int32_t)idx < listed && at >= 0 && at < a.table_width;
            seen = in_kv ? min(rq.kv_len - (at * (int32_t)a.page_size.d + (int32_t)in_page), kKT) : 0;
            page = table[in_kv ? at : 0];
            if constexpr (SHARED) {
                key_l = at * (int32_t)a.page_size.d + (int32_t)in_page;
                mask_l = (uint32_t)__builtin_amdgcn_readfirstlane((int)entry_mask);
            }
        } else if constexpr (SEL) {
            const uint32_t idx = fast_div((uint32_t)entry, a.page_size);
            in_page = (uint32_t)entry - idx * a.page_size.d;
            const bool is = (int32_t)idx < listed && entry_page >= 0 && entry_page < a.table_width;
            const int32_t at = is ? entry_page : 0;
            in_kv = is && at * (int32_t)a.page_size.d + (int32_t)in_page < rq.kv_len;
            page = table[at];
        } else {
            const int32_t key = tile * kKT + (lane & 31);
            in_kv = key < rq.kv_len;
            const uint32_t k = (uint32_t)min(key, rq.kv_len - 1);
            const uint32_t idx = fast_div(k, a.page_size);
            in_page = k - idx * a.page_size.d;
            page = table[idx];
        }
    };
    // off: the row's place in 16-byte units (of a row that is not there: the pool's first); returns a
    // bit per key whose row is there
    uint32_t ko[2], vo[8];                                     // places of the rows that this lane loads from
    float ks_n = 1.f, vs_n = 1.f;                              // BLK: the scales of the lane's key's page
    const char *kt_p = kp, *vt_p = vp;                         // WHOLE: the tile's first rows, and the lane's places behind them
    uint32_t k_lane[2] = {}, v_lane[8] = {};
    if constexpr (WHOLE) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
            k_lane[t] = (uint32_t)(16 * t + (lane >> 2)) * a.s_tok * 16 + (F8 && !Ge::PAIR ? 8 : 16) * (lane & 3);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v_lane[j] = (uint32_t)((j >> 2) * 16 + 4 * g + (j & 3)) * a.s_tok * 16 + (uint32_t)(min(n, Ge::NC - 1) * (F8 ? E : 2 * E));
    }
    auto place = [&]() __attribute__((always_inline)) {
        if constexpr (WHOLE) {
            const int32_t pg = __builtin_amdgcn_readfirstlane(page);
            const bool ok = in_kv && (uint32_t)pg < (uint32_t)a.n_pages;
            key_n = key_l;
            mask_n = mask_l;
            off = ok ? (uint32_t)pg * a.s_page + in_page * a.s_tok : 0u;
            kt_p = kp + (uint64_t)off * 16;
            vt_p = vp + (uint64_t)off * 16;
            if constexpr (BLK) {
                const float2 sc = *(const float2 *)(a.kscale + 2 * ((int64_t)(ok ? pg : 0) * a.n_heads + head));
                ks_n = sc.x;
                vs_n = sc.y;
            }
            return ok ? bits_to(seen - 1) : 0u;
        }
        const bool ok = in_kv && (uint32_t)page < (uint32_t)a.n_pages;
        off = (ok ? (uint32_t)page : 0u) * a.s_page + (ok ? in_page : 0u) * a.s_tok;
        if constexpr (BLK) {
            const float2 sc = *(const float2 *)(a.kscale + 2 * ((int64_t)(ok ? page : 0) * a.n_heads + head));
            ks_n = sc.x;
            vs_n = sc.y;
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) ko[t] = (uint32_t)__shfl((int)off, 16 * t + n);
        // V rows in the order of S^T's registers: place j of lane group g is key 4 g + j, 16 + 4 g + j - 4
#pragma unroll
        for (int j = 0; j < 8; ++j) vo[j] = (uint32_t)__shfl((int)off, (j >> 2) * 16 + 4 * g + (j & 3));
        return (uint32_t)__ballot(ok);
    };
    uint32_t kr[2][Ge::KW], vr[8][Ge::VW];
    auto load_k = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const char *p = WHOLE ? kt_p + k_lane[t] : kp + (uint64_t)ko[t] * 16 + (F8 && !Ge::PAIR ? 8 : 16) * g;
            if constexpr (!F8 || Ge::PAIR) {
#pragma unroll
                for (int s = 0; s < Ge::KW / 4; ++s) {
                    const u32x4_t x = *(const u32x4_t *)(p + 64 * s);
                    kr[t][4 * s] = x[0]; kr[t][4 * s + 1] = x[1]; kr[t][4 * s + 2] = x[2]; kr[t][4 * s + 3] = x[3];
                }
            } else {
#pragma unroll
                for (int s = 0; s < Ge::NS; ++s) {
                    const u32x2_t x = *(const u32x2_t *)(p + 32 * s);
                    kr[t][2 * s] = x[0]; kr[t][2 * s + 1] = x[1];
                }
            }
        }
    };
    // WHOLE: four lanes that follow one another read 64 bytes of one row, and the operand's lane (row n, piece g) has them
    // from lane 4 n + g.  (Rows that stay in the caches, as neighbouring tokens' pages do, are bound by the lines that the
    // first cache looks up: with every lane on its own row 4 times as many.)
    auto k_of = [&](uint32_t x) __attribute__((always_inline)) {
        return WHOLE ? (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (4 * n + g), (int)x) : x;
    };
    auto load_v = [&]() __attribute__((always_inline)) {
        const int c = min(n, Ge::NC - 1);                      // 96: lanes 12 .. 15 repeat lane 11, unused
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const char *p = WHOLE ? vt_p + v_lane[j] : vp + (uint64_t)vo[j] * 16 + c * (F8 ? E : 2 * E);
            if constexpr (Ge::VW == 4) {
                const u32x4_t x = *(const u32x4_t *)p;
                vr[j][0] = x[0]; vr[j][1] = x[1]; vr[j][2] = x[2]; vr[j][3] = x[3];
            } else if constexpr (Ge::VW == 2) {
                const u32x2_t x = *(const u32x2_t *)p;
                vr[j][0] = x[0]; vr[j][1] = x[1];
            } else {
                vr[j][0] = *(const uint32_t *)p;
            }
        }
    };
    auto sees = [&](int32_t key, int32_t p) __attribute__((always_inline)) {
        return key <= p && (a.window == 0 || key > p - a.window || key < a.n_sinks);
    };
    // every key of the tile is there and seen by every row
    auto whole_tile = [&](int32_t k0, uint32_t there) __attribute__((always_inline)) {
        if (SHARED) return there == 0xffffffffu && key + kKT - 1 <= p_lo && mask + 1 == 1u << rq.q_len;
        if (SEL) return there == 0xffffffffu;                  // (one position: there are the keys that it sees)
        return there == 0xffffffffu && k0 + kKT - 1 <= p_lo &&
               (a.window == 0 || k0 > p_hi - a.window || k0 + kKT <= a.n_sinks);
    };

    f32x4_t o[E];
    float m, l;
    const int32_t v0 = part_begin(kt.n, it.part, it.parts) + wave;
    uint32_t there, there_n, odd;
    // SHARED: keys that are there and finite need no care where only some rows see them.  Whether V held others shows in
    // the sums; then they are formed again, with care.
    for (bool careful = !SHARED;; careful = true) {
    m = -HUGE_VALF;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // A tile's K and V are requested while the tile before it is worked on: K as soon as its registers
    // have met the queries, V as soon as its own have become operands.
    there = there_n = odd = 0;
    if (v0 < v1) {
        if constexpr (SEL) peek(v0);
        look_up(kt.tile(v0));
        if constexpr (SEL) peek(v0 + NW);
        there = place();
        if constexpr (SHARED) {
            key = key_n;
            mask = mask_n;
        }
        load_k();
        load_v();
        if (v0 + NW < v1) look_up(kt.tile(v0 + NW));
        if constexpr (SEL) peek(v0 + 2 * NW);
    }
    for (int32_t v = v0; v < v1; v += NW) {
        const int32_t k0 = kt.tile(v) * kKT;
        const bool whole = whole_tile(k0, there);
        const float vs_v = vs_n;
        f32x4_t s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            const float ks = !BLK ? 1.f : WHOLE ? ks_n : __shfl(ks_n, 16 * t + n);
#pragma unroll
            for (int st = 0; st < Ge::NS; ++st) {
                bf16x8_t kf;
                if constexpr (F8) {
                    const uint32_t x = k_of(kr[t][2 * st]), y = k_of(kr[t][2 * st + 1]);
                    kf = frag(e4m3_pair<false>(x, ks), e4m3_pair<true>(x, ks), e4m3_pair<false>(y, ks), e4m3_pair<true>(y, ks));
                } else {
                    kf = frag(k_of(kr[t][4 * st]), k_of(kr[t][4 * st + 1]), k_of(kr[t][4 * st + 2]), k_of(kr[t][4 * st + 3]));
                }
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[st], s[t], 0, 0, 0);
            }
        }
        if (v + NW < v1) {
            there_n = place();
            if (v + 2 * NW < v1) look_up(kt.tile(v + 2 * NW));
            if constexpr (SEL) peek(v + 3 * NW);
            load_k();
        }
        uint32_t p2[4];                                    // exp2(s - m) as the operand of P V
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s[e >> 2][e & 3] * c2;
        if (!whole) {
            asm volatile("");                              // a branch, not selects on every tile
            // key k0 + 4 g + c is register e's, c = 16 (e >> 2) + (e & 3)
            const uint32_t vis = SHARED ? (there & bits_to(pos - key) & (0u - ((mask >> own) & 1u))) >> (4 * g)
                                 : SEL  ? there >> (4 * g)
                                        : visible(pos - k0 - 4 * g, there >> (4 * g), a.window, a.n_sinks - k0 - 4 * g);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = keep_if(vis, 16 * (e >> 2) + (e & 3), x[e]);
        }
        float mx = x[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mx = fmaxf(mx, x[e]);
        // sums are rescaled only where some row's maximum grows
        if (__any(mx > m)) {
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            mx = fmaxf(mx, m);
            const float al = __builtin_amdgcn_exp2f(m - (mx == -HUGE_VALF ? 0.f : mx));
            m = mx;
            l *= al;
#pragma unroll
            for (int i = 0; i < E; ++i) o[i] *= al;
        }
        const float ref = m == -HUGE_VALF ? 0.f : m;   // nothing seen so far: every weight is zero
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = __builtin_amdgcn_exp2f(x[e] - ref);
            sum += x[e];
        }
        l += sum;
#pragma unroll
        for (int q = 0; q < 4; ++q) p2[q] = pack_bf16(x[2 * q], x[2 * q + 1]);
        if (!whole && (careful || there != 0xffffffffu)) {
            // In a tile with a key that some row does not see a NaN or infinity of V would meet zero
            // weights: it becomes a zero here and reaches the rows that see it after the last tile.
            // Rows that are not there become zeros as well.
            asm volatile("");
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t is = 0u - ((there >> ((j >> 2) * 16 + 4 * g + (j & 3))) & 1u);
#pragma unroll
                for (int w = 0; w < Ge::VW; ++w) {
                    const uint32_t bad = F8 ? nan_bytes(vr[j][w]) : not_finite_halves(vr[j][w]);
                    odd |= bad & is;
                    vr[j][w] &= ~bad & is;
                }
            }
        }
        // V as bf16 pairs of channels
        uint32_t vb[8][E / 2];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float vs = !BLK ? 1.f : WHOLE ? vs_v : __shfl(vs_v, (j >> 2) * 16 + 4 * g + (j & 3));
#pragma unroll
            for (int w = 0; w < E / 2; ++w) {
                if constexpr (F8)
                    vb[j][w] = (w & 1) ? e4m3_pair<true>(vr[j][w >> 1], vs) : e4m3_pair<false>(vr[j][w >> 1], vs);
                else
                    vb[j][w] = vr[j][w];
            }
        }
#pragma unroll
        for (int i = 0; i < E; ++i) {
            uint32_t f[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                f[q] = __builtin_amdgcn_perm(vb[2 * q + 1][i >> 1], vb[2 * q][i >> 1], (i & 1) ? 0x07060302u : 0x05040100u);
            const bf16x8_t vf = frag(f[0], f[1], f[2], f[3]);
            o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, frag(p2[0], p2[1], p2[2], p2[3]),
                                                              o[i], 0, 0, 0);
        }
        if (v + NW < v1) load_v();
        there = there_n;
        if constexpr (SHARED) {
            key = key_n;
            mask = mask_n;
        }
    }
    if (careful) break;
    float zero = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) zero = __builtin_fmaf(o[i][r], 0.f, zero);
    if (!__any(zero != 0.f)) break;
    }
    if (__any(odd != 0)) {
        // NaNs and infinities of V that were left out of tiles which some row does not see whole: they
        // come to the rows that see their keys (whatever finite weight they have)
#pragma unroll 1
        for (int32_t v = v0; v < v1; v += NW) {
            const int32_t k0 = kt.tile(v) * kKT;
            if constexpr (SEL) peek(v);
            look_up(kt.tile(v));
            there = place();
            if constexpr (SHARED) {
                key = key_n;
                mask = mask_n;
            }
            if (whole_tile(k0, there)) continue;
#pragma unroll 1
            for (int kk = 0; kk < kKT; ++kk) {
                if (!((there >> kk) & 1)) continue;
                const char *vrow = WHOLE ? vt_p + (uint32_t)kk * a.s_tok * 16 : vp + (uint64_t)(uint32_t)__shfl((int)off, kk) * 16;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int c = min(4 * g + r, Ge::NC - 1) * E;
#pragma unroll
                    for (int i = 0; i < E; i += 2) {
                        const uint32_t u = F8 ? e4m3_pair<false>(*(const uint16_t *)(vrow + c + i)) : *(const uint32_t *)(vrow + 2 * (c + i));
                        const bool see = SHARED ? key + kk <= pos && ((mask >> own) & 1) : SEL || sees(k0 + kk, pos);
                        if (see && not_finite(u & 0xffffu)) o[i][r] += bf_lo(u);
                        if (see && not_finite(u & 0xffff0000u)) o[i + 1][r] += bf_hi(u);
                    }
                }
            }
        }
    }

    // ---- the waves' results, joined in their order
    const float vs = EL == kE4m3 ? a.vscale[head] : 1.f;
    float lt = l;
    lt += __shfl_xor(lt, 16);
    lt += __shfl_xor(lt, 32);
    if (g == 0) {
        ml[wave][n][0] = m;
        ml[wave][n][1] = lt;
    }
    __syncthreads();
    float mx = ml[0][n][0];
#pragma unroll
    for (int w = 1; w < NW; ++w) mx = fmaxf(mx, ml[w][n][0]);
    const float f = __builtin_amdgcn_exp2f(m - (mx == -HUGE_VALF ? 0.f : mx));
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int c = 4 * g + r;
        if (c < Ge::NC) {
#pragma unroll
            for (int i = 0; i < E; i += 4)
                *(float4 *)&ol[wave][n][E * c + i] = make_float4(o[i][r] * f, o[i + 1][r] * f,
                                                                o[i + 2][r] * f, o[i + 3][r] * f);
        }
    }
    __syncthreads();
    const int row = tid / (D / 8), ch = tid % (D / 8) * 8;
    if (row < 16 && row < n_rows) {
        float mr = ml[0][row][0];
#pragma unroll
        for (int w = 1; w < NW; ++w) mr = fmaxf(mr, ml[w][row][0]);
        const float ref = mr == -HUGE_VALF ? 0.f : mr;
        float lr = 0.f, y[8] = {};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            lr += ml[w][row][1] * __builtin_amdgcn_exp2f(ml[w][row][0] - ref);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] += ol[w][row][ch + e];
        }
        if (it.parts > 1) {
            float *w = cl.ws + ((int64_t)(it.slot + it.part) * a.n_heads + head) * (M * (D + 2));
            *(float4 *)(w + row * D + ch) = make_float4(y[0], y[1], y[2], y[3]);
            *(float4 *)(w + row * D + ch + 4) = make_float4(y[4], y[5], y[6], y[7]);
            if (ch == 0) {
                w[M * D + row] = mr;
                w[M * D + M + row] = lr;
            }
        } else {
            const float inv = lr == 0.f ? 0.f : vs / lr;
            const int32_t tok = (int32_t)fast_div((uint32_t)(row0 + row), a.G), u = row0 + row - tok * G;
            uint16_t *out = a.out + (int64_t)(rq.row0 + tok) * a.o_tok + (int64_t)(head * G + u) * a.o_head + ch;
            if (lr == 0.f) {
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = 0.f;
            }
            *(uint4 *)out = make_uint4(pack_bf16(y[0] * inv, y[1] * inv), pack_bf16(y[2] * inv, y[3] * inv),
                                       pack_bf16(y[4] * inv, y[5] * inv), pack_bf16(y[6] * inv, y[7] * inv));
            if (a.lse && ch == 0)
                a.lse[(int64_t)(rq.row0 + tok) * (a.n_heads * G) + head * G + u] =
                    lr == 0.f ? -HUGE_VALF : 0.6931471805599453f * (mr + __log2f(lr));
        }
    }
}

// ------------------------------------------------------------------ joining parts

// The partial sums of parts p0 .. p1 - 1 of a row, by one wave, brought to the maximum of all parts: lane
// l < D / 4 gets four channels' sum in t, every lane the weights' sum in lt and the maximum in mx.  Lane p
// holds the weight of part p (64 parts at a time); 4 D bytes of a part are D / 4 lanes' loads,
// so NP parts are added at once, slot p0 takes parts p0, p0 + NP, ..., and the slots are added at the
// end: always the same order.
// Eight loads on their way together: one single token over 131,072 keys in 171 parts 117 us instead of 136.
template <int D, int M>
__device__ __forceinline__ void join_parts(const float *w0, int64_t step, int rr, int parts, int p0, int p1, f32x4_t &t, float &lt,
                                           float &mx) {
    constexpr int LP = D / 4, NP = 64 / LP, U = 8;
    const int lane = threadIdx.x & 63;
    const int ch = lane % LP * 4, slot = lane / LP;
    mx = -HUGE_VALF;
    for (int p = lane; p < parts; p += 64) mx = fmaxf(mx, w0[p * step + M * D + rr]);
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) mx = fmaxf(mx, __shfl_xor(mx, s));
    const float ref = mx == -HUGE_VALF ? 0.f : mx;
    lt = 0.f;
    f32x4_t y = {0.f, 0.f, 0.f, 0.f};
    for (int pb = p0; pb < p1; pb += 64) {
        const int np = min(64, p1 - pb);
        float f = 0.f;
        if (lane < np) {
            const float *w = w0 + (pb + lane) * step + M * D + rr;
            f = __builtin_amdgcn_exp2f(w[0] - ref);
            lt += w[M] * f;
        }
        const float *x0 = w0 + pb * step + rr * D + ch;
        for (int q = 0; q < np; q += U * NP) {
            f32x4_t x[U];
#pragma unroll
            for (int i = 0; i < U; ++i) x[i] = *(const f32x4_t *)(x0 + min(q + i * NP + slot, np - 1) * step);
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int p = q + i * NP + slot;
                const float fq = __shfl(f, min(p, 63));
                if (slot < NP && p < np) y += x[i] * fq;
            }
        }
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) lt += __shfl_xor(lt, s);
    t = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < NP; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] += __shfl(y[e], s * LP + lane % LP);
}

template <int D> struct JoinLds { f32x4_t t[4][D / 4]; float lt[4]; };

// The rows of one item: four, a wave each, or, of a tile in many parts, one, whose parts the waves share.
template <int D, int M, int EL>
__device__ __forceinline__ void join_rows(const PagedArgs &a, const PagedClass &cl, const Item &it, const Request &rq, int head,
                                          JoinLds<D> &lds) {
    constexpr int LP = D / 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool wide = it.parts > kWideParts;
    const int rr = wide ? it.part : 4 * it.part + wave;
    const int32_t G = (int32_t)a.G.d;
    const int32_t row0 = it.tile * M;
    const int32_t n_rows = (int32_t)min((int64_t)rq.q_len * G - row0, (int64_t)M);
    const float *w0 = cl.ws + ((int64_t)it.slot * a.n_heads + head) * (M * (D + 2));
    const int64_t step = (int64_t)a.n_heads * (M * (D + 2));
    f32x4_t t = {0.f, 0.f, 0.f, 0.f};
    float lt = 0.f, mx = 0.f;
    if (rr < n_rows) {
        const int p0 = wide ? it.parts * wave / 4 : 0, p1 = wide ? it.parts * (wave + 1) / 4 : it.parts;
        join_parts<D, M>(w0, step, rr, it.parts, p0, p1, t, lt, mx);
    }
    if (wide) {                                                // the waves' sums, in their order
        if (lane < LP) lds.t[wave][lane] = t;
        if (lane == 0) lds.lt[wave] = lt;
        __syncthreads();
        if (wave > 0) return;
        const int l = lane < LP ? lane : 0;
        t = lds.t[0][l];
        lt = lds.lt[0];
#pragma unroll
        for (int w = 1; w < 4; ++w) {
            t += lds.t[w][l];
            lt += lds.lt[w];
        }
    }
    if (rr >= n_rows || lane >= LP) return;
    const float inv = (EL == kE4m3 ? a.vscale[head] : 1.f) / lt;
    const int32_t tok = (int32_t)fast_div((uint32_t)(row0 + rr), a.G), u = row0 + rr - tok * G;
    uint16_t *out = a.out + (int64_t)(rq.row0 + tok) * a.o_tok + (int64_t)(head * G + u) * a.o_head + 4 * lane;
    *(u32x2_t *)out = lt == 0.f ? u32x2_t{0u, 0u} : u32x2_t{pack_bf16(t[0] * inv, t[1] * inv), pack_bf16(t[2] * inv, t[3] * inv)};
    if (a.lse && lane == 0)
        a.lse[(int64_t)(rq.row0 + tok) * (a.n_heads * G) + head * G + u] =
            lt == 0.f ? -HUGE_VALF : 0.6931471805599453f * (mx + __log2f(lt));
}

}  // namespace
}  // namespace cb
