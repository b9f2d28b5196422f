// cb_attn_paged.hip -- attention of new tokens over pages on gfx950.
//
// For a row (new token, query head) with query q and the visible keys j:
//     s_j = scale q . k_j,  m = max s_j,  l = sum exp(s_j - m),  o = sum exp(s_j - m) v_j / l,
// formed in one pass over the keys: a new maximum m' rescales l and o by
// exp(m - m').  In log2 units throughout (scale carries log2 e).
//
// Rows of one request and KV head are (token, head of its group) pairs, so the
// group's query heads share every K and V row read.  The weights exp(s_j - m)
// are rounded to bf16 as the matrix cores' operand (2^-8 of a weight, below the
// output's own rounding where the values do not cancel) and summed unrounded;
// scores, sums and outputs are fp32.  Against 64 bits the outputs are off by 0.17%
// (decode) to 0.19% (a 2,048-token chunk) in norm, 0.166% of it their own rounding:
// weights in full would need a second product with V for what bf16 leaves out, half
// of the matrix work again.  m is the running maximum itself, so the largest weight
// is 1 (tile_body: to half an ulp of m), which the rounding hardly touches: with a
// maximum that may lag by 2^8, which spares rescaling, a chunk took 1.3% less and
// its outputs were off by 0.22%.
//
// rows_body: requests of few rows, 16 of them a workgroup.  Each wave has its
//   own key tiles of 32 keys, from memory straight into matrix-core operands:
//   S^T = K Q^T (16x16x32): lane l holds row n = l & 15 and, of key subtile t,
//     keys 16 t + 4 g + r, g = l >> 4, r = 0 .. 3: the statistics of a row are
//     per-lane numbers.
//   O^T = V^T P^T with the 32 keys in the order that S^T leaves them (4 g + r,
//     16 + 4 g + r): the P operand is S^T's registers rounded in place.  The V
//     operand (eight keys of one channel) comes from eight 16-byte pieces of
//     eight rows, transposed in registers (v_perm); channel E c + i goes to
//     output row c of product i, so a lane ends with E consecutive channels.
//   No LDS and no barrier until the waves' results are joined.  K of the next
//   tile is requested when K of this one has met the queries, V when V has
//   become operands, table entries a tile earlier.  Bound by memory: 64 single
//   tokens over 512 .. 16,384 keys (8 heads of 128, 8 query heads each, 1.36 GB)
//   250 us, 5.4 TB/s; in e4m3 pages, 8 over 65,536 .. 131,072 (1.57 GB), 312 us,
//   5.0 TB/s (a copy of 2 GiB runs at 4.9 TB/s here, both directions counted).
//   Two waves per SIMD are enough: with registers for three the calls took 274
//   and 344 us, 252 and 336 with two.  Requested at the top of a tile instead of
//   a tile ahead, K and V took the kernel from 245 and 319 to 270 and 375 us.
//
// tile_body: the other requests, 32 rows a wave, 128 or 256 a workgroup, K and
//   V tiles of 64 keys in LDS, two of them.
//   S^T = K Q^T (32x32x16): lane l holds row l & 31 and, of each 32 keys, those
//     with bit 2 = l >> 5.  O^T = V^T P^T takes P from these registers as
//     above; its V operand comes out of LDS transposed (ds_read_b64_tr_b16).
//   While a tile is worked on the next is on its way, and the table entries of
//   the one after are on theirs.  bf16 rows of 64 or 128 channels go to LDS by
//   its own loads (2.14 -> 2.07 ms below, and 370 -> 312 us for 8 new tokens of
//   64 requests over 512 .. 16,384 keys), others through registers: e4m3 becomes
//   bf16 on the way, and rows of 96 channels get their padding there.  A tile's
//   products with V run beside the weights of its next 16 keys.
//   Bound by the board's power: 2,048 tokens x 64 query heads over 32,768 keys
//   in 8 heads of 128 take 2.01 .. 2.20 ms from board to board, 0.97 .. 1.06
//   PFLOP/s (a bf16 matrix product of 8192^3: 1.21 .. 1.45), e4m3 1.99; heads of 96
//   1.82 ms, of 64 1.42 (the weights' work is the same, the products are half).  At
//   128 channels 1.32 kW and 2.01 GHz of 2.4 with the matrix units busy in 47 - 49% of
//   the cycles; four sums and maxima instead of one, other orders of the products
//   and wave priorities change nothing.
//   No LDS bank meets twice (with V's rows 288 bytes apart a quarter of the LDS
//   cycles were conflicts).
//
// Division of work: a row tile's keys go in `parts` to workgroups of their own
//   (cb_paged_rules.h), whose partial sums attn_join_kernel adds in an order that
//   depends on their number alone.  Every workgroup finds its row tile and part from the
//   requests' lengths by itself: sums over the requests by data-parallel moves,
//   about 2 us, instead of a plan that a caller would have to keep in step.
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
// Two e4m3 values (exact in bf16).
template <bool HI> __device__ __forceinline__ uint32_t e4m3_pair(uint32_t u) {
    const bf16x2_t v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, 1.0f, HI);
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

template <int D, bool F8, int NW>
__device__ __forceinline__ void rows_body(const PagedArgs &a, const PagedClass &cl, uint32_t block, SchedLds<NW> &sched,
                                          RowsLds<D, NW> &lds) {
    using Ge = Geo<D, F8>;
    constexpr int M = 16, E = Ge::E;
    auto &ol = lds.o;
    auto &ml = lds.ml;
    const int head = (int)(block % (uint32_t)a.n_heads);
    Item it;
    if (!find_item<M, kKT, false, NW>(a, cl, block / (uint32_t)a.n_heads, sched, it)) return;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, g = lane >> 4;
    const Request rq = request(a, it.req);
    const int32_t G = (int32_t)a.G.d;
    const int64_t rows = (int64_t)rq.q_len * G;                // at most M tiles of them exist: fits 32 bits below
    const int32_t row0 = it.tile * M;
    const int32_t n_rows = (int32_t)min(rows - row0, (int64_t)M);
    const int32_t tok0 = (int32_t)fast_div((uint32_t)row0, a.G), tok1 = (int32_t)fast_div((uint32_t)(row0 + n_rows - 1), a.G);
    const int32_t p_lo = rq.kv_len - rq.q_len + tok0, p_hi = rq.kv_len - rq.q_len + tok1;
    const KeyTiles kt = key_tiles(p_lo, p_hi, a.window, a.n_sinks, kKT);
    const int32_t v1 = part_begin(kt.n, it.part + 1, it.parts);
    const int32_t *table = a.table + it.req * a.table_stride;
    const char *kp = a.k + head * a.s_head, *vp = a.v + head * a.s_head;

    // queries: row n (rows behind the last repeat it)
    bf16x8_t qf[Ge::NS];
    int32_t pos;
    {
        const int32_t row = row0 + min(n, n_rows - 1);
        const int32_t tok = (int32_t)fast_div((uint32_t)row, a.G), u = row - tok * G;
        pos = rq.kv_len - rq.q_len + tok;
        const uint16_t *q = a.q + (int64_t)(rq.row0 + tok) * a.q_tok + (int64_t)(head * G + u) * a.q_head;
#pragma unroll
        for (int s = 0; s < Ge::NS; ++s) qf[s] = *(const bf16x8_t *)(q + Ge::chan(s, g));
    }
    const float c2 = F8 ? a.scale_log2 * a.kscale[head] : a.scale_log2;

    // where the rows of a tile's keys are: lane's key 32 tile + (lane & 31), a tile ahead of the loads
    int32_t page = 0;
    uint32_t in_page = 0, off = 0;
    bool in_kv = false;
    auto look_up = [&](int32_t tile) __attribute__((always_inline)) {
        const int32_t key = tile * kKT + (lane & 31);
        in_kv = key < rq.kv_len;
        const uint32_t k = (uint32_t)min(key, rq.kv_len - 1);
        const uint32_t idx = fast_div(k, a.page_size);
        in_page = k - idx * a.page_size.d;
        page = table[idx];
    };
    // off: the row's place in 16-byte units (of a row that is not there: the pool's first); returns a
    // bit per key whose row is there
    uint32_t ko[2], vo[8];                                     // places of the rows that this lane loads from
    auto place = [&]() __attribute__((always_inline)) {
        const bool ok = in_kv && (uint32_t)page < (uint32_t)a.n_pages;
        off = (ok ? (uint32_t)page : 0u) * a.s_page + (ok ? in_page : 0u) * a.s_tok;
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
            const char *p = kp + (uint64_t)ko[t] * 16;
            if constexpr (!F8 || Ge::PAIR) {
#pragma unroll
                for (int s = 0; s < Ge::KW / 4; ++s) {
                    const u32x4_t x = *(const u32x4_t *)(p + 64 * s + 16 * g);
                    kr[t][4 * s] = x[0]; kr[t][4 * s + 1] = x[1]; kr[t][4 * s + 2] = x[2]; kr[t][4 * s + 3] = x[3];
                }
            } else {
#pragma unroll
                for (int s = 0; s < Ge::NS; ++s) {
                    const u32x2_t x = *(const u32x2_t *)(p + 32 * s + 8 * g);
                    kr[t][2 * s] = x[0]; kr[t][2 * s + 1] = x[1];
                }
            }
        }
    };
    auto load_v = [&]() __attribute__((always_inline)) {
        const int c = min(n, Ge::NC - 1);                      // 96: lanes 12 .. 15 repeat lane 11, unused
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const char *p = vp + (uint64_t)vo[j] * 16 + c * (F8 ? E : 2 * E);
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
        return there == 0xffffffffu && k0 + kKT - 1 <= p_lo &&
               (a.window == 0 || k0 > p_hi - a.window || k0 + kKT <= a.n_sinks);
    };

    f32x4_t o[E];
    float m, l;
    m = -HUGE_VALF;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    // A tile's K and V are requested while the tile before it is worked on: K as soon as its registers
    // have met the queries, V as soon as its own have become operands.
    const int32_t v0 = part_begin(kt.n, it.part, it.parts) + wave;
    uint32_t there = 0, there_n = 0;
    uint32_t odd = 0;
    if (v0 < v1) {
        look_up(kt.tile(v0));
        there = place();
        load_k();
        load_v();
        if (v0 + NW < v1) look_up(kt.tile(v0 + NW));
    }
    for (int32_t v = v0; v < v1; v += NW) {
        const int32_t k0 = kt.tile(v) * kKT;
        const bool whole = whole_tile(k0, there);
        f32x4_t s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < Ge::NS; ++st) {
                bf16x8_t kf;
                if constexpr (F8) {
                    const uint32_t x = kr[t][2 * st], y = kr[t][2 * st + 1];
                    kf = frag(e4m3_pair<false>(x), e4m3_pair<true>(x), e4m3_pair<false>(y), e4m3_pair<true>(y));
                } else {
                    kf = frag(kr[t][4 * st], kr[t][4 * st + 1], kr[t][4 * st + 2], kr[t][4 * st + 3]);
                }
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[st], s[t], 0, 0, 0);
            }
        }
        if (v + NW < v1) {
            there_n = place();
            if (v + 2 * NW < v1) look_up(kt.tile(v + 2 * NW));
            load_k();
        }
        uint32_t p2[4];                                    // exp2(s - m) as the operand of P V
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s[e >> 2][e & 3] * c2;
        if (!whole) {
            asm volatile("");                              // a branch, not selects on every tile
            // key k0 + 4 g + c is register e's, c = 16 (e >> 2) + (e & 3)
            const uint32_t vis = visible(pos - k0 - 4 * g, there >> (4 * g), a.window, a.n_sinks - k0 - 4 * g);
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
        if (!whole) {
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
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int w = 0; w < E / 2; ++w) {
                if constexpr (F8)
                    vb[j][w] = (w & 1) ? e4m3_pair<true>(vr[j][w >> 1]) : e4m3_pair<false>(vr[j][w >> 1]);
                else
                    vb[j][w] = vr[j][w];
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
    }
    if (__any(odd != 0)) {
        // NaNs and infinities of V that were left out of tiles which some row does not see whole: they
        // come to the rows that see their keys (whatever finite weight they have)
#pragma unroll 1
        for (int32_t v = v0; v < v1; v += NW) {
            const int32_t k0 = kt.tile(v) * kKT;
            look_up(kt.tile(v));
            there = place();
            if (whole_tile(k0, there)) continue;
#pragma unroll 1
            for (int kk = 0; kk < kKT; ++kk) {
                if (!((there >> kk) & 1)) continue;
                const char *vrow = vp + (uint64_t)(uint32_t)__shfl((int)off, kk) * 16;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int c = min(4 * g + r, Ge::NC - 1) * E;
#pragma unroll
                    for (int i = 0; i < E; i += 2) {
                        const uint32_t u = F8 ? e4m3_pair<false>(*(const uint16_t *)(vrow + c + i)) : *(const uint32_t *)(vrow + 2 * (c + i));
                        const bool see = sees(k0 + kk, pos);
                        if (see && not_finite(u & 0xffffu)) o[i][r] += bf_lo(u);
                        if (see && not_finite(u & 0xffff0000u)) o[i + 1][r] += bf_hi(u);
                    }
                }
            }
        }
    }

    // ---- the waves' results, joined in their order
    const float vs = F8 ? a.vscale[head] : 1.f;
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

// ------------------------------------------------------------------ tile kernel

typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

// Key of accumulator register v in lane half h of S^T's 32-key subtile.
__device__ __forceinline__ int acc_key(int v, int h) { return 8 * (v >> 2) + 4 * h + (v & 3); }

// A NaN among the three is the maximum (v_maximum3_f32: no extra instruction quiets its operands).
__device__ __forceinline__ float max3(float a, float b, float c) {
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

// The maximum over lanes l and l ^ 32.
__device__ __forceinline__ float both_halves_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __builtin_elementwise_maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

typedef __attribute__((address_space(3))) char lds_char_t;
// 16 bytes per lane from memory to LDS at m0 + 16 lane, counted by vmcnt.  A load to LDS may follow a write of M0
// one wait state later at the earliest, and the compiler does not see into the statement: it waits itself.
// The compiler keeps nothing in M0 here.
__device__ __forceinline__ void copy16(const void *from, uint32_t m0) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(m0) : "memory");
}

template <int D> struct TileLds {
    // bytes between rows of K and V: 16 rows' 16-byte pieces, and 4 rows' 64 bytes, in 64 banks each
    static constexpr int KS = 2 * D + 16, VS = D == 96 ? 192 : 2 * D + 64;
    char kv[2][kTileKT * (KS + VS)];
    int32_t odd;
};

template <int D, bool F8, int NW>
__device__ __forceinline__ void tile_body(const PagedArgs &a, const PagedClass &cl, uint32_t block, SchedLds<NW> &sched,
                                          TileLds<D> &tl) {
    constexpr int M = 32 * NW, NT = 64 * NW, KT = kTileKT, NS = D / 16, ND = D / 32;
    constexpr bool DMA = !F8 && D != 96;                       // rows go to LDS as they are, by its own loads
    constexpr int KS = DMA ? 2 * D : TileLds<D>::KS, VS = DMA ? 2 * D : TileLds<D>::VS;
    constexpr int CPR = F8 ? D / 16 : D / 8;                   // 16-byte pieces of a row in memory
    constexpr int NP = (KT * CPR + NT - 1) / NT;               // pieces of a thread, for each of K and V
    constexpr bool RAGGED = KT * CPR % NT != 0;
    constexpr int STAGE = KT * (KS + VS);
    char *lds = tl.kv[0];
    int32_t &odd = tl.odd;
    const int head = (int)(block % (uint32_t)a.n_heads);
    Item it;
    if (!find_item<M, KT, false, NW>(a, cl, block / (uint32_t)a.n_heads, sched, it)) return;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, h = lane >> 5;
    const Request rq = request(a, it.req);
    const int32_t G = (int32_t)a.G.d;
    const int32_t row0 = it.tile * M;
    const int32_t n_rows = (int32_t)min((int64_t)rq.q_len * G - row0, (int64_t)M);
    const int32_t base = rq.kv_len - rq.q_len;                 // position of new token 0
    const int32_t p_lo = base + (int32_t)fast_div((uint32_t)row0, a.G);
    const int32_t p_hi = base + (int32_t)fast_div((uint32_t)(row0 + n_rows - 1), a.G);
    const KeyTiles kt = key_tiles(p_lo, p_hi, a.window, a.n_sinks, KT);
    const int32_t v0 = part_begin(kt.n, it.part, it.parts), v1 = part_begin(kt.n, it.part + 1, it.parts);
    const int32_t *table = a.table + it.req * a.table_stride;
    const char *kp = a.k + head * a.s_head, *vp = a.v + head * a.s_head;
    // weights are exp2(c2 s - m) with c2 > 0: a negative scale turns the queries' signs, and a zero
    // one becomes the least number (a masked score, -infinity, stays what it is)
    float c2 = F8 ? a.scale_log2 * a.kscale[head] : a.scale_log2;
    const uint32_t flip = c2 < 0.f ? 0x80008000u : 0u;
    c2 = fmaxf(fabsf(c2), 1.17549435e-38f);
    if (tid == 0) odd = 0;

    // queries of this wave's 32 rows (rows behind the last repeat it)
    bf16x8_t qf[NS];
    int32_t pos;                                           // of the lane's rows
    const int w0 = 32 * wave;
    {
        const int32_t row = row0 + min(w0 + n, n_rows - 1);
        const int32_t tok = (int32_t)fast_div((uint32_t)row, a.G), u = row - tok * G;
        pos = base + tok;
        const uint16_t *q = a.q + (int64_t)(rq.row0 + tok) * a.q_tok + (int64_t)(head * G + u) * a.q_head;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const uint4 x = *(const uint4 *)(q + 16 * s + 8 * h);
            qf[s] = frag(x.x ^ flip, x.y ^ flip, x.z ^ flip, x.w ^ flip);
        }
    }
    const int32_t s_lo = __builtin_amdgcn_readfirstlane(pos);
    const int32_t s_hi = __builtin_amdgcn_readlane(pos, 31);

    // the places of a tile's 64 rows: lane l looks up key l, a tile ahead of the loads that use it
    int32_t page = 0;
    uint32_t in_page = 0;
    bool in_kv = false;
    auto look_up = [&](int32_t tile) __attribute__((always_inline)) {
        const int32_t key = tile * KT + lane;
        in_kv = key < rq.kv_len;
        const uint32_t k = (uint32_t)min(key, rq.kv_len - 1);
        const uint32_t idx = fast_div(k, a.page_size);
        in_page = k - idx * a.page_size.d;
        page = table[idx];
    };
    auto place = [&](uint64_t &there) __attribute__((always_inline)) {
        const bool ok = in_kv && (uint32_t)page < (uint32_t)a.n_pages;
        there = __ballot(ok);
        return (ok ? (uint32_t)page : 0u) * a.s_page + (ok ? in_page : 0u) * a.s_tok;
    };
    // By LDS's own loads piece p of a tile lands in place p: rows without gaps, their 16-byte pieces in
    // an order of their own, so that the operands' reads meet no bank twice.  Row r has K's piece c in
    // place c ^ f(r), f = r mod 16 (64 channels: r / 2 mod 8), and V's in place c ^ 4 (r mod 4) (64
    // channels: c ^ 4 (r / 2 mod 2)).
    const int my_row = tid / CPR, my_c = tid - my_row * CPR;
    const int k_piece = 16 * (my_c ^ (D == 128 ? my_row & 15 : my_row >> 1 & 7));
    const int v_piece = 16 * (my_c ^ (D == 128 ? 4 * (my_row & 3) : 4 * (my_row >> 1 & 1)));
    u32x4_t kr[NP], vr[NP];
    auto load = [&](uint32_t off, int st) __attribute__((always_inline)) {
        uint32_t ro[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) ro[i] = (uint32_t)__shfl((int)off, (tid + NT * i) / CPR & 63);
        __builtin_amdgcn_sched_barrier(0);                     // one trip to the other lanes for all of them
        if constexpr (DMA) {
            const uint32_t to = (uint32_t)(uintptr_t)(lds_char_t *)(lds + st * STAGE) + 1024 * wave;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                copy16(kp + (uint64_t)ro[i] * 16 + k_piece, __builtin_amdgcn_readfirstlane(to + 16 * NT * i));
                copy16(vp + (uint64_t)ro[i] * 16 + v_piece, __builtin_amdgcn_readfirstlane(to + 16 * NT * i + KT * KS));
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int id = tid + NT * i;
            const int row = id / CPR, c = id - row * CPR;
            const uint64_t at = (uint64_t)ro[i] * 16 + 16 * c;
            if (RAGGED && id >= KT * CPR) continue;
            kr[i] = *(const u32x4_t *)(kp + at);
            vr[i] = *(const u32x4_t *)(vp + at);
        }
    };
    // In a tile with a key that some row does not see (edge) a NaN or infinity of V would meet zero
    // weights: it becomes a zero here and reaches the rows that see it after the last tile.  V's rows
    // that are not there become zeros as well.
    auto store = [&](int st, uint64_t there, bool edge) __attribute__((always_inline)) {
        char *ks = lds + st * STAGE, *vs = ks + KT * KS;
        if constexpr (DMA) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wave's pieces have landed
            if (!edge) return;
#pragma unroll
            for (int i = 0; i < NP; ++i) vr[i] = *(const u32x4_t *)(vs + 16 * (tid + NT * i));
        }
        if (edge) {
            uint32_t found = 0;
            asm volatile("");
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int id = tid + NT * i, row = id / CPR;
                if (RAGGED && id >= KT * CPR) continue;
                const uint32_t is = 0u - (uint32_t)((there >> (row & 63)) & 1);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint32_t bad = F8 ? nan_bytes(vr[i][w]) : not_finite_halves(vr[i][w]);
                    found |= bad & is;
                    vr[i][w] &= ~bad & is;
                }
            }
            if (found) odd = 1;
        }
        if constexpr (DMA) {
#pragma unroll
            for (int i = 0; i < NP; ++i) *(u32x4_t *)(vs + 16 * (tid + NT * i)) = vr[i];
            return;
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int id = tid + NT * i;
            if (RAGGED && id >= KT * CPR) continue;
            const int row = id / CPR, c = id - row * CPR;
            if constexpr (F8) {
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const uint32_t k0 = kr[i][2 * w], k1 = kr[i][2 * w + 1], x0 = vr[i][2 * w], x1 = vr[i][2 * w + 1];
                    *(uint4 *)(ks + row * KS + 32 * c + 16 * w) =
                        make_uint4(e4m3_pair<false>(k0), e4m3_pair<true>(k0), e4m3_pair<false>(k1), e4m3_pair<true>(k1));
                    *(uint4 *)(vs + row * VS + 32 * c + 16 * w) =
                        make_uint4(e4m3_pair<false>(x0), e4m3_pair<true>(x0), e4m3_pair<false>(x1), e4m3_pair<true>(x1));
                }
            } else {
                *(u32x4_t *)(ks + row * KS + 16 * c) = kr[i];
                *(u32x4_t *)(vs + row * VS + 16 * c) = vr[i];
            }
        }
    };
    // every key of the tile is there and seen by every row, of the wave and of the workgroup
    auto seen = [&](int32_t k0, uint64_t there, int32_t lo, int32_t hi) __attribute__((always_inline)) {
        return there == ~0ull && k0 <= lo - (KT - 1) && (k0 > (a.window == 0 ? INT32_MIN : hi - a.window) || k0 <= a.n_sinks - KT);
    };
    auto next_tile = [&](int32_t t) __attribute__((always_inline)) { return t + 1 == kt.sink ? kt.first : t + 1; };

    f32x16_t o[ND];
    float m, l;
    m = -HUGE_VALF;
    l = 0.f;
#pragma unroll
    for (int q = 0; q < ND; ++q) o[q] = f32x16_t{};
    // The exponent is fma(s, c2, -m) with m = c2 max s rounded: off by up to half an ulp of m, alike for every
    // key of a row, so it cancels against the sum of the weights as long as it is small.  Where some row's |m| passes 2^24 it
    // is not (2^32 would overflow the weights): from there the scores take c2, rounded, before.
    bool far = false;
    // K operand: key n, channels 16 q + 8 h .. + 7, at k_at ^ 32 q (rows without gaps) or k_at + 32 q.
    // V^T operand: keys 16 kk + 4 h + {0 .. 3} and + 8, channel 32 q + (lane & 31), at v_at ^ 64 q or
    // v_at + 64 q.
    const int r4 = (lane >> 2) & 3, f_n = D == 128 ? n & 15 : n >> 1 & 7;
    const int k_at = n * KS + (DMA ? 16 * (h ^ f_n) : 16 * h);
    const int v_at = (4 * h + r4) * VS + 32 * ((lane >> 4) & 1) + 8 * (lane & 3) + (DMA ? (D == 128 ? 64 * r4 : 64 * (r4 >> 1)) : 0);
    auto k_place = [&](int q) __attribute__((always_inline)) { return DMA ? k_at ^ 32 * q : k_at + 32 * q; };
    auto v_place = [&](int q) __attribute__((always_inline)) { return DMA ? v_at ^ 64 * q : v_at + 64 * q; };

    auto read_v = [&](const char *vs, int kk, bf16x8_t *f) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < ND; ++q) {
            const char *pp = vs + v_place(q) + 16 * kk * VS;
            const s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)pp);
            const s16x4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(pp + 8 * VS));
            typedef __attribute__((ext_vector_type(8))) short s16x8_t;
            const s16x8_t v8 = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
            f[q] = __builtin_bit_cast(bf16x8_t, v8);
        }
    };

    uint64_t there = 0, there_n = 0;
    int32_t t0 = kt.tile(v0), t1 = next_tile(t0), t2 = next_tile(t1);   // this tile and the two behind it
    if (v0 < v1) {
        look_up(t0);
        const uint32_t off = place(there);
        if (v0 + 1 < v1) look_up(t1);
        load(off, 0);
        __syncthreads();                                       // odd is set
        store(0, there, !seen(t0 * KT, there, p_lo, p_hi));
    }
    __syncthreads();
    for (int32_t v = v0; v < v1; ++v) {
        const int st = (v - v0) & 1;
        const int32_t k0 = t0 * KT;
        // (the table entries first: what waits for them later does not wait for the rows)
        uint32_t off = 0;
        if (v + 1 < v1) off = place(there_n);
        if (v + 2 < v1) look_up(t2);
        if (v + 1 < v1) load(off, st ^ 1);
        const char *ks = lds + st * STAGE, *vs = ks + KT * KS;
        f32x16_t s[2];
        s[0] = s[1] = f32x16_t{};
#pragma unroll
        for (int q = 0; q < NS; ++q) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const bf16x8_t kf = *(const bf16x8_t *)(ks + k_place(q) + 32 * t * KS);
                s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[q], s[t], 0, 0, 0);
            }
        }
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int i = 0; i < 2 * NS - 4; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
        if (!seen(k0, there, s_lo, s_hi)) {
            asm volatile("");                                  // a branch, not selects on every tile
            // key k0 + 4 h + c is register e's, c = 32 (e >> 4) + acc_key(e & 15, 0)
            const int32_t p = pos - k0 - 4 * h;
            const uint64_t bits = there >> (4 * h);
            const uint32_t vis[2] = {visible(p, (uint32_t)bits, a.window, a.n_sinks - k0 - 4 * h),
                                     visible(p - 32, (uint32_t)(bits >> 32), a.window, a.n_sinks - k0 - 4 * h - 32)};
#pragma unroll
            for (int e = 0; e < 32; ++e)
                s[e >> 4][e & 15] = keep_if(vis[e >> 4], acc_key(e & 15, 0), s[e >> 4][e & 15]);
        }
        bf16x8_t vf[2][ND];
        read_v(vs, 0, vf[0]);
        __builtin_amdgcn_sched_barrier(0);
        uint32_t pk[16];
        float mx = max3(s[0][0], s[0][1], s[0][2]);
#pragma unroll
        for (int e = 3; e < 31; e += 2) mx = max3(mx, s[e >> 4][e & 15], s[(e + 1) >> 4][(e + 1) & 15]);
        mx = max3(mx, s[1][15], s[1][15]);
        mx = both_halves_max(mx) * c2;
        // sums are rescaled only where some row's maximum grows
        if (__any(mx > m)) {
            const float mn = fmaxf(m, mx);
            const float al = __builtin_amdgcn_exp2f(m - (mn == -HUGE_VALF ? 0.f : mn));
            m = mn;
            l *= al;
#pragma unroll
            for (int q = 0; q < ND; ++q) o[q] *= al;
            far = __any(fabsf(m == -HUGE_VALF ? 0.f : m) > 16777216.f);
        }
        const float ref = m == -HUGE_VALF ? 0.f : m;
        float ce = c2;
        if (far) {
#pragma unroll
            for (int e = 0; e < 32; ++e) s[e >> 4][e & 15] *= c2;
            ce = 1.f;
        }
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float x0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 3][2 * e & 15], ce, -ref));
            const float x1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 3][(2 * e & 15) + 1], ce, -ref));
            sum += x0;
            sum += x1;
            pk[e] = pack_bf16(x0, x1);
        }
        l += sum;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            if (kk < 3) read_v(vs, kk + 1, vf[(kk + 1) & 1]);
#pragma unroll
            for (int q = 0; q < ND; ++q)
                o[q] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    vf[kk & 1][q], frag(pk[4 * kk], pk[4 * kk + 1], pk[4 * kk + 2], pk[4 * kk + 3]),
                    o[q], 0, 0, 0);
        }
        // a quarter of the weights, then its products beside the next quarter's
        __builtin_amdgcn_sched_group_barrier(0x406, 28, 1);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            if (kk < 3) __builtin_amdgcn_sched_group_barrier(0x100, 2 * ND, 1);
#pragma unroll
            for (int q = 0; q < ND; ++q) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
                if (kk < 3) __builtin_amdgcn_sched_group_barrier(0x406, (28 + ND - 1) / ND, 1);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (v + 1 < v1) store(st ^ 1, there_n, !seen(t1 * KT, there_n, p_lo, p_hi));
        there = there_n;
        t0 = t1;
        t1 = t2;
        t2 = next_tile(t2);
        __syncthreads();
    }
    if (odd) {
        // NaNs and infinities of V that were left out of tiles which some row does not see whole: they
        // come to the rows that see their keys (whatever finite weight they have)
#pragma unroll 1
        for (int32_t v = v0; v < v1; ++v) {
            const int32_t k0 = kt.tile(v) * KT;
            look_up(kt.tile(v));
            const uint32_t off = place(there);
            if (seen(k0, there, p_lo, p_hi)) continue;
#pragma unroll 1
            for (int kk = 0; kk < KT; ++kk) {
                if (!((there >> kk) & 1)) continue;
                const char *vrow = vp + (uint64_t)(uint32_t)__shfl((int)off, kk) * 16;
                const int32_t key = k0 + kk;
                const bool see = key <= pos && (a.window == 0 || key > pos - a.window || key < a.n_sinks);
#pragma unroll
                for (int q = 0; q < ND; ++q)
#pragma unroll
                    for (int r = 0; r < 16; r += 2) {
                        const int c = 32 * q + acc_key(r, h);
                        const uint32_t u = F8 ? e4m3_pair<false>(*(const uint16_t *)(vrow + c)) : *(const uint32_t *)(vrow + 2 * c);
                        if (see && not_finite(u & 0xffffu)) o[q][r] += bf_lo(u);
                        if (see && not_finite(u & 0xffff0000u)) o[q][r + 1] += bf_hi(u);
                    }
            }
        }
    }

    const float vsc = F8 ? a.vscale[head] : 1.f;
    const int rr = w0 + n;
    const float lr = l + __shfl_xor(l, 32);
    if (rr >= n_rows) return;
    if (it.parts > 1) {
        float *w = cl.ws + ((int64_t)(it.slot + it.part) * a.n_heads + head) * (M * (D + 2));
#pragma unroll
        for (int q = 0; q < ND; ++q)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *(float4 *)(w + rr * D + 32 * q + acc_key(r, h)) =
                    make_float4(o[q][r], o[q][r + 1], o[q][r + 2], o[q][r + 3]);
        if (h == 0) {
            w[M * D + rr] = m;
            w[M * D + M + rr] = lr;
        }
    } else {
        const int32_t tok = (int32_t)fast_div((uint32_t)(row0 + rr), a.G), u = row0 + rr - tok * G;
        uint16_t *out = a.out + (int64_t)(rq.row0 + tok) * a.o_tok + (int64_t)(head * G + u) * a.o_head;
        const float inv = vsc / lr;
#pragma unroll
        for (int q = 0; q < ND; ++q)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                uint2 y = make_uint2(pack_bf16(o[q][r] * inv, o[q][r + 1] * inv),
                                     pack_bf16(o[q][r + 2] * inv, o[q][r + 3] * inv));
                if (lr == 0.f) y = make_uint2(0u, 0u);
                *(uint2 *)(out + 32 * q + acc_key(r, h)) = y;
            }
        if (a.lse && h == 0)
            a.lse[(int64_t)(rq.row0 + tok) * (a.n_heads * G) + head * G + u] =
                lr == 0.f ? -HUGE_VALF : 0.6931471805599453f * (m + __log2f(lr));
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
template <int D, int M, bool F8>
__device__ __forceinline__ void join_rows(const PagedArgs &a, const PagedClass &cl, const Item &it, int head, JoinLds<D> &lds) {
    constexpr int LP = D / 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool wide = it.parts > kWideParts;
    const int rr = wide ? it.part : 4 * it.part + wave;
    const Request rq = request(a, it.req);
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
    const float inv = (F8 ? a.vscale[head] : 1.f) / lt;
    const int32_t tok = (int32_t)fast_div((uint32_t)(row0 + rr), a.G), u = row0 + rr - tok * G;
    uint16_t *out = a.out + (int64_t)(rq.row0 + tok) * a.o_tok + (int64_t)(head * G + u) * a.o_head + 4 * lane;
    *(u32x2_t *)out = lt == 0.f ? u32x2_t{0u, 0u} : u32x2_t{pack_bf16(t[0] * inv, t[1] * inv), pack_bf16(t[2] * inv, t[3] * inv)};
    if (a.lse && lane == 0)
        a.lse[(int64_t)(rq.row0 + tok) * (a.n_heads * G) + head * G + u] =
            lt == 0.f ? -HUGE_VALF : 0.6931471805599453f * (mx + __log2f(lt));
}

// Blocks go round while there are more items.
template <int D, int M, int KT, bool F8>
__device__ __forceinline__ void join_body(const PagedArgs &a, const PagedClass &cl, uint32_t block, uint32_t blocks,
                                          SchedLds<4> &sched, JoinLds<D> &lds) {
    for (uint32_t b = block;; b += blocks) {
        const uint32_t idx = b / (uint32_t)a.n_heads;
        Item it;
        if (!find_item<M, KT, true, 4>(a, cl, idx, sched, it)) return;
        join_rows<D, M, F8>(a, cl, it, (int)(b - idx * a.n_heads), lds);
        __syncthreads();                                       // the item and the sums have been read
    }
}

// ------------------------------------------------------------------ kernels

template <int D, bool F8>
__global__ __launch_bounds__(256) void attn_rows_kernel(PagedArgs a) {
    __shared__ SchedLds<4> sched;
    __shared__ __attribute__((aligned(16))) RowsLds<D, 4> lds;
    rows_body<D, F8, 4>(a, a.rows, blockIdx.x, sched, lds);
}

// The requests with few rows and the others in one launch, runs of the two in turn, so that a compute
// unit has products of the one beside loads of the other; a tile, which takes longer, first.  With fewer
// than a run of either kind all tiles come first.  64 single tokens over 1,024 .. 8,192 keys beside a chunk
// of 512 (8 heads of 128, 8 query heads each): 252 us, 272 with all tiles first, 272 with runs of 8; 24
// beside three chunks of 515 with windows of 1,024, which have no whole run: 53, 72 with runs of 8.
template <int D, bool F8, int NW>
__global__ __launch_bounds__(64 * NW, 2) void attn_tile_kernel(PagedArgs a) {
    __shared__ SchedLds<NW> sched;
    __shared__ __attribute__((aligned(16))) union { RowsLds<D, NW> rows; TileLds<D> tile; } lds;
    const uint32_t pairs = min(a.tile.blocks, a.rows.blocks) / kRun, run = blockIdx.x / kRun;
    uint32_t b;
    bool tile;
    if (run < 2 * pairs) {
        tile = !(run & 1);
        b = run / 2 * kRun + blockIdx.x % kRun;
    } else {
        b = blockIdx.x - pairs * kRun;
        tile = b < a.tile.blocks;
        if (!tile) b -= a.tile.blocks - pairs * kRun;
    }
    if (tile) tile_body<D, F8, NW>(a, a.tile, b, sched, lds.tile);
    else rows_body<D, F8, NW>(a, a.rows, b, sched, lds.rows);
}

template <int D, bool F8, int NW>
__global__ __launch_bounds__(256) void attn_join_kernel(PagedArgs a) {
    __shared__ SchedLds<4> sched;
    __shared__ JoinLds<D> lds;
    if (blockIdx.x < a.tile.join_blocks) join_body<D, 32 * NW, kTileKT, F8>(a, a.tile, blockIdx.x, a.tile.join_blocks, sched, lds);
    else join_body<D, 16, kKT, F8>(a, a.rows, blockIdx.x - a.tile.join_blocks, a.rows.join_blocks, sched, lds);
}

constexpr int kSmallRows = 16;          // rows of a request up to which rows_body takes it beside tile_body
// ... and alone, when no request is said to have more.  64 requests over 512 .. 16,384 keys (8 heads of 128),
// rows_body and tile_body: 16 rows each 228 and 231 us, 24 rows 276 and 298, 32 rows 281 and 300, 40 rows
// 349 and 305, 64 rows 451 and 313; the same with 4 query heads a KV head as with 8.
constexpr int kFewRows = 32;
constexpr int kTileTarget = 512;        // workgroups of tile_body (of 128 rows) that long rows are divided into
constexpr int kJoinBlocks = 2048;

// The blocks of a class of requests and its part of the workspace.
template <int D, int M, int KT>
bool prepare_class(const PagedArgs &a, PagedClass &c, int target, int64_t row_min, int64_t row_max, char *&ws, int64_t &ws_bytes) {
    const int64_t slot = (int64_t)M * (D + 2) * 4;
    c.row_min = row_min;
    c.row_max = row_max;
    c.target = (int32_t)std::min<int64_t>(target, ws_bytes / (2 * slot));
    // no row is long enough to be divided
    const int32_t most = (int32_t)std::min<int64_t>((int64_t)a.table_width * a.page_size.d, INT32_MAX);
    if (parts_of(key_tiles_bound(most, M, a.window, a.n_sinks, KT), part_min(KT), split_min(KT)) == 1) c.target = 0;
    c.ws = (float *)ws;
    ws += 2 * slot * c.target;
    ws_bytes -= 2 * slot * c.target;
    const int64_t tiles = row_tiles_bound(a.n_tokens, a.n_reqs, a.G.d, M, row_max);
    const int64_t blocks = (tiles + c.target / a.n_heads) * a.n_heads;
    const int64_t join = std::min<int64_t>(tiles, c.target / a.n_heads) * M * a.n_heads;
    if (blocks > INT32_MAX / 2 || join > INT32_MAX / 2) return false;
    c.blocks = (uint32_t)blocks;
    c.join_blocks = (uint32_t)std::min<int64_t>(join, kJoinBlocks);
    return true;
}

// Rows up to which a request goes to rows_body in a launch of tile_body: none where no other request could be
// beside it, or where one token has more.
int32_t least_rows(int32_t G, int32_t n_reqs) { return G <= kSmallRows && n_reqs > 1 ? kSmallRows : 0; }

template <int D, bool F8, int NW>
hipError_t launch_tiles(PagedArgs a, char *w, int64_t ws_bytes, hipStream_t s) {
    constexpr int M = 32 * NW;
    const int64_t least = least_rows((int32_t)a.G.d, a.n_reqs);
    if (least > 0 && !prepare_class<D, 16, kKT>(a, a.rows, kTarget, 0, least, w, ws_bytes)) return hipErrorInvalidValue;
    if (!prepare_class<D, M, kTileKT>(a, a.tile, kTileTarget * 4 / NW, least, INT64_MAX, w, ws_bytes)) return hipErrorInvalidValue;
    hipLaunchKernelGGL((attn_tile_kernel<D, F8, NW>), dim3(a.tile.blocks + a.rows.blocks), dim3(64 * NW), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
    const uint32_t join = a.tile.join_blocks + a.rows.join_blocks;
    if (join > 0) hipLaunchKernelGGL((attn_join_kernel<D, F8, NW>), dim3(join), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <int D, bool F8>
hipError_t launch(PagedArgs a, int32_t max_q_len, void *ws, int64_t ws_bytes, hipStream_t s) {
    char *w = (char *)ws;
    const int64_t rows = (int64_t)max_q_len * a.G.d;
    if constexpr (D != 96) {
        // 256 rows share a tile's way to LDS where there are two such workgroups for every compute unit
        // and the requests are alike (their tokens fill three quarters of n_reqs x max_q_len).  A chunk
        // of 2,048 x 8 rows in 8 heads over 32,768 keys: 2.09 ms, 2.20 with 128 rows; three chunks of
        // 515 x 4 beside 24 single tokens: 64 us, 54 with 128 rows.  Heads of 96, whose 1.5 pieces a
        // thread leave half the loads of the second empty: 1.93 and 1.77 ms.
        if (rows >= 256 && (int64_t)a.n_tokens * a.G.d * a.n_heads >= 2 * 256 * 256 &&
            4 * (int64_t)a.n_tokens >= 3 * (int64_t)a.n_reqs * max_q_len)
            return launch_tiles<D, F8, 8>(a, w, ws_bytes, s);
    }
    if (rows > kFewRows) return launch_tiles<D, F8, 4>(a, w, ws_bytes, s);
    // few rows everywhere: rows_body alone, whatever the lengths turn out to be
    if (!prepare_class<D, 16, kKT>(a, a.rows, kTarget, 0, INT64_MAX, w, ws_bytes)) return hipErrorInvalidValue;
    hipLaunchKernelGGL((attn_rows_kernel<D, F8>), dim3(a.rows.blocks), dim3(256), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
    if (a.rows.join_blocks > 0) hipLaunchKernelGGL((attn_join_kernel<D, F8, 4>), dim3(a.rows.join_blocks), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

int64_t attn_paged_workspace_bytes(int32_t d, int32_t G, int32_t n_reqs, int32_t max_q_len) {
    const int64_t rows = (int64_t)2 * kTarget * 16 * (d + 2) * 4, tile = (int64_t)2 * kTileTarget * 128 * (d + 2) * 4;
    if ((int64_t)max_q_len * G <= kFewRows) return rows;
    return (least_rows(G, n_reqs) > 0 ? rows : 0) + tile;
}

hipError_t launch_attn_paged(const PagedArgs &a, int32_t d, bool f8, int32_t max_q_len, void *ws, int64_t ws_bytes,
                             hipStream_t s) {
    switch (d * 2 + f8) {
        case 128: return launch<64, false>(a, max_q_len, ws, ws_bytes, s);
        case 129: return launch<64, true>(a, max_q_len, ws, ws_bytes, s);
        case 192: return launch<96, false>(a, max_q_len, ws, ws_bytes, s);
        case 193: return launch<96, true>(a, max_q_len, ws, ws_bytes, s);
        case 256: return launch<128, false>(a, max_q_len, ws, ws_bytes, s);
        case 257: return launch<128, true>(a, max_q_len, ws, ws_bytes, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace cb
