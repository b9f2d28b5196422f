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
// Pages with scales of their own (powers of two): the scales of a tile's keys are read
//   when their rows are requested and are operands of the conversion to bf16, K's by the
//   lanes that have the key's row, V's by the places of the product: no instruction more
//   per element, no rounding.  64 single tokens over 512 .. 16,384 keys in pages of 16
//   (0.61 GB) 133 us, 4.6 TB/s (135 with accumulators beside the vector registers, which
//   cost moves); 2,048 tokens x 64 query heads over 32,768 keys 2.07 .. 2.37 ms by board.
//
// Division of work: a row tile's keys go in `parts` to workgroups of their own
//   (cb_paged_rules.h), whose partial sums attn_join_kernel adds in an order that
//   depends on their number alone.  Every workgroup finds its row tile and part from the
//   requests' lengths by itself: sums over the requests by data-parallel moves,
//   about 2 us, instead of a plan that a caller would have to keep in step.
#include "cb_serve_internal.h"
#include "cb_paged_rules.h"
#include "cb_attn_rows.h"

namespace cb {
namespace {

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

template <int D, int EL, int NW>
__device__ __forceinline__ void tile_body(const PagedArgs &a, const PagedClass &cl, uint32_t block, SchedLds<NW> &sched,
                                          TileLds<D> &tl) {
    constexpr bool F8 = EL != kBf16, BLK = EL == kBlocks;
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
    float c2 = EL == kE4m3 ? a.scale_log2 * a.kscale[head] : a.scale_log2;
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
    float ks_n = 1.f, vs_n = 1.f;                              // BLK: the scales of the lane's key's page
    auto place = [&](uint64_t &there) __attribute__((always_inline)) {
        const bool ok = in_kv && (uint32_t)page < (uint32_t)a.n_pages;
        there = __ballot(ok);
        if constexpr (BLK) {
            const float2 sc = *(const float2 *)(a.kscale + 2 * ((int64_t)(ok ? page : 0) * a.n_heads + head));
            ks_n = sc.x;
            vs_n = sc.y;
        }
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
        float sk[NP], sv[NP];                                  // (before the lanes without a last piece part)
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int row = (tid + NT * i) / CPR & 63;
            sk[i] = BLK ? __shfl(ks_n, row) : 1.f;
            sv[i] = BLK ? __shfl(vs_n, row) : 1.f;
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int id = tid + NT * i;
            if (RAGGED && id >= KT * CPR) continue;
            const int row = id / CPR, c = id - row * CPR;
            if constexpr (F8) {
                const float f = sk[i], y = sv[i];
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const uint32_t k0 = kr[i][2 * w], k1 = kr[i][2 * w + 1], x0 = vr[i][2 * w], x1 = vr[i][2 * w + 1];
                    *(uint4 *)(ks + row * KS + 32 * c + 16 * w) =
                        make_uint4(e4m3_pair<false>(k0, f), e4m3_pair<true>(k0, f), e4m3_pair<false>(k1, f), e4m3_pair<true>(k1, f));
                    *(uint4 *)(vs + row * VS + 32 * c + 16 * w) =
                        make_uint4(e4m3_pair<false>(x0, y), e4m3_pair<true>(x0, y), e4m3_pair<false>(x1, y), e4m3_pair<true>(x1, y));
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

    const float vsc = EL == kE4m3 ? a.vscale[head] : 1.f;
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

// Blocks go round while there are more items.
template <int D, int M, int KT, int EL>
__device__ __forceinline__ void join_body(const PagedArgs &a, const PagedClass &cl, uint32_t block, uint32_t blocks,
                                          SchedLds<4> &sched, JoinLds<D> &lds) {
    for (uint32_t b = block;; b += blocks) {
        const uint32_t idx = b / (uint32_t)a.n_heads;
        Item it;
        if (!find_item<M, KT, true, 4>(a, cl, idx, sched, it)) return;
        join_rows<D, M, EL>(a, cl, it, request(a, it.req), (int)(b - idx * a.n_heads), lds);
        __syncthreads();                                       // the item and the sums have been read
    }
}

// ------------------------------------------------------------------ kernels

template <int D, int EL>
__global__ __launch_bounds__(256, EL == kBlocks ? 2 : 1) void attn_rows_kernel(PagedArgs a) {
    __shared__ SchedLds<4> sched;
    __shared__ __attribute__((aligned(16))) RowsLds<D, 4> lds;
    rows_body<D, EL, 4, kAll>(a, a.rows, blockIdx.x, sched, lds);
}

// The requests with few rows and the others in one launch, runs of the two in turn, so that a compute
// unit has products of the one beside loads of the other; a tile, which takes longer, first.  With fewer
// than a run of either kind all tiles come first.  64 single tokens over 1,024 .. 8,192 keys beside a chunk
// of 512 (8 heads of 128, 8 query heads each): 252 us, 272 with all tiles first, 272 with runs of 8; 24
// beside three chunks of 515 with windows of 1,024, which have no whole run: 53, 72 with runs of 8.
template <int D, int EL, int NW>
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
    if (tile) tile_body<D, EL, NW>(a, a.tile, b, sched, lds.tile);
    else rows_body<D, EL, NW, kAll>(a, a.rows, b, sched, lds.rows);
}

template <int D, int EL, int NW>
__global__ __launch_bounds__(256) void attn_join_kernel(PagedArgs a) {
    __shared__ SchedLds<4> sched;
    __shared__ JoinLds<D> lds;
    if (blockIdx.x < a.tile.join_blocks) join_body<D, 32 * NW, kTileKT, EL>(a, a.tile, blockIdx.x, a.tile.join_blocks, sched, lds);
    else join_body<D, 16, kKT, EL>(a, a.rows, blockIdx.x - a.tile.join_blocks, a.rows.join_blocks, sched, lds);
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

template <int D, int EL, int NW>
hipError_t launch_tiles(PagedArgs a, char *w, int64_t ws_bytes, hipStream_t s) {
    constexpr int M = 32 * NW;
    const int64_t least = least_rows((int32_t)a.G.d, a.n_reqs);
    if (least > 0 && !prepare_class<D, 16, kKT>(a, a.rows, kTarget, 0, least, w, ws_bytes)) return hipErrorInvalidValue;
    if (!prepare_class<D, M, kTileKT>(a, a.tile, kTileTarget * 4 / NW, least, INT64_MAX, w, ws_bytes)) return hipErrorInvalidValue;
    hipLaunchKernelGGL((attn_tile_kernel<D, EL, NW>), dim3(a.tile.blocks + a.rows.blocks), dim3(64 * NW), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
    const uint32_t join = a.tile.join_blocks + a.rows.join_blocks;
    if (join > 0) hipLaunchKernelGGL((attn_join_kernel<D, EL, NW>), dim3(join), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <int D, int EL>
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
            return launch_tiles<D, EL, 8>(a, w, ws_bytes, s);
    }
    if (rows > kFewRows) return launch_tiles<D, EL, 4>(a, w, ws_bytes, s);
    // few rows everywhere: rows_body alone, whatever the lengths turn out to be
    if (!prepare_class<D, 16, kKT>(a, a.rows, kTarget, 0, INT64_MAX, w, ws_bytes)) return hipErrorInvalidValue;
    hipLaunchKernelGGL((attn_rows_kernel<D, EL>), dim3(a.rows.blocks), dim3(256), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
    if (a.rows.join_blocks > 0) hipLaunchKernelGGL((attn_join_kernel<D, EL, 4>), dim3(a.rows.join_blocks), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

int64_t attn_paged_workspace_bytes(int32_t d, int32_t G, int32_t n_reqs, int32_t max_q_len) {
    const int64_t rows = (int64_t)2 * kTarget * 16 * (d + 2) * 4, tile = (int64_t)2 * kTileTarget * 128 * (d + 2) * 4;
    if ((int64_t)max_q_len * G <= kFewRows) return rows;
    return (least_rows(G, n_reqs) > 0 ? rows : 0) + tile;
}

hipError_t launch_attn_paged(const PagedArgs &a, int32_t d, int32_t dtype, int32_t max_q_len, void *ws, int64_t ws_bytes,
                             hipStream_t s) {
    switch (d * 4 + dtype) {
        case 256 + CB_PAGES_BF16: return launch<64, kBf16>(a, max_q_len, ws, ws_bytes, s);
        case 256 + CB_PAGES_E4M3: return launch<64, kE4m3>(a, max_q_len, ws, ws_bytes, s);
        case 256 + CB_PAGES_E4M3_BLOCKS: return launch<64, kBlocks>(a, max_q_len, ws, ws_bytes, s);
        case 384 + CB_PAGES_BF16: return launch<96, kBf16>(a, max_q_len, ws, ws_bytes, s);
        case 384 + CB_PAGES_E4M3: return launch<96, kE4m3>(a, max_q_len, ws, ws_bytes, s);
        case 384 + CB_PAGES_E4M3_BLOCKS: return launch<96, kBlocks>(a, max_q_len, ws, ws_bytes, s);
        case 512 + CB_PAGES_BF16: return launch<128, kBf16>(a, max_q_len, ws, ws_bytes, s);
        case 512 + CB_PAGES_E4M3: return launch<128, kE4m3>(a, max_q_len, ws, ws_bytes, s);
        case 512 + CB_PAGES_E4M3_BLOCKS: return launch<128, kBlocks>(a, max_q_len, ws, ws_bytes, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace cb
