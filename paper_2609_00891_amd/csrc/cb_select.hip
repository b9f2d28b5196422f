// cb_select.hip -- which pages every query attends to, by a bound on their scores, on
// gfx950.
//
// With lo_i and hi_i the least and greatest of channel i over a page's keys, no key of
// it scores more with a query q than sum_i max(q_i lo_i, q_i hi_i) = sum_i (q+_i hi_i +
// q-_i lo_i), q+ = max(q, 0), q- = min(q, 0).  A page's score for a token and KV head is
// the sum of these bounds over the group's query heads, and so one product of
// (sum q-, sum q+) with (lo, hi).
//
// Choices are whole numbers: two pages whose scores differ in the last places of 32
// bits must not change places with the order of a sum.  A score is therefore the sum
// in 64 bits, where products are exact and sums are but for cancellations beyond 2^37,
// rounded once to 32; equal ones go to the lower page.  But only pages near the border
// need so much: first come estimates, whose error is bounded, then the scores of the
// pages that the bound leaves undecided.
//
// estimates_kernel: 16 tokens of a request and one head a workgroup, 16 pages a wave at
//   a time, by 16x16x32 products in bf16.  A token's sum over its heads (fp32; terms of
//   one sign, off by G 2^-24) is split into two bf16 numbers (off by 2^-18); the products of 32
//   channels start from zero and the steps are added in fp32, so that no sum of more
//   than 64 terms is formed in a matrix instruction.  Together they are off by less than
//   (2^-16 + G 2^-23) S, S = sum |q| |bound|, which a third product forms.  The bounds are read four lanes to 64
//   bytes of a page and handed to the operand's lanes.
// choose_wave_kernel: a wave per token and head, its keys (estimates as numbers of their
//   order) in LDS.  The n_selected-th largest is found by counts of eight bits, from the first
//   in which they differ (bit by bit the two calls below took 2 and 5 us more); pages further than
//   twice the error above it are taken, as far below it are not,
//   and of the others, where they are more than are needed, the wave forms the scores.
// scores_kernel and choose_kernel: tables of more than 8,192 entries.  All scores in 64
//   bits by 16x16x4 products, and a workgroup per token and head that finds the
//   threshold by bytes with counts in LDS.  1,024 new tokens over 65,535 keys in 8-bit pages of
//   8, 8,192 entries: 575 us, over 65,560 keys (8,195 entries) 1,076.  The host knows the table's
//   width alone, so what counts is that and not the entries in use, for the LDS of a wave too:
//   the two calls below 61 and 44 us in tables as wide as their contexts, 61 and 82 in tables of
//   8,192 entries, 102 and 93 in tables of 8,200.
//
// Bound by latency and HBM: 48 single tokens over 4,096 .. 65,536 keys in pages of 32 (8
// heads of 128, 8 query heads each, 0.15 GB) 61 us with the bounds of the step's pages (40
// of them the estimates, 16 the choices), 1,024 new tokens over 32,768 keys in 8-bit pages
// of 64 44 (22 and 18); the choices' last rows, whose open pages are scored, end them.  With
// scores of all pages in 64 bits 62 (bounds in the last cache) and 70 (47 and 55 of them
// the scores), chosen by workgroups that read the keys again for every byte 140 and 97.
#include "cb_serve_internal.h"
#include "cb_attn_rows.h"

namespace cb {
namespace {

typedef __attribute__((ext_vector_type(4))) double f64x4_t;

constexpr int kTokens = 16;             // of a request that share the bounds read
constexpr int kPages = 256;             // pages of a workgroup
constexpr int kWaveTable = 8192;        // table entries up to which a wave has a row's keys (32 KB)
constexpr uint32_t kUnknown = 0xff800000u;   // key of an estimate that says nothing (and of the scores +infinity and NaN)

// A number's place in the order of all (a NaN counts as the greatest, both zeros are one), at least 1 and below all ones.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x == x ? x : HUGE_VALF);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// What a workgroup of one head has: 16 tokens of a request and some of the pages up to the last one's own.
struct Work { Request rq; int32_t req, tok0, n_tok, base, first, end; };   // base: the first token's position
__device__ __forceinline__ bool find_work(const SelectArgs &s, Work &w) {
    const PagedArgs &a = s.a;
    int32_t tile = 0;
    const auto tiles_of = [](int32_t q) { return (uint32_t)(q + kTokens - 1) / kTokens; };
    if (!find_tile(a, blockIdx.x / (uint32_t)a.n_heads, tiles_of, w.rq, w.req, tile)) return false;
    w.tok0 = tile * kTokens;
    w.n_tok = min(w.rq.q_len - w.tok0, kTokens);
    // (tokens of this round)
    if (w.rq.row0 + w.tok0 >= s.tok1 || w.rq.row0 + w.tok0 + w.n_tok <= s.tok0) return false;
    w.base = w.rq.kv_len - w.rq.q_len + w.tok0;
    const int32_t p_hi = w.base + w.n_tok - 1;
    if (p_hi < 0) return false;
    w.first = (int32_t)blockIdx.y * kPages;
    w.end = min(w.first + kPages, (int32_t)fast_div((uint32_t)p_hi, a.page_size) + 1);
    return w.first < w.end;
}

// The key of page i for token t of the workgroup, or none where it is no candidate.
__device__ __forceinline__ void write_key(const SelectArgs &s, const Work &w, int head, int t, int32_t i, bool ok, uint32_t key) {
    const PagedArgs &a = s.a;
    const int32_t tok = w.rq.row0 + w.tok0 + t, pos = w.base + t;
    if (t >= w.n_tok || pos < 0 || tok < s.tok0 || tok >= s.tok1) return;
    const int32_t own = (int32_t)fast_div((uint32_t)pos, a.page_size);
    if (i > own) return;
    if (i < s.n_first || i > own - s.n_last) key = 0xffffffffu;
    s.keys[((int64_t)(tok - s.tok0) * a.n_heads + head) * a.table_width + i] = ok ? key : 0u;
}

template <int D, int EL>
__global__ __launch_bounds__(256, 4) void estimates_kernel(SelectArgs s) {
    constexpr bool F8 = EL != kBf16;
    constexpr int NP = 2 * D * (F8 ? 1 : 2) / 64;              // pieces of 64 bytes of a page's bounds
    constexpr int QS = 2 * D + 8;                              // (16 tokens' pieces of 16 bytes in 64 banks)
    const PagedArgs &a = s.a;
    // every token's sum q-, sum q+ over the group as two bf16 numbers
    __shared__ __attribute__((aligned(16))) uint16_t parts[2][kTokens * QS];
    const int head = (int)(blockIdx.x % (uint32_t)a.n_heads), tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, g = lane >> 4;
    Work wk;
    if (!find_work(s, wk)) return;

    // the bounds of 16 pages: lane l has 16 bytes of every piece of page i0 + l / 4, requested while those before are
    // worked on
    const int32_t *table = a.table + wk.req * a.table_stride;
    int32_t page = 0;
    auto look_up = [&](int32_t i0) __attribute__((always_inline)) { page = table[min(i0 + (lane >> 2), wk.end - 1)]; };
    u32x4_t ahead[NP];
    float scale_n = 1.f;
    uint64_t ok_n = 0;
    auto load = [&](int32_t i0) __attribute__((always_inline)) {
        const bool ok = i0 + (lane >> 2) < wk.end && (uint32_t)page < (uint32_t)a.n_pages;
        ok_n = __ballot(ok);
        const int64_t at = (int64_t)(ok ? page : 0) * a.n_heads + head;
        const char *x = s.bounds + at * (2 * D * (F8 ? 1 : 2)) + 16 * (lane & 3);
#pragma unroll
        for (int p = 0; p < NP; ++p) ahead[p] = *(const u32x4_t *)(x + 64 * p);
        if (EL == kBlocks) scale_n = a.kscale[2 * at];
    };
    int32_t i0 = wk.first + 16 * wave;
    if (i0 < wk.end) {
        look_up(i0);
        load(i0);
        if (i0 + 64 < wk.end) look_up(i0 + 64);
    }

    // a thread has 8 channels of a token
    const int32_t G = (int32_t)a.G.d;
    for (int u = tid; u < kTokens * (D / 8); u += 256) {
        const int t = u / (D / 8), c = u % (D / 8) * 8;
        float lo[8] = {}, hi[8] = {};
        if (t < wk.n_tok) {
            const uint16_t *q = a.q + (int64_t)(wk.rq.row0 + wk.tok0 + t) * a.q_tok + (int64_t)head * G * a.q_head + c;
#pragma unroll 8
            for (int h = 0; h < G; ++h) {
                const u32x4_t x = *(const u32x4_t *)(q + h * a.q_head);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = e & 1 ? bf_hi(x[e >> 1]) : bf_lo(x[e >> 1]);
                    // (a NaN goes to both)
                    lo[e] += __builtin_elementwise_minimum(v, 0.f);
                    hi[e] += __builtin_elementwise_maximum(v, 0.f);
                }
            }
        }
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            const float *y = z ? hi : lo;
            uint32_t h[4], m[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                h[e] = pack_bf16(y[2 * e], y[2 * e + 1]);
                m[e] = pack_bf16(y[2 * e] - bf_lo(h[e]), y[2 * e + 1] - bf_hi(h[e]));
            }
            *(uint4 *)&parts[0][t * QS + z * D + c] = make_uint4(h[0], h[1], h[2], h[3]);
            *(uint4 *)&parts[1][t * QS + z * D + c] = make_uint4(m[0], m[1], m[2], m[3]);
        }
    }
    __syncthreads();

    uint32_t most[4] = {0, 0, 0, 0};                           // the bits of the largest S of the lane's tokens
    // the lane's token's parts of its channels; read from LDS for every 16 pages
    int q_at = n * QS + (F8 ? 16 : 8) * g;
    for (; i0 < wk.end; i0 += 64) {
        asm volatile("" : "+v"(q_at));
        u32x4_t w[NP];
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int e = 0; e < 4; ++e) w[p][e] = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (4 * n + g), (int)ahead[p][e]);
        const float scale = EL == kBlocks ? __uint_as_float(__float_as_uint(__shfl(scale_n, 4 * n)) & 0x7f800000u) : 1.f;
        const bool ok = (ok_n >> (4 * n)) & 1;
        if (i0 + 64 < wk.end) {
            load(i0 + 64);
            if (i0 + 128 < wk.end) look_up(i0 + 128);
        }
        f32x4_t sum = {0.f, 0.f, 0.f, 0.f}, size = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int st = 0; st < (F8 ? 2 : 1); ++st) {
                uint32_t b[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (F8) b[e] = e & 1 ? e4m3_pair<true>(w[p][2 * st + (e >> 1)]) : e4m3_pair<false>(w[p][2 * st + (e >> 1)]);
                    else b[e] = w[p][e];
                }
                const int at = q_at + (F8 ? 64 * p + 8 * st : 32 * p);
                const u32x4_t h = *(const u32x4_t *)&parts[0][at], m = *(const u32x4_t *)&parts[1][at];
                const bf16x8_t bf = frag(b[0], b[1], b[2], b[3]);
                f32x4_t step = {0.f, 0.f, 0.f, 0.f};
                step = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(h[0], h[1], h[2], h[3]), bf, step, 0, 0, 0);
                step = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(m[0], m[1], m[2], m[3]), bf, step, 0, 0, 0);
                sum += step;
                const uint32_t k = 0x7fff7fffu;
                size = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(h[0] & k, h[1] & k, h[2] & k, h[3] & k),
                                                               frag(b[0] & k, b[1] & k, b[2] & k, b[3] & k), size, 0, 0, 0);
            }
        const int32_t i = i0 + n;
        if (i >= wk.end) continue;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            // lane's tokens 4 g + k; an estimate says nothing where its terms leave fp32's range
            const float size_k = size[k] * scale;
            const bool good = size_k >= 0x1p-100f && size_k <= 0x1p126f && scale >= 0x1p-100f && scale <= 0x1p100f;
            if (good && ok) most[k] = max(most[k], __float_as_uint(size_k));
            write_key(s, wk, head, 4 * g + k, i, ok, good ? order_of(sum[k] * scale) : kUnknown);
        }
    }
    // the largest S of every token, one number for each wave
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) most[k] = max(most[k], (uint32_t)__shfl_xor((int)most[k], o));
        const int32_t t = 4 * g + k, tok = wk.rq.row0 + wk.tok0 + t;
        if (n == 0 && t < wk.n_tok && tok >= s.tok0 && tok < s.tok1)
            s.sizes[((int64_t)(tok - s.tok0) * a.n_heads + head) * s.slots + 4 * blockIdx.y + wave] = __uint_as_float(most[k]);
    }
}

template <int D, int EL>
__global__ __launch_bounds__(256) void scores_kernel(SelectArgs s) {
    constexpr bool F8 = EL != kBf16;
    constexpr int E = F8 ? 16 : 8, NP = 2 * D / (4 * E);       // channels of a piece, pieces of a lane
    constexpr int QS = 2 * D + 2;                              // (16 tokens' pairs of sums in 64 banks)
    const PagedArgs &a = s.a;
    __shared__ __attribute__((aligned(16))) double sums[kTokens * QS];   // of every token: sum q-, sum q+ over the group
    const int head = (int)(blockIdx.x % (uint32_t)a.n_heads), tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, g = lane >> 4;
    Work wk;
    if (!find_work(s, wk)) return;
    const int32_t G = (int32_t)a.G.d;
    for (int u = tid; u < kTokens * (D / 8); u += 256) {
        const int t = u / (D / 8), c = u % (D / 8) * 8;
        double lo[8] = {}, hi[8] = {};
        if (t < wk.n_tok) {
            const uint16_t *q = a.q + (int64_t)(wk.rq.row0 + wk.tok0 + t) * a.q_tok + (int64_t)head * G * a.q_head + c;
#pragma unroll 4
            for (int h = 0; h < G; ++h) {
                const u32x4_t x = *(const u32x4_t *)(q + h * a.q_head);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = e & 1 ? bf_hi(x[e >> 1]) : bf_lo(x[e >> 1]);
                    lo[e] += (double)__builtin_elementwise_minimum(v, 0.f);
                    hi[e] += (double)__builtin_elementwise_maximum(v, 0.f);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            sums[t * QS + c + e] = lo[e];
            sums[t * QS + D + c + e] = hi[e];
        }
    }
    __syncthreads();
    const int32_t *table = a.table + wk.req * a.table_stride;
    int q_at = n * QS + E * g;
    for (int32_t i0 = wk.first + 16 * wave; i0 < wk.end; i0 += 64) {
        asm volatile("" : "+v"(q_at));
        const double *qa = sums + q_at;
        const int32_t i = i0 + n;                              // the lane's page
        const int32_t page = i < wk.end ? table[i] : -1;
        const bool ok = (uint32_t)page < (uint32_t)a.n_pages;
        const int64_t at = (int64_t)(ok ? page : 0) * a.n_heads + head;
        const char *x = s.bounds + at * (2 * D * (F8 ? 1 : 2)) + 16 * g;
        u32x4_t w[NP];
#pragma unroll
        for (int p = 0; p < NP; ++p) w[p] = *(const u32x4_t *)(x + 64 * p);
        const float scale = EL == kBlocks ? __uint_as_float(__float_as_uint(a.kscale[2 * at]) & 0x7f800000u) : 1.f;
        f64x4_t acc = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                uint32_t u;
                if constexpr (F8) u = (e & 2) ? e4m3_pair<true>(w[p][e >> 2]) : e4m3_pair<false>(w[p][e >> 2]);
                else u = w[p][e >> 1];
                acc = __builtin_amdgcn_mfma_f64_16x16x4f64(qa[4 * E * p + e], (double)((e & 1) ? bf_hi(u) : bf_lo(u)), acc, 0, 0, 0);
            }
        if (i >= wk.end) continue;
#pragma unroll
        for (int k = 0; k < 4; ++k) write_key(s, wk, head, g + 4 * k, i, ok, order_of((float)(acc[k] * (double)scale)));
    }
}

// The row (token, head) of a choice: the candidates' number, its keys and its list; false for a token of no request.
__device__ __forceinline__ bool choice(const SelectArgs &s, int32_t t, int32_t head, int32_t &req, int32_t &n, const uint32_t *&keys,
                                       int32_t *&out) {
    const PagedArgs &a = s.a;
    const int32_t tok = s.tok0 + t;
    Request rq;
    if (!request_of(a, tok, req, rq)) return false;
    const int32_t pos = rq.kv_len - rq.q_len + (tok - rq.row0);
    n = pos < 0 ? 0 : (int32_t)fast_div((uint32_t)pos, a.page_size) + 1;
    keys = s.keys + ((int64_t)t * a.n_heads + head) * a.table_width;
    out = s.selected + ((int64_t)tok * a.n_heads + head) * s.n_selected;
    return true;
}

// The greatest number and the bits of all lanes' numbers, by data-parallel moves.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    x = max(x, moved<0x111, 0xf>(x));   // row_shr:1, 2, 4, 8
    x = max(x, moved<0x112, 0xf>(x));
    x = max(x, moved<0x114, 0xf>(x));
    x = max(x, moved<0x118, 0xf>(x));
    x = max(x, moved<0x142, 0xa>(x));   // row_bcast:15, 31
    x = max(x, moved<0x143, 0xc>(x));
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
__device__ __forceinline__ uint32_t wave_or(uint32_t x) {
    x |= moved<0x111, 0xf>(x);
    x |= moved<0x112, 0xf>(x);
    x |= moved<0x114, 0xf>(x);
    x |= moved<0x118, 0xf>(x);
    x |= moved<0x142, 0xa>(x);
    x |= moved<0x143, 0xc>(x);
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// Keys of a row in LDS, of one wave: lane l has keys 4 l .. 4 l + 3 of every 256, absent ones 0.  (In registers they make
// code of thousands of instructions that every workgroup runs once: 28 us where this form, bit by bit, took 22.)
struct Keys {
    uint4 *k;
    int groups;                                                // of 256

    // keys that reach x, counted lane by lane, then over the wave
    __device__ __forceinline__ int at_least(uint32_t x) const {
        const int lane = threadIdx.x;
        uint32_t c = 0;
#pragma unroll 4
        for (int j = 0; j < groups; ++j) {
            const uint4 v = k[64 * j + lane];
            c += (v.x >= x ? 1u : 0u) + (v.y >= x ? 1u : 0u) + (v.z >= x ? 1u : 0u) + (v.w >= x ? 1u : 0u);
        }
        return __builtin_amdgcn_readlane((int)wave_sums(c), 63);
    }
    // The largest number that n keys reach, or one that just n reach (exact: true); more than n keys are not 0, fewer
    // or just n all ones.  By counts of eight bits at a time (in `bins`, 256 words of LDS) until few enough keys are
    // left that each lane has one.
    __device__ __forceinline__ uint32_t threshold(int n, uint32_t *bins, bool &exact) const {
        // bits that all keys but 0 and all ones share are the threshold's too
        const int lane = threadIdx.x;
        uint32_t all = ~0u, any = 0, ones = 0;
#pragma unroll 4
        for (int j = 0; j < groups; ++j) {
            const uint4 v = k[64 * j + lane];
            const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                all &= among(u[c]) ? u[c] : ~0u;
                any |= among(u[c]) ? u[c] : 0u;
                ones += u[c] == ~0u ? 1u : 0u;
            }
        }
        int need = n - __builtin_amdgcn_readlane((int)wave_sums(ones), 63);
        exact = true;
        if (need == 0) return ~0u;
        all = ~wave_or(~all);
        any = wave_or(any);
        const int top = 31 - __builtin_clz((all ^ any) | 1u);      // the highest bit in which two differ
        uint32_t x = top == 31 ? 0u : any & ~((2u << top) - 1);    // the threshold's bits from bit `low` on
        int low = top + 1, count;
        do {
            const int w = min(low, 8);
            low -= w;
            __syncthreads();
            *(uint4 *)&bins[4 * lane] = make_uint4(0, 0, 0, 0);
            __syncthreads();
            for (int j = 0; j < groups; ++j) {
                const uint4 v = k[64 * j + lane];
                const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (among(u[c]) && ((u[c] ^ x) >> low) >> w == 0) atomicAdd(&bins[(u[c] >> low) & ((1u << w) - 1)], 1u);
            }
            __syncthreads();
            // a lane has four bins, the first lane the largest numbers
            const uint4 v = *(const uint4 *)&bins[4 * (63 - lane)];
            const int own = (int)(v.x + v.y + v.z + v.w), sum = (int)wave_sums((uint32_t)own);
            const int from = __builtin_ctzll(__ballot(sum >= need));
            int rest = need - (sum - own), bin = 4 * (63 - lane) + 3, c = (int)v.w;
            if (rest > c) { rest -= c; --bin; c = (int)v.z;
                if (rest > c) { rest -= c; --bin; c = (int)v.y;
                    if (rest > c) { rest -= c; --bin; c = (int)v.x; } } }
            need = __builtin_amdgcn_readlane(rest, from);
            count = __builtin_amdgcn_readlane(c, from);
            x |= (uint32_t)__builtin_amdgcn_readlane(bin, from) << low;
            if (count == need) return x;
        } while (low > 0 && count > 64);
        exact = false;
        if (low == 0) return x;
        // a key for each lane
        __syncthreads();
        int at = 0;
        for (int j = 0; j < groups; ++j) {
            const uint4 v = k[64 * j + lane];
            const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const bool is = among(u[c]) && (u[c] ^ x) >> low == 0;
                const uint64_t has = __ballot(is);
                if (is) bins[at + __builtin_popcountll(has & ((1ull << lane) - 1))] = u[c];
                at += __builtin_popcountll(has);
            }
        }
        __syncthreads();
        const uint32_t mine = lane < count ? bins[lane] : 0u;
        int before = 0;                                            // larger ones, and equal ones of earlier lanes
        for (int p = 0; p < count; ++p) {
            const uint32_t other = (uint32_t)__builtin_amdgcn_readlane((int)mine, p);
            before += other > mine || (other == mine && p < lane) ? 1 : 0;
        }
        x = (uint32_t)__builtin_amdgcn_readlane((int)mine, __builtin_ctzll(__ballot(lane < count && before == need - 1)));
        exact = __builtin_popcountll(__ballot(mine >= x)) == need;
        return x;
    }
    // neither 0 nor all ones
    static __device__ __forceinline__ bool among(uint32_t u) { return u - 1 < ~0u - 1; }
    // the smallest key that reaches x, and whether a key is y
    __device__ __forceinline__ uint32_t first_from(uint32_t x, uint32_t y, bool &found) const {
        uint32_t m = ~0u;
        bool is = false;
#pragma unroll 4
        for (int j = 0; j < groups; ++j) {
            const uint4 v = k[64 * j + threadIdx.x];
            const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                m = u[c] >= x ? min(m, u[c]) : m;
                is |= u[c] == y;
            }
        }
        found = __any(is);
        return ~wave_max(~m);
    }
};

// The scores of pages of one row by its wave, four at a time by 16 lanes each: a lane has d / 8 of the 2 d elements of
// (sum q-, sum q+) and of a page's bounds.  (Few waves come here, and run this code once: it is kept short.  With a page
// to the whole wave, two bytes a lane, it was twice as long, and the rows that need it took 7,000 cycles more: 65 us the first call above.)
struct Scores {
    double q[16];
    const uint32_t *x;                                         // the lane's channels of the group's first head
    uint32_t v[8];                                             // and of a head
    int d, words;                                              // dwords of a lane's bf16 numbers
    const int32_t *table;

    // Requests the first heads' queries; heads go to the lanes' groups in turn.
    __device__ __forceinline__ Scores(const SelectArgs &s, int32_t req, int32_t tok, int32_t head) {
        const PagedArgs &a = s.a;
        d = s.head_dim;
        words = d / 16;
        table = a.table + req * a.table_stride;
        x = (const uint32_t *)(a.q + (int64_t)tok * a.q_tok + (int64_t)head * (int)a.G.d * a.q_head + (threadIdx.x & 7) * (d / 8));
        fetch(a, 0);
    }
    __device__ __forceinline__ void fetch(const PagedArgs &a, int h0) {
        const int h = h0 + (int)(threadIdx.x >> 4), G = (int)a.G.d;
#pragma unroll
        for (int w = 0; w < 8; ++w) v[w] = w < words ? x[min(h, G - 1) * (a.q_head / 2) + w] : 0u;
    }
    __device__ __forceinline__ void sums(const PagedArgs &a) {
        const int G = (int)a.G.d;
        const uint32_t sign = (threadIdx.x & 8) ? 0u : 0x80000000u;    // min(y, 0) = -max(-y, 0); a NaN goes to both
#pragma unroll
        for (int e = 0; e < 16; ++e) q[e] = 0.0;
#pragma unroll 1
        for (int h0 = 0; h0 < G; h0 += 4) {
            uint32_t now[8];
#pragma unroll
            for (int w = 0; w < 8; ++w) now[w] = h0 + (int)(threadIdx.x >> 4) < G ? v[w] : 0u;
            if (h0 + 4 < G) fetch(a, h0 + 4);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t u = e & 1 ? now[e >> 1] & 0xffff0000u : now[e >> 1] << 16;
                const float y = __builtin_elementwise_maximum(__uint_as_float(u ^ sign), 0.f);
                q[e] += (double)__uint_as_float(__float_as_uint(y) ^ sign);
            }
        }
        // over the four groups
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            q[e] = both<16>(q[e]);
            q[e] = both<32>(q[e]);
        }
    }
    // The sum of a lane's number and that of the lane 16, or 32, places from it.
    template <int N> static __device__ __forceinline__ double both(double y) {
        const uint64_t u = __builtin_bit_cast(uint64_t, y);
        const uint32_t lo = (uint32_t)u, hi = (uint32_t)(u >> 32);
        const auto l = N == 16 ? __builtin_amdgcn_permlane16_swap(lo, lo, false, false) : __builtin_amdgcn_permlane32_swap(lo, lo, false, false);
        const auto h = N == 16 ? __builtin_amdgcn_permlane16_swap(hi, hi, false, false) : __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
        return __builtin_bit_cast(double, (uint64_t)h[0] << 32 | l[0]) + __builtin_bit_cast(double, (uint64_t)h[1] << 32 | l[1]);
    }
    // In lane 16 g + 15 the key of page i of group g (a place in the table).
    __device__ __forceinline__ uint32_t key(const SelectArgs &s, int32_t head, int32_t i) const {
        const PagedArgs &a = s.a;
        const int64_t at = (int64_t)min((uint32_t)table[i], (uint32_t)a.n_pages - 1) * a.n_heads + head;
        const int64_t e0 = at * 2 * d + (threadIdx.x & 15) * (d / 8);
        const float scale = s.dtype == CB_PAGES_E4M3_BLOCKS ? a.kscale[2 * at] : 1.f;
        uint32_t u[8];
        if (s.dtype == CB_PAGES_BF16) {
            const uint32_t *b = (const uint32_t *)(s.bounds + 2 * e0);
#pragma unroll
            for (int w = 0; w < 8; ++w) u[w] = w < words ? b[w] : 0u;
        } else {
            const uint32_t *b = (const uint32_t *)(s.bounds + e0);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t y = 2 * w < words ? b[w] : 0u;
                u[2 * w] = e4m3_pair<false>(y);
                u[2 * w + 1] = e4m3_pair<true>(y);
            }
        }
        double sum = 0.0;
#pragma unroll
        for (int w = 0; w < 8; ++w) sum += q[2 * w] * (double)bf_lo(u[w]) + q[2 * w + 1] * (double)bf_hi(u[w]);
        sum += moved<0x111, 0xf>(sum);   // row_shr:1, 2, 4, 8
        sum += moved<0x112, 0xf>(sum);
        sum += moved<0x114, 0xf>(sum);
        sum += moved<0x118, 0xf>(sum);
        return order_of((float)(sum * (double)__uint_as_float(__float_as_uint(scale) & 0x7f800000u)));
    }
};

constexpr int kScored = 64;             // pages whose scores are formed at a time

// The places of the keys from lo to hi, of kScored of them from the one of number `from` on, in their order; returns how
// many there are.
__device__ __forceinline__ int between(const Keys &row, uint32_t lo, uint32_t hi, int from, int32_t *place) {
    const int lane = threadIdx.x;
    int rank = 0;
    for (int j = 0; j < row.groups; ++j) {
        const uint4 v = row.k[64 * j + lane];
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
        int mine = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) mine += u[c] >= lo && u[c] <= hi ? 1 : 0;
        if (!__any(mine)) continue;
        const int sum = (int)wave_sums((uint32_t)mine);
        int at = rank + sum - mine - from;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if (u[c] < lo || u[c] > hi) continue;
            if (at >= 0 && at < kScored) place[at] = 256 * j + 4 * lane + c;
            ++at;
        }
        rank += __builtin_amdgcn_readlane(sum, 63);
    }
    return rank;
}

// Rows whose keys fit LDS, a wave each.
__global__ __launch_bounds__(64) void choose_wave_kernel(SelectArgs s) {
    extern __shared__ __attribute__((aligned(16))) uint4 lds[];
    __shared__ int32_t place[kScored];
    __shared__ __attribute__((aligned(16))) uint32_t bins[256];
    const int lane = threadIdx.x;
    const int32_t t = (int32_t)blockIdx.x, head = (int32_t)blockIdx.y;
    int32_t req, n;
    const uint32_t *keys;
    int32_t *out;
    if (!choice(s, t, head, req, n, keys, out)) return;
    const float *sizes = s.sizes + ((int64_t)t * s.a.n_heads + head) * s.slots;
    uint32_t most = 0;
    for (int i = lane; i < 4 * ((n + kPages - 1) / kPages); i += 64) most = max(most, __float_as_uint(sizes[i]));
    const Keys row = {lds, (n + 255) / 256};
    uint32_t *key_at = (uint32_t *)lds;
    for (int j0 = 0; j0 < row.groups; j0 += 8) {               // (2,048 keys on their way together)
        uint32_t u[8][4];
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (j0 + j < row.groups) u[j][c] = keys[min(256 * (j0 + j) + 64 * c + lane, n - 1)];
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int i = 256 * (j0 + j) + 64 * c + lane;
                if (j0 + j < row.groups) key_at[i] = i < n ? u[j][c] : 0u;
            }
    }
    __syncthreads();
    // taken are the keys above `least` and the first `equal` of just that
    uint32_t least = 0;
    int equal = 0;
    if (row.at_least(1) > s.n_selected) {
        bool exact, unknown;
        const uint32_t border = row.first_from(row.threshold(s.n_selected, bins, exact), kUnknown, unknown);
        if (border == ~0u) {
            least = ~0u - 1;                                   // those always taken are all
        } else {
            // pages whose estimates are within the errors of the n_selected-th: between lo and hi
            most = wave_max(most);
            const float at = value_of(border);
            // (each of two estimates off by (2^-16 + G 2^-23) S, and two scores that round to one number)
            const float far = 2.f * (0x1p-16f + 0x1p-23f * (float)s.a.G.d) * __uint_as_float(most) + 0x1p-22f * fabsf(at);
            const uint32_t lo = unknown ? 1u : order_of(at - far), hi = unknown ? ~0u - 1 : order_of(at + far);
            if (row.at_least(lo) == s.n_selected) {
                least = lo - 1;
            } else {
                // Those above are taken, those below are not, and of those between as many as are needed.
                Scores scores(s, req, s.tok0 + t, head);
                // the key of the lane's page of `count` that `place` has
                auto score = [&](int count) __attribute__((always_inline)) {
                    uint32_t mine = 0;
#pragma unroll 1
                    for (int p0 = 0; p0 < count; p0 += 4) {
                        const uint32_t key = scores.key(s, head, place[min(p0 + (lane >> 4), count - 1)]);
                        const uint32_t x = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (16 * (lane & 3) + 15), (int)key);
                        mine = lane >> 2 == p0 >> 2 ? x : mine;
                    }
                    return mine;
                };
                const int open = between(row, lo, hi, 0, place);
                scores.sums(s.a);
                if (open <= kScored) {
                    const int need = s.n_selected - row.at_least(hi + 1);
                    __syncthreads();
                    const uint32_t mine = score(open);
                    // how many come before the lane's: those with a larger key, or an equal one and a lower place
                    int before = 0;
                    for (int p = 0; p < open; ++p) {
                        const uint32_t other = (uint32_t)__builtin_amdgcn_readlane((int)mine, p);
                        before += other > mine || (other == mine && p < lane) ? 1 : 0;
                    }
                    if (lane < open) key_at[place[lane]] = before < need ? ~0u : 0u;
                    least = hi;
                } else {
                    // (rows of infinities, or of many pages that are nearly alike) the open keys become scores, which are
                    // neither 0 nor all ones
                    for (int i = lane; i < 256 * row.groups; i += 64) {
                        const uint32_t k = key_at[i];
                        key_at[i] = k > hi ? ~0u : k >= lo ? k : 0u;
                    }
                    for (int from = 0; from < open; from += kScored) {
                        __syncthreads();
                        between(row, 1, ~0u - 1, from, place);
                        __syncthreads();
                        const int count = min(open - from, kScored);
                        const uint32_t mine = score(count);
                        if (lane < count) key_at[place[lane]] = mine;
                    }
                    __syncthreads();
                    least = row.threshold(s.n_selected, bins, exact);
                    if (exact) least -= 1;
                    else equal = s.n_selected - row.at_least(least + 1);
                }
                __syncthreads();
            }
        }
    }
    int n_out = 0, n_equal = 0;
    for (int j = 0; j < row.groups; ++j) {
        const uint4 v = row.k[64 * j + lane];
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
        uint32_t mine = 0;                                     // keys above, and 2^16 for each of just that
#pragma unroll
        for (int c = 0; c < 4; ++c) mine += u[c] > least ? 1u : equal > 0 && u[c] == least ? 0x10000u : 0u;
        const uint32_t sum = wave_sums(mine), all = (uint32_t)__builtin_amdgcn_readlane((int)sum, 63);
        int above = n_out + (int)((sum - mine) & 0xffff), same = n_equal + (int)((sum - mine) >> 16);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const bool is = equal > 0 && u[c] == least;
            if (u[c] > least || (is && same < equal)) out[above + min(same, equal)] = 256 * j + 4 * lane + c;
            above += u[c] > least ? 1 : 0;
            same += is ? 1 : 0;
        }
        n_out += (int)(all & 0xffff);
        n_equal += (int)(all >> 16);
    }
    for (int i = n_out + min(n_equal, equal) + lane; i < s.n_selected; i += 64) out[i] = -1;
}

// Rows of any number of candidates, a workgroup each.
__global__ __launch_bounds__(256) void choose_kernel(SelectArgs s) {
    __shared__ uint32_t hist[256], wsum[4], found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int32_t req, n;
    const uint32_t *keys;
    int32_t *out;
    if (!choice(s, (int32_t)blockIdx.x, (int32_t)blockIdx.y, req, n, keys, out)) return;

    // the sum over the workgroup
    auto total_of = [&](uint32_t x) __attribute__((always_inline)) {
        x = wave_sums(x);
        __syncthreads();
        if (lane == 63) wsum[wave] = x;
        __syncthreads();
        return wsum[0] + wsum[1] + wsum[2] + wsum[3];
    };
    uint32_t some = 0;
    for (int32_t i = tid; i < n; i += 256) some += keys[i] != 0;
    some = total_of(some);
    // the threshold and how many pages of just that key are taken
    uint32_t least = 0, equal = 0;
    if (some > (uint32_t)s.n_selected) {
        uint32_t rest = (uint32_t)s.n_selected;
        for (int shift = 24; shift >= 0; shift -= 8) {
            hist[tid] = 0;
            __syncthreads();
            const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
            for (int32_t i = tid; i < n; i += 256) {
                const uint32_t k = keys[i];
                if ((k & mask) == least) atomicAdd(&hist[k >> shift & 255], 1u);
            }
            __syncthreads();
            // thread t has byte 255 - t: counts from the largest byte on
            const uint32_t c = hist[255 - tid];
            uint32_t sum = wave_sums(c);
            if (lane == 63) wsum[wave] = sum;
            __syncthreads();
            for (int w = 0; w < wave; ++w) sum += wsum[w];
            if (sum >= rest && sum - c < rest) {
                found[0] = (uint32_t)(255 - tid);
                found[1] = rest - (sum - c);
            }
            __syncthreads();
            least |= found[0] << shift;
            rest = found[1];
        }
        equal = rest;
    }
    // pages above it, and the first equal ones, in their order
    uint32_t n_out = 0, n_equal = 0;
    for (int32_t i0 = 0; i0 < n; i0 += 256) {
        const uint32_t k = i0 + tid < n ? keys[i0 + tid] : 0u;
        const bool same = equal > 0 && k == least;
        const uint64_t eq = __ballot(same), gt = __ballot(k > least);
        const uint64_t below = (1ull << lane) - 1;
        __syncthreads();
        if (lane == 0) wsum[wave] = (uint32_t)__builtin_popcountll(eq) << 16 | (uint32_t)__builtin_popcountll(gt);
        __syncthreads();
        uint32_t e0 = n_equal, g0 = n_out, all_e = 0, all_g = 0;
        for (int w = 0; w < 4; ++w) {
            if (w < wave) {
                e0 += wsum[w] >> 16;
                g0 += wsum[w] & 0xffff;
            }
            all_e += wsum[w] >> 16;
            all_g += wsum[w] & 0xffff;
        }
        e0 += (uint32_t)__builtin_popcountll(eq & below);
        g0 += (uint32_t)__builtin_popcountll(gt & below);
        if (k > least || (same && e0 < equal)) out[g0 + min(e0, equal)] = i0 + tid;
        n_out += all_g;
        n_equal += all_e;
    }
    for (uint32_t i = n_out + min(n_equal, equal) + tid; i < (uint32_t)s.n_selected; i += 256) out[i] = -1;
}

template <int D, int EL> hipError_t launch(SelectArgs s, char *ws, int64_t ws_bytes, hipStream_t stream) {
    const PagedArgs &a = s.a;
    const int64_t each = select_row_bytes(a.table_width) * a.n_heads;
    const int64_t round = std::min<int64_t>(std::min<int64_t>(a.n_tokens, 1 << 20), each > 0 ? ws_bytes / each : a.n_tokens);
    const int64_t tiles = std::min<int64_t>((int64_t)a.n_tokens / kTokens + a.n_reqs, a.n_tokens);
    const int64_t blocks = ((int64_t)a.table_width + kPages - 1) / kPages;
    s.keys = (uint32_t *)ws;
    s.sizes = (float *)ws + round * a.n_heads * a.table_width;
    s.slots = (int32_t)blocks * 4;
    const bool waves = a.table_width <= kWaveTable;
    const unsigned lds = (unsigned)((a.table_width + 255) / 256 * 1024);
    for (int64_t t = 0; t < a.n_tokens; t += round) {
        s.tok0 = (int32_t)t;
        s.tok1 = (int32_t)std::min<int64_t>(t + round, a.n_tokens);
        const unsigned tokens = (unsigned)(s.tok1 - s.tok0);
        if (blocks > 0)
            hipLaunchKernelGGL((waves ? estimates_kernel<D, EL> : scores_kernel<D, EL>),
                               dim3((unsigned)(tiles * a.n_heads), (unsigned)blocks), dim3(256), 0, stream, s);
        if (waves) hipLaunchKernelGGL(choose_wave_kernel, dim3(tokens, (unsigned)a.n_heads), dim3(64), lds, stream, s);
        else hipLaunchKernelGGL(choose_kernel, dim3(tokens, (unsigned)a.n_heads), dim3(256), 0, stream, s);
    }
    return hipGetLastError();
}

}  // namespace

int64_t select_row_bytes(int32_t table_width) {
    return 4 * ((int64_t)table_width + 4 * (((int64_t)table_width + kPages - 1) / kPages));
}

hipError_t launch_page_select(const SelectArgs &s, int32_t d, int32_t dtype, void *ws, int64_t ws_bytes, hipStream_t stream) {
    char *w = (char *)ws;
    switch (d * 4 + dtype) {
        case 256 + CB_PAGES_BF16: return launch<64, kBf16>(s, w, ws_bytes, stream);
        case 256 + CB_PAGES_E4M3: return launch<64, kE4m3>(s, w, ws_bytes, stream);
        case 256 + CB_PAGES_E4M3_BLOCKS: return launch<64, kBlocks>(s, w, ws_bytes, stream);
        case 384 + CB_PAGES_BF16: return launch<96, kBf16>(s, w, ws_bytes, stream);
        case 384 + CB_PAGES_E4M3: return launch<96, kE4m3>(s, w, ws_bytes, stream);
        case 384 + CB_PAGES_E4M3_BLOCKS: return launch<96, kBlocks>(s, w, ws_bytes, stream);
        case 512 + CB_PAGES_BF16: return launch<128, kBf16>(s, w, ws_bytes, stream);
        case 512 + CB_PAGES_E4M3: return launch<128, kE4m3>(s, w, ws_bytes, stream);
        case 512 + CB_PAGES_E4M3_BLOCKS: return launch<128, kBlocks>(s, w, ws_bytes, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace cb
