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
// bits must not change places with the order of a sum.  The products are formed and
// summed in 64 bits, where they are exact but for cancellations beyond 2^37, and the
// result is rounded once to 32; equal ones go to the lower page.
//
// scores_kernel: 16 tokens of a request and one head a workgroup, 16 pages a wave at a
//   time, by 16x16x4 products in 64 bits.  The order of the 2 d channels is free: a lane
//   takes 16-byte pieces of a page's bounds as they lie in memory and the tokens' sums
//   accordingly.  Written are 32-bit keys in the order of the scores, 0 for pages that
//   are not there, all ones for those that are always taken.
// choose_kernel: a workgroup per token and head finds the n_selected-th largest key
//   by its bytes, from the highest, by counts in LDS, and writes the pages above it, and
//   as many equal ones as fit, in their order.
#include "cb_serve_internal.h"
#include "cb_attn_rows.h"
#include <cstdlib>

namespace cb {
namespace {

typedef __attribute__((ext_vector_type(4))) double f64x4_t;


// Tile `idx` of all requests' token tiles of T, and its request, every wave for itself.
template <int T>
__device__ __forceinline__ bool find_tile(const PagedArgs &a, uint32_t idx, Request &rq, int32_t &req, int32_t &tile) {
    const int lane = threadIdx.x & 63;
    uint32_t before = 0;
    for (int r0 = 0; r0 < a.n_reqs; r0 += 64) {
        const Request r = request(a, min(r0 + lane, a.n_reqs - 1));
        const uint32_t n = r0 + lane < a.n_reqs ? (uint32_t)(r.q_len + T - 1) / T : 0;
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

// A number's place in the order of all (a NaN counts as the greatest, both zeros are one), at least 1 and below all ones.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x == x ? x : HUGE_VALF);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// T tokens of a request share the bounds read: 16, or 4 where requests have few.
template <int D, int EL, int T, int NW>
__global__ __launch_bounds__(64 * NW) void scores_kernel(SelectArgs s) {
    constexpr int NT = 64 * NW, STEP = 16 * NW;                // threads, pages that the waves have at a time
    constexpr bool F8 = EL != kBf16;
    constexpr int E = F8 ? 16 : 8, NP = 2 * D / (4 * E);       // channels of a piece, pieces of a lane
    constexpr int QS = 2 * D + 2;                              // (16 tokens' pairs of sums in 64 banks)
    const PagedArgs &a = s.a;
    __shared__ __attribute__((aligned(16))) double sums[T * QS];   // of every token: sum q-, sum q+ over the group
    const int head = (int)blockIdx.y, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, g = lane >> 4;
    int32_t req = 0, tile = 0;
    Request rq;
    if (!find_tile<T>(a, blockIdx.x, rq, req, tile)) return;
    const int32_t tok0 = tile * T, n_tok = min(rq.q_len - tok0, T);
    // (tokens of this round)
    if (rq.row0 + tok0 >= s.tok1 || rq.row0 + tok0 + n_tok <= s.tok0) return;
    const int32_t base = rq.kv_len - rq.q_len + tok0, p_hi = base + n_tok - 1;
    if (p_hi < 0) return;
    const int32_t every = (int32_t)fast_div((uint32_t)p_hi, a.page_size) + 1;
    const int32_t first = (int32_t)blockIdx.z * s.per, end = min(first + s.per, every);
    if (first >= end) return;

    // the bounds of 16 pages, lane's page i0 + n: pieces of 16 bytes, requested while those before are worked on
    const int32_t *table = a.table + req * a.table_stride;
    int32_t page = 0;
    auto look_up = [&](int32_t i0) __attribute__((always_inline)) { page = table[min(i0 + n, end - 1)]; };
    u32x4_t ahead[NP];
    float scale_n = 1.f;
    bool ok_n = false;
    auto load = [&](int32_t i0) __attribute__((always_inline)) {
        ok_n = i0 + n < end && (uint32_t)page < (uint32_t)a.n_pages;
        const int64_t at = (int64_t)(ok_n ? page : 0) * a.n_heads + head;
        const char *x = s.bounds + at * (2 * D * (F8 ? 1 : 2)) + 16 * g;
#pragma unroll
        for (int p = 0; p < NP; ++p) ahead[p] = *(const u32x4_t *)(x + 64 * p);
        if (EL == kBlocks) scale_n = a.kscale[2 * at];
    };
    int32_t i0 = first + 16 * wave;
    if (i0 < end) {
        look_up(i0);
        load(i0);
        if (i0 + STEP < end) look_up(i0 + STEP);
    }

    // sums over the group's heads: a thread has 8 channels of a token, and where there are fewer of these than threads,
    // every HS-th head
    constexpr int HS = T == 4 ? NW : NW / 4;
    const int32_t G = (int32_t)a.G.d;
    for (int u = tid / HS; u < T * (D / 8); u += NT / HS) {
        const int t = u / (D / 8), c = u % (D / 8) * 8;
        double lo[8] = {}, hi[8] = {};
        if (t < n_tok) {
            const uint16_t *q = a.q + (int64_t)(rq.row0 + tok0 + t) * a.q_tok + (int64_t)head * G * a.q_head + c;
#pragma unroll 4
            for (int h = tid % HS; h < G; h += HS) {
                const u32x4_t x = *(const u32x4_t *)(q + h * a.q_head);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = e & 1 ? bf_hi(x[e >> 1]) : bf_lo(x[e >> 1]);
                    // (a NaN goes to both)
                    lo[e] += (double)__builtin_elementwise_minimum(v, 0.f);
                    hi[e] += (double)__builtin_elementwise_maximum(v, 0.f);
                }
            }
        }
#pragma unroll
        for (int o = 1; o < HS; o <<= 1) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                lo[e] += __shfl_xor(lo[e], o);
                hi[e] += __shfl_xor(hi[e], o);
            }
        }
        if (tid % HS == 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sums[t * QS + c + e] = lo[e];
                sums[t * QS + D + c + e] = hi[e];
            }
        }
    }
    __syncthreads();

    // the lane's token's sums of its channels; read from LDS for every 16 pages (registers for them would leave two waves a
    // SIMD)
    int q_at = (n & (T - 1)) * QS + E * g;
    for (; i0 < end; i0 += STEP) {
        asm volatile("" : "+v"(q_at));
        const double *qa = sums + q_at;
        u32x4_t w[NP];
#pragma unroll
        for (int p = 0; p < NP; ++p) w[p] = ahead[p];
        const float scale = EL == kBlocks ? __uint_as_float(__float_as_uint(scale_n) & 0x7f800000u) : 1.f;
        const bool ok = ok_n;
        if (i0 + STEP < end) {
            load(i0 + STEP);
            if (i0 + 2 * STEP < end) look_up(i0 + 2 * STEP);
        }
        f64x4_t acc = {0.0, 0.0, 0.0, 0.0};
        double few[2] = {0.0, 0.0};
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                uint32_t u;
                if constexpr (F8) u = (e & 2) ? e4m3_pair<true>(w[p][e >> 2]) : e4m3_pair<false>(w[p][e >> 2]);
                else u = w[p][e >> 1];
                const double b = (double)((e & 1) ? bf_hi(u) : bf_lo(u));
                if constexpr (T == 16) acc = __builtin_amdgcn_mfma_f64_16x16x4f64(qa[4 * E * p + e], b, acc, 0, 0, 0);
                else few[e & 1] = __builtin_amdgcn_mfma_f64_4x4x4f64(qa[4 * E * p + e], b, few[e & 1], 0, 0, 0);
            }
        if (T == 4) acc[0] = few[0] + few[1];
        const int32_t i = i0 + n;
        if (i >= end) continue;
#pragma unroll
        for (int k = 0; k < T / 4; ++k) {
            const int t = g + 4 * k, tok = rq.row0 + tok0 + t;
            const int32_t pos = base + t;
            if (t >= n_tok || pos < 0 || tok < s.tok0 || tok >= s.tok1) continue;
            const int32_t own = (int32_t)fast_div((uint32_t)pos, a.page_size);
            if (i > own) continue;
            uint32_t key = order_of((float)(acc[k] * (double)scale));
            if (i < s.n_first || i > own - s.n_last) key = 0xffffffffu;
            s.keys[((int64_t)(tok - s.tok0) * a.n_heads + head) * a.table_width + i] = ok ? key : 0u;
        }
    }
}

// The row (token, head) of a choice: the candidates' number, its keys and its list; false for a token of no request.
__device__ __forceinline__ bool choice(const SelectArgs &s, int32_t t, int32_t head, int32_t &n, const uint32_t *&keys, int32_t *&out) {
    const PagedArgs &a = s.a;
    const int32_t tok = s.tok0 + t, req = request_of(a, tok);
    if (req < 0) return false;
    const Request rq = request(a, req);
    if (tok < rq.row0 || tok >= rq.row0 + rq.q_len) return false;
    const int32_t pos = rq.kv_len - rq.q_len + (tok - rq.row0);
    n = pos < 0 ? 0 : (int32_t)fast_div((uint32_t)pos, a.page_size) + 1;
    keys = s.keys + ((int64_t)t * a.n_heads + head) * a.table_width;
    out = s.selected + ((int64_t)tok * a.n_heads + head) * s.n_selected;
    return true;
}

// Rows of up to 64 K candidates, a wave each, keys in registers.
template <int K>
__global__ __launch_bounds__(256) void choose_wave_kernel(SelectArgs s) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t t = (int32_t)blockIdx.x, head = (int32_t)blockIdx.y * 4 + wave;
    if (head >= s.a.n_heads) return;
    int32_t n;
    const uint32_t *keys;
    int32_t *out;
    if (!choice(s, t, head, n, keys, out)) return;
    uint32_t k[K];
#pragma unroll
    for (int j = 0; j < K; ++j) k[j] = 64 * j + lane < n ? keys[64 * j + lane] : 0u;
    // counts lane by lane, then over the wave
    auto at_least = [&](uint32_t x) __attribute__((always_inline)) {
        uint32_t c = 0;
#pragma unroll
        for (int j = 0; j < K; ++j) c += k[j] >= x ? 1u : 0u;
        return __builtin_amdgcn_readlane((int)wave_sums(c), 63);
    };
    // taken are the keys above `least` and the first `equal` of just that
    uint32_t least = 0;
    int equal = 0;
    if (at_least(1) > s.n_selected) {
        // the scores' keys (neither those always taken nor the absent): bits that all of them share are the threshold's too
        uint32_t all = ~0u, any = 0;
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const bool is = k[j] - 1 < 0xfffffffeu;
            all &= is ? k[j] : ~0u;
            any |= is ? k[j] : 0u;
        }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            all &= (uint32_t)__shfl_xor((int)all, o);
            any |= (uint32_t)__shfl_xor((int)any, o);
        }
        all = (uint32_t)__builtin_amdgcn_readfirstlane((int)all);
        any = (uint32_t)__builtin_amdgcn_readfirstlane((int)any);
        const int top = 31 - __builtin_clz((all ^ any) | 1u);        // the highest bit in which two differ
        least = top == 31 ? 0u : any & ~((2u << top) - 1);
        // the largest number that n_selected keys reach, from that bit on; or one that just so many reach
        for (int bit = top; bit >= 0; --bit) {
            const uint32_t x = least | 1u << bit;
            const int c = at_least(x);
            if (c < s.n_selected) continue;
            least = x;
            equal = -1;
            if (c == s.n_selected) break;
            equal = 0;
        }
        if (equal < 0) {
            least -= 1;
            equal = 0;
        } else {
            equal = s.n_selected - at_least(least + 1);
        }
    }
    int n_out = 0, n_equal = 0;
    const uint64_t below = (1ull << lane) - 1;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const bool above = k[j] > least, same = equal > 0 && k[j] == least;
        const uint64_t gt = __ballot(above), eq = __ballot(same);
        const int e = n_equal + __builtin_popcountll(eq & below);
        if (above || (same && e < equal)) out[n_out + __builtin_popcountll(gt & below) + min(e, equal)] = 64 * j + lane;
        n_out += __builtin_popcountll(gt);
        n_equal += __builtin_popcountll(eq);
    }
    for (int i = n_out + min(n_equal, equal) + lane; i < s.n_selected; i += 64) out[i] = -1;
}

// Rows of any number of candidates, a workgroup each.
__global__ __launch_bounds__(256) void choose_kernel(SelectArgs s) {
    __shared__ uint32_t hist[256], wsum[4], found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int32_t n;
    const uint32_t *keys;
    int32_t *out;
    if (!choice(s, (int32_t)blockIdx.x, (int32_t)blockIdx.y, n, keys, out)) return;

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

template <int D, int EL> hipError_t launch(SelectArgs s, uint32_t *ws, int64_t ws_bytes, hipStream_t stream) {
    const PagedArgs &a = s.a;
    const int64_t each = (int64_t)a.n_heads * a.table_width * 4;
    const int64_t round = std::min<int64_t>(std::min<int64_t>(a.n_tokens, 1 << 20), each > 0 ? ws_bytes / each : a.n_tokens);
    const bool few = (int64_t)a.n_tokens <= 4 * (int64_t)a.n_reqs;
    const int T = few ? 4 : 16;
    const int64_t tiles = std::min<int64_t>((int64_t)a.n_tokens / T + a.n_reqs, a.n_tokens);
    s.per = getenv("CBP") ? atoi(getenv("CBP")) : 256;
    const int64_t blocks = ((int64_t)a.table_width + s.per - 1) / s.per;
    if (round < 1 || blocks > 65535) return hipErrorInvalidValue;
    s.keys = ws;
    for (int64_t t = 0; t < a.n_tokens; t += round) {
        s.tok0 = (int32_t)t;
        s.tok1 = (int32_t)std::min<int64_t>(t + round, a.n_tokens);
        if (blocks > 0)
{ const bool w8 = getenv("CBW") && atoi(getenv("CBW")) == 8;
            hipLaunchKernelGGL((w8 ? few ? scores_kernel<D, EL, 4, 8> : scores_kernel<D, EL, 16, 8> : few ? scores_kernel<D, EL, 4, 4> : scores_kernel<D, EL, 16, 4>),
                               dim3((unsigned)tiles, (unsigned)a.n_heads, (unsigned)blocks), dim3(w8 ? 512 : 256), 0, stream, s); }
        const auto waves = a.table_width <= 512 ? choose_wave_kernel<8> : a.table_width <= 1024 ? choose_wave_kernel<16>
                           : a.table_width <= 2048 ? choose_wave_kernel<32> : nullptr;
        const unsigned tokens = (unsigned)(s.tok1 - s.tok0);
        if (waves) hipLaunchKernelGGL(waves, dim3(tokens, (unsigned)(a.n_heads + 3) / 4), dim3(256), 0, stream, s);
        else hipLaunchKernelGGL(choose_kernel, dim3(tokens, (unsigned)a.n_heads), dim3(256), 0, stream, s);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_page_select(const SelectArgs &s, int32_t d, int32_t dtype, void *ws, int64_t ws_bytes, hipStream_t stream) {
    uint32_t *w = (uint32_t *)ws;
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
