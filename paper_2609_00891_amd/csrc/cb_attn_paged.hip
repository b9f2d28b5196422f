// cb_attn_paged.hip -- attention of new tokens over pages on gfx950.
//
// For a row (new token, query head) with query q and the visible keys j:
//     s_j = scale q . k_j,  m = max s_j,  l = sum exp(s_j - m),  o = sum exp(s_j - m) v_j / l,
// formed in one pass over the keys: a new maximum m' rescales l and o by
// exp(m - m').  In log2 units throughout (scale carries log2 e).
//
// Rows of one request and KV head are (token, head of its group) pairs, so the
// group's query heads share every K and V row read.  Row tiles of 16 MT rows.
//
// attn_rows_kernel: four waves, each with its own key tiles of 32 keys, from
//   memory straight into matrix-core operands:
//   S^T = K Q^T (16x16x32): lane l holds row n = l & 15 and, of key subtile t,
//     keys 16 t + 4 g + r, g = l >> 4, r = 0 .. 3: the statistics of a row are
//     per-lane numbers.
//   O^T = V^T P^T with the 32 keys in the order that S^T leaves them (4 g + r,
//     16 + 4 g + r): the P operand is S^T's registers rounded in place.  The V
//     operand (eight keys of one channel) comes from eight 16-byte pieces of
//     eight rows, transposed in registers (v_perm); channel E c + i goes to
//     output row c of product i, so a lane ends with E consecutive channels.
//   No LDS and no barrier until the waves' results are joined.
//
// Division of work: a row tile's keys go in `parts` to workgroups of their own
//   (cb_paged_rules.h), whose partial sums attn_join_kernel adds in the order
//   of the parts.  Every workgroup finds its row tile and part from the
//   requests' lengths by itself.
#include "cb_internal.h"
#include "cb_paged_rules.h"

namespace cb {
namespace {

typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;

#ifndef CB_SCHED
#define CB_SCHED 0
#endif
constexpr int kKT = 32;                 // keys of a tile
constexpr int kPartMin = 8;             // least key tiles of a part: two for each of the four waves
constexpr int kTarget = 2048;           // workgroups that long rows are divided into

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
// The bits of the bf16 values, and of the e4m3 ones, that are infinities or NaNs.
__device__ __forceinline__ uint32_t not_finite_halves(uint32_t u) {
    return ((u & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((u & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}
__device__ __forceinline__ uint32_t nan_bytes(uint32_t u) {
    uint32_t r = 0;
#pragma unroll
    for (int b = 0; b < 32; b += 8) r |= ((u >> b) & 0x7fu) == 0x7fu ? 0xffu << b : 0u;
    return r;
}
// Two e4m3 values (exact in bf16).
template <bool HI> __device__ __forceinline__ uint32_t e4m3_pair(uint32_t u) {
    const bf16x2_t v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, 1.0f, HI);
    return __builtin_bit_cast(uint32_t, v);
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
struct SchedLds { int64_t wsum[4]; Item item; int32_t found; };

// The row tile and part of index `idx` (JOIN: of the idx-th row tile in more
// than one part), or false behind the last.
template <int M, int KT, bool JOIN>
__device__ __forceinline__ bool find_item(const PagedArgs &a, int64_t idx, SchedLds &sh, Item &out) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    auto work_of = [&](int r) __attribute__((always_inline)) {
        RequestWork w = {0, 0, 0};
        if (r < a.n_reqs) {
            const Request q = request(a, r);
            w = request_work(q.q_len, q.kv_len, (int32_t)a.G.d, M, KT, a.c.row_min, a.c.row_max, a.window, a.n_sinks);
        }
        return w;
    };
    if (tid == 0) sh.found = 0;
    int64_t W = 0;
    for (int r = tid; r < a.n_reqs; r += 256) {
        const RequestWork w = work_of(r);
        W += w.tiles * w.bound;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) W += __shfl_xor(W, o);
    if (lane == 0) sh.wsum[wave] = W;
    __syncthreads();
    W = sh.wsum[0] + sh.wsum[1] + sh.wsum[2] + sh.wsum[3];
    const int64_t c = part_tiles(W, a.n_heads, a.c.target, kPartMin);
    int64_t n_before = 0;
    int32_t s_before = 0;
    for (int r0 = 0; r0 < a.n_reqs; r0 += 256) {
        const RequestWork w = work_of(r0 + tid);
        const int32_t parts = parts_of(w.bound, c);
        const int64_t n = JOIN ? (parts > 1 ? w.tiles : 0) : (int64_t)w.tiles * parts;
        const int32_t s = parts > 1 ? w.tiles * parts : 0;
        int64_t ni = n;
        int32_t si = s;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t u = __shfl_up(ni, o);
            const int32_t t = __shfl_up(si, o);
            if (lane >= o) { ni += u; si += t; }
        }
        __syncthreads();                                      // the last round's sums have been read
        if (lane == 63) sh.wsum[wave] = ni << 24 | si;        // slots are fewer than 2^24 (see parts_of)
        __syncthreads();
        int64_t total = 0;
        int32_t s_total = 0;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int64_t x = sh.wsum[v];
            if (v < wave) { ni += x >> 24; si += (int32_t)(x & 0xffffff); }
            total += x >> 24;
            s_total += (int32_t)(x & 0xffffff);
        }
        const int64_t first = n_before + ni - n;
        if (idx >= first && idx < first + n) {
            const int32_t k = (int32_t)(idx - first);
            const int32_t tile = JOIN ? k : k / parts;
            sh.item = {r0 + tid, tile, JOIN ? 0 : k - tile * parts, parts, s_before + si - s + tile * parts};
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

template <int D, int MT, bool F8>
__global__ __launch_bounds__(256) void attn_rows_kernel(PagedArgs a) {
    using Ge = Geo<D, F8>;
    constexpr int M = 16 * MT, E = Ge::E;
    constexpr int OS = D + 4;                                  // floats between rows of the joined results
    __shared__ SchedLds sched;
    __shared__ __attribute__((aligned(16))) float ol[4][16][OS];
    __shared__ float ml[4][16][2];
    const int head = (int)(blockIdx.x % (uint32_t)a.n_heads);
    Item it;
    if (!find_item<M, kKT, false>(a, blockIdx.x / (uint32_t)a.n_heads, sched, it)) return;

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

    // queries: row n of subtile mt (rows behind the last repeat it)
    bf16x8_t qf[MT][Ge::NS];
    int32_t pos[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int32_t row = row0 + min(16 * mt + n, n_rows - 1);
        const int32_t tok = (int32_t)fast_div((uint32_t)row, a.G), u = row - tok * G;
        pos[mt] = rq.kv_len - rq.q_len + tok;
        const uint16_t *q = a.q + (int64_t)(rq.row0 + tok) * a.q_tok + (int64_t)(head * G + u) * a.q_head;
#pragma unroll
        for (int s = 0; s < Ge::NS; ++s) qf[mt][s] = *(const bf16x8_t *)(q + Ge::chan(s, g));
    }
    const float c2 = F8 ? a.scale_log2 * a.kscale[head] : a.scale_log2;

    // where the rows of a tile's keys are: lane's key 32 tile + (lane & 31), its place in 16-byte units
    uint32_t off = 0, there = 0;                               // there: bit per key, its page is in the pool
    auto locate = [&](int32_t tile) __attribute__((always_inline)) {
        const int32_t key = tile * kKT + (lane & 31);
        bool ok = key < rq.kv_len;
        off = 0;
        if (ok) {
            const uint32_t idx = fast_div((uint32_t)key, a.page_size);
            const int32_t page = table[idx];
            ok = page >= 0 && page < a.n_pages;
            if (ok) off = (uint32_t)page * a.s_page + ((uint32_t)key - idx * a.page_size.d) * a.s_tok;
        }
        there = (uint32_t)__ballot(ok);
    };
    uint32_t kr[2][Ge::KW], vr[8][Ge::VW];
    auto load_k = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const char *p = kp + (uint64_t)(uint32_t)__shfl((int)off, 16 * t + n) * 16;
            if constexpr (!F8 || Ge::PAIR) {
#pragma unroll
                for (int s = 0; s < Ge::KW / 4; ++s) {
                    const uint4 x = *(const uint4 *)(p + 64 * s + 16 * g);
                    kr[t][4 * s] = x.x; kr[t][4 * s + 1] = x.y; kr[t][4 * s + 2] = x.z; kr[t][4 * s + 3] = x.w;
                }
            } else {
#pragma unroll
                for (int s = 0; s < Ge::NS; ++s) {
                    const uint2 x = *(const uint2 *)(p + 32 * s + 8 * g);
                    kr[t][2 * s] = x.x; kr[t][2 * s + 1] = x.y;
                }
            }
        }
    };
    // V rows in the order of S^T's registers: place j of lane group g is key 4 g + j, 16 + 4 g + j - 4
    auto load_v = [&]() __attribute__((always_inline)) {
        const int c = min(n, Ge::NC - 1);                      // 96: lanes 12 .. 15 repeat lane 11, unused
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const char *p = vp + (uint64_t)(uint32_t)__shfl((int)off, (j >> 2) * 16 + 4 * g + (j & 3)) * 16 + c * (F8 ? E : 2 * E);
            if constexpr (Ge::VW == 4) {
                const uint4 x = *(const uint4 *)p;
                vr[j][0] = x.x; vr[j][1] = x.y; vr[j][2] = x.z; vr[j][3] = x.w;
            } else if constexpr (Ge::VW == 2) {
                const uint2 x = *(const uint2 *)p;
                vr[j][0] = x.x; vr[j][1] = x.y;
            } else {
                vr[j][0] = *(const uint32_t *)p;
            }
        }
    };

    f32x4_t o[MT][E];
    float m[MT], l[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        m[mt] = -HUGE_VALF;
        l[mt] = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) o[mt][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    for (int32_t v = part_begin(kt.n, it.part, it.parts) + wave; v < v1; v += 4) {
        const int32_t k0 = kt.tile(v) * kKT;
        locate(kt.tile(v));
        load_k();
        load_v();
        // every key of the tile is seen by every row
        const bool whole = there == 0xffffffffu && k0 + kKT - 1 <= p_lo &&
                           (a.window == 0 || k0 > p_hi - a.window || k0 + kKT <= a.n_sinks);
        uint32_t p2[MT][4];                                    // exp2(s - m) as the operand of P V
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
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
                    s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[mt][st], s[t], 0, 0, 0);
                }
            }
            float x[8];
            float mx = m[mt];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = s[e >> 2][e & 3] * c2;
            if (!whole) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int kk = (e >> 2) * 16 + 4 * g + (e & 3), key = k0 + kk;
                    const bool see = ((there >> kk) & 1) && key <= pos[mt] &&
                                     (a.window == 0 || key > pos[mt] - a.window || key < a.n_sinks);
                    x[e] = see ? x[e] : -HUGE_VALF;
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) mx = fmaxf(mx, x[e]);
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float ref = mx == -HUGE_VALF ? 0.f : mx;     // nothing seen so far: every weight is zero
            const float al = __builtin_amdgcn_exp2f(m[mt] - ref);
            m[mt] = mx;
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = __builtin_amdgcn_exp2f(x[e] - ref);
                sum += x[e];
            }
            l[mt] = l[mt] * al + sum;
#pragma unroll
            for (int q = 0; q < 4; ++q) p2[mt][q] = pack_bf16(x[2 * q], x[2 * q + 1]);
#pragma unroll
            for (int i = 0; i < E; ++i) o[mt][i] *= al;
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
        bool odd = false;
        if (!whole) {
            // rows that are not there are zeros; and a NaN or infinity of V must not meet the zero
            // weight of a row that does not see its key
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool is = (there >> ((j >> 2) * 16 + 4 * g + (j & 3))) & 1;
#pragma unroll
                for (int w = 0; w < E / 2; ++w) {
                    vb[j][w] = is ? vb[j][w] : 0u;
                    odd |= not_finite(vb[j][w]);
                }
            }
            odd = __ballot(odd) != 0;
        }
        if (!odd) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                uint32_t f[4];
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    f[q] = __builtin_amdgcn_perm(vb[2 * q + 1][i >> 1], vb[2 * q][i >> 1], (i & 1) ? 0x07060302u : 0x05040100u);
                const bf16x8_t vf = frag(f[0], f[1], f[2], f[3]);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
                    o[mt][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, frag(p2[mt][0], p2[mt][1], p2[mt][2], p2[mt][3]),
                                                                      o[mt][i], 0, 0, 0);
            }
        } else {
            // one key after the other, for the rows that see it only
            for (int kk = 0; kk < kKT; ++kk) {
                if (!((there >> kk) & 1)) continue;
                const int src = 16 * ((kk & 15) >> 2) + n, key = k0 + kk, e = (kk >> 4) * 4 + (kk & 3);
                const uint32_t at = (uint32_t)__shfl((int)off, kk);
                float pk[MT];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const uint32_t w = e < 2 ? p2[mt][0] : e < 4 ? p2[mt][1] : e < 6 ? p2[mt][2] : p2[mt][3];
                    const float pw = (e & 1) ? bf_hi(w) : bf_lo(w);
                    pk[mt] = __shfl(pw, src);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int c = 4 * g + r;
                    if (c >= Ge::NC) continue;
                    float vv[E];
                    const char *p = vp + (uint64_t)at * 16 + c * (F8 ? E : 2 * E);
#pragma unroll
                    for (int w = 0; w < E / 2; ++w) {
                        uint32_t u;
                        if constexpr (F8) u = e4m3_pair<false>(*(const uint16_t *)(p + 2 * w));
                        else u = *(const uint32_t *)(p + 4 * w);
                        vv[2 * w] = bf_lo(u);
                        vv[2 * w + 1] = bf_hi(u);
                    }
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        const bool see = key <= pos[mt] && (a.window == 0 || key > pos[mt] - a.window || key < a.n_sinks);
#pragma unroll
                        for (int i = 0; i < E; ++i)
                            if (see) o[mt][i][r] = __builtin_fmaf(pk[mt], vv[i], o[mt][i][r]);
                    }
                }
            }
        }
    }

    // ---- the four waves' results, joined in their order
    const float vs = F8 ? a.vscale[head] : 1.f;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        float lt = l[mt];
        lt += __shfl_xor(lt, 16);
        lt += __shfl_xor(lt, 32);
        if (mt > 0) __syncthreads();                           // the last subtile's results have been read
        if (g == 0) {
            ml[wave][n][0] = m[mt];
            ml[wave][n][1] = lt;
        }
        __syncthreads();
        const float mx = fmaxf(fmaxf(ml[0][n][0], ml[1][n][0]), fmaxf(ml[2][n][0], ml[3][n][0]));
        const float f = __builtin_amdgcn_exp2f(m[mt] - (mx == -HUGE_VALF ? 0.f : mx));
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int c = 4 * g + r;
            if (c < Ge::NC) {
#pragma unroll
                for (int i = 0; i < E; i += 4)
                    *(float4 *)&ol[wave][n][E * c + i] = make_float4(o[mt][i][r] * f, o[mt][i + 1][r] * f,
                                                                    o[mt][i + 2][r] * f, o[mt][i + 3][r] * f);
            }
        }
        __syncthreads();
        const int row = tid / (D / 8), ch = tid % (D / 8) * 8, rr = 16 * mt + row;
        if (row < 16 && rr < n_rows) {
            const float mr = fmaxf(fmaxf(ml[0][row][0], ml[1][row][0]), fmaxf(ml[2][row][0], ml[3][row][0]));
            const float ref = mr == -HUGE_VALF ? 0.f : mr;
            float lr = 0.f, y[8] = {};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                lr += ml[w][row][1] * __builtin_amdgcn_exp2f(ml[w][row][0] - ref);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] += ol[w][row][ch + e];
            }
            if (it.parts > 1) {
                float *w = a.c.ws + ((int64_t)(it.slot + it.part) * a.n_heads + head) * (M * (D + 2));
                *(float4 *)(w + rr * D + ch) = make_float4(y[0], y[1], y[2], y[3]);
                *(float4 *)(w + rr * D + ch + 4) = make_float4(y[4], y[5], y[6], y[7]);
                if (ch == 0) {
                    w[M * D + rr] = mr;
                    w[M * D + M + rr] = lr;
                }
            } else {
                const float inv = lr == 0.f ? 0.f : vs / lr;
                const int32_t tok = (int32_t)fast_div((uint32_t)(row0 + rr), a.G), u = row0 + rr - tok * G;
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

template <int D, int RT, bool F8>
__global__ __launch_bounds__(256, RT == 1 ? 2 : 1) void attn_tile_kernel(PagedArgs a) {
    constexpr int M = 128 * RT, KT = 64, NS = D / 16, ND = D / 32;
    constexpr int KS = 2 * D + 16, VS = 2 * D + 32;            // bytes between rows of K and V in LDS
    constexpr int CPR = F8 ? D / 16 : D / 8;                   // 16-byte pieces of a row in memory
    constexpr int NP = (KT * CPR + 255) / 256;                 // pieces of a thread, for each of K and V
    constexpr bool RAGGED = KT * CPR % 256 != 0;
    constexpr int STAGE = KT * (KS + VS);
    constexpr float kLag = 8.f;
    __shared__ SchedLds sched;
    __shared__ int32_t odd;
    __shared__ __attribute__((aligned(16))) char lds[2 * STAGE];
    const int head = (int)(blockIdx.x % (uint32_t)a.n_heads);
    Item it;
    if (!find_item<M, KT, false>(a, blockIdx.x / (uint32_t)a.n_heads, sched, it)) return;

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

    // queries of this wave's RT subtiles of 32 rows (rows behind the last repeat it)
    bf16x8_t qf[RT][NS];
    int32_t pos[RT];                                           // of the lane's rows
    const int w0 = 32 * RT * wave;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int32_t row = row0 + min(w0 + 32 * rt + n, n_rows - 1);
        const int32_t tok = (int32_t)fast_div((uint32_t)row, a.G), u = row - tok * G;
        pos[rt] = base + tok;
        const uint16_t *q = a.q + (int64_t)(rq.row0 + tok) * a.q_tok + (int64_t)(head * G + u) * a.q_head;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const uint4 x = *(const uint4 *)(q + 16 * s + 8 * h);
            qf[rt][s] = frag(x.x ^ flip, x.y ^ flip, x.z ^ flip, x.w ^ flip);
        }
    }
    const int32_t s_lo = __builtin_amdgcn_readfirstlane(pos[0]);
    const int32_t s_hi = __builtin_amdgcn_readlane(pos[RT - 1], 31);

    // the places of a tile's 64 rows: lane l looks up key l
    auto locate = [&](int32_t tile, uint64_t &there) __attribute__((always_inline)) {
        const int32_t key = tile * KT + lane;
        bool ok = key < rq.kv_len;
        uint32_t off = 0;
        if (ok) {
            const uint32_t idx = fast_div((uint32_t)key, a.page_size);
            const int32_t page = table[idx];
            ok = page >= 0 && page < a.n_pages;
            if (ok) off = (uint32_t)page * a.s_page + ((uint32_t)key - idx * a.page_size.d) * a.s_tok;
        }
        there = __ballot(ok);
        return off;
    };
    uint4 kr[NP], vr[NP];
    auto load = [&](uint32_t off) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int id = tid + 256 * i;
            const int row = id / CPR, c = id - row * CPR;
            const uint64_t at = (uint64_t)(uint32_t)__shfl((int)off, row & 63) * 16 + 16 * c;
            if (RAGGED && id >= KT * CPR) continue;
            kr[i] = *(const uint4 *)(kp + at);
            vr[i] = *(const uint4 *)(vp + at);
        }
    };
    // In a tile with a key that some row does not see (edge) a NaN or infinity of V would meet zero
    // weights: it becomes a zero here and reaches the rows that see it after the last tile.  V's rows
    // that are not there become zeros as well.
    auto store = [&](int st, uint64_t there, bool edge) __attribute__((always_inline)) {
        char *ks = lds + st * STAGE, *vs = ks + KT * KS;
        if (edge) {
            asm volatile("");
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int id = tid + 256 * i, row = id / CPR;
                const bool is = (there >> (row & 63)) & 1;
                uint32_t v4[4] = {vr[i].x, vr[i].y, vr[i].z, vr[i].w};
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t bad;                              // the bits of the values that are no number
                    if constexpr (F8) bad = nan_bytes(v4[w]);
                    else bad = not_finite_halves(v4[w]);
                    if (is && bad) odd = 1;
                    v4[w] = is ? v4[w] & ~bad : 0u;
                }
                vr[i] = make_uint4(v4[0], v4[1], v4[2], v4[3]);
            }
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int id = tid + 256 * i;
            if (RAGGED && id >= KT * CPR) continue;
            const int row = id / CPR, c = id - row * CPR;
            if constexpr (F8) {
                const uint32_t k4[4] = {kr[i].x, kr[i].y, kr[i].z, kr[i].w}, v4[4] = {vr[i].x, vr[i].y, vr[i].z, vr[i].w};
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const uint32_t k0 = k4[2 * w], k1 = k4[2 * w + 1], x0 = v4[2 * w], x1 = v4[2 * w + 1];
                    *(uint4 *)(ks + row * KS + 32 * c + 16 * w) =
                        make_uint4(e4m3_pair<false>(k0), e4m3_pair<true>(k0), e4m3_pair<false>(k1), e4m3_pair<true>(k1));
                    *(uint4 *)(vs + row * VS + 32 * c + 16 * w) =
                        make_uint4(e4m3_pair<false>(x0), e4m3_pair<true>(x0), e4m3_pair<false>(x1), e4m3_pair<true>(x1));
                }
            } else {
                *(uint4 *)(ks + row * KS + 16 * c) = kr[i];
                *(uint4 *)(vs + row * VS + 16 * c) = vr[i];
            }
        }
    };
    // every key of the tile is there and seen by every row from position lo to hi
    auto seen = [&](int32_t k0, uint64_t there, int32_t lo, int32_t hi) __attribute__((always_inline)) {
        return there == ~0ull && k0 + KT - 1 <= lo && (a.window == 0 || k0 > hi - a.window || k0 + KT <= a.n_sinks);
    };

    f32x16_t o[RT][ND];
    float m[RT], l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = -HUGE_VALF;
        l[rt] = 0.f;
#pragma unroll
        for (int q = 0; q < ND; ++q) o[rt][q] = f32x16_t{};
    }
    // V^T operand: keys 16 kk + 4 h + {0 .. 3} and + 8, channel 32 q + (lane & 31)
    const int vt = (4 * h + ((lane >> 2) & 3)) * VS + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);

    uint64_t there = 0, there_n = 0;
    if (v0 < v1) {
        load(locate(kt.tile(v0), there));
        __syncthreads();                                       // odd is set
        store(0, there, !seen(kt.tile(v0) * KT, there, p_lo, p_hi));
    }
    __syncthreads();
    for (int32_t v = v0; v < v1; ++v) {
        const int st = (v - v0) & 1;
        const int32_t k0 = kt.tile(v) * KT;
        if (v + 1 < v1) load(locate(kt.tile(v + 1), there_n));
        const char *ks = lds + st * STAGE, *vs = ks + KT * KS;
        f32x16_t s[RT][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) s[rt][t] = f32x16_t{};
#pragma unroll
            for (int q = 0; q < NS; ++q) {
                const bf16x8_t kf = *(const bf16x8_t *)(ks + (32 * t + n) * KS + 32 * q + 16 * h);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                    s[rt][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[rt][q], s[rt][t], 0, 0, 0);
            }
        }
#if CB_SCHED & 1
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int i = 0; i < 2 * NS - 4; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, RT, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4 * RT, 0);
#endif
        if (!seen(k0, there, s_lo, s_hi)) {
            asm volatile("");                                  // a branch, not selects on every tile
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                // key k0 + 4 h + c is register e's, c = 32 (e >> 4) + acc_key(e & 15, 0)
                const int hi = pos[rt] - k0 - 4 * h, lo = a.window == 0 ? INT32_MIN : hi - a.window;
                const int sink = a.n_sinks - k0 - 4 * h;
                const uint64_t bits = there >> (4 * h);
                const uint32_t bit2[2] = {(uint32_t)bits, (uint32_t)(bits >> 32)};
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    const int c = 32 * (e >> 4) + acc_key(e & 15, 0);
                    const bool see = (bit2[e >> 4] & (1u << (c & 31))) && c <= hi && (c > lo || c < sink);
                    s[rt][e >> 4][e & 15] = see ? s[rt][e >> 4][e & 15] : -HUGE_VALF;
                }
            }
        }
        uint32_t pk[RT][16];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float mx = max3(s[rt][0][0], s[rt][0][1], s[rt][0][2]);
#pragma unroll
            for (int e = 3; e < 31; e += 2) mx = max3(mx, s[rt][e >> 4][e & 15], s[rt][(e + 1) >> 4][(e + 1) & 15]);
            mx = max3(mx, s[rt][1][15], s[rt][1][15]);
            mx = max3(mx, __shfl_xor(mx, 32), mx) * c2;
            // the maximum in use may lag the true one by 2^kLag in weight: sums are rescaled seldom
            if (__any(mx > m[rt] + kLag)) {
                const float mn = fmaxf(m[rt], mx);
                const float al = __builtin_amdgcn_exp2f(m[rt] - (mn == -HUGE_VALF ? 0.f : mn));
                m[rt] = mn;
                l[rt] *= al;
#pragma unroll
                for (int q = 0; q < ND; ++q) o[rt][q] *= al;
            }
            const float ref = m[rt] == -HUGE_VALF ? 0.f : m[rt];
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float x0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][e >> 3][2 * e & 15], c2, -ref));
                const float x1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][e >> 3][(2 * e & 15) + 1], c2, -ref));
                sum += x0;
                sum += x1;
                pk[rt][e] = pack_bf16(x0, x1);
            }
            l[rt] += sum;
        }
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
#pragma unroll
            for (int q = 0; q < ND; ++q) {
                const char *pp = vs + vt + 16 * kk * VS + 64 * q;
                const s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)pp);
                const s16x4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(pp + 8 * VS));
                typedef __attribute__((ext_vector_type(8))) short s16x8_t;
                const s16x8_t v8 = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                    o[rt][q] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        __builtin_bit_cast(bf16x8_t, v8),
                        frag(pk[rt][4 * kk], pk[rt][4 * kk + 1], pk[rt][4 * kk + 2], pk[rt][4 * kk + 3]), o[rt][q], 0, 0, 0);
            }
        }
#if CB_SCHED & 2
        // a quarter of the weights, then its products beside the next quarter
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 1);
        __builtin_amdgcn_sched_group_barrier(0x402, 28, 1);
#pragma unroll
        for (int i = 0; i < 3; ++i) {
#pragma unroll
            for (int q = 0; q < ND; ++q) {
                __builtin_amdgcn_sched_group_barrier(0x008, RT, 1);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
                __builtin_amdgcn_sched_group_barrier(0x402, 28 / ND, 1);
            }
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 2 * RT, 1);
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 1);
        __builtin_amdgcn_sched_group_barrier(0x008, 2 * RT, 1);
#endif
        if (v + 1 < v1) store(st ^ 1, there_n, !seen(kt.tile(v + 1) * KT, there_n, p_lo, p_hi));
        there = there_n;
        __syncthreads();
    }
    if (odd) {
        // NaNs and infinities of V that were left out of tiles which some row does not see whole: they
        // come to the rows that see their keys (whatever finite weight they have)
#pragma unroll 1
        for (int32_t v = v0; v < v1; ++v) {
            const int32_t k0 = kt.tile(v) * KT;
            const uint32_t off = locate(kt.tile(v), there);
            if (seen(k0, there, p_lo, p_hi)) continue;
#pragma unroll 1
            for (int kk = 0; kk < KT; ++kk) {
                if (!((there >> kk) & 1)) continue;
                const char *vrow = vp + (uint64_t)(uint32_t)__shfl((int)off, kk) * 16;
                const int32_t key = k0 + kk;
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const bool see = key <= pos[rt] && (a.window == 0 || key > pos[rt] - a.window || key < a.n_sinks);
#pragma unroll
                    for (int q = 0; q < ND; ++q)
#pragma unroll
                        for (int r = 0; r < 16; r += 2) {
                            const int c = 32 * q + acc_key(r, h);
                            const uint32_t u = F8 ? e4m3_pair<false>(*(const uint16_t *)(vrow + c)) : *(const uint32_t *)(vrow + 2 * c);
                            if (see && not_finite(u & 0xffffu)) o[rt][q][r] += bf_lo(u);
                            if (see && not_finite(u & 0xffff0000u)) o[rt][q][r + 1] += bf_hi(u);
                        }
                }
            }
        }
    }

    const float vsc = F8 ? a.vscale[head] : 1.f;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int rr = w0 + 32 * rt + n;
        const float lr = l[rt] + __shfl_xor(l[rt], 32);
        if (rr >= n_rows) continue;
        if (it.parts > 1) {
            float *w = a.c.ws + ((int64_t)(it.slot + it.part) * a.n_heads + head) * (M * (D + 2));
#pragma unroll
            for (int q = 0; q < ND; ++q)
#pragma unroll
                for (int r = 0; r < 16; r += 4)
                    *(float4 *)(w + rr * D + 32 * q + acc_key(r, h)) =
                        make_float4(o[rt][q][r], o[rt][q][r + 1], o[rt][q][r + 2], o[rt][q][r + 3]);
            if (h == 0) {
                w[M * D + rr] = m[rt];
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
                    uint2 y = make_uint2(pack_bf16(o[rt][q][r] * inv, o[rt][q][r + 1] * inv),
                                         pack_bf16(o[rt][q][r + 2] * inv, o[rt][q][r + 3] * inv));
                    if (lr == 0.f) y = make_uint2(0u, 0u);
                    *(uint2 *)(out + 32 * q + acc_key(r, h)) = y;
                }
            if (a.lse && h == 0)
                a.lse[(int64_t)(rq.row0 + tok) * (a.n_heads * G) + head * G + u] =
                    lr == 0.f ? -HUGE_VALF : 0.6931471805599453f * (m[rt] + __log2f(lr));
        }
    }
}

// ------------------------------------------------------------------ joining parts

// One workgroup per 16 rows of a row tile that went in parts: their partial
// sums, brought to the common maximum and added in the order of the parts.
template <int D, int M, int KT, bool F8>
__global__ __launch_bounds__(256) void attn_join_kernel(PagedArgs a) {
    __shared__ SchedLds sched;
    const int head = (int)(blockIdx.x % (uint32_t)a.n_heads);
    Item it;
    const int64_t idx = blockIdx.x / (uint32_t)a.n_heads;
    if (!find_item<M, KT, true>(a, idx / (M / 16), sched, it)) return;
    const int tid = threadIdx.x;
    const Request rq = request(a, it.req);
    const int32_t G = (int32_t)a.G.d;
    const int32_t row0 = it.tile * M;
    const int32_t n_rows = (int32_t)min((int64_t)rq.q_len * G - row0, (int64_t)M);
    const int rr = (int)(idx % (M / 16)) * 16 + tid / (D / 8), ch = tid % (D / 8) * 8;
    if (tid >= 2 * D || rr >= n_rows) return;
    const float *w0 = a.c.ws + ((int64_t)it.slot * a.n_heads + head) * (M * (D + 2));
    const int64_t step = (int64_t)a.n_heads * (M * (D + 2));
    float mx = -HUGE_VALF;
    for (int p = 0; p < it.parts; ++p) mx = fmaxf(mx, w0[p * step + M * D + rr]);
    const float ref = mx == -HUGE_VALF ? 0.f : mx;
    float lr = 0.f, y[8] = {};
    for (int p = 0; p < it.parts; ++p) {
        const float *w = w0 + p * step;
        const float f = __builtin_amdgcn_exp2f(w[M * D + rr] - ref);
        const float4 x0 = *(const float4 *)(w + rr * D + ch), x1 = *(const float4 *)(w + rr * D + ch + 4);
        lr += w[M * D + M + rr] * f;
        y[0] += x0.x * f; y[1] += x0.y * f; y[2] += x0.z * f; y[3] += x0.w * f;
        y[4] += x1.x * f; y[5] += x1.y * f; y[6] += x1.z * f; y[7] += x1.w * f;
    }
    const float inv = lr == 0.f ? 0.f : (F8 ? a.vscale[head] : 1.f) / lr;
    if (lr == 0.f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = 0.f;
    }
    const int32_t tok = (int32_t)fast_div((uint32_t)(row0 + rr), a.G), u = row0 + rr - tok * G;
    uint16_t *out = a.out + (int64_t)(rq.row0 + tok) * a.o_tok + (int64_t)(head * G + u) * a.o_head + ch;
    *(uint4 *)out = make_uint4(pack_bf16(y[0] * inv, y[1] * inv), pack_bf16(y[2] * inv, y[3] * inv),
                               pack_bf16(y[4] * inv, y[5] * inv), pack_bf16(y[6] * inv, y[7] * inv));
    if (a.lse && ch == 0)
        a.lse[(int64_t)(rq.row0 + tok) * (a.n_heads * G) + head * G + u] =
            lr == 0.f ? -HUGE_VALF : 0.6931471805599453f * (mx + __log2f(lr));
}

constexpr int kSmallRows = 16;          // rows of a request up to which attn_rows_kernel takes it beside the tile kernel
constexpr int kTileTarget = 512;        // workgroups of the tile kernel that long rows are divided into
#ifndef CB_RT
#define CB_RT 1
#endif
constexpr int kRT = CB_RT, kTileM = 128 * kRT;

// One kernel over its requests, and the joining of their parts.
template <int D, int M, int KT, bool F8, typename K>
hipError_t launch_class(PagedArgs a, K kernel, int target, int64_t row_min, int64_t row_max, char *&ws, int64_t &ws_bytes,
                        hipStream_t s) {
    const int64_t slot = (int64_t)M * (D + 2) * 4;
    a.c.row_min = row_min;
    a.c.row_max = row_max;
    a.c.target = (int32_t)std::min<int64_t>(target, ws_bytes / (2 * slot));
    // no row is long enough to be divided
    if ((int64_t)a.table_width * a.page_size.d <= (int64_t)kPartMin * KT) a.c.target = 0;
    a.c.ws = (float *)ws;
    ws += 2 * slot * a.c.target;
    ws_bytes -= 2 * slot * a.c.target;
    const int64_t tiles = row_tiles_bound(a.n_tokens, a.n_reqs, a.G.d, M);
    const int64_t items = (tiles + a.c.target / a.n_heads) * a.n_heads;
    const int64_t join = std::min<int64_t>(tiles, a.c.target / a.n_heads) * (M / 16) * a.n_heads;
    if (items > INT32_MAX || join > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL(kernel, dim3((unsigned)items), dim3(256), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
    if (join > 0) hipLaunchKernelGGL((attn_join_kernel<D, M, KT, F8>), dim3((unsigned)join), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <int D, bool F8>
hipError_t launch(PagedArgs a, int32_t max_q_len, void *ws, int64_t ws_bytes, hipStream_t s) {
    const int64_t G = a.G.d;
    char *w = (char *)ws;
    // few rows everywhere: the rows kernel alone, whatever the lengths turn out to be
    if ((int64_t)max_q_len * G <= 32)
        return launch_class<D, 16, kKT, F8>(a, attn_rows_kernel<D, 1, F8>, kTarget, 0, INT64_MAX, w, ws_bytes, s);
    int64_t least = 0;
    if (G <= kSmallRows && a.n_reqs > 1) {
        least = kSmallRows;
        if (hipError_t e = launch_class<D, 16, kKT, F8>(a, attn_rows_kernel<D, 1, F8>, kTarget, 0, least, w, ws_bytes, s)) return e;
    }
    return launch_class<D, kTileM, 64, F8>(a, attn_tile_kernel<D, kRT, F8>, kTileTarget, least, INT64_MAX, w, ws_bytes, s);
}

}  // namespace

int64_t attn_paged_workspace_bytes(int32_t d, int32_t G, int32_t n_tokens, int32_t n_reqs, int32_t max_q_len) {
    const int64_t rows = (int64_t)2 * kTarget * 16 * (d + 2) * 4, tile = (int64_t)2 * kTileTarget * kTileM * (d + 2) * 4;
    return (int64_t)max_q_len * G <= 32 ? rows : rows + tile;
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
