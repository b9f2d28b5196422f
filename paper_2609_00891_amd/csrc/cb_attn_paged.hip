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
template <int M, bool JOIN>
__device__ __forceinline__ bool find_item(const PagedArgs &a, int64_t idx, SchedLds &sh, Item &out) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    auto work_of = [&](int r) __attribute__((always_inline)) {
        RequestWork w = {0, 0, 0};
        if (r < a.n_reqs) {
            const Request q = request(a, r);
            w = request_work(q.q_len, q.kv_len, (int32_t)a.G.d, M, kKT, a.c.row_min, a.c.row_max, a.window, a.n_sinks);
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
    if (!find_item<M, false>(a, blockIdx.x / (uint32_t)a.n_heads, sched, it)) return;

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

// ------------------------------------------------------------------ joining parts

// One workgroup per 16 rows of a row tile that went in parts: their partial
// sums, brought to the common maximum and added in the order of the parts.
template <int D, int M, bool F8>
__global__ __launch_bounds__(256) void attn_join_kernel(PagedArgs a) {
    __shared__ SchedLds sched;
    const int head = (int)(blockIdx.x % (uint32_t)a.n_heads);
    Item it;
    const int64_t idx = blockIdx.x / (uint32_t)a.n_heads;
    if (!find_item<M, true>(a, idx / (M / 16), sched, it)) return;
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

template <int D, bool F8>
hipError_t launch(PagedArgs a, void *ws, int64_t ws_bytes, hipStream_t s) {
    constexpr int M = 16;
    const int64_t G = a.G.d;
    const int64_t slot = (int64_t)M * (D + 2) * 4;
    a.c.row_min = 0;
    a.c.row_max = INT64_MAX;
    a.c.target = (int32_t)(ws ? std::min<int64_t>(kTarget, ws_bytes / (2 * slot)) : 0);
    a.c.ws = (float *)ws;
    // no row is long enough to be divided
    if ((int64_t)a.table_width * a.page_size.d <= (int64_t)kPartMin * kKT) a.c.target = 0;
    const int64_t tiles = row_tiles_bound(a.n_tokens, a.n_reqs, G, M);
    const int64_t items = (tiles + a.c.target / a.n_heads) * a.n_heads;
    const int64_t join = std::min<int64_t>(tiles, a.c.target / a.n_heads) * (M / 16) * a.n_heads;
    if (items > INT32_MAX || join > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((attn_rows_kernel<D, 1, F8>), dim3((unsigned)items), dim3(256), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
    if (join > 0) hipLaunchKernelGGL((attn_join_kernel<D, M, F8>), dim3((unsigned)join), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

int64_t attn_paged_workspace_bytes(int32_t d, int32_t G, int32_t n_tokens, int32_t n_reqs, int32_t max_q_len) {
    return (int64_t)2 * kTarget * 16 * (d + 2) * 4;
}

hipError_t launch_attn_paged(const PagedArgs &a, int32_t d, bool f8, int32_t max_q_len, void *ws, int64_t ws_bytes,
                             hipStream_t s) {
    switch (d * 2 + f8) {
        case 128: return launch<64, false>(a, ws, ws_bytes, s);
        case 129: return launch<64, true>(a, ws, ws_bytes, s);
        case 192: return launch<96, false>(a, ws, ws_bytes, s);
        case 193: return launch<96, true>(a, ws, ws_bytes, s);
        case 256: return launch<128, false>(a, ws, ws_bytes, s);
        case 257: return launch<128, true>(a, ws, ws_bytes, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace cb
