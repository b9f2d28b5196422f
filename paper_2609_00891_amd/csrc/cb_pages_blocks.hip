// cb_pages_blocks.hip -- pages whose 8-bit rows have a scale for every page, head
// and K or V on gfx950: rows written into them, pages read back into rows, and
// the least and greatest key channels of pages.
//
// A block, the K or V rows of one page and head, stores x as e4m3(x / 2^e) with its
// scale 2^e: a power of two, so that x 2^-e is exact, rounding happens once, and an
// element stands for a number that bf16 holds exactly, which the conversion
// instruction forms with 2^e as its operand at no cost (floats lose nothing by a scale
// that is up to 2 too large: they have one exponent less below, not one bit less).
// e is the least number with max |x| <= M 2^e over the finite values of the rows as
// they come, M = 448, the largest e4m3 number.  A turn (a, b) -> (a c - b s, b c + a s)
// makes a channel larger by up to sqrt(2): M = 316 for keys that are turned, so the
// scale is found from the rows' own bits, by whole-number maxima, and does not depend
// on positions or roundings.
//
// A step's new tokens of a request lie in consecutive places of consecutive pages.
// One workgroup takes one (request, page) and a group of (layer, head) rows, so no
// other touches its scales: a page that the step begins gets the scale of its new
// rows, one that it continues the larger of its own and theirs, and where that grew
// the codes that are there already go over to it (exactly, but for codes that become
// denormal).  No atomics, no pass before, no workspace.
#include "cb_serve_internal.h"
#include "cb_rows_device.h"

namespace cb {
namespace {

typedef __attribute__((ext_vector_type(2))) uint16_t u16x2_t;

// 2^-64 448 is far below any cache's values, and 2^119 448 below the largest bf16 number, so that what a finite code
// stands for is finite.
constexpr int kEMin = -64, kEMax = 119;
constexpr uint32_t kMantPlain = 96, kMantTurned = 30;          // mantissa bits of 448 and 316 in bf16 (2^8 1.75, 2^8 1.234375)

// The bits of the bf16 values that are infinities or NaNs (an exponent of all ones carries into the sign's place).
__device__ __forceinline__ uint32_t not_finite_halves(uint32_t u) {
    const uint32_t t = ((u & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
    return t | (t - (t >> 15));
}
// The larger magnitudes, half by half, of m and of the finite values of u.
__device__ __forceinline__ uint32_t max_finite(uint32_t m, uint32_t u) {
    const uint32_t x = u & 0x7fff7fffu & ~not_finite_halves(u);
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, m), __builtin_bit_cast(u16x2_t, x)));
}
__device__ __forceinline__ uint32_t max_finite(uint32_t m, const uint4 &v) {
    return max_finite(max_finite(max_finite(max_finite(m, v.x), v.y), v.z), v.w);
}
// The least e from kEMin to kEMax with |x| <= M 2^e, from the bits of |x|.
__device__ __forceinline__ int exponent_for(uint32_t bits, uint32_t mant) {
    return min(max((int)(bits >> 7) - 127 - 8 + ((bits & 127) > mant ? 1 : 0), kEMin), kEMax);
}
__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// Two e4m3 values times 2^e (the scale's exponent is all that counts), as bf16.
template <bool HI> __device__ __forceinline__ uint32_t e4m3_pair(uint32_t u, float scale) {
    const bf16x2_t v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, scale, HI);
    return __builtin_bit_cast(uint32_t, v);
}
// To e4m3, nearest even; what is no number or beyond the largest becomes a NaN.
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
    return (uint32_t)r;
}

// ------------------------------------------------------------------ who does what

// Page `index` of request `req`, which holds n tokens of the step from place `at` on, the first of them row tok0.
struct SpanItem { int32_t req, index, at, n, kv_len; int64_t tok0; };

struct Span { int32_t first, pages; };                         // pages that the last q tokens of a request lie in

__device__ __forceinline__ Span span_of(const SpanArgs &a, int r) {
    Span s = {0, 0};
    if (r >= a.n_reqs) return s;
    const int32_t q = a.q_lens[r], kv = a.kv_lens[r];
    if (q <= 0 || kv < q || kv > a.most) return s;
    if (a.row_starts) {
        const int64_t b = a.row_starts[r];
        if (b < 0 || b + q > a.n_tokens) return s;
    }
    s.first = (int32_t)fast_div((uint32_t)(kv - q), a.page_size);
    s.pages = (int32_t)fast_div((uint32_t)(kv - 1), a.page_size) - s.first + 1;
    return s;
}

// The idx-th of all requests' pages, or false behind the last.  Every wave finds it for itself: a lane has four
// requests, 256 at a time, their pages summed across the lanes.
__device__ __forceinline__ bool find_span(const SpanArgs &a, uint32_t idx, SpanItem &out) {
    const int lane = threadIdx.x & 63;
    uint32_t before = 0;
    for (int r0 = 0; r0 < a.n_reqs; r0 += 256) {
        Span s[4];
        uint32_t n = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[i] = span_of(a, r0 + 4 * lane + i);
            n += (uint32_t)s[i].pages;
        }
        uint32_t sum = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t u = (uint32_t)__shfl_up((int)sum, o);
            if (lane >= o) sum += u;
        }
        const uint32_t total = (uint32_t)__builtin_amdgcn_readlane((int)sum, 63);
        if (idx - before < total) {
            uint32_t k = idx - before - (sum - n);
            const uint64_t mine = __ballot(k < n);             // (below the lane's first: wraps)
            if (mine == 0) return false;
            int req = r0 + 4 * lane, index = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (k < (uint32_t)s[i].pages) {
                    req = r0 + 4 * lane + i;
                    index = s[i].first + (int)k;
                    break;
                }
                k -= (uint32_t)s[i].pages;
            }
            const int from = __builtin_ctzll(mine);
            out.req = __builtin_amdgcn_readlane(req, from);
            out.index = __builtin_amdgcn_readlane(index, from);
            const int32_t q = a.q_lens[out.req], kv = a.kv_lens[out.req], ps = (int32_t)a.page_size.d;
            const int32_t begin = out.index * ps, pos = max(begin, kv - q);
            out.kv_len = kv;
            out.at = pos - begin;
            out.n = min(ps - out.at, kv - pos);
            out.tok0 = a.row_starts ? (int64_t)a.row_starts[out.req] + (pos - (kv - q)) : 0;
            return true;
        }
        before += total;
    }
    return false;
}

// How the 256 threads of a workgroup share the n rows of a page: a team of S threads (a power of two) has one
// (layer, head) row at a time, a thread of it P pairs of 16-byte chunks at a time, unit u = pair u mod 2^lgc
// of token u >> lgc; where the page has more units than P S they are taken in `turns`.
template <int P> struct Team {
    int lgc, lgS, S, j, slot, teams, turns, n, nc2;
    __device__ __forceinline__ Team(int n_tok, int nc2_, int lgc_) : lgc(lgc_), n(n_tok), nc2(nc2_) {
        const int units = n << lgc;                            // (a page has at most 2^24 tokens)
        lgS = lgc;
        while (lgS < 8 && (1 << lgS) < units) ++lgS;
        S = 1 << lgS;
        j = threadIdx.x & (S - 1);
        slot = threadIdx.x >> lgS;
        teams = 256 >> lgS;
        turns = (units + P * S - 1) / (P * S);
    }
    __device__ __forceinline__ bool unit(int turn, int p, int &i, int &c) const {
        const int u = j + S * (p + P * turn);
        i = u >> lgc;
        c = u & ((1 << lgc) - 1);
        return i < n && c < nc2;
    }
};

__device__ __forceinline__ int64_t row_place(const RowsArgs &a, int64_t tok) {
    const uint32_t seq = fast_div((uint32_t)tok, a.seq_len);
    return seq * a.is.seq + (int64_t)((uint32_t)tok - seq * a.seq_len.d) * a.is.tok;
}

// ------------------------------------------------------------------ rows into pages

template <bool ROPE, int P>
__global__ __launch_bounds__(256) void page_quant_kernel(RowsArgs a, SpanArgs span, float *scales) {
    __shared__ uint32_t sh_max[2][4], sh_old[2][4];
    int parity = 0;                                            // which of the two places in LDS
    for (uint32_t item = blockIdx.x;; item += gridDim.x) {
        SpanItem it;
        if (!find_span(span, item, it)) return;
        const int32_t page = span.table[it.req * span.table_stride + it.index];
        if ((uint32_t)page >= (uint32_t)span.n_pages) continue;
        const int nc2 = (int)a.nc2.d, H = (int)a.n_heads.d, LH = a.n_lh, QH = a.n_qh;
        const Team<P> tm(it.n, nc2, a.lgc);
        const int row0 = blockIdx.y * a.group, row1 = min(row0 + a.group, a.n_rows);
        const int wave = threadIdx.x >> 6;
        // places and angles of the thread's units, kept where one turn is all
        int64_t in_at[P], out_at[P], tok[P];
        int cc[P];
        bool ok[P];
        Angles an[P];
        auto units = [&](int turn, bool angles) __attribute__((always_inline)) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                int i;
                ok[p] = tm.unit(turn, p, i, cc[p]);
                tok[p] = it.tok0 + i;
                in_at[p] = ok[p] ? row_place(a, tok[p]) : 0;
                out_at[p] = page * a.os.seq + (int64_t)(it.at + i) * a.os.tok;
                if (ROPE && angles && ok[p]) an[p] = load_angles(a.rope, tok[p], cc[p], nc2, a.sign);
            }
        };
        const bool one = tm.turns == 1;
        if (one) units(0, row0 < LH + QH);
        for (int base = row0; base < row1; base += tm.teams) {
            const int row = base + tm.slot;
            const bool live = row < row1, is_q = row >= LH && row < LH + QH;
            const int kv = row >= LH + QH, lh = kv ? row - LH - QH : row;
            const int l = is_q ? 0 : (int)fast_div((uint32_t)lh, a.n_heads), h = is_q ? 0 : lh - l * H;
            const bool turned = ROPE && !kv;
            const uint16_t *x = is_q ? a.q + (row - LH) * a.q_head : a.in + l * a.is.layer + kv * a.is.kv + h * a.is.head;
            ChunkPair v[P];
            auto fetch = [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    v[p] = {};
                    if (!ok[p] || !live) continue;
                    const uint16_t *r = x + (is_q ? tok[p] * a.q_tok : in_at[p]);
                    v[p].a = *(const uint4 *)(r + 8 * cc[p]);
                    v[p].b = *(const uint4 *)(r + 8 * (cc[p] + nc2));
                }
            };
            // the largest magnitude of the block's new rows
            uint32_t m = 0;
            for (int turn = 0; turn < tm.turns; ++turn) {
                if (!one) units(turn, false);
                fetch();
#pragma unroll
                for (int p = 0; p < P; ++p) m = max_finite(max_finite(m, v[p].a), v[p].b);
            }
            m = max(m & 0xffffu, m >> 16);
            for (int s = 1; s < min(tm.S, 64); s <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, s));
            float *sc = scales + ((((int64_t)(a.layer0 + l) * span.n_pages + page) * H + h) * 2 + kv);
            const bool goes_on = it.at > 0 && live && !is_q;
            uint32_t was = 0;                                      // the exponent's bits of the block's scale so far
            if (tm.S <= 64) {
                if (goes_on) was = __float_as_uint(*sc);
            } else {
                // (one wave of the team reads the scale, so that none does after another has written it)
                if ((tm.j >> 6) == 0 && goes_on) was = __float_as_uint(*sc);
                if ((threadIdx.x & 63) == 0) {
                    sh_max[parity][wave] = m;
                    sh_old[parity][wave] = was;
                }
                __syncthreads();
                const int w0 = tm.slot * (tm.S / 64);
                was = sh_old[parity][w0];
                for (int w = 0; w < tm.S / 64; ++w) m = max(m, sh_max[parity][w0 + w]);
                parity ^= 1;
            }
            if (!live) continue;
            int e = exponent_for(m, turned ? kMantTurned : kMantPlain);
            if (goes_on) {
                const int e_old = min(max((int)((was >> 23) & 255) - 127, kEMin), kEMax);
                e = max(e, e_old);
                if (e > e_old) {                                   // what is there goes over to the larger scale
                    const float f = power(max(e_old - e, -126));
                    for (int u = tm.j; u < it.at << tm.lgc; u += tm.S) {
                        const int i = u >> tm.lgc, c = u & ((1 << tm.lgc) - 1);
                        if (c >= nc2) continue;
                        uint4 *o = (uint4 *)((uint8_t *)a.out + l * a.os.layer + kv * a.os.kv + h * a.os.head + page * a.os.seq +
                                             (int64_t)i * a.os.tok + 16 * c);
                        const uint4 w = *o;
                        const uint32_t in[4] = {w.x, w.y, w.z, w.w};
                        uint32_t out[4];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const uint32_t y0 = e4m3_pair<false>(in[q], f), y1 = e4m3_pair<true>(in[q], f);
                            out[q] = to_e4m3(bf_lo(y0), bf_hi(y0), bf_lo(y1), bf_hi(y1));
                        }
                        *o = make_uint4(out[0], out[1], out[2], out[3]);
                    }
                }
            }
            if (tm.j == 0 && !is_q) *sc = power(e);
            const float inv = power(-e);
            for (int turn = 0; turn < tm.turns; ++turn) {
                if (!one) {
                    units(turn, turned);
                    fetch();
                }
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    if (!ok[p]) continue;
                    float y0[8], y1[8];
                    if (turned) {
                        cb::turn(v[p], an[p], a.rope.style, y0, y1);
                    } else {
                        unpack8(v[p].a, y0);
                        unpack8(v[p].b, y1);
                    }
                    if (is_q) {
                        uint16_t *o = a.q_out + tok[p] * a.qo_tok + (row - LH) * a.qo_head;
                        *(uint4 *)(o + 8 * cc[p]) = pack8(y0);
                        *(uint4 *)(o + 8 * (cc[p] + nc2)) = pack8(y1);
                    } else {
                        uint8_t *o = (uint8_t *)a.out + l * a.os.layer + kv * a.os.kv + h * a.os.head + out_at[p];
                        *(uint2 *)(o + 8 * cc[p]) = make_uint2(to_e4m3(y0[0] * inv, y0[1] * inv, y0[2] * inv, y0[3] * inv),
                                                             to_e4m3(y0[4] * inv, y0[5] * inv, y0[6] * inv, y0[7] * inv));
                        *(uint2 *)(o + 8 * (cc[p] + nc2)) = make_uint2(to_e4m3(y1[0] * inv, y1[1] * inv, y1[2] * inv, y1[3] * inv),
                                                                     to_e4m3(y1[4] * inv, y1[5] * inv, y1[6] * inv, y1[7] * inv));
                    }
                }
            }
        }
    }
}

// ------------------------------------------------------------------ pages into rows

enum { kBf16, kE4m3, kBlocks };

// a.in: the rows that are written; a.out: the pool that is read.
template <int KIND, bool ROPE, int P>
__global__ __launch_bounds__(256) void page_read_kernel(RowsArgs a, SpanArgs span, const float *scales) {
    for (uint32_t item = blockIdx.x;; item += gridDim.x) {
        SpanItem it;
        if (!find_span(span, item, it)) return;
        const int32_t page = span.table[it.req * span.table_stride + it.index];
        if ((uint32_t)page >= (uint32_t)span.n_pages) continue;
        const int nc2 = (int)a.nc2.d, H = (int)a.n_heads.d, LH = a.n_lh;
        const Team<P> tm(it.n, nc2, a.lgc);
        const int row0 = blockIdx.y * a.group, row1 = min(row0 + a.group, a.n_rows);
        for (int turn = 0; turn < tm.turns; ++turn) {
            int64_t in_at[P], out_at[P];
            int cc[P];
            bool ok[P];
            Angles an[P];
#pragma unroll
            for (int p = 0; p < P; ++p) {
                int i;
                ok[p] = tm.unit(turn, p, i, cc[p]);
                in_at[p] = ok[p] ? row_place(a, it.tok0 + i) : 0;
                out_at[p] = page * a.os.seq + (int64_t)(it.at + i) * a.os.tok;
                if (ROPE && ok[p] && row0 < LH) an[p] = load_angles(a.rope, it.tok0 + i, cc[p], nc2, a.sign);
            }
            for (int row = row0 + tm.slot; row < row1; row += tm.teams) {
                const int kv = row >= LH, lh = kv ? row - LH : row;
                const int l = (int)fast_div((uint32_t)lh, a.n_heads), h = lh - l * H;
                const bool turned = ROPE && !kv;
                float sc = 1.f;
                if (KIND == kE4m3) sc = scales[((a.layer0 + l) * 2 + kv) * H + h];
                if (KIND == kBlocks) sc = scales[(((int64_t)(a.layer0 + l) * span.n_pages + page) * H + h) * 2 + kv];
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    if (!ok[p]) continue;
                    const int64_t from = l * a.os.layer + kv * a.os.kv + h * a.os.head + out_at[p];
                    uint16_t *o = (uint16_t *)a.in + l * a.is.layer + kv * a.is.kv + h * a.is.head + in_at[p];
                    ChunkPair v;
                    if (KIND == kBf16) {
                        const uint16_t *x = (const uint16_t *)a.out + from;
                        v.a = *(const uint4 *)(x + 8 * cc[p]);
                        v.b = *(const uint4 *)(x + 8 * (cc[p] + nc2));
                    } else {
                        // e4m3 numbers (times a power of two) are bf16 numbers
                        const uint8_t *x = (const uint8_t *)a.out + from;
                        const uint2 w0 = *(const uint2 *)(x + 8 * cc[p]), w1 = *(const uint2 *)(x + 8 * (cc[p] + nc2));
                        const float f = KIND == kBlocks ? sc : 1.f;
                        v.a = make_uint4(e4m3_pair<false>(w0.x, f), e4m3_pair<true>(w0.x, f), e4m3_pair<false>(w0.y, f), e4m3_pair<true>(w0.y, f));
                        v.b = make_uint4(e4m3_pair<false>(w1.x, f), e4m3_pair<true>(w1.x, f), e4m3_pair<false>(w1.y, f), e4m3_pair<true>(w1.y, f));
                    }
                    if (turned || KIND == kE4m3) {
                        float y0[8], y1[8];
                        if (turned) {
                            cb::turn(v, an[p], a.rope.style, y0, y1);
                        } else {
                            unpack8(v.a, y0);
                            unpack8(v.b, y1);
                        }
                        if (KIND == kE4m3) {
#pragma unroll
                            for (int q = 0; q < 8; ++q) {
                                y0[q] *= sc;
                                y1[q] *= sc;
                            }
                        }
                        v.a = pack8(y0);
                        v.b = pack8(y1);
                    }
                    *(uint4 *)(o + 8 * cc[p]) = v.a;
                    *(uint4 *)(o + 8 * (cc[p] + nc2)) = v.b;
                }
            }
        }
    }
}

// ------------------------------------------------------------------ bounds of pages

// A NaN among the two is the result.
__device__ __forceinline__ float least(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ __forceinline__ float greatest(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// A wave has the K rows of one (page, layer, head): a lane a 16-byte chunk of every 64 >> lgc-th token.
template <bool F8>
__global__ __launch_bounds__(256) void page_bounds_kernel(BoundsArgs a, SpanArgs span) {
    constexpr int E = F8 ? 16 : 8;                             // channels of a chunk
    const int lane = threadIdx.x & 63, lh = blockIdx.y * 4 + (threadIdx.x >> 6);
    const int c = lane & ((1 << a.lgc) - 1), slot = lane >> a.lgc, slots = 64 >> a.lgc;
    const int H = (int)a.n_heads.d, l = (int)fast_div((uint32_t)lh, a.n_heads), h = lh - l * H;
    if (lh >= a.n_lh) return;
    for (uint32_t item = blockIdx.x;; item += gridDim.x) {
        SpanItem it;
        if (!find_span(span, item, it)) return;
        const int32_t page = span.table[it.req * span.table_stride + it.index];
        if ((uint32_t)page >= (uint32_t)span.n_pages) continue;
        const int n = min((int)span.page_size.d, it.kv_len - it.index * (int)span.page_size.d);
        const char *x = a.k + l * a.s_layer + page * a.s_page + h * a.s_head + 16 * c;
        float lo[E], hi[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            lo[e] = HUGE_VALF;
            hi[e] = -HUGE_VALF;
        }
        if (c < a.chunks) {
            for (int t = slot; t < n; t += slots) {
                const uint4 v = *(const uint4 *)(x + t * a.s_tok);
                const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t y[2] = {u[w], 0};
                    if (F8) {
                        y[0] = e4m3_pair<false>(u[w], 1.f);
                        y[1] = e4m3_pair<true>(u[w], 1.f);
                    }
#pragma unroll
                    for (int k = 0; k < (F8 ? 2 : 1); ++k) {
                        const int e = (F8 ? 4 : 2) * w + 2 * k;
                        lo[e] = least(lo[e], bf_lo(y[k]));
                        hi[e] = greatest(hi[e], bf_lo(y[k]));
                        lo[e + 1] = least(lo[e + 1], bf_hi(y[k]));
                        hi[e + 1] = greatest(hi[e + 1], bf_hi(y[k]));
                    }
                }
            }
        }
        for (int s = 1 << a.lgc; s < 64; s <<= 1) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                lo[e] = least(lo[e], __shfl_xor(lo[e], s));
                hi[e] = greatest(hi[e], __shfl_xor(hi[e], s));
            }
        }
        if (slot == 0 && c < a.chunks) {
            char *o = a.bounds + (((int64_t)(a.layer0 + l) * span.n_pages + page) * H + h) * (32 * a.chunks) + 16 * c;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const float *y = b ? hi : lo;
                uint4 w;
                if (F8) {
                    w = make_uint4(to_e4m3(y[0], y[1], y[2], y[3]), to_e4m3(y[4], y[5], y[6], y[7]),
                                   to_e4m3(y[8 % E], y[9 % E], y[10 % E], y[11 % E]), to_e4m3(y[12 % E], y[13 % E], y[14 % E], y[15 % E]));
                } else {
                    w = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
                }
                *(uint4 *)(o + 16 * a.chunks * b) = w;
            }
        }
    }
}

// Pages that the new tokens of a call can lie in together, unless requests share rows: a page has at least one token,
// all but a request's first and last a whole page.  (Workgroups go round while there are more.)
int64_t span_bound(const SpanArgs &s) {
    const int64_t b = s.n_tokens / s.page_size.d + 2 * (int64_t)s.n_reqs;
    return b < s.n_tokens ? b : s.n_tokens;
}

// Pairs of chunks of a thread: as many as let 256 threads hold a page's row in registers, up to 4.
int pairs_for(const RowsArgs &a, const SpanArgs &s) {
    const int64_t units = (int64_t)s.page_size.d << a.lgc;
    return units <= 256 ? 1 : units <= 512 ? 2 : 4;
}

int log2_up(int n) {
    int l = 0;
    while ((1 << l) < n) ++l;
    return l;
}

// Rows of a page that one workgroup takes: up to 16, which share its places and angles, while the launch fills the chip.
bool cut(RowsArgs &a, const SpanArgs &s, dim3 &grid) {
    const int64_t items = span_bound(s);
    a.lgc = log2_up((int)a.nc2.d);
    a.group = 16;
    while (a.group > 1 && items * ((a.n_rows + a.group - 1) / a.group) < 2048) a.group /= 2;
    while ((a.n_rows + a.group - 1) / a.group > 65535) a.group *= 2;
    if (items > INT32_MAX) return false;
    grid = dim3((unsigned)(items < 1 ? 1 : items), (unsigned)((a.n_rows + a.group - 1) / a.group));
    return true;
}

}  // namespace

hipError_t launch_page_quant(RowsArgs a, const SpanArgs &span, bool rope, float *scales, hipStream_t s) {
    dim3 grid;
    if (!cut(a, span, grid)) return hipErrorInvalidValue;
    switch (pairs_for(a, span) * 2 + rope) {
        case 2: hipLaunchKernelGGL((page_quant_kernel<false, 1>), grid, dim3(256), 0, s, a, span, scales); break;
        case 3: hipLaunchKernelGGL((page_quant_kernel<true, 1>), grid, dim3(256), 0, s, a, span, scales); break;
        case 4: hipLaunchKernelGGL((page_quant_kernel<false, 2>), grid, dim3(256), 0, s, a, span, scales); break;
        case 5: hipLaunchKernelGGL((page_quant_kernel<true, 2>), grid, dim3(256), 0, s, a, span, scales); break;
        case 8: hipLaunchKernelGGL((page_quant_kernel<false, 4>), grid, dim3(256), 0, s, a, span, scales); break;
        default: hipLaunchKernelGGL((page_quant_kernel<true, 4>), grid, dim3(256), 0, s, a, span, scales); break;
    }
    return hipGetLastError();
}

hipError_t launch_page_read(RowsArgs a, const SpanArgs &span, bool rope, int32_t dtype, const float *scales, hipStream_t s) {
    dim3 grid;
    if (!cut(a, span, grid)) return hipErrorInvalidValue;
    const auto kernel = dtype == CB_PAGES_BF16   ? rope ? page_read_kernel<kBf16, true, 2> : page_read_kernel<kBf16, false, 2>
                        : dtype == CB_PAGES_E4M3 ? rope ? page_read_kernel<kE4m3, true, 2> : page_read_kernel<kE4m3, false, 2>
                                                 : rope ? page_read_kernel<kBlocks, true, 2> : page_read_kernel<kBlocks, false, 2>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a, span, scales);
    return hipGetLastError();
}

hipError_t launch_page_bounds(BoundsArgs a, const SpanArgs &span, bool f8, int32_t max_q_len, hipStream_t s) {
    a.lgc = log2_up(a.chunks);
    const int64_t each = (int64_t)max_q_len / span.page_size.d + 2;
    int64_t items = (each < max_q_len ? each : max_q_len) * span.n_reqs;
    if (items < 1) items = 1;
    if (items > 65536) items = 65536;
    const dim3 grid((unsigned)items, (unsigned)((a.n_lh + 3) / 4));
    if (f8) hipLaunchKernelGGL(page_bounds_kernel<true>, grid, dim3(256), 0, s, a, span);
    else hipLaunchKernelGGL(page_bounds_kernel<false>, grid, dim3(256), 0, s, a, span);
    return hipGetLastError();
}

}  // namespace cb
