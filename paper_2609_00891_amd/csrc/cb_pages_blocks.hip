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
//
// page_quant_kernel: a page's tokens are spread over teams of threads that have one row at a time, in registers between
//   the search of its maximum and its writing; the next row is on its way meanwhile, and the barrier between the waves of
//   a team waits for LDS alone.  Everything about a row is one number for a wave (teams of whole waves), the conversions
//   take bf16 pairs and the scale as they are.  Bound by HBM: 64 layers of four mapped caches of up to 2,048 tokens, keys
//   turned (2.65 GB), 565 us, 4.7 TB/s (a copy of 2 GiB: 4.9).  With rows that differed within a wave (64-bit products
//   for every address, in vector instructions) 845 us, with values unpacked, scaled and masked one by one 767, with two rows ahead 616.
// page_read_kernel: the same search and places without a maximum: 40 layers of 8,191 tokens turned back (2.0 GB) 390 us,
//   5.2 TB/s; from e4m3 pages with one scale a head the same, from bf16 pages 520 us (2.7 GB).
// page_bounds_kernel: the pages of a step 5-7 us, a launch.  Whole contexts, 40 layers of 8,191 tokens of 8 heads of 128: 123 us
//   in bf16 pages of 64 (0.69 GB, 5.6 TB/s) and 185 in pages of 16; 85 and 262 in 8-bit ones: of a small
//   page a wave reads 4 or 2 KB behind a search of its own.
#include "cb_serve_internal.h"
#include "cb_paged_rules.h"
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
// The larger magnitudes, half by half, of m and of u's values, or of its finite ones alone.
template <bool FINITE> __device__ __forceinline__ uint32_t max_halves(uint32_t m, uint32_t u) {
    uint32_t x = u & 0x7fff7fffu;
    if (FINITE) x &= ~not_finite_halves(u);
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, m), __builtin_bit_cast(u16x2_t, x)));
}
template <bool FINITE> __device__ __forceinline__ uint32_t max_halves(uint32_t m, const uint4 &v) {
    return max_halves<FINITE>(max_halves<FINITE>(max_halves<FINITE>(max_halves<FINITE>(m, v.x), v.y), v.z), v.w);
}
// The maximum over a wave, by data-parallel moves (in its last lane, read from there).
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t max_moved(uint32_t x) {
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    x = max_moved<0x111, 0xf>(x);   // row_shr:1, 2, 4, 8
    x = max_moved<0x112, 0xf>(x);
    x = max_moved<0x114, 0xf>(x);
    x = max_moved<0x118, 0xf>(x);
    x = max_moved<0x142, 0xa>(x);   // row_bcast:15, 31
    x = max_moved<0x143, 0xc>(x);
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
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
// Over the scale 2^e and to e4m3, nearest even; what is no number or beyond the largest becomes a NaN.  (The conversions take
// the scale's exponent; with every bf16 number they give what a product with 2^-e and a rounding give.)
typedef __attribute__((ext_vector_type(2))) short s16x2_t;
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d, float scale = 1.f) {
    s16x2_t r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, scale, true);
    return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ uint32_t to_e4m3(uint32_t ab, uint32_t cd, float scale) {
    s16x2_t r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2_t, ab), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2_t, cd), scale, true);
    return __builtin_bit_cast(uint32_t, r);
}

// Four codes times a power of two, rounded to e4m3 again.
__device__ __forceinline__ uint32_t shifted(uint32_t codes, float f) {
    return to_e4m3(e4m3_pair<false>(codes, f), e4m3_pair<true>(codes, f), 1.f);
}

// A kernel's arguments, read anew: a workgroup that goes from its rows' work to the next search does not hold both in
// scalar registers (which spilled by the hundred).
template <typename T> __device__ __forceinline__ const T &arguments() {
    auto p = (const __attribute__((address_space(4))) T *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const T *)p;
}

// ------------------------------------------------------------------ who does what

// Page `index` of request `req`, which holds n tokens of the step from place `at` on, the first of them row tok0; whether
// there may be another for the workgroup.
struct SpanItem { int32_t req, index, at, n, kv_len; int64_t tok0; bool more; };

// The idx-th of the pages that the last q_lens[r] tokens of all requests lie in, or false behind the last.  Every wave finds
// it for itself: a lane has four requests, 256 at a time, loaded together, their pages summed across the lanes.
template <bool ROWS>
__device__ __forceinline__ bool find_span(const SpanArgs &a, uint32_t idx, SpanItem &out) {
    const int lane = threadIdx.x & 63;
    const int32_t ps = (int32_t)a.page_size.d;
    uint32_t before = 0;
    for (int r0 = 0; r0 < a.n_reqs; r0 += 256) {
        int32_t q[4], kv[4], b[4], first[4];
        uint32_t pages[4], n = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = min(r0 + 4 * lane + i, a.n_reqs - 1);
            q[i] = a.q_lens[r];
            kv[i] = a.kv_lens[r];
            b[i] = ROWS ? a.row_starts[r] : 0;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool is = r0 + 4 * lane + i < a.n_reqs && q[i] > 0 && kv[i] >= q[i] && kv[i] <= a.most &&
                            (!ROWS || (b[i] >= 0 && (int64_t)b[i] + q[i] <= a.n_tokens));
            first[i] = (int32_t)fast_div((uint32_t)(kv[i] - q[i]), a.page_size);
            pages[i] = is ? fast_div((uint32_t)(kv[i] - 1), a.page_size) - (uint32_t)first[i] + 1 : 0;
            n += pages[i];
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
            int i = 0;
            int32_t qi = q[0], kvi = kv[0], bi = b[0], fi = first[0];
#pragma unroll
            for (int j = 0; j < 3; ++j) {
                const bool past = i == j && k >= pages[j];
                k -= past ? pages[j] : 0;
                i = past ? j + 1 : i;
                qi = past ? q[j + 1] : qi;
                kvi = past ? kv[j + 1] : kvi;
                bi = past ? b[j + 1] : bi;
                fi = past ? first[j + 1] : fi;
            }
            const int from = __builtin_ctzll(mine);
            out.req = r0 + 4 * from + __builtin_amdgcn_readlane(i, from);
            out.index = __builtin_amdgcn_readlane(fi + (int)k, from);
            const int32_t tokens = __builtin_amdgcn_readlane(qi, from);
            out.kv_len = __builtin_amdgcn_readlane(kvi, from);
            const int32_t begin = out.index * ps, old = out.kv_len - tokens, pos = max(begin, old);
            out.at = pos - begin;
            out.n = min(ps - out.at, out.kv_len - pos);
            out.tok0 = (int64_t)__builtin_amdgcn_readlane(bi, from) + (pos - old);
            out.more = idx + gridDim.x - before < total || r0 + 256 < a.n_reqs;
            return true;
        }
        before += total;
    }
    return false;
}

// How the 256 threads of a workgroup share the n rows of a page: a team of S threads (a power of two) has one
// (layer, head) row at a time, a thread of it P pairs of 16-byte chunks at a time, unit u = pair u mod 2^lgc
// of token u >> lgc; where the page has more units than P S they are taken in `turns`.  WIDE: teams of whole waves, so
// that everything about a row is one number for the wave.
template <bool WIDE, int P> struct Team {
    int lgc, lgS, S, j, slot, teams, turns, n, nc2;
    __device__ __forceinline__ Team(int n_tok, int nc2_, int lgc_) : lgc(lgc_), n(n_tok), nc2(nc2_) {
        const int units = n << lgc;                            // (a page has at most 2^24 tokens)
        lgS = WIDE ? 6 : lgc;
        while (lgS < 8 && (1 << lgS) < units) ++lgS;
        S = 1 << lgS;
        j = threadIdx.x & (S - 1);
        slot = threadIdx.x >> lgS;
        if (WIDE) slot = __builtin_amdgcn_readfirstlane(slot);
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

// A barrier for what waves exchange in LDS: rows on their way from and to memory stay on it.
__device__ __forceinline__ void meet() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// ------------------------------------------------------------------ rows into pages

struct SpanRowsArgs {
    RowsArgs rows;
    SpanArgs span;
    float *scales;
};

// ONE: no page has more units than a team takes in one turn.
template <bool ROPE, bool WIDE, bool ONE, int P>
__global__ __launch_bounds__(256) void page_quant_kernel(SpanRowsArgs) {
    __shared__ uint32_t sh_max[2][4], sh_old[2][4];
    int parity = 0;                                            // which of the two places in LDS
    SpanItem it;
    it.more = true;
    for (uint32_t item = blockIdx.x; it.more; item += gridDim.x) {
        int32_t page;
        {
            const SpanArgs &span = arguments<SpanRowsArgs>().span;
            if (!find_span<true>(span, item, it)) return;
            page = span.table[it.req * span.table_stride + it.index];
            if ((uint32_t)page >= (uint32_t)span.n_pages) continue;
        }
        const SpanRowsArgs &args = arguments<SpanRowsArgs>();
        const RowsArgs &a = args.rows;
        const int nc2 = (int)a.nc2.d, H = (int)a.n_heads.d, LH = a.n_lh, QH = a.n_qh;
        const Team<WIDE, P> tm(it.n, nc2, a.lgc);
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
                if (ROPE && angles && ok[p]) an[p] = load_angles<true>(a.rope, tok[p], cc[p], nc2, a.sign);
            }
        };
        // a (layer, head) row, or a query's
        struct Row { const uint16_t *x; int l, h, kv; bool live, is_q; };
        auto row_at = [&](int row) __attribute__((always_inline)) {
            Row r;
            r.live = row < row1;
            r.is_q = row >= LH && row < LH + QH;
            r.kv = row >= LH + QH;
            const int lh = r.kv ? row - LH - QH : row;
            r.l = r.is_q ? 0 : (int)fast_div((uint32_t)lh, a.n_heads);
            r.h = r.is_q ? row - LH : lh - r.l * H;
            r.x = r.is_q ? a.q + r.h * a.q_head : a.in + r.l * a.is.layer + r.kv * a.is.kv + r.h * a.is.head;
            return r;
        };
        auto fetch = [&](const Row &r, ChunkPair (&v)[P]) __attribute__((always_inline)) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                v[p] = {};
                if (!ok[p] || !r.live) continue;
                const uint16_t *x = r.x + (r.is_q ? tok[p] * a.q_tok : in_at[p]);
                v[p].a = *(const uint4 *)(x + 8 * cc[p]);
                v[p].b = *(const uint4 *)(x + 8 * (cc[p] + nc2));
            }
        };
        const bool one = ONE || tm.turns == 1;
        const int turns = one ? 1 : tm.turns;
        ChunkPair v[P], ahead[P];
        Row row = row_at(row0 + tm.slot);
        if (one) {
            units(0, row0 < LH + QH);
            fetch(row, v);
        }
        for (int base = row0; base < row1; base += tm.teams) {
            const Row next = row_at(base + tm.teams + tm.slot);
            if (one && base + tm.teams < row1) fetch(next, ahead);     // on their way while this row is worked on
            const bool turned = ROPE && !row.kv;
            // the largest magnitude of the block's new rows, of the finite ones where that is none
            float *sc = args.scales + ((((int64_t)(a.layer0 + row.l) * args.span.n_pages + page) * H + row.h) * 2 + row.kv);
            const bool goes_on = it.at > 0 && row.live && !row.is_q;
            uint32_t was = 0;                                      // the bits of the block's scale so far
            if (goes_on && (tm.S <= 64 || (tm.j >> 6) == 0)) was = __float_as_uint(*sc);
            uint32_t m = 0;
            for (int pass = 0; pass < 2; ++pass) {
                m = 0;
                for (int turn = 0; turn < turns; ++turn) {
                    if (!one) {
                        units(turn, false);
                        fetch(row, v);
                    }
                    if (pass == 0) {
#pragma unroll
                        for (int p = 0; p < P; ++p) m = max_halves<false>(max_halves<false>(m, v[p].a), v[p].b);
                    } else {
#pragma unroll
                        for (int p = 0; p < P; ++p) m = max_halves<true>(max_halves<true>(m, v[p].a), v[p].b);
                    }
                }
                m = max(m & 0xffffu, m >> 16);
                if (WIDE) {
                    m = wave_max(m);
                } else {
                    for (int s = 1; s < min(tm.S, 64); s <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, s));
                }
                bool again = __any(m >= 0x7f80u);
                if (tm.S > 64) {
                    // (one wave of the team reads the scale, so that none does after another has written it)
                    if ((threadIdx.x & 63) == 0) {
                        sh_max[parity][wave] = m;
                        sh_old[parity][wave] = was;
                    }
                    meet();
                    const int w0 = tm.slot * (tm.S / 64);
                    was = sh_old[parity][w0];
                    for (int w = 0; w < tm.S / 64; ++w) m = max(m, sh_max[parity][w0 + w]);
                    // (alike for all teams, which meet at the barrier)
                    again = max(max(sh_max[parity][0], sh_max[parity][1]), max(sh_max[parity][2], sh_max[parity][3])) >= 0x7f80u;
                    parity ^= 1;
                    if (WIDE) {
                        m = (uint32_t)__builtin_amdgcn_readfirstlane((int)m);
                        was = (uint32_t)__builtin_amdgcn_readfirstlane((int)was);
                    }
                }
                if (!again) break;
            }
            if (row.live) {
                int e = exponent_for(m, turned ? kMantTurned : kMantPlain);
                uint8_t *block = (uint8_t *)a.out + row.l * a.os.layer + row.kv * a.os.kv + row.h * a.os.head;
                if (goes_on) {
                    const int e_old = min(max((int)((was >> 23) & 255) - 127, kEMin), kEMax);
                    e = max(e, e_old);
                    if (e > e_old) {                               // what is there goes over to the larger scale
                        const float f = power(max(e_old - e, -126));
                        for (int u = tm.j; u < it.at << tm.lgc; u += tm.S) {
                            const int i = u >> tm.lgc, c = u & ((1 << tm.lgc) - 1);
                            if (c >= nc2) continue;
                            uint4 *o = (uint4 *)(block + page * a.os.seq + (int64_t)i * a.os.tok + 16 * c);
                            const uint4 w = *o;
                            *o = make_uint4(shifted(w.x, f), shifted(w.y, f), shifted(w.z, f), shifted(w.w, f));
                        }
                    }
                }
                const float scale = power(e);
                if (tm.j == 0 && !row.is_q) *sc = scale;
                for (int turn = 0; turn < turns; ++turn) {
                    if (!one) {
                        units(turn, turned);
                        fetch(row, v);
                    }
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        if (!ok[p]) continue;
                        float y0[8], y1[8];
                        if (turned) cb::turn(v[p], an[p], a.rope.style, y0, y1);
                        if (row.is_q) {
                            uint16_t *o = a.q_out + tok[p] * a.qo_tok + row.h * a.qo_head;
                            *(uint4 *)(o + 8 * cc[p]) = pack8(y0);
                            *(uint4 *)(o + 8 * (cc[p] + nc2)) = pack8(y1);
                            continue;
                        }
                        uint2 w0, w1;
                        if (turned) {
                            w0 = make_uint2(to_e4m3(y0[0], y0[1], y0[2], y0[3], scale), to_e4m3(y0[4], y0[5], y0[6], y0[7], scale));
                            w1 = make_uint2(to_e4m3(y1[0], y1[1], y1[2], y1[3], scale), to_e4m3(y1[4], y1[5], y1[6], y1[7], scale));
                        } else {
                            w0 = make_uint2(to_e4m3(v[p].a.x, v[p].a.y, scale), to_e4m3(v[p].a.z, v[p].a.w, scale));
                            w1 = make_uint2(to_e4m3(v[p].b.x, v[p].b.y, scale), to_e4m3(v[p].b.z, v[p].b.w, scale));
                        }
                        uint8_t *o = block + out_at[p];
                        *(uint2 *)(o + 8 * cc[p]) = w0;
                        *(uint2 *)(o + 8 * (cc[p] + nc2)) = w1;
                    }
                }
            }
            row = next;
            if (one) {
#pragma unroll
                for (int p = 0; p < P; ++p) v[p] = ahead[p];
            }
        }
    }
}

// ------------------------------------------------------------------ pages into rows

enum { kBf16, kE4m3, kBlocks };

// a.in: the rows that are written; a.out: the pool that is read.
template <int KIND, bool ROPE, bool WIDE, int P>
__global__ __launch_bounds__(256) void page_read_kernel(SpanRowsArgs) {
    SpanItem it;
    it.more = true;
    for (uint32_t item = blockIdx.x; it.more; item += gridDim.x) {
        int32_t page;
        {
            const SpanArgs &span = arguments<SpanRowsArgs>().span;
            if (!find_span<true>(span, item, it)) return;
            page = span.table[it.req * span.table_stride + it.index];
            if ((uint32_t)page >= (uint32_t)span.n_pages) continue;
        }
        const SpanRowsArgs &args = arguments<SpanRowsArgs>();
        const RowsArgs &a = args.rows;
        const int nc2 = (int)a.nc2.d, H = (int)a.n_heads.d, LH = a.n_lh;
        const Team<WIDE, P> tm(it.n, nc2, a.lgc);
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
                if (ROPE && ok[p] && row0 < LH) an[p] = load_angles<true>(a.rope, it.tok0 + i, cc[p], nc2, a.sign);
            }
            for (int row = row0 + tm.slot; row < row1; row += tm.teams) {
                const int kv = row >= LH, lh = kv ? row - LH : row;
                const int l = (int)fast_div((uint32_t)lh, a.n_heads), h = lh - l * H;
                const bool turned = ROPE && !kv;
                float sc = 1.f;
                if (KIND == kE4m3) sc = args.scales[((a.layer0 + l) * 2 + kv) * H + h];
                if (KIND == kBlocks) sc = args.scales[(((int64_t)(a.layer0 + l) * args.span.n_pages + page) * H + h) * 2 + kv];
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
    SpanItem it;
    it.more = true;
    for (uint32_t item = blockIdx.x; it.more; item += gridDim.x) {
        if (!find_span<false>(span, item, it)) return;
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
            // (eight tokens' chunks on their way together; behind the last, it again)
            for (int t0 = slot; t0 < n; t0 += 8 * slots) {
                uint4 v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = *(const uint4 *)(x + min(t0 + i * slots, n - 1) * a.s_tok);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t u[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
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

// The launch of a call on spans of pages.
struct Cut { dim3 grid; bool wide; int pairs; };
Cut cut(RowsArgs &a, const SpanArgs &s) {
    const SpanCut c = span_cut(s.n_tokens, s.n_reqs, (int32_t)s.page_size.d, (int32_t)a.nc2.d * 16, a.n_rows);
    a.lgc = c.lgc;
    a.group = c.group;
    return {dim3((unsigned)c.blocks, (unsigned)c.groups), c.wide, c.pairs};
}

template <bool ROPE>
auto quant_kernel(const Cut &c) {
    return !c.wide        ? page_quant_kernel<ROPE, false, false, 1>
           : c.pairs == 1 ? page_quant_kernel<ROPE, true, true, 1>
           : c.pairs == 2 ? page_quant_kernel<ROPE, true, true, 2>
           : c.pairs == 4 ? page_quant_kernel<ROPE, true, true, 4>
                          : page_quant_kernel<ROPE, true, false, 2>;
}
template <int KIND>
auto read_kernel(const Cut &c, bool rope) {
    return c.wide ? rope ? page_read_kernel<KIND, true, true, 2> : page_read_kernel<KIND, false, true, 2>
                  : rope ? page_read_kernel<KIND, true, false, 1> : page_read_kernel<KIND, false, false, 1>;
}

}  // namespace

hipError_t launch_page_quant(RowsArgs a, const SpanArgs &span, bool rope, float *scales, hipStream_t s) {
    const Cut c = cut(a, span);
    hipLaunchKernelGGL(rope ? quant_kernel<true>(c) : quant_kernel<false>(c), c.grid, dim3(256), 0, s, SpanRowsArgs{a, span, scales});
    return hipGetLastError();
}

hipError_t launch_page_read(RowsArgs a, const SpanArgs &span, bool rope, int32_t dtype, const float *scales, hipStream_t s) {
    const Cut c = cut(a, span);
    const auto kernel = dtype == CB_PAGES_BF16   ? read_kernel<kBf16>(c, rope)
                        : dtype == CB_PAGES_E4M3 ? read_kernel<kE4m3>(c, rope)
                                                 : read_kernel<kBlocks>(c, rope);
    hipLaunchKernelGGL(kernel, c.grid, dim3(256), 0, s, SpanRowsArgs{a, span, const_cast<float *>(scales)});
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
