// cb_pages.hip -- pages of a serving receiver on gfx950: the tables of a step,
// rotary positions with several axes, and the write of rows into pages.
//
// page_tables_kernel: sums of the requests' lengths give every request its
//   token rows and its free pages.  The sums are over at most 4096 requests, so
//   every workgroup forms them itself (wave scans, 256 requests at a time) and
//   then fills its share of the tokens and new table entries by binary search
//   in LDS: one launch, no pass that waits for another.  Bound by latency: 64
//   requests of one token 4.3 us, 512 requests of 273,000 tokens (2.3 MB of
//   tables) 10.6 us.
//
// rows_kernel: one thread per (token, pair of 16-byte chunks) -- channels
//   8c .. 8c+7 and the chunk d/16 further on, which holds their half-split
//   partners -- and a group of consecutive (layer, head) rows.  The token's slot
//   and angles are read once for the group; products in fp32 from the exact
//   bf16 values and the fp32 table, one rounding to the output's type.
//   HBM-bound: every row is read once and written once.  40 layers of 12,282
//   tokens turned back (8 heads of 128, 4.0 GB) 0.78 .. 0.80 ms, 5.0 TB/s; a mapped
//   cache of 64 layers x 4,096 tokens into 16-bit pages (2.1 GB) 0.41 ms, 5.2
//   TB/s; four of up to 2,048 tokens into 8-bit pages, keys turned (2.4 GB),
//   0.49 ms, 4.8 TB/s.
#include "cb_serve_internal.h"
#include "cb_paged_rules.h"
#include "cb_rows_device.h"

namespace cb {
namespace {

// ------------------------------------------------------------------ page tables

constexpr int kTokensPerThread = 4;

// Inclusive sum over the 256 threads of a workgroup; *total gets the whole.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t *wsum, int64_t *total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t u = __shfl_up(v, o);
        if (lane >= o) v += u;
    }
    __syncthreads();                                          // wsum of the previous scan has been read
    if (lane == 63) wsum[wave] = v;
    __syncthreads();
    int64_t t = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < wave) v += wsum[w];
        t += wsum[w];
    }
    *total = t;
    return v;
}

// Last index i in [0, n) with key[i] <= x (key[0] = 0 <= x, not decreasing).
__device__ __forceinline__ int last_le(const int32_t *key, int n, int32_t x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (key[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ __launch_bounds__(256) void page_tables_kernel(PageTablesArgs a) {
    extern __shared__ int32_t lds[];
    int32_t *start = lds;                                     // [n_reqs + 1] token rows before a request
    int32_t *base = lds + a.n_reqs + 1;                       // [n_reqs] new pages before it
    uint8_t *why = (uint8_t *)(base + a.n_reqs);              // [n_reqs] info
    __shared__ int64_t wsum[4];
    const int tid = threadIdx.x;
    const bool first = blockIdx.x == 0;
    const int64_t ps = a.page_size.d;
    int64_t c_tok = 0, c_page = 0;
    for (int r0 = 0; r0 < a.n_reqs; r0 += 256) {
        const int r = r0 + tid;
        const bool is = r < a.n_reqs;
        const int32_t ctx = is ? a.ctx_lens[r] : 0, q = is ? a.q_lens[r] : 0;
        const bool bad = ctx < 0 || q < 0;
        int64_t total;
        const int64_t t1 = c_tok + block_scan(bad ? 0 : q, wsum, &total);
        c_tok += total;
        const int64_t t0 = t1 - (bad ? 0 : q);
        const int64_t have = bad ? 0 : ((int64_t)ctx + ps - 1) / ps;
        const int64_t all = bad ? 0 : ((int64_t)ctx + q + ps - 1) / ps;
        int info = bad ? 3 : all > a.table_width ? 2 : t1 > a.max_tokens ? 4 : 0;
        const int64_t need = info ? 0 : all - have;
        const int64_t p1 = c_page + block_scan(need, wsum, &total);
        c_page += total;
        if (need > 0 && p1 > a.n_free) info = 1;
        if (is) {
            start[r] = (int32_t)min(t0, (int64_t)a.max_tokens);
            base[r] = (int32_t)min(p1 - need, (int64_t)a.n_free);
            why[r] = (uint8_t)info;
            if (first) {
                a.q_starts[r] = start[r];
                a.kv_lens[r] = info ? 0 : ctx + q;
                a.info[r] = info;
            }
        }
    }
    // Pages are given out up to the first request that found the list used up: its base, the least of
    // those refused for it.
    __shared__ int32_t given;
    if (tid == 0) {
        start[a.n_reqs] = (int32_t)min(c_tok, (int64_t)a.max_tokens);
        given = (int32_t)min(c_page, (int64_t)INT32_MAX);
    }
    __syncthreads();
    for (int r = tid; r < a.n_reqs; r += 256)
        if (why[r] == 1) atomicMin(&given, base[r]);
    __syncthreads();
    const int32_t n_new = given;
    if (first && tid == 0) {
        a.q_starts[a.n_reqs] = start[a.n_reqs];
        a.n_used[0] = n_new;
    }
    __syncthreads();
    const int64_t n_thr = (int64_t)gridDim.x * 256;
    // new table entries
    for (int64_t e = (int64_t)blockIdx.x * 256 + tid; e < n_new; e += n_thr) {
        // requests that need no page share the base of the next that does, so the last base at or
        // before e is that of the request that gets page e
        const int r = last_le(base, a.n_reqs, (int32_t)e);
        const int64_t have = ((int64_t)a.ctx_lens[r] + ps - 1) / ps;
        a.block_table[r * a.table_stride + have + (e - base[r])] = a.free_pages[e];
    }
    // slots and positions
    const int32_t n_tok = start[a.n_reqs];
    for (int64_t t = (int64_t)blockIdx.x * 256 + tid; t < a.max_tokens; t += n_thr) {
        int32_t slot = -1, pos = -1;
        if (t < n_tok) {
            const int r = last_le(start, a.n_reqs, (int32_t)t);
            if (why[r] == 0) {
                const int32_t ctx = a.ctx_lens[r];
                pos = ctx + (int32_t)(t - start[r]);
                const uint32_t idx = fast_div((uint32_t)pos, a.page_size);
                const uint32_t have = (uint32_t)(((int64_t)ctx + ps - 1) / ps);
                const int32_t page = idx < have ? a.block_table[r * a.table_stride + idx]
                                                : a.free_pages[base[r] + (int32_t)(idx - have)];
                const int64_t s = (int64_t)page * ps + (pos - (int64_t)idx * ps);
                slot = page < 0 || s > INT32_MAX ? -1 : (int32_t)s;
            }
        }
        a.slots[t] = slot;
        a.positions[t] = pos;
    }
}

// ------------------------------------------------------------------ rows: turn, copy, write into pages

// x * inv to e4m3, nearest even, clamped to the largest value; a NaN fails both comparisons and stays.
__device__ __forceinline__ float clamp_e4m3(float x) { return x > 448.f ? 448.f : x < -448.f ? -448.f : x; }
__device__ __forceinline__ uint2 pack8_e4m3(const float y[8], float inv) {
    int r[2] = {0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        r[h] = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_e4m3(y[4 * h] * inv), clamp_e4m3(y[4 * h + 1] * inv), r[h], false);
        r[h] = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_e4m3(y[4 * h + 2] * inv), clamp_e4m3(y[4 * h + 3] * inv), r[h], true);
    }
    return make_uint2((uint32_t)r[0], (uint32_t)r[1]);
}

// The value of another lane.
__device__ __forceinline__ uint4 exchange(const uint4 &v, int lane) {
    return make_uint4((uint32_t)__shfl((int)v.x, lane), (uint32_t)__shfl((int)v.y, lane), (uint32_t)__shfl((int)v.z, lane),
                      (uint32_t)__shfl((int)v.w, lane));
}

// Rows of a token, in this order: K rows (layer, head), then query rows, then V rows.  blockIdx.y takes
// a.group of them; a wave takes a.tok_per_wave tokens.
// PAIRS: two tokens' lanes exchange halves of rows (rows_cut in cb_paged_rules.h, with what it measured).
template <bool ROPE, bool F8, bool PAIRS>
__global__ __launch_bounds__(256) void rows_kernel(RowsArgs a) {
    static_assert(!(F8 && PAIRS), "8-bit pages have no pairs");
    const int nc2 = (int)a.nc2.d, lane = threadIdx.x & 63;
    const int tl = (int)fast_div((uint32_t)lane, a.nc2), c = lane - tl * nc2;
    if (tl >= a.tok_per_wave) return;                          // (an even number: of a pair both stay)
    const int64_t tok = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * a.tok_per_wave + tl;
    const int odd = PAIRS ? tl & 1 : 0, other = lane + (odd ? -nc2 : nc2);
    // where the rows of the lane's token, or of the pair's two, come from and go
    constexpr int NT = PAIRS ? 2 : 1;
    int64_t in_tok[NT], out_tok[NT];
    bool ok[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int64_t t = tok - odd + i;
        ok[i] = t < a.n_tokens;
        in_tok[i] = out_tok[i] = 0;
        if (!ok[i]) continue;
        const uint32_t seq = fast_div((uint32_t)t, a.seq_len);
        const uint32_t in_seq = (uint32_t)t - seq * a.seq_len.d;
        in_tok[i] = seq * a.is.seq + (int64_t)in_seq * a.is.tok;
        if (a.slots) {
            const int32_t slot = a.slots[t];
            ok[i] = slot >= 0 && slot < a.n_slots;
            const uint32_t page = fast_div((uint32_t)slot, a.page_size);
            out_tok[i] = page * a.os.seq + (int64_t)((uint32_t)slot - page * a.page_size.d) * a.os.tok;
        } else {
            out_tok[i] = seq * a.os.seq + (int64_t)in_seq * a.os.tok;
        }
    }
    if (!ok[0] && !ok[NT - 1]) return;                         // both lanes of a pair
    const int row0 = blockIdx.y * a.group, row1 = min(row0 + a.group, a.n_rows);
    const int LH = a.n_lh, QH = a.n_qh;
    Angles an = {};
    if (ROPE && row0 < LH + QH && ok[odd]) an = load_angles<F8>(a.rope, tok, c, nc2, a.sign);
    // the two 16-byte chunks of a row that the lane reads, or one of each of the pair's rows
    const int p0 = PAIRS ? odd * nc2 + c : c, p1 = PAIRS ? p0 : c + nc2;
    for (int row = row0; row < row1; ++row) {
        const bool is_q = row >= LH && row < LH + QH;
        const int kv = row >= LH + QH;
        const int lh = kv ? row - LH - QH : row;
        const int l = is_q ? 0 : (int)fast_div((uint32_t)lh, a.n_heads), h = is_q ? 0 : lh - l * (int)a.n_heads.d;
        const uint16_t *x = is_q ? a.q + (tok - odd) * a.q_tok + (row - LH) * a.q_head
                                 : a.in + l * a.is.layer + kv * a.is.kv + h * a.is.head;
        const uint16_t *x0 = x + (is_q ? 0 : in_tok[0]), *x1 = x + (is_q ? (PAIRS ? a.q_tok : 0) : in_tok[NT - 1]);
        ChunkPair v = {};
        if (ok[0]) v.a = *(const uint4 *)(x0 + 8 * p0);
        if (ok[NT - 1]) v.b = *(const uint4 *)(x1 + 8 * p1);
        if constexpr (PAIRS) {
            const uint4 got = exchange(odd ? v.a : v.b, other);
            if (odd) v.a = got; else v.b = got;
        }
        float y0[8], y1[8];
        const bool turned = ROPE && !kv;
        if (turned) {
            turn(v, an, a.rope.style, y0, y1);
        } else if (F8) {
            unpack8(v.a, y0);
            unpack8(v.b, y1);
        }
        if (F8 && !is_q) {
            const float inv = 1.0f / a.scales[((a.layer0 + l) * 2 + kv) * (int)a.n_heads.d + h];
            uint8_t *o = (uint8_t *)a.out + l * a.os.layer + kv * a.os.kv + h * a.os.head;
            *(uint2 *)(o + out_tok[0] + 8 * c) = pack8_e4m3(y0, inv);
            *(uint2 *)(o + out_tok[0] + 8 * (c + nc2)) = pack8_e4m3(y1, inv);
        } else {
            uint16_t *o = is_q ? a.q_out + (tok - odd) * a.qo_tok + (row - LH) * a.qo_head
                               : (uint16_t *)a.out + l * a.os.layer + kv * a.os.kv + h * a.os.head;
            uint16_t *o0 = o + (is_q ? 0 : out_tok[0]), *o1 = o + (is_q ? (PAIRS ? a.qo_tok : 0) : out_tok[NT - 1]);
            uint4 w0 = turned ? pack8(y0) : v.a, w1 = turned ? pack8(y1) : v.b;
            if constexpr (PAIRS) {
                const uint4 got = exchange(odd ? w0 : w1, other);
                if (odd) w0 = got; else w1 = got;
            }
            if (ok[0]) *(uint4 *)(o0 + 8 * p0) = w0;
            if (ok[NT - 1]) *(uint4 *)(o1 + 8 * p1) = w1;
        }
    }
}

}  // namespace

hipError_t launch_page_tables(const PageTablesArgs &a, hipStream_t s) {
    const int64_t most = a.max_tokens > a.n_free ? a.max_tokens : a.n_free;
    int64_t blocks = (most + 256 * kTokensPerThread - 1) / (256 * kTokensPerThread);
    if (blocks < 1) blocks = 1;
    if (blocks > 512) blocks = 512;
    const size_t bytes = (size_t)(2 * a.n_reqs + 1) * 4 + (size_t)a.n_reqs;
    hipLaunchKernelGGL(page_tables_kernel, dim3((unsigned)blocks), dim3(256), bytes, s, a);
    return hipGetLastError();
}

hipError_t launch_rows(RowsArgs a, bool rope, bool f8, hipStream_t s) {
    if (a.n_tokens == 0 || a.n_rows == 0) return hipSuccess;
    const RowsCut cut = rows_cut(a.n_tokens, a.n_rows, 16 * (int)a.nc2.d, f8);
    a.tok_per_wave = cut.tok_per_wave;
    a.group = cut.group;
    const dim3 grid((unsigned)cut.blocks, (unsigned)cut.groups);
    const bool pairs = cut.pairs;
    const auto kernel = f8 ? rope ? rows_kernel<true, true, false> : rows_kernel<false, true, false>
                        : pairs ? rope ? rows_kernel<true, false, true> : rows_kernel<false, false, true>
                                : rope ? rows_kernel<true, false, false> : rows_kernel<false, false, false>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace cb
