// cb_attn_selected.hip -- attention of every token over the pages that were selected
// for it, on gfx950.
//
// Every token and KV head has a list of pages of its own, so what tokens could share
// is the group's query heads: a row tile is one token's (up to 16) query heads of one KV
// head, and rows_body (cb_attn_rows.h) reads the listed pages' keys as one list, 32 at a
// time, each wave its own, from memory straight into matrix-core operands.  The list's
// entry is read three tiles ahead of its keys, the table's two, so no load waits for
// another.  The lists' length and not the contexts' decides the work, and the host knows
// it: keys are divided among workgroups where rows are few, and joined in a second launch.
//
// A key tile in one page (pages of whole tiles) has one place, scale and set of visible keys for its wave
// (kSelectedWhole): no lane asks another for them and the loads' addresses are scalars.  Then K's rows can be read four
// lanes to 64 bytes: neighbouring tokens choose much the same pages, which stay in the caches, and the first cache's
// lookups bind where every lane reads a row of its own.
//
// Tokens of one request that follow one another choose much the same pages, and one token's query heads rarely fill a
// row tile: where a call has rows enough, a tile takes as many tokens as have their heads in it, reads the pages that any of
// them chose once, ascending, and every row sees those of its own token (kSelectedShared).  The lists are sorted in LDS,
// each workgroup for itself.  Only some rows see such keys: with a weight of zero a finite V does no harm, and whether
// there was another shows in the sums, which are then formed again with those zeroed.
//
// 512 tokens of one request, 64 pages of 64 tokens each, a scale for every page (8 heads of 128, 8 query heads each): 400 us
// with a place for every lane, 371 with places for the wave, 273 with K's rows read four lanes together, 218 with two
// tokens a tile.  (In pages of 16, 256 of them, every lane has a place of its own: 388, in bf16 600 where pages of 64 take 260.)
// What binds it then is the vector work on rows, conversions, V's transpose and exponentials, and the
// last workgroups (2,048 on 768 places); its products are 56 us at the rate of large ones.  48 single tokens, 64 pages of
// 32 each: 80-84 us, 5 TB/s, at its bytes (83 at the rate of a copy); in 8-bit pages 51 (42), 128 pages of 16 each 87, in 8 bits 58.
#include "cb_serve_internal.h"
#include "cb_paged_rules.h"
#include "cb_attn_rows.h"

namespace cb {
namespace {

template <int D, int EL, int KEYS>
__global__ __launch_bounds__(256, 2) void attn_selected_kernel(PagedArgs a) {
    __shared__ SchedLds<4> sched;
    __shared__ __attribute__((aligned(16))) RowsLds<D, 4> lds;
    rows_body<D, EL, 4, KEYS>(a, a.rows, blockIdx.x, sched, lds);
}

// Blocks take four rows of a tile, or one where a workgroup joins it.
template <int D, int EL>
__global__ __launch_bounds__(256) void attn_selected_join_kernel(PagedArgs a, FastDiv per) {
    __shared__ JoinLds<D> lds;
    const uint32_t head = blockIdx.x % (uint32_t)a.n_heads, idx = blockIdx.x / (uint32_t)a.n_heads;
    const uint32_t unit = fast_div(idx, per);
    Item it;
    Request rq;
    if (!selected_item(a, unit * a.sel_parts.d, it, rq)) return;
    it.part = (int32_t)(idx - unit * per.d);
    join_rows<D, 16, EL>(a, a.rows, it, rq, (int)head, lds);
}

constexpr int64_t kSlot = 16;           // rows of a partial result

template <int D, int EL>
hipError_t launch(PagedArgs a, void *ws, int64_t ws_bytes, hipStream_t s) {
    const SelectedCut cut = selected_cut(a.n_tokens, a.n_heads, (int32_t)a.G.d, (int32_t)a.page_size.d, a.n_selected);
    const int64_t units = (int64_t)a.n_tokens * cut.tiles, slot = kSlot * (D + 2) * 4;
    const int64_t fits = ws_bytes / (units * a.n_heads * slot);
    const int32_t parts = fits < 2 ? 1 : (int32_t)std::min<int64_t>(cut.parts, fits);
    a.rows.ws = (float *)ws;
    a.sel_parts = make_fastdiv((uint32_t)parts);
    a.sel_tiles = make_fastdiv((uint32_t)cut.tiles);
    // tiles of 32 keys in one page each, their rows within 2^31 bytes
    const bool whole = a.page_size.d % kKT == 0 && a.s_tok < (1u << 21);
    // (places of all keys of a tile's lists are below 2^30)
    const int32_t entries = std::min<int32_t>(kSharedEntries, (1 << 30) / (int32_t)a.page_size.d);
    const int32_t share = whole && parts == 1 ? shared_tokens(a.n_tokens, a.n_reqs, a.n_heads, (int32_t)a.G.d, a.n_selected, entries) : 1;
    if (share > 1) {
        a.sel_tokens = make_fastdiv((uint32_t)share);
        const int64_t tiles = std::min<int64_t>(a.n_tokens, a.n_tokens / share + a.n_reqs);
        hipLaunchKernelGGL((attn_selected_kernel<D, EL, kSelectedShared>), dim3((unsigned)(tiles * a.n_heads)), dim3(256), 0, s, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((whole ? attn_selected_kernel<D, EL, kSelectedWhole> : attn_selected_kernel<D, EL, kSelected>),
                       dim3((unsigned)(units * parts * a.n_heads)), dim3(256), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
    if (parts > 1) {
        const uint32_t rows = std::min<uint32_t>(a.G.d, 16), per = parts > kWideParts ? rows : (rows + 3) / 4;
        hipLaunchKernelGGL((attn_selected_join_kernel<D, EL>), dim3((unsigned)(units * per * a.n_heads)), dim3(256), 0, s, a,
                           make_fastdiv(per));
    }
    return hipGetLastError();
}

}  // namespace

int64_t attn_selected_workspace_bytes(int64_t n_tokens, int32_t n_heads, int32_t G, int32_t d, int32_t page_size,
                                      int32_t n_selected) {
    const SelectedCut cut = selected_cut(n_tokens, n_heads, G, page_size, n_selected);
    return cut.parts > 1 ? n_tokens * cut.tiles * cut.parts * n_heads * kSlot * ((int64_t)d + 2) * 4 : 0;
}

hipError_t launch_attn_selected(const PagedArgs &a, int32_t d, int32_t dtype, void *ws, int64_t ws_bytes, hipStream_t s) {
    switch (d * 4 + dtype) {
        case 256 + CB_PAGES_BF16: return launch<64, kBf16>(a, ws, ws_bytes, s);
        case 256 + CB_PAGES_E4M3: return launch<64, kE4m3>(a, ws, ws_bytes, s);
        case 256 + CB_PAGES_E4M3_BLOCKS: return launch<64, kBlocks>(a, ws, ws_bytes, s);
        case 384 + CB_PAGES_BF16: return launch<96, kBf16>(a, ws, ws_bytes, s);
        case 384 + CB_PAGES_E4M3: return launch<96, kE4m3>(a, ws, ws_bytes, s);
        case 384 + CB_PAGES_E4M3_BLOCKS: return launch<96, kBlocks>(a, ws, ws_bytes, s);
        case 512 + CB_PAGES_BF16: return launch<128, kBf16>(a, ws, ws_bytes, s);
        case 512 + CB_PAGES_E4M3: return launch<128, kE4m3>(a, ws, ws_bytes, s);
        case 512 + CB_PAGES_E4M3_BLOCKS: return launch<128, kBlocks>(a, ws, ws_bytes, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace cb
