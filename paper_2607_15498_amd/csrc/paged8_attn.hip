// Attention of new tokens over pages of e4m3 codes, gfx950: bf16 queries, and the host side of both.
#include "paged8_attn.h"

namespace vr {

template <>
__device__ __forceinline__ void few_rows<Coded<uint16_t>>(const Piece<Coded<uint16_t>>& P, uint8_t* smem, int rows, bool cut, int64_t rec_row) {
    few_rows8<uint16_t>(P, smem, rows, cut, rec_row);
}
template <>
__device__ __forceinline__ void many_rows<Coded<uint16_t>>(const Piece<Coded<uint16_t>>& P, uint8_t* smem, int32_t row0, int32_t rows,
                                                           bool cut, int64_t rec_row) {
    many_rows8<uint16_t>(P, smem, row0, rows, cut, rec_row);
}

hipError_t launch_paged8_bf16(const AttnArgs& a, int groups, hipStream_t st) { return launch_paged<Coded<uint16_t>>(a, groups, st); }

// ---- host ------------------------------------------------------------------------------------
size_t paged8_attn_ws_bytes(int64_t T, int S, int G, int H, int dtype, int64_t cap) {
    const int64_t rows = max_records(T, S, G, H / G, cap, costs8_of(dtype == VARRATE_BF16).lmin);
    return rows ? (size_t)rows * (D + 2) * 4 + SHARES_BYTES : 0;
}

hipError_t launch_paged8_attn(const varrate_pages8& pg, const varrate_batch& b, int dtype, const void* q, int64_t q_stride, int H,
                              int causal, int window, float scale, void* out, int64_t out_stride, float* lse, void* ws, hipStream_t st) {
    AttnArgs a = {};
    a.q = q;
    a.out = out;
    a.k = pg.k;
    a.v = pg.v;
    a.kscale = (const uint8_t*)pg.k_scale;
    a.vscale = (const uint8_t*)pg.v_scale;
    a.lse = lse;
    a.table = b.table;
    a.kv_len = b.kv_len;
    a.q_start = b.q_start;
    a.rec = (float*)ws;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.table_stride = b.table_stride;
    a.T = (int32_t)b.T;
    a.S = b.S;
    a.cap = b.width * pg.page;
    a.n_pages = (int32_t)pg.n_pages;
    a.G = pg.G;
    a.Hg = H / pg.G;
    a.shift = __builtin_ctz((unsigned)pg.page);
    a.causal = causal;
    a.window = window;
    a.costs = costs8_of(dtype == VARRATE_BF16);
    split_scale(scale, a.c, a.c_lo);
    a.most_units = max_units(b.T, b.S, pg.G, a.Hg);
    a.rec_rows = max_records(b.T, b.S, pg.G, a.Hg, a.cap, a.costs.lmin);
    const int groups = max_groups(b.T, b.S, pg.G, a.Hg, a.cap, a.costs.lmin);
    return dtype == VARRATE_BF16 ? launch_paged8_bf16(a, groups, st) : launch_paged8_f32(a, groups, st);
}

}  // namespace vr
