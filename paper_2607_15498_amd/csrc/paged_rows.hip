// Row operators of the uncompressed cache, gfx950: RMS norm and position rotation of query and key
// rows, appending key and value rows to a paged cache (keys rotated on the way), and gathering a
// sequence's rows out of its pages.  All of them read every row once and write it once; memory bounds
// them for many rows and latency for few.
//
// A row (128 values) belongs to 8 lanes: lane j holds values 8 j .. 8 j + 7 and 64 + 8 j .. 64 + 8 j + 7,
// so the pairs (i, i + 64) of the rotation stay within the lane, every access of a lane is 16 bytes and
// the 8 lanes of a bf16 row read whole 128-byte lines.
#include "vr_internal.h"
#include "vr_pages.h"

namespace vr {
namespace {

// cos and sin of pos x theta (radians; the exact product's fraction of a turn) to fp32: whole turns and
// quarters are removed in fp64, where a position of 2^31 still leaves 2^-24 of a turn at theta = 1, and
// the rest, at most an eighth of a turn, goes through the two Taylor series (x <= pi / 4: the first
// terms left out, x^13 / 13! and x^14 / 14!, are below 2^-36).
__device__ __forceinline__ float2 turn_of(int32_t pos, float theta) {
    double t = (double)pos * ((double)theta * 0.15915494309189533576888);
    t -= rint(t);
    const double quarter = rint(4.0 * t);
    const double x = (t - 0.25 * quarter) * 6.28318530717958647692, x2 = x * x;
    double s = 1.0 / 39916800.0, c = 1.0 / 479001600.0;
    s = -s * x2 + 1.0 / 362880.0;
    s = s * x2 - 1.0 / 5040.0;
    s = s * x2 + 1.0 / 120.0;
    s = s * x2 - 1.0 / 6.0;
    s = (s * x2 + 1.0) * x;
    c = c * x2 - 1.0 / 3628800.0;
    c = c * x2 + 1.0 / 40320.0;
    c = c * x2 - 1.0 / 720.0;
    c = c * x2 + 1.0 / 24.0;
    c = c * x2 - 0.5;
    c = c * x2 + 1.0;
    const int k = (int)quarter & 3;
    const double cc = k & 1 ? s : c, ss = k & 1 ? c : s;
    return float2{(float)(k == 1 || k == 2 ? -cc : cc), (float)(k >= 2 ? -ss : ss)};
}

// 8 values and back.  ONCE: non-temporal.  Append reads and writes so (32768 tokens of 8 + 8 heads: 51.7 -> 46 us, its
// loads or stores alone 51.4 and 48.6); norm and rotation (16384 tokens of 28 + 4 heads: 47 -> 54) and gather (42 -> 48) do not.
struct Half8 { float x[8]; };
template <bool ONCE, typename V> __device__ __forceinline__ V take(const V* p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(p);
    else return *p;
}
template <bool ONCE, typename V> __device__ __forceinline__ void give(V* p, V v) {
    if constexpr (ONCE) __builtin_nontemporal_store(v, p);
    else *p = v;
}
template <bool ONCE = false> __device__ __forceinline__ Half8 load8(const uint16_t* p) {
    const u32x4 w = take<ONCE>((const u32x4*)p);
    Half8 v;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        v.x[2 * k] = bf_lo(w[k]);
        v.x[2 * k + 1] = bf_hi(w[k]);
    }
    return v;
}
template <bool ONCE = false> __device__ __forceinline__ Half8 load8(const float* p) {
    const f32x4 a = take<ONCE>((const f32x4*)p), b = take<ONCE>((const f32x4*)(p + 4));
    return Half8{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
}
template <bool ONCE> __device__ __forceinline__ void store8(uint16_t* p, const Half8& v) {
    give<ONCE>((u32x4*)p, u32x4{cvt_bf16x2(v.x[0], v.x[1]), cvt_bf16x2(v.x[2], v.x[3]), cvt_bf16x2(v.x[4], v.x[5]),
                                cvt_bf16x2(v.x[6], v.x[7])});
}
template <bool ONCE> __device__ __forceinline__ void store8(float* p, const Half8& v) {
    give<ONCE>((f32x4*)p, f32x4{v.x[0], v.x[1], v.x[2], v.x[3]});
    give<ONCE>((f32x4*)(p + 4), f32x4{v.x[4], v.x[5], v.x[6], v.x[7]});
}

// the sum of a row's squares, in each of its 8 lanes
__device__ __forceinline__ float squares(const Half8& x0, const Half8& x1) {
    float sq = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) sq = fmaf(x0.x[k], x0.x[k], fmaf(x1.x[k], x1.x[k], sq));
    sq += shfl_xor_f(sq, 1);
    sq += shfl_xor_f(sq, 2);
    return sq + shfl_xor_f(sq, 4);
}

constexpr int TPB_MAX = 16;

// Two kinds of rows of every token: Ha heads of `a`, then Hb heads of `b`.
struct RowArgs {
    const void *a, *b;
    void *ao, *bo;                   // norm and rotation: rows; append: the pools of keys and values
    int64_t a_stride, b_stride, ao_stride, bo_stride;    // elements between tokens
    const float *wa, *wb;            // norm weights, null: no norm
    int64_t wa_stride, wb_stride;    // elements between heads' weights
    const float* theta;              // null: no rotation
    const int32_t* pos;
    float eps;
    int32_t T, Ha, Hb, tpb, hpb;
    // append
    const int32_t *table, *kv_len, *q_start;
    int64_t table_stride;
    int32_t S, cap, n_pages, shift;
};

// grid (token blocks, head blocks): tpb tokens x hpb heads a workgroup, 32 rows at a time.
// PAGED: keys (a) rotated and values (b) copied into the slots of their sequences' pages.
template <typename ET, bool PAGED>
__global__ __launch_bounds__(256) void row_kernel(RowArgs p) {
    __shared__ float2 cs[TPB_MAX][64];
    __shared__ int64_t slot[TPB_MAX];        // PAGED: page x G x page size + slot, -1: none
    const int h0 = (int)blockIdx.y * p.hpb, Hs = p.Ha + p.Hb;
    const int nh = Hs - h0 < p.hpb ? Hs - h0 : p.hpb;
    const int64_t step = (int64_t)gridDim.x * p.tpb;
    for (int64_t at0 = (int64_t)blockIdx.x * p.tpb; at0 < p.T; at0 += step) {
        const int32_t t0 = (int32_t)at0;
        const int nt = p.T - t0 < p.tpb ? p.T - t0 : p.tpb;
        if (PAGED || p.theta) {
            for (int i = threadIdx.x; i < nt * 64; i += 256) {
                const int t = i >> 6;
                int32_t at = -1;
                if constexpr (PAGED) {
                    const int s = find_seq(p.q_start, p.S, t0 + t);
                    if (s >= 0) {
                        const SeqRange r = seq_range(p.q_start[s], p.q_start[s + 1], p.kv_len[s], p.T, p.cap);
                        at = r.klen - r.qlen + (t0 + t - r.q0);
                        // a length beyond the table would move the rows: nothing is written for it
                        if (p.kv_len[s] > p.cap || p.kv_len[s] < 0) at = -1;
                    }
                    if ((i & 63) == 0) {
                        const int32_t pg = at < 0 ? -1 : good_page(p.table[s * p.table_stride + (at >> p.shift)], p.n_pages);
                        slot[t] = pg < 0 ? -1 : (((int64_t)pg * p.Ha) << p.shift) + (at & ((1 << p.shift) - 1));
                    }
                } else at = p.pos[t0 + t];
                if (p.theta) cs[t][i & 63] = turn_of(at, p.theta[i & 63]);
            }
            __syncthreads();
        }
        const int j = threadIdx.x & 7;
        for (int i = threadIdx.x >> 3; i < nt * nh; i += 32) {
            // norm and rotation: in the order of the rows; append: a head's tokens together, as they lie in its page
            const int t = PAGED ? i % nt : i / nh, hd = h0 + (PAGED ? i / nt : i % nh);
            const bool second = hd >= p.Ha;
            const int hh = second ? hd - p.Ha : hd;
            const ET* src = (second ? (const ET*)p.b + (int64_t)(t0 + t) * p.b_stride
                                    : (const ET*)p.a + (int64_t)(t0 + t) * p.a_stride) + (int64_t)hh * D + 8 * j;
            ET* dst;
            if constexpr (PAGED) {
                if (slot[t] < 0) continue;
                dst = (ET*)(second ? p.bo : p.ao) + (slot[t] + ((int64_t)hh << p.shift)) * D + 8 * j;
            } else {
                dst = (second ? (ET*)p.bo + (int64_t)(t0 + t) * p.bo_stride
                              : (ET*)p.ao + (int64_t)(t0 + t) * p.ao_stride) + (int64_t)hh * D + 8 * j;
            }
            Half8 x0 = load8<PAGED>(src), x1 = load8<PAGED>(src + 64);
            if constexpr (!PAGED) {
                const float* w = second ? p.wb : p.wa;
                if (w) {                         // the same for the 8 lanes of a row
                    w += hh * (second ? p.wb_stride : p.wa_stride) + 8 * j;
                    const Half8 w0 = load8(w), w1 = load8(w + 64);
                    float sq = squares(x0, x1), eps = p.eps;
                    // Squares beyond fp32's range (or of values below 2^-40, where eps does not hide what they lack): of the
                    // row times a power of two, and eps times its square, which leave y as it is.
                    const bool large = sq > 3.4e38f;
                    if (large || (sq < 0x1p-80f && eps < 0x1p-100f)) {
                        const float s = large ? 0x1p-70f : 0x1p100f;
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            x0.x[k] *= s;
                            x1.x[k] *= s;
                        }
                        sq = squares(x0, x1);
                        eps = eps * s * s;
                    }
                    const float r = 1.0f / sqrtf(sq * (1.0f / D) + eps);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        x0.x[k] *= r * w0.x[k];
                        x1.x[k] *= r * w1.x[k];
                    }
                }
            }
            if (p.theta && !(PAGED && second)) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float2 q = cs[t][8 * j + k];
                    const float u = x0.x[k], v = x1.x[k];
                    x0.x[k] = u * q.x - v * q.y;
                    x1.x[k] = u * q.y + v * q.x;
                }
            }
            store8<PAGED>(dst, x0);
            store8<PAGED>(dst + 64, x1);
        }
        if (at0 + step < p.T) __syncthreads();             // the tables are written again
    }
}

// Few rows: a token and 32 of its rows a workgroup, so that they spread over the card.  Many: about 128 rows a workgroup
// share their tokens' angles; append's workgroups find their slots first, and more that are smaller hide that
// better.  Rows a workgroup 64 / 128 / 256: norm and rotation of 16384 tokens of 28 + 4 heads 47.5 / 45.8 / 50 us (5.8 TB/s
// of reading and writing); append of 32768 tokens of 8 + 8 heads 51.3 / 54.4 / 60 us, 53.6 / 57 / 60 with a token's heads
// together instead (46 us, 5.8 TB/s, since its accesses are non-temporal).
template <typename ET, bool PAGED>
hipError_t launch_rows(RowArgs p, hipStream_t st) {
    const int Hs = p.Ha + p.Hb;
    const bool many = (int64_t)p.T * Hs >= 32 * 1024;
    constexpr int per = PAGED ? 64 : 128;
    p.tpb = !many ? 1 : (per + Hs - 1) / Hs < TPB_MAX ? (per + Hs - 1) / Hs : TPB_MAX;
    p.hpb = many ? Hs : Hs < 32 ? Hs : 32;
    const int64_t blocks = ((int64_t)p.T + p.tpb - 1) / p.tpb;
    const dim3 grid((unsigned)(blocks < 1 << 20 ? blocks : 1 << 20), (unsigned)((Hs + p.hpb - 1) / p.hpb));
    row_kernel<ET, PAGED><<<grid, 256, 0, st>>>(p);
    return hipGetLastError();
}

// ---- gather -------------------------------------------------------------------------------------
// 16 bytes of a key row and of a value row a thread and step, in the order of the output.
// 32768 tokens of 8 heads: 41 us, 6.5 TB/s of reading and writing; 777 in fp32: 4.2 us, all latency.
__global__ __launch_bounds__(256) void gather_kernel(const uint4* __restrict__ k, const uint4* __restrict__ v,
                                                     uint4* __restrict__ K, uint4* __restrict__ V,
                                                     const int32_t* __restrict__ table, int64_t n, int G, int n_pages,
                                                     int shift, int pieces /* of a row */) {
    const int64_t total = n * G * pieces;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int c = (int)(i % pieces);
        const int64_t row = i / pieces;
        const int g = (int)(row % G);
        const int64_t t = row / G;
        const int32_t pg = good_page(table[t >> shift], n_pages);
        uint4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
        if (pg >= 0) {
            const int64_t at = (((((int64_t)pg * G + g) << shift) + (t & ((1 << shift) - 1))) * pieces) + c;
            a = k[at];
            b = v[at];
        }
        K[i] = a;
        V[i] = b;
    }
}

}  // namespace

hipError_t launch_norm_rotate(int dtype, const NormRotate& n, hipStream_t st) {
    RowArgs p = {};
    p.a = n.q;
    p.b = n.k;
    p.ao = n.q_out;
    p.bo = n.k_out;
    p.a_stride = n.q_stride;
    p.b_stride = n.k_stride;
    p.ao_stride = n.qo_stride;
    p.bo_stride = n.ko_stride;
    p.wa = n.wq;
    p.wb = n.wk;
    p.wa_stride = n.wq_stride;
    p.wb_stride = n.wk_stride;
    p.theta = n.theta;
    p.pos = n.pos;
    p.eps = n.eps;
    p.T = (int32_t)n.T;
    p.Ha = n.H;
    p.Hb = n.G;
    return dtype == VARRATE_BF16 ? launch_rows<uint16_t, false>(p, st) : launch_rows<float, false>(p, st);
}

hipError_t launch_paged_append(const varrate_pages& pg, const varrate_batch& b, const void* k, int64_t k_stride,
                               const void* v, int64_t v_stride, const float* theta, hipStream_t st) {
    RowArgs p = {};
    p.a = k;
    p.b = v;
    p.ao = pg.k;
    p.bo = pg.v;
    p.a_stride = k_stride;
    p.b_stride = v_stride;
    p.theta = theta;
    p.T = (int32_t)b.T;
    p.Ha = p.Hb = pg.G;
    p.table = b.table;
    p.kv_len = b.kv_len;
    p.q_start = b.q_start;
    p.table_stride = b.table_stride;
    p.S = b.S;
    p.cap = b.width * pg.page;
    p.n_pages = (int32_t)pg.n_pages;
    p.shift = __builtin_ctz((unsigned)pg.page);
    return pg.dtype == VARRATE_BF16 ? launch_rows<uint16_t, true>(p, st) : launch_rows<float, true>(p, st);
}

hipError_t launch_paged_gather(const varrate_pages& pg, const int32_t* table, int64_t n, void* K, void* V, hipStream_t st) {
    const int pieces = D * (pg.dtype == VARRATE_BF16 ? 2 : 4) / 16;
    const int64_t blocks = (n * pg.G * pieces + 255) / 256;
    gather_kernel<<<(unsigned)(blocks < 16384 ? blocks : 16384), 256, 0, st>>>(
        (const uint4*)pg.k, (const uint4*)pg.v, (uint4*)K, (uint4*)V, table, n, pg.G, (int)pg.n_pages,
        __builtin_ctz((unsigned)pg.page), pieces);
    return hipGetLastError();
}

}  // namespace vr
