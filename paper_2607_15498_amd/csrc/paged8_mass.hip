// The weight that each cached key is paid by the batch's new tokens, gfx950:
//   out[s][g][t] = (mass[s][g][t] if t is older than the call, else 0) + sum_r exp(scale <q_r, k_t> - lse_r)
// over the rows r (new token, query head) of KV head g that see key t.  The rows' sums are known (the attention gives their
// logarithms), so one pass over the keys does, and a key belongs to one wave that goes through all rows in order: nothing is
// added by atomics and nothing is joined.
//
// A wave has NK blocks of 32 keys, decoded into bf16 fragments that stay in registers, and takes 32 rows at a time: S^T = K Q^T
// leaves a lane one row and 16 keys of a block, whose weights it adds up; a key's 32 lanes are added at the end.
#include "paged8_attn.h"

namespace vr {
namespace {

struct MassArgs {
    AttnArgs a;
    const float *lse, *mass;
    float* out;
    int64_t L;
    // how many of a sequence's keys there are masses for
    __device__ __forceinline__ int32_t keys(const SeqRange& r) const { return r.klen < L ? r.klen : (int32_t)L; }
};

template <typename Q, int NK>
__global__ __launch_bounds__(256) void paged8_mass_kernel(MassArgs m) {
    typedef Form<Coded<Q>> F;
    constexpr int KEYS = 128 * NK;                         // of a workgroup
    const AttnArgs& a = m.a;
    const int lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5, wave = first_lane((int)(threadIdx.x >> 6));
    const int H = a.G * a.Hg, sh = a.shift - 5;
    const SeqRange first = load_range(a, lane);
    Search from;
    for (int64_t u = blockIdx.x;; u += gridDim.x) {
        Found f;
        if (!find(a, first, u, from, f, [&](const SeqRange& r) { return (int64_t)((m.keys(r) + KEYS - 1) / KEYS) * a.G; })) return;
        const SeqRange r = {first_lane(f.r.q0), first_lane(f.r.qlen), first_lane(f.r.klen)};
        const int s = first_lane(f.s), in = first_lane((int)(u - f.base)), g = in % a.G;
        const int32_t base = in / a.G * KEYS + 32 * NK * wave;
        const int32_t klen = m.keys(r);
        if (base >= klen) continue;
        // keys: block b is base + 32 b ..; lane's key l32, dims 16 (2 j + h) .. of piece j
        u32x4 kf[NK][F::NF];
        uint32_t there = 0;                                // blocks with a page
#pragma unroll
        for (int b = 0; b < NK; ++b) {
            const int32_t t = base + 32 * b;
            int32_t pg = -1;
            if (t < klen) pg = first_lane(good_page(a.table[s * a.table_stride + (t >> a.shift)], a.n_pages));
#pragma unroll
            for (int k = 0; k < F::NF; ++k) kf[b][k] = u32x4{0, 0, 0, 0};
            if (pg < 0) continue;
            there |= 1u << b;
            const int64_t head = (int64_t)pg * a.G + g;
            const float scale = __uint_as_float((uint32_t)a.kscale[(head << sh) + ((t >> 5) & ((1 << sh) - 1))] << 23);
            const uint8_t* row = (const uint8_t*)a.k + ((head << a.shift) + (t & ((1 << a.shift) - 1)) + l32) * D + 16 * h;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const u32x4 w = load16(row + 32 * j);
                kf[b][2 * j] = decode8(uint2{w[0], w[1]}, scale);
                kf[b][2 * j + 1] = decode8(uint2{w[2], w[3]}, scale);
            }
        }
        f32x16 sum[NK];
#pragma unroll
        for (int b = 0; b < NK; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[b][i] = 0.f;
        // the new tokens that see some of these keys, [i0, i1)
        const int32_t old = r.klen - r.qlen, last = base + 32 * NK < klen ? base + 32 * NK - 1 : klen - 1;
        int32_t i0 = 0, i1 = r.qlen;
        if (a.causal && base > old) i0 = base - old;
        if (a.window && (int64_t)last + a.window - old < i1) i1 = last + a.window - old;
        const int64_t rows = (int64_t)r.qlen * a.Hg, end = i1 > i0 ? (int64_t)i1 * a.Hg : 0;
        for (int64_t r0 = (int64_t)i0 * a.Hg & ~(int64_t)31; r0 < end; r0 += 32) {
            const int64_t mine = r0 + l32;
            const bool real = mine < rows;
            const int32_t tok = (int32_t)((real ? mine : r0) / a.Hg), hd = g * a.Hg + (int32_t)((real ? mine : r0) % a.Hg);
            u32x4 qf[F::NP][F::NF];
            const Q* src = (const Q*)a.q + (int64_t)(r.q0 + tok) * a.q_stride + (int64_t)hd * D;
            load_query<Q>(src, h, qf);
            const float lse = real ? m.lse[(int64_t)(r.q0 + tok) * H + hd] : INFINITY;
            // exp(scale x - lse) = exp2(c x - z), both products' roundings carried along
            const float z = lse == -INFINITY ? INFINITY : lse * LOG2E;
            const float z_lo = fabsf(z) < INFINITY ? fmaf(lse, LOG2E, -z) + lse * LOG2E_LO : 0.f;
            int32_t lo, hi;
            row_keys(r, tok, a.causal, a.window, lo, hi);
            if (!real) hi = lo = 0;
#pragma unroll
            for (int b = 0; b < NK; ++b) {
                if (!(there >> b & 1u)) continue;
                f32x16 sc;
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
                for (int p = F::NP - 1; p >= 0; --p)
#pragma unroll
                    for (int k = 0; k < F::NF; ++k) sc = mfma32(kf[b][k], qf[p][k], sc);
                const int32_t t0 = base + 32 * b;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    sc[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], a.c, -z) + fmaf(sc[i], a.c_lo, -z_lo));
                if (__any(lo > t0 || hi < t0 + 32)) {
                    const uint32_t at = (uint32_t)(t0 + 4 * h - lo), n = (uint32_t)(hi > lo ? hi - lo : 0);
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (at + 8 * (i >> 2) + (i & 3) >= n) sc[i] = 0.f;
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[b][i] += sc[i];
            }
        }
        // a key's 32 lanes: halves of the keys change hands four times, then a lane has one key
        const int64_t at = ((int64_t)s * a.G + g) * m.L;
#pragma unroll
        for (int b = 0; b < NK; ++b) {
#pragma unroll
            for (int half = 8, bit = 16; half >= 1; half >>= 1, bit >>= 1) {
                const bool up = l32 & bit;
#pragma unroll
                for (int i = 0; i < half; ++i) {
                    const float give = up ? sum[b][i] : sum[b][i + half], keep = up ? sum[b][i + half] : sum[b][i];
                    sum[b][i] = keep + __shfl_xor(give, bit, WAVE);
                }
            }
            const float x = sum[b][0] + __shfl_xor(sum[b][0], 1, WAVE);
            const int i = l32 >> 1;                        // bit 16 of the lane chose 8, 8 chose 4, 4 chose 2, 2 chose 1
            const int32_t t = base + 32 * b + 8 * (i >> 2) + 4 * h + (i & 3);
            if (!(l32 & 1) && t < klen) m.out[at + t] = (t < old ? m.mass[at + t] : 0.f) + x;
        }
    }
}

template <typename Q>
hipError_t launch_mass(const MassArgs& m, hipStream_t st) {
    const AttnArgs& a = m.a;
    // many rows a sequence: two blocks of keys a wave share the rows' fragments
    const bool many = (int64_t)a.T * a.Hg >= (int64_t)128 * a.S;
    const int64_t keys = many ? 256 : 128, units = ((a.cap < m.L ? a.cap : m.L) + keys - 1) / keys * a.G * a.S;
    const unsigned grid = (unsigned)(units < 4096 ? units : 4096);
    if (many) paged8_mass_kernel<Q, 2><<<grid, 256, 0, st>>>(m);
    else paged8_mass_kernel<Q, 1><<<grid, 256, 0, st>>>(m);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged8_mass(const varrate_pages8& pg, const varrate_batch& b, int dtype, const void* q, int64_t q_stride, int H,
                              int causal, int window, float scale, const float* lse, const float* mass, float* out, int64_t L,
                              hipStream_t st) {
    MassArgs m = {};
    AttnArgs& a = m.a;
    a.q = q;
    a.k = pg.k;
    a.kscale = (const uint8_t*)pg.k_scale;
    a.table = b.table;
    a.kv_len = b.kv_len;
    a.q_start = b.q_start;
    a.q_stride = q_stride;
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
    split_scale(scale, a.c, a.c_lo);
    m.lse = lse;
    m.mass = mass;
    m.out = out;
    m.L = L;
    return dtype == VARRATE_BF16 ? launch_mass<uint16_t>(m, st) : launch_mass<float>(m, st);
}

}  // namespace vr
