// The weight that each cached key is paid by the batch's new tokens, gfx950:
//   out[s][g][t] = (mass[s][g][t] if t is older than the call, else 0) + sum_r exp(scale <q_r, k_t> - lse_r)
// over the rows r (new token, query head) of KV head g that see key t.  The rows' sums are known (the attention gives their
// logarithms), so one pass over the keys does, and a key belongs to one wave that goes through all rows in order: nothing is
// added by atomics and nothing is joined.
//
// A workgroup has 128 U keys and stages the rows that see them in shared memory, as the products take them; its waves bring
// their keys through rings of their own, 32 at a time.  S^T = K Q^T leaves a lane one row and 16 keys, whose weights it adds up over
// the staged rows; then a key's 32 lanes are added.
//   Few rows (single tokens): rings of four tiles, up to 16 rows in products of 16 x 16; the reads of the keys bound it (8 tokens over
//   16384 of 4 KV heads of 7: 16.2 us of the card, 32.6 over 32768, 4.9 TB/s, and 6.8 over 128; with 32 x 32 products 3 more;
//   fragments read from memory into registers, a wave's keys at a time, 42).  Many: 160 rows (fp32 32) are staged at once, and the
//   exponentials and the products bound it, with what the next rows' staging waits for (1024 tokens over 16384 of 8 heads of 4: 225 us,
//   590 TFLOP/s, matrix cores busy for 23% of the time and vector instructions for 50%; a window of 32 over 32768: 18 us, over 128 8).
#include "paged8_attn.h"

namespace vr {
namespace {

// exp(scale x - lse) = exp2(c x - z) 2^-(what z, lse log2 e, lacks of it): z and that factor.  lse's rounding, 2^-24 of it, is an exponent's
// error, so that a weight could be anything between nothing and infinity.  Rows whose |z| is 2^8 and more pay a key 1 at most: LARGE in
// the number of their first key takes them where masks are looked at, which costs the others next to nothing (1024 tokens over 17408:
// 343 -> 345 us; a bound for every score 360).  From |z| = FAR on fp32's steps are 1 and more, and z is taken 2^-20 of it lower, so that the
// key whose score is the row's largest is paid 1, and so are those that are as near to it as the sums of a score's products, taken in
// another order by the attention, are to each other (fp32 queries, 100 rows: up to more than 2^-22).
constexpr int32_t LARGE = 1 << 30;                         // (no key's number)
constexpr float FAR = 0x1p24f;
__device__ __forceinline__ float2 subtracted(float lse) {
    const float z = lse * LOG2E, lack = fmaf(lse, LOG2E, -z) + lse * LOG2E_LO, most = __builtin_elementwise_minimum(z, 0x1.fffffep127f);
    const bool far = fabsf(z) >= FAR;
    const float low = far ? fmaf(fabsf(most), -0x1p-20f, most) : z;
    return float2{z == -INFINITY ? INFINITY : low, __builtin_amdgcn_exp2f(far ? 0.f : -lack)};      // (no sum: nothing is paid)
}
// (NaN stays NaN)
__device__ __forceinline__ float paid_most(float x, float most) { return __builtin_elementwise_minimum(x, most); }

struct MassArgs {
    AttnArgs a;
    const float *lse, *mass;
    float* out;
    int64_t L;
    // how many of a sequence's keys there are masses for
    __device__ __forceinline__ int32_t keys(const SeqRange& r) const { return r.klen < L ? r.klen : (int32_t)L; }
};

constexpr int MOST_U = 8;
template <typename Q>
struct MassForm {
    typedef Form<Coded<Q>> F;
    static constexpr int FRAGS = F::NP * F::NF * 1024;     // a block of 32 rows
    static constexpr int RING_FEW = F::NP == 1 ? 4 : 3, RING_MANY = 2;
    static constexpr int RB_MANY = F::NP == 1 ? 5 : 1;
    static constexpr int SUMS = 4 * MOST_U * 32 * 4, ROWS = RB_MANY * 32 * 16;
    static constexpr int FEW = FRAGS + 4 * RING_FEW * F::KB, MANY = RB_MANY * FRAGS + 4 * RING_MANY * F::KB;
    static constexpr int LDS = SUMS + ROWS + (FEW > MANY ? FEW : MANY);
    static_assert(LDS <= 80 * 1024, "two workgroups a CU");
};

template <int CTRL> __device__ __forceinline__ float dpp(float x) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, true));
}
// What a wave's lanes have of 16 keys each (lane 32 h + i: key 8 (k / 4) + 4 h + k % 4 in x[k]), added over i: lane i ends with the
// key of k = i / 2.  Pairs of lanes exchange halves of what they have.
__device__ __forceinline__ float sum_lanes(f32x16 x) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < 8; ++k) {                          // lanes 16 apart
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x[k]), __float_as_uint(x[k + 8]), false, false);
        x[k] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)                            // i and 15 - i
        x[k] = (lane & 8 ? x[k + 4] : x[k]) + dpp<0x140>(lane & 8 ? x[k] : x[k + 4]);
#pragma unroll
    for (int k = 0; k < 2; ++k)                            // i and 7 - i
        x[k] = (lane & 4 ? x[k + 2] : x[k]) + dpp<0x141>(lane & 4 ? x[k] : x[k + 2]);
    const float y = (lane & 2 ? x[1] : x[0]) + dpp<0x4E>(lane & 2 ? x[0] : x[1]);
    return y + dpp<0xB1>(y);
}

// The same of 8 keys, lane 16 q + i: key 16 (k / 4) + 4 q + k % 4 in x[k], added over i: lane i ends with the key of k = i / 2.
__device__ __forceinline__ float sum_lanes16(float (&x)[8]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = (lane & 8 ? x[k + 4] : x[k]) + dpp<0x140>(lane & 8 ? x[k] : x[k + 4]);
#pragma unroll
    for (int k = 0; k < 2; ++k) x[k] = (lane & 4 ? x[k + 2] : x[k]) + dpp<0x141>(lane & 4 ? x[k] : x[k + 2]);
    const float y = (lane & 2 ? x[1] : x[0]) + dpp<0x4E>(lane & 2 ? x[0] : x[1]);
    return y + dpp<0xB1>(y);
}

// A wave's tiles: number i is keys first + 128 i .. + 31, i < U; page and scale of tile i in lane i.
template <typename Q>
struct Tiles {
    Piece<Coded<Q>> P;
    int32_t first, page;
    float scale;
    int U;
    uint32_t ring0;
    uint8_t* ring;
    template <int R> __device__ __forceinline__ void issue(int i) const {
        const int32_t pg = i < U ? __builtin_amdgcn_readlane(page, i & 63) : -1;
        const uint8_t* k = P.rows_at(P.kbase, pg, first + 128 * i);
#pragma unroll
        for (int v = 0; v < 4; ++v) P.template bring1<false, R != 2>(k, P.advance(pg), v, 0, ring0 + i % R * 4096);
    }
    template <int R> __device__ __forceinline__ void begin() const {
#pragma unroll
        for (int i = 0; i + 1 < R; ++i) issue<R>(i);
    }
    // Weights of nb blocks of staged rows, added to the wave's sums.
    template <int R>
    __device__ __forceinline__ void weigh(const u32x4* frag, const float4* row_of, int nb, float* sums) const {
        typedef Form<Coded<Q>> F;
        typedef MassForm<Q> M;
        const AttnArgs& a = P.a;
        for (int i = 0; i < U; ++i) {
            wait_lds();                                    // the tile before has been read
            issue<R>(i + R - 1);
            wait_loads<4 * (R - 1)>();
            if (__builtin_amdgcn_readlane(page, i) < 0) continue;
            const int32_t t0 = first + 128 * i;
            const uint8_t* kt = ring + i % R * 4096;
            const float sc_k = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scale), i));
            u32x4 kf[F::NF];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const u32x4 w = *reinterpret_cast<const u32x4*>(kt + (P.kaddr ^ (32u * j)));
                kf[2 * j] = decode8(uint2{w[0], w[1]}, sc_k);
                kf[2 * j + 1] = decode8(uint2{w[2], w[3]}, sc_k);
            }
            f32x16 sum;
#pragma unroll
            for (int k = 0; k < 16; ++k) sum[k] = 0.f;
            // bf16: a block's fragments are read while the exponentials of the block before are taken (as the compiler has it, they are
            // read where they are used, one after another: 1024 tokens over 16384 248 -> 235 us)
            u32x4 qf[F::NP][F::NF];
            float4 w;
            auto read = [&](int rb) {
#pragma unroll
                for (int p = 0; p < F::NP; ++p)
#pragma unroll
                    for (int k = 0; k < F::NF; ++k) qf[p][k] = frag[((rb * F::NP + p) * F::NF + k) * 64 + P.lane];
            };
            read(0);
            for (int rb = 0; rb < nb; ++rb) {
                w = row_of[rb * 32 + P.l32];
                f32x16 x;
#pragma unroll
                for (int k = 0; k < 16; ++k) x[k] = 0.f;
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int p = F::NP - 1; p >= 0; --p)
#pragma unroll
                    for (int k = 0; k < F::NF; ++k) x = mfma32(kf[k], qf[p][k], x);
                __builtin_amdgcn_sched_barrier(0);
                if (M::RB_MANY > 1) read(rb + 1 < nb ? rb + 1 : rb);
                __builtin_amdgcn_sched_barrier(0);
                const int32_t lo = __float_as_int(w.z), hi = __float_as_int(w.w);
#pragma unroll
                for (int k = 0; k < 16; ++k) x[k] = __builtin_amdgcn_exp2f(fmaf(x[k], a.c_lo, fmaf(x[k], a.c, -w.x)));
                if (__builtin_expect(__any(lo > t0 || hi < t0 + 32), 0)) {
                    const int32_t from = lo & ~LARGE;
                    const uint32_t at = (uint32_t)(t0 + 4 * P.h - from), n = (uint32_t)(hi - from);
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (at + 8 * (k >> 2) + (k & 3) >= n) x[k] = 0.f;
                    if (__builtin_expect(__any(lo & LARGE), 0)) {
                        const float most = 1.f / w.y;
#pragma unroll
                        for (int k = 0; k < 16; ++k) x[k] = paid_most(x[k], most);
                    }
                }
#pragma unroll
                for (int k = 0; k < 16; ++k) sum[k] = fmaf(x[k], w.y, sum[k]);
            }
            const float mine = sum_lanes(sum);
            const int k = P.l32 >> 1;
            if (!(P.l32 & 1)) sums[32 * i + 8 * (k >> 2) + 4 * P.h + (k & 3)] += mine;
        }
        wait_loads<0>();
        wait_lds();
    }
    // Up to 16 rows: products of 16 x 16, half of the work.  frag [NP][4][64]: lane 16 q + i has dims 16 (q + 4 j) + 8 b .. of row i in
    // number 2 j + b.
    template <int R>
    __device__ __forceinline__ void weigh16(const u32x4* frag, const float4* row_of, float* sums) const {
        typedef Form<Coded<Q>> F;
        const AttnArgs& a = P.a;
        const int i16 = P.lane & 15, q4 = P.lane >> 4;
        const uint32_t kaddr = (uint32_t)(i16 * F::ROWB + (q4 ^ P.swizzle(i16)) * 16);
        u32x4 qf[F::NP][4];
#pragma unroll
        for (int p = 0; p < F::NP; ++p)
#pragma unroll
            for (int k = 0; k < 4; ++k) qf[p][k] = frag[(p * 4 + k) * 64 + P.lane];
        const float4 w = row_of[i16];
        const int32_t lo = __float_as_int(w.z), hi = __float_as_int(w.w);
        for (int i = 0; i < U; ++i) {
            wait_lds();                                    // the tile before has been read
            issue<R>(i + R - 1);
            wait_loads<4 * (R - 1)>();
            if (__builtin_amdgcn_readlane(page, i) < 0) continue;
            const int32_t t0 = first + 128 * i;
            const uint8_t* kt = ring + i % R * 4096;
            const float sc_k = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scale), i));
            f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
            u32x4 kf[2][4];
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const u32x4 c = *reinterpret_cast<const u32x4*>(kt + 2048 * n + (kaddr ^ (64u * j)));
                    kf[n][2 * j] = decode8(uint2{c[0], c[1]}, sc_k);
                    kf[n][2 * j + 1] = decode8(uint2{c[2], c[3]}, sc_k);
                }
#pragma unroll
            for (int p = F::NP - 1; p >= 0; --p)
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int n = 0; n < 2; ++n) s[n] = mfma(kf[n][k], qf[p][k], s[n]);
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float y = s[k >> 2][k & 3];
                x[k] = __builtin_amdgcn_exp2f(fmaf(y, a.c_lo, fmaf(y, a.c, -w.x)));
            }
            if (__builtin_expect(__any(lo > t0 || hi < t0 + 32), 0)) {
                const int32_t from = lo & ~LARGE;
                const uint32_t at = (uint32_t)(t0 + 4 * q4 - from), n = (uint32_t)(hi - from);
                const float most = 1.f / w.y;
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = at + 16 * (k >> 2) + (k & 3) >= n ? 0.f : paid_most(x[k], most);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] *= w.y;
            const float mine = sum_lanes16(x);
            const int k = i16 >> 1;
            if (!(i16 & 1)) sums[32 * i + 16 * (k >> 2) + 4 * q4 + (k & 3)] += mine;
        }
        wait_loads<0>();
        wait_lds();
    }
};

template <typename Q>
__global__ __launch_bounds__(256, 2) void paged8_mass_kernel(MassArgs m) {
    typedef MassForm<Q> M;
    typedef Form<Coded<Q>> F;
    extern __shared__ __align__(1024) uint8_t smem[];
    const AttnArgs& a = m.a;
    const int lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5, wave = first_lane((int)(threadIdx.x >> 6));
    const int H = a.G * a.Hg;
    float* sums = reinterpret_cast<float*>(smem + M::LDS - M::SUMS) + wave * MOST_U * 32;
    float4* row_of = reinterpret_cast<float4*>(smem + M::LDS - M::SUMS - M::ROWS);   // what is subtracted, its rest as a factor, keys seen
    const SeqRange first = load_range(a, lane);
    // tiles a wave: as many as leave the card two workgroups a CU
    constexpr int ENOUGH = 8 * 2 * SLOTS;                  // (no sequence counts for more, so that 32 bits do)
    int32_t all = 0;
    float claimed = 0.f;                                   // rows, by all sequences together
    for (int s0 = 0; s0 < a.S; s0 += 64) {
        const SeqRange r = s0 ? load_range(a, s0 + lane) : first;
        const int32_t n = (m.keys(r) + 127) / 128;
        all += n < ENOUGH ? n : ENOUGH;
        claimed += (float)r.qlen;
    }
    for (int k = 1; k < (a.S < WAVE ? a.S : WAVE); k <<= 1) {
        all += __shfl_xor(all, k, WAVE);
        claimed += __shfl_xor(claimed, k, WAVE);
    }
    // More rows than there are (and more than rounding adds): starts fall, up to S / 2 times the work of any call.  Nothing is done.
    if (first_lane(claimed) > 1.01f * (float)a.T) return;
    all = first_lane(all);
    all = (all < ENOUGH ? all : ENOUGH) * a.G;
    const int U = all >= ENOUGH ? 8 : all >= 4 * 2 * SLOTS ? 4 : all >= 2 * 2 * SLOTS ? 2 : 1, per = 128 * U;
    Search from;
    for (int64_t u = blockIdx.x;; u += gridDim.x) {
        Found f;
        if (!find(a, first, u, from, f, [&](const SeqRange& r) { return (int64_t)((m.keys(r) + per - 1) / per) * a.G; })) return;
        f.r = SeqRange{first_lane(f.r.q0), first_lane(f.r.qlen), first_lane(f.r.klen)};
        f.s = first_lane(f.s);
        const SeqRange r = f.r;
        const int in = first_lane((int)(u - f.base)), g = in % a.G;
        const int32_t klen = m.keys(r), top = in / a.G * per, old = r.klen - r.qlen;
        const int64_t at = ((int64_t)f.s * a.G + g) * m.L;
        // the new tokens that see some of these keys, [i0, i1)
        const int32_t last = top + per < klen ? top + per - 1 : klen - 1;
        int32_t i0 = 0, i1 = r.qlen;
        if (a.causal && top > old) i0 = top - old;
        if (a.window && (int64_t)last + a.window - old < i1) i1 = last + a.window - old;
        const int64_t rows = (int64_t)r.qlen * a.Hg, end = i1 > i0 ? (int64_t)i1 * a.Hg : 0;
        int64_t c0 = (int64_t)i0 * a.Hg & ~(int64_t)31;
        const bool few = end - c0 <= 32, half = rows <= 16;
        Tiles<Q> T = {Piece<Coded<Q>>(a, f, g, 0, klen, lane), top + 32 * wave, -1, 1.f, U, 0, nullptr};
        T.ring = smem + (few ? M::FRAGS + wave * M::RING_FEW * F::KB : M::RB_MANY * M::FRAGS + wave * M::RING_MANY * F::KB);
        T.ring0 = first_lane((int)(uint32_t)(size_t)(__attribute__((address_space(3))) uint8_t*)T.ring);
        if (lane < U) {
            const int32_t t = T.first + 128 * lane;
            if (t < klen) T.page = T.P.page_of(T.P.raw_page(t), t);
            T.scale = T.P.scale_of(T.page, t, false);
        }
        // the sums begin with what older keys have been paid (asked for before the keys, used behind them)
        float paid[MOST_U / 2];
#pragma unroll
        for (int i = 0; i < MOST_U / 2; ++i) {
            const int32_t t = T.first + 128 * (2 * i + h) + l32;
            paid[i] = 2 * i + h < U && t < klen && t < old ? m.mass[at + t] : 0.f;
        }
        auto begin_sums = [&]() {
#pragma unroll
            for (int i = 0; i < MOST_U / 2; ++i)
                if (2 * i + h < U) sums[32 * (2 * i + h) + l32] = paid[i];
        };
        if (c0 >= end) begin_sums();
        bool begun = false;
        // The rows of a stage, a fourth of the dims a wave, and the sums of every fourth block's: asked for while the stage before is
        // used (1024 tokens over 1024: 134 -> 110 us; asked for behind the last tile's loads instead, they spill).
        u32x4 raw[M::RB_MANY][2][sizeof(Q) / 2];
        float lse[(M::RB_MANY + 3) / 4];
        auto row_at = [&](int64_t c, int rb, bool& real, int32_t& tok, int32_t& hd) {
            const int64_t mine = c + 32 * rb + l32;
            real = mine < rows;
            const uint32_t row = (uint32_t)(real ? mine : rows - 1);
            tok = (int32_t)(row / (uint32_t)a.Hg);
            hd = g * a.Hg + (int32_t)(row % (uint32_t)a.Hg);
        };
        auto ask = [&](int64_t c) {
#pragma unroll
            for (int rb = 0; rb < M::RB_MANY; ++rb) {
                if (c + 32 * rb >= end) break;
                bool real;
                int32_t tok, hd;
                row_at(c, rb, real, tok, hd);
                const Q* src = (const Q*)a.q + (int64_t)(r.q0 + tok) * a.q_stride + (int64_t)hd * D + 16 * (2 * wave + h);
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int e = 0; e < (int)sizeof(Q) / 2; ++e) raw[rb][k][e] = load16((const uint8_t*)(src + 8 * k) + 16 * e);
                if ((rb & 3) == wave) lse[rb >> 2] = m.lse[(int64_t)(r.q0 + tok) * H + hd];
            }
        };
        u32x4* frag = reinterpret_cast<u32x4*>(smem);      // [RB][NP][NF][64]
        if (!half && c0 < end) ask(c0);
        for (; c0 < end; c0 += 32 * M::RB_MANY) {
            const int nb = few ? 1 : end - c0 < 32 * M::RB_MANY ? (int)((end - c0 + 31) / 32) : M::RB_MANY;
            if (few) T.template begin<M::RING_FEW>();
            else T.template begin<M::RING_MANY>();
            auto put_row = [&](int rb, int l, bool real, int32_t tok, float z0) {
                const float2 z = subtracted(z0);
                int32_t lo, hi;
                row_keys(r, tok, a.causal, a.window, lo, hi);
                if (!real || hi < lo) lo = hi = 0;
                if (fabsf(z.x) >= 0x1p8f && z.x < INFINITY) lo |= LARGE;
                row_of[rb * 32 + l] = float4{z.x, z.y, __int_as_float(lo), __int_as_float(hi)};
            };
            if (half) {
                const int32_t mine = (lane & 15) < rows ? lane & 15 : 0, tok = mine / a.Hg, hd = g * a.Hg + mine % a.Hg;
                load_query16((const Q*)a.q + (int64_t)(r.q0 + tok) * a.q_stride + (int64_t)hd * D, lane >> 4, wave,
                             [&](int p, const u32x4& x) { frag[(p * 4 + wave) * 64 + lane] = x; });
                if (wave == 0 && lane < 16) put_row(0, lane, lane < rows, tok, m.lse[(int64_t)(r.q0 + tok) * H + hd]);
            } else {
#pragma unroll
                for (int rb = 0; rb < M::RB_MANY; ++rb) {
                    if (rb >= nb) break;
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        query_parts((const Q*)&raw[rb][k], [&](int p, const u32x4& x) {
                            frag[((rb * F::NP + p) * F::NF + 2 * wave + k) * 64 + lane] = x;
                        });
                    if ((rb & 3) != wave || h) continue;
                    bool real;
                    int32_t tok, hd;
                    row_at(c0, rb, real, tok, hd);
                    put_row(rb, l32, real, tok, lse[rb >> 2]);
                }
            }
            if (!begun) begin_sums();
            begun = true;
            __syncthreads();
            if (!half && c0 + 32 * M::RB_MANY < end) ask(c0 + 32 * M::RB_MANY);
            if (half) T.template weigh16<M::RING_FEW>(frag, row_of, sums);
            else if (few) T.template weigh<M::RING_FEW>(frag, row_of, nb, sums);
            else T.template weigh<M::RING_MANY>(frag, row_of, nb, sums);
            __syncthreads();                               // the rows have been read
        }
        for (int i = 0; i < U; i += 2) {
            const int32_t t = T.first + 128 * (i + h) + l32;
            if (i + h < U && t < klen) m.out[at + t] = sums[32 * (i + h) + l32];
        }
    }
}

template <typename Q>
hipError_t launch_mass(const MassArgs& m, hipStream_t st) {
    const AttnArgs& a = m.a;
    const void* fn = (const void*)paged8_mass_kernel<Q>;
    const hipError_t e = ensure_lds_limit(fn, MassForm<Q>::LDS);
    if (e != hipSuccess) return e;
    const int64_t units = ((a.cap < m.L ? a.cap : m.L) + 127) / 128 * a.G * a.S;
    paged8_mass_kernel<Q><<<(unsigned)(units < 2 * SLOTS ? units : 2 * SLOTS), 256, MassForm<Q>::LDS, st>>>(m);
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
