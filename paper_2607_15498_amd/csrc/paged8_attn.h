// Attention over pages of e4m3 codes: what its bf16 and fp32 queries share.  paged_attn.h has the rest: the call's cut,
// masks, running sums, stages and the second launch.
//
// A code times its block's power of two is a bf16 number, so that keys and values are turned into bf16 fragments in
// registers without an error, the scale with the conversion, and everything behind that is the raw cache's.  fp32 queries
// and weights are three bf16 parts each (8 + 8 + 8 bits, cut off rather than rounded, so that the parts are exact), whose products
// the matrix cores sum in fp32.
//   The scaled products of codes themselves (f8f6f4), with queries in parts, take no conversions, but sum their 64 products to
//   about 12 bits only (errors up to 3e-4 of the sum of magnitudes, measured), too few for scores.
//
// A row is 128 bytes; row r's 16-byte piece c lies at place c ^ f(r), f(r) = bits 1, 3 and 2 of r as 2, 4 and 1: 16 rows'
// reads of one piece (keys) and 8 rows' of two (values, transposed 8 x 16 bytes at a time) fall into different banks.
#pragma once
#include "paged_agpr.h"

namespace vr {

// Nothing of the compiler's stays in a0 .. a191 across this.  (It may place what lives long in AGPRs, of which the bf16 kernel's
// many-rows form names these.)
template <typename Q> __device__ __forceinline__ void keep_out() {
    if constexpr (sizeof(Q) == 2) asm volatile("" ::: PA_AGPRS);
}

typedef int pa_i32x2 __attribute__((ext_vector_type(2)));

// 8 codes times scale, as a bf16 fragment
__device__ __forceinline__ u32x4 decode8(uint2 w, float scale) {
    u32x4 f;
    f[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w.x, scale, false));
    f[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w.x, scale, true));
    f[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w.y, scale, false));
    f[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w.y, scale, true));
    return f;
}
// the upper halves of two numbers, packed, and what they lack
__device__ __forceinline__ uint32_t cut2(float& a, float& b) {
    const uint32_t x = __float_as_uint(a) & 0xFFFF0000u, y = __float_as_uint(b) & 0xFFFF0000u;
    a -= __uint_as_float(x);
    b -= __uint_as_float(y);
    return x >> 16 | y;
}

// 8 dims of a row's query as a B operand, in parts; put(part, fragment)
template <typename Q, typename A>
__device__ __forceinline__ void query_parts(const Q* at, A&& put) {
    if constexpr (sizeof(Q) == 2) put(0, load16(at));
    else {
        float x[8];
        *reinterpret_cast<f32x4*>(x) = *reinterpret_cast<const f32x4*>(at);
        *reinterpret_cast<f32x4*>(x + 4) = *reinterpret_cast<const f32x4*>(at + 4);
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            u32x4 f;
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = cut2(x[2 * e], x[2 * e + 1]);
            put(p, f);
        }
    }
}
// A row's query (src): fragments 2 j and 2 j + 1 are dims 16 (2 j + h) .. of 8 each; put(part, k, fragment)
template <typename Q, typename A>
__device__ __forceinline__ void load_query(const Q* src, int h, int j, A&& put) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
        query_parts(src + 16 * (2 * j + h) + 8 * b, [&](int p, const u32x4& f) { put(p, 2 * j + b, f); });
}
// ... for products of 16 rows: fragment k = 2 j + b is dims 16 (q + 4 j) + 8 b ..; put(part, fragment)
template <typename Q, typename A>
__device__ __forceinline__ void load_query16(const Q* src, int q, int k, A&& put) {
    query_parts(src + 16 * (q + 4 * (k >> 1)) + 8 * (k & 1), put);
}

template <typename Q>
struct Piece<Coded<Q>> : PieceOf<Coded<Q>> {
    typedef Form<Coded<Q>> F;
    typedef PieceOf<Coded<Q>> P;
    using P::a;
    using P::g;
    using P::h;
    using P::l32;
    using P::lane;
    using P::r;
    using P::sees;
    using typename P::Seen;
    uint32_t off0, kaddr, vaddr;

    __device__ __forceinline__ Piece(const AttnArgs& a_, const Found& f, int g_, int32_t lo_, int32_t hi_, int lane_)
        : P(a_, f, g_, lo_, hi_, lane_) {
        const int lrow = lane >> 3;
        off0 = (uint32_t)(lrow * F::ROWB + ((lane & 7) ^ swizzle(lrow)) * 16);
        kaddr = (uint32_t)(l32 * F::ROWB + (h ^ swizzle(l32)) * 16);
        const int rr = (lane & 15) >> 1, row = 8 * (rr >> 2) + 4 * h + (rr & 3);
        vaddr = (uint32_t)(row * F::ROWB + (((lane >> 4) & 1) ^ swizzle(row)) * 16 + (lane & 1) * 8);
    }
    static __device__ __forceinline__ int swizzle(int row) { return (row & 2) | ((row >> 2) & 1) | ((row >> 1) & 4); }
    __device__ __forceinline__ Piece anew() const {
        Piece p = *this;
        asm volatile("" : "+v"(p.lane), "+v"(p.l32), "+v"(p.h));
        return p;
    }
    // the scale of the block of key t on page p (1 where there is none)
    __device__ __forceinline__ float scale_of(int32_t p, int32_t t, bool values) const {
        if (p < 0) return 1.f;
        const int sh = a.shift - 5;
        const uint8_t* at = values ? a.vscale : a.kscale;
        return __uint_as_float((uint32_t)at[(((int64_t)p * a.G + g) << sh) + ((t >> 5) & ((1 << sh) - 1))] << 23);
    }
    // 1 KB number v of the rows at src into LDS; row 0 of number 0 is row 4 `quad` of its block
    template <bool VALUES, bool ONCE = false>
    __device__ __forceinline__ void bring1(const uint8_t* src, int adv, int v, int quad, uint32_t dst) const {
        lds_load<ONCE>(src + v * adv, off0 ^ (((uint32_t)(quad >> 1) + v) & 1u) << 6, dst + v * 1024);
    }
    // values behind the end in the rows [r0, r1) of a tile of keys from t0 on: not read as data
    __device__ __forceinline__ void clear_tail(int32_t t0, int32_t r0, int32_t r1, uint8_t* vt) const {
        const int32_t end = r.klen - t0, from = end > r0 ? end : r0;
        for (int i = lane; i < (r1 - from) * F::PPR; i += 64)
            *reinterpret_cast<uint4*>(vt + from * F::ROWB + 16 * i) = uint4{0, 0, 0, 0};
    }
    // The third parts of fp32 queries lie in shared memory, [NF][64]: in registers they leave too few.
    static constexpr int HELD = F::NP == 1 ? 1 : 2;
    __device__ __forceinline__ void query(u32x4 (&qf)[HELD][F::NF], u32x4* low, int64_t token, int head) const {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            load_query((const Q*)a.q + token * a.q_stride + (int64_t)head * D, h, j, [&](int p, int k, const u32x4& f) {
                if (p < HELD) qf[p][k] = f;
                else low[k * 64 + lane] = f;
            });
    }
    // scores of 32 rows of fp32 with 32 keys of one scale
    __device__ __forceinline__ void scores(const uint8_t* kt, float scale, const u32x4 (&qf)[HELD][F::NF], const u32x4* low, f32x16& sc) const {
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(kt + (kaddr ^ (32u * j)));
            const u32x4 kf[2] = {decode8(uint2{w[0], w[1]}, scale), decode8(uint2{w[2], w[3]}, scale)};
#pragma unroll
            for (int k = 0; k < 2; ++k) sc = mfma32(kf[k], low[(2 * j + k) * 64 + lane], sc);
#pragma unroll
            for (int p = HELD - 1; p >= 0; --p)
#pragma unroll
                for (int k = 0; k < 2; ++k) sc = mfma32(kf[k], qf[p][2 * j + k], sc);
        }
    }
    // ... of any 32 rows, their fragments in shared memory, with NT blocks of keys side by side
    template <int NT>
    __device__ __forceinline__ void scores_of(const uint8_t* kt, const float (&scale)[NT], const u32x4* query, f32x16 (&sc)[NT]) const {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[n][i] = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u32x4 kf[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const u32x4 w = *reinterpret_cast<const u32x4*>(kt + n * F::KB + (kaddr ^ (32u * j)));
                kf[n][0] = decode8(uint2{w[0], w[1]}, scale[n]);
                kf[n][1] = decode8(uint2{w[2], w[3]}, scale[n]);
            }
#pragma unroll
            for (int p = F::NP - 1; p >= 0; --p)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const u32x4 q = query[(p * F::NF + 2 * j + k) * 64 + lane];
#pragma unroll
                    for (int n = 0; n < NT; ++n) sc[n] = mfma32(kf[n][k], q, sc[n]);
                }
        }
    }
    // codes of a V^T fragment: keys r0 + 4 h + 0..3 and r0 + 8 + 4 h + 0..3, dim 32 dt + l32
    __device__ __forceinline__ uint2 vcodes(const uint8_t* vt, int r0, int dt) const {
        return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
            (__attribute__((address_space(3))) pa_i32x2*)(vt + (vaddr ^ (32u * dt)) + r0 * F::ROWB)));
    }
    static __device__ __forceinline__ uint32_t finite(uint32_t x) { return Piece<uint16_t>::finite(x); }
    // acc += V^T P^T of 32 keys of one scale; p: the weights' parts, packed in pairs.  Of the values that are numbers alone: never,
    // always, or with `odd`.
    enum Finite { NEVER, ALWAYS, ODD };
    template <int WP, Finite FINITE>
    __device__ __forceinline__ void values(const uint8_t* vt, float scale, const u32x4 (&p)[WP][2], f32x16 (&acc)[4], bool odd = false) const {
#pragma unroll
        for (int mm = 0; mm < 2; ++mm)
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) {
                u32x4 f = decode8(vcodes(vt, 16 * mm, dt), scale);
                if constexpr (FINITE != NEVER)
                    if (FINITE == ALWAYS || odd)
#pragma unroll
                        for (int k = 0; k < 4; ++k) f[k] = finite(f[k]);
#pragma unroll
                for (int n = WP - 1; n >= 0; --n) acc[dt] = mfma32(f, p[n][mm], acc[dt]);
            }
    }
    // As the raw cache's: NaN (codes have no infinities) among values of keys that some row does not see.
    __device__ __forceinline__ bool odd_values(const uint8_t* vt) const {
        uint32_t odd = 0;
        for (int i = lane; i < F::KB / 16; i += 64) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(vt + 16 * i);
#pragma unroll
            for (int k = 0; k < 4; ++k) odd |= ((w[k] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
        }
        return __ballot(odd != 0) != 0;
    }
    // add(dt, i, x): x to the lane's sum of dim 32 dt + 8 (i / 4) + 4 h + i % 4
    template <typename A>
    __device__ __forceinline__ void add_odd(const uint8_t* vt, int32_t t0, Seen s, uint32_t gm, A&& add) const {
#pragma unroll 1
        for (int kk = 0; kk < 32; ++kk) {
            const bool see = sees(t0 + kk, s) && (gm >> (kk >> 4) & 1u);
#pragma unroll
            for (int n = 0; n < 16; ++n) {                 // four dims
                const int byte = 8 * n + 4 * h;
                const uint32_t w = *reinterpret_cast<const uint32_t*>(vt + kk * F::ROWB + (((byte >> 4) ^ swizzle(kk)) << 4) + (byte & 15));
#pragma unroll
                for (int k = 0; k < 4; ++k) add(n >> 2, 4 * (n & 3) + k, see && (w >> (8 * k) & 0x7Fu) == 0x7Fu ? NAN : 0.f);
            }
        }
    }
};

// A step's weights of a row, in place, and their sum (of the weights themselves, so that its logarithm is the row's).
template <typename Q>
__device__ __forceinline__ void weights8(f32x16& sc, const Running& run, const AttnArgs& a, float& l) {
    if (__any(beyond(run.off))) weights32(sc, l, [&](float x) { return run.weight_of(x, a.c, a.c_lo); });
    else if constexpr (sizeof(Q) == 2) weights32(sc, l, [&](float x) { return __builtin_amdgcn_exp2f(fmaf(x, a.c, run.off)); });
    else weights32(sc, l, [&](float x) { return weight32(x, a.c, a.c_lo, run.off); });
}
// As the value products take them: fp32 in three exact parts,
__device__ __forceinline__ void parts_of(f32x16& sc, u32x4 (&p)[3][2]) {
#pragma unroll
    for (int n = 0; n < 3; ++n)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float x = sc[2 * k], y = sc[2 * k + 1];
            p[n][k >> 2][k & 3] = cut2(x, y);
            sc[2 * k] = x;
            sc[2 * k + 1] = y;
        }
}
// bf16 rounded and what that takes away, rounded: 2^-17 of a weight is missing.
__device__ __forceinline__ void parts_of(f32x16& sc, u32x4 (&p)[2][2]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t w = p[0][k >> 2][k & 3] = cvt_bf16x2(sc[2 * k], sc[2 * k + 1]);
        p[1][k >> 2][k & 3] = cvt_bf16x2(sc[2 * k] - bf_lo(w), sc[2 * k + 1] - bf_hi(w));
    }
}

// Few rows: each wave takes every WAVES-th group of NT x 32 keys out of a ring of two of its own, and the waves' sums are joined
// at the end.  bf16, one wave a SIMD: two tiles at a time, whose products and exponentials do not wait for each other (one token
// over 131072 of 8 KV heads, tile by tile out of a ring of four: 72 us, what keys are more read at 4.9 TB/s; two at a time
// 66; with the queries in shared memory 60 - 62, 6.8 TB/s).
template <typename Q>
__device__ __forceinline__ void few_rows8(const Piece<Coded<Q>>& P, uint8_t* smem, int rows, bool cut, int64_t rec_row) {
    typedef Form<Coded<Q>> F;
    constexpr int NW = F::WAVES, NT = F::FEW_TILES, L = NT * F::KB / 1024, step = 32 * NT * NW, GROUP = 2 * NT * F::KB;
    const AttnArgs& a = P.a;
    const SeqRange& r = P.r;
    const int wave = first_lane((int)(threadIdx.x >> 6)), lane = P.lane, l32 = P.l32, h = P.h;
    const int Hg = a.Hg, g = P.g, lo = P.lo, hi = P.hi;
    uint8_t* ring = smem + wave * 2 * GROUP;
    const uint32_t ring0 = first_lane((int)(uint32_t)(size_t)(__attribute__((address_space(3))) uint8_t*)ring);
    // bf16: weights in two parts; up to 16 rows leave half of a product's columns to the second, the same rows again
    const bool halves = F::NP == 1 && rows <= 16;
    const int col = halves ? l32 & 15 : l32, myrow = col < rows ? col : 0, tok = myrow / Hg;
    const float rest = col < l32 ? -1.f : 0.f;
    int32_t mylo, myhi, firsthi, lastlo, x;
    row_keys(r, tok, a.causal, a.window, mylo, myhi);
    const auto seen = P.seen(mylo, myhi);
    row_keys(r, 0, a.causal, a.window, x, firsthi);
    row_keys(r, (rows - 1) / Hg, a.causal, a.window, lastlo, x);
    // the rows' fragments lie in shared memory, [NP][NF][64]: in registers they leave too few for two tiles
    const u32x4* query = reinterpret_cast<const u32x4*>(smem + NW * 2 * GROUP);
    if (wave < 4)
        load_query((const Q*)a.q + (int64_t)(r.q0 + tok) * a.q_stride + (int64_t)(g * Hg + myrow % Hg) * D, h, wave,
                   [&](int p, int k, const u32x4& f) { const_cast<u32x4*>(query)[(p * F::NF + k) * 64 + lane] = f; });
    Running run;
    const float slack = SLACK / a.c;
    f32x16 acc[4];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[dt][i] = 0.f;

    // pages and scales of the wave's next 32 tiles: lane 2 i has the page and the keys' scale of tile i, lane 2 i + 1 the values'
    constexpr int WINDOW = 32 / NT;                        // groups
    int32_t window = 0;
    float scales = 1.f;
    int at = WINDOW;
    int32_t page[NT];                                      // of the group that is on its way
    float ks[NT], vs[NT];
    auto issue = [&](int32_t t, int slot) {
        if (at == WINDOW) {
            const int32_t tl = t + (lane / (2 * NT)) * step + (lane / 2 % NT) * 32;
            window = tl < hi ? P.page_of(P.raw_page(tl), tl) : -1;
            scales = P.scale_of(window, tl, lane & 1);
            at = 0;
        }
        const uint32_t dst = ring0 + slot * GROUP;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int l = 2 * (NT * at + n);
            page[n] = __builtin_amdgcn_readlane(window, l);
            ks[n] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scales), l));
            vs[n] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scales), l + 1));
        }
        ++at;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const uint8_t* src = P.rows_at(kv ? P.vbase : P.kbase, page[n], t + 32 * n);
                const int adv = P.advance(page[n]);
#pragma unroll
                for (int i = 0; i < F::KB / 1024; ++i)
                    P.template bring1<false, true>(src, adv, i, 0, dst + (kv * NT + n) * F::KB + 0);
            }
    };
    int32_t t0 = (lo & ~(32 * NT - 1)) + 32 * NT * wave;
    if (t0 < hi) issue(t0, 0);
    __syncthreads();                                       // the queries are there
    for (int st = 0; t0 < hi; t0 += step, st ^= 1) {
        uint8_t* kt = ring + st * GROUP;
        uint8_t* vt = kt + NT * F::KB;
        int32_t pg[NT];
        float ksc[NT], vsc[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            pg[n] = page[n];
            ksc[n] = ks[n];
            vsc[n] = vs[n];
        }
        keep_out<Q>();
        wait_lds();                                        // the group before has been read
        issue(t0 + step, st ^ 1);                          // (behind the piece: zeros, so that the counts stay)
        bool masked = t0 < lastlo || t0 < lo || t0 + 32 * NT > firsthi || t0 + 32 * NT > hi;
#pragma unroll
        for (int n = 0; n < NT; ++n) masked = masked || pg[n] < 0;
        wait_loads<3 * L>();
        f32x16 sc[NT];
        P.template scores_of<NT>(kt, ksc, query, sc);
        keep_out<Q>();
        __builtin_amdgcn_sched_barrier(0);                 // (what lies between two of these fits the registers)
        if (masked)
#pragma unroll
            for (int n = 0; n < NT; ++n) P.anew().mask(sc[n], t0 + 32 * n, seen, pg[n] >= 0 ? 3u : 0u);
        float mt = P.most(sc[0]);
#pragma unroll
        for (int n = 1; n < NT; ++n) mt = fmaxf(mt, P.most(sc[n]));
        if (__any(mt > run.m + slack)) {
            const float f = run.raise(mt, a.c);
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[dt][i] *= f;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) weights8<Q>(sc[n], run, a, run.l);
        __builtin_amdgcn_sched_barrier(0);
        wait_loads<2 * L>();
        bool odd = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) P.clear_tail(t0 + 32 * n, 0, 32, vt + n * F::KB);
        if (masked)
#pragma unroll
            for (int n = 0; n < NT; ++n) odd = odd || P.anew().odd_values(vt + n * F::KB);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint8_t* v = vt + n * F::KB;
            keep_out<Q>();
            __builtin_amdgcn_sched_barrier(0);
            if (halves) {                                  // lanes 16 .. 31 (and 48 ..) have what the rounding takes away
                u32x4 p[1][2];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float e0 = sc[n][2 * k], e1 = sc[n][2 * k + 1];
                    const uint32_t w = cvt_bf16x2(e0, e1);
                    p[0][k >> 2][k & 3] = cvt_bf16x2(fmaf(rest, bf_lo(w), e0), fmaf(rest, bf_hi(w), e1));
                }
                if (odd) P.anew().template values<1, Piece<Coded<Q>>::ALWAYS>(v, vsc[n], p, acc);
                else P.template values<1, Piece<Coded<Q>>::NEVER>(v, vsc[n], p, acc);
            } else {
                constexpr int WP = F::NP == 1 ? 2 : 3;
                u32x4 p[WP][2];
                parts_of(sc[n], p);
                // fp32: one copy of the code, for whose two the registers do not do
                if constexpr (F::NP == 3) P.template values<WP, Piece<Coded<Q>>::ODD>(v, vsc[n], p, acc, odd);
                else if (odd) P.anew().template values<WP, Piece<Coded<Q>>::ALWAYS>(v, vsc[n], p, acc);
                else P.template values<WP, Piece<Coded<Q>>::NEVER>(v, vsc[n], p, acc);
            }
            if (odd)
                P.anew().add_odd(v, t0 + 32 * n, seen, pg[n] >= 0 ? 3u : 0u, [&](int dt, int i, float y) { acc[dt][i] += y; });
        }
    }
    wait_loads<0>();
    run.l = xsum32(run.l);
    __syncthreads();                                       // every wave is done with its ring
    float* js = (float*)smem;                              // [NW][32][132] sums
    float* jm = js + NW * 32 * 132;                        // [NW][32][2]
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<f32x4*>(js + (wave * 32 + l32) * 132 + 32 * dt + 2 * i + 4 * h) =
                f32x4{acc[dt][i], acc[dt][i + 1], acc[dt][i + 2], acc[dt][i + 3]};
    if (h == 0) *reinterpret_cast<float2*>(jm + (wave * 32 + l32) * 2) = float2{run.m, run.l};
    __syncthreads();
    // A thread's PER dims: of one of 32 rows, or half as many of one of 16 and of its rests
    constexpr int PER = 64 / NW;
    const int of_row = halves ? 2 * D / PER : D / PER, row = (int)threadIdx.x / of_row, own = halves ? PER / 2 : PER;
    const int d0 = (int)threadIdx.x % of_row * own;
    if (row < rows) {
        float mw[NW], lw[NW], M = -INFINITY, Ls = 0.f, o[PER];
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float2 v = *reinterpret_cast<const float2*>(jm + (w * 32 + row) * 2);
            mw[w] = v.x;
            lw[w] = v.y;
            M = fmaxf(M, v.x);
        }
        const float to = off_of(M, a.c);
#pragma unroll
        for (int i = 0; i < PER; ++i) o[i] = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = rescale(mw[w], M, to, a.c);
            Ls = fmaf(f, lw[w], Ls);
#pragma unroll
            for (int i = 0; i < PER; i += 4) {
                const int at4 = halves && i >= PER / 2 ? 16 * 132 + i - PER / 2 : i;
                const f32x4 v = *reinterpret_cast<const f32x4*>(js + (w * 32 + row) * 132 + d0 + at4);
#pragma unroll
                for (int k = 0; k < 4; ++k) o[i + k] = fmaf(f, v[k], o[i + k]);
            }
        }
        if (halves)                                        // (an infinite sum times a rest is no number)
#pragma unroll
            for (int i = 0; i < PER / 2; ++i) o[i] += fabsf(o[i]) < INFINITY ? o[i + PER / 2] : 0.f;
        if (cut) {
            float* dst = a.rec + (rec_row + row) * D + d0;
#pragma unroll
            for (int i = 0; i < PER; i += 4)
                if (i < own) *reinterpret_cast<f32x4*>(dst + i) = f32x4{o[i], o[i + 1], o[i + 2], o[i + 3]};
            if (d0 == 0) *reinterpret_cast<float2*>(a.rec + a.rec_rows * D + (rec_row + row) * 2) = float2{M, Ls};
        } else {
            const float inv = Ls == 0.f ? 0.f : 1.f / Ls;
            const int64_t token = r.q0 + row / Hg;
            const int head = g * Hg + row % Hg;
            Q* dst = (Q*)a.out + token * a.out_stride + (int64_t)head * D + d0;
#pragma unroll
            for (int i = 0; i < PER; i += 4)
                if (i < own) store4<Q>(dst + i, o[i] * inv, o[i + 1] * inv, o[i + 2] * inv, o[i + 3] * inv);
            if (a.lse && d0 == 0) a.lse[token * (a.G * Hg) + head] = lse_of<F::NP == 1>(M, Ls, a);
        }
    }
    __syncthreads();                                       // the rings are free again
}

hipError_t launch_paged8_bf16(const AttnArgs& a, int groups, hipStream_t st);
hipError_t launch_paged8_f32(const AttnArgs& a, int groups, hipStream_t st);

}  // namespace vr
