// The fp32 kernel of the paged attention (paged_attn.hip).  Its products take 16 times as long as bf16's, so its
// forms go one step after another, with two waves a SIMD: while one takes exponentials or waits for a fragment, the
// other's products run.  Many rows: 32 a wave.
#include "paged_attn.h"

namespace vr {

__device__ __forceinline__ f32x4 mfma16(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// Few rows: each of the 8 waves takes every eighth tile of 16 keys, keys and values 8 KB each of its own, and their
// sums are joined at the end.  Products of 16 x 16: up to 16 rows (NB = 1) cost half as much as 32, and then
// the matrix cores need 15 us of the 50 us that reading 32768 tokens of 8 heads takes.
//   S^T = K Q^T: lane 16 q + i gives dims 16 c + 4 q + e of key i and of row i, product e of every c;
//     receives keys 4 q + v of row i.
//   O^T = V^T P^T: lane gives dim 64 half + 4 i + e of key 4 q + v (values of 16 bytes, a row's adjacent) and the
//     weight that it holds; receives dims 64 half + 16 q + 4 v + e of row i.
template <int NB>
__device__ __forceinline__ void few_rows_of(const Piece<float>& P, uint8_t* smem, int rows, bool cut, int64_t rec_row) {
    constexpr int NW = Form<float>::WAVES, ROWB = 512, TB = 16 * ROWB;
    const AttnArgs& a = P.a;
    const SeqRange& r = P.r;
    const int wave = first_lane((int)(threadIdx.x >> 6)), lane = P.lane, i16 = lane & 15, q4 = lane >> 4;
    const int Hg = a.Hg, g = P.g, lo = P.lo, hi = P.hi;
    uint8_t* kt = smem + wave * 2 * TB;
    uint8_t* vt = kt + TB;
    const uint32_t kdst = first_lane((int)(uint32_t)(size_t)(__attribute__((address_space(3))) uint8_t*)kt);
    int32_t firsthi, lastlo, x;
    row_keys(r, 0, a.causal, a.window, x, firsthi);
    row_keys(r, (rows - 1) / Hg, a.causal, a.window, lastlo, x);
    typename Piece<float>::Seen seen[NB];
    u32x4 qf[NB][8];
    f32x4 acc[NB][2][4];
    Running run[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int row = 16 * b + i16 < rows ? 16 * b + i16 : 0, tok = row / Hg;
        int32_t rlo, rhi;
        row_keys(r, tok, a.causal, a.window, rlo, rhi);
        seen[b] = P.seen(rlo, rhi);
        const uint8_t* src = (const uint8_t*)((const float*)a.q + (int64_t)(r.q0 + tok) * a.q_stride + (int64_t)(g * Hg + row % Hg) * D);
#pragma unroll
        for (int c = 0; c < 8; ++c) qf[b][c] = load16(src + (4 * c + q4) * 16);
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[b][half][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const uint32_t kaddr = (uint32_t)(i16 * ROWB + (q4 ^ (((i16 & 3) << 2) | (i16 >> 2))) * 16);
    const float slack = SLACK / a.c;

    // pages of the wave's next 64 tiles, one a lane
    constexpr int L = TB / 1024, step = 16 * NW;
    int32_t window = 0, page = -1;
    int at = 64;
    auto fetch = [&](int32_t t) {
        if (at == 64) {
            const int32_t tl = t + lane * step;
            window = P.page_of(P.raw_page(tl), tl);
            at = 0;
        }
        page = __builtin_amdgcn_readlane(window, at++);
    };
    auto bring_keys = [&](int32_t t) {
        const uint8_t* src = P.rows_at(P.kbase, page, t);
#pragma unroll
        for (int v = 0; v < L; ++v) P.bring1<false, true>(src, P.advance(page), v, 0, kdst);
    };
    auto bring_values = [&](int32_t t) {
        const uint8_t* src = P.rows_at(P.vbase, page, t);
#pragma unroll
        for (int v = 0; v < L; ++v) lds_load<true>(src + v * P.advance(page), 16u * (uint32_t)lane, kdst + TB + v * 1024);
    };
    int32_t t0 = (lo & ~15) + 16 * wave;
    if (t0 < hi) {
        fetch(t0);
        bring_keys(t0);
        bring_values(t0);
    }
    for (; t0 < hi; t0 += step) {
        const bool paged = page >= 0, more = t0 + step < hi;
        const bool masked = t0 < lastlo || t0 < lo || t0 + 16 > firsthi || t0 + 16 > hi || !paged;
        wait_loads<L>();
        // several sums of 32 or 64 products: shorter chains round less (one token over 512: 1.3e-6 -> 3.4e-7 relative)
        constexpr int NS = NB == 1 ? 4 : 2;
        f32x4 sc[NB], part[NB][NS];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < NS; ++e) part[b][e] = f32x4{0.f, 0.f, 0.f, 0.f};
        auto kfrag = [&](int c) { return *reinterpret_cast<const u32x4*>(kt + (kaddr ^ (64u * (c & 3))) + 256 * (c >> 2)); };
        u32x4 kf[2] = {kfrag(0)};
#pragma unroll
        for (int c = 0; c < 8; ++c) {                      // the next fragment is read before the products of this one
            if (c < 7) kf[(c + 1) & 1] = kfrag(c + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    part[b][e % NS] = mfma16(__uint_as_float(kf[c & 1][e]), __uint_as_float(qf[b][c][e]), part[b][e % NS]);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                sc[b][v] = part[b][0][v] + part[b][1][v];
                if constexpr (NS == 4) sc[b][v] += part[b][2][v] + part[b][3][v];
            }
        wait_lds();                                        // the keys have been read
        if (more) {
            fetch(t0 + step);
            bring_keys(t0 + step);
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            if (masked)
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    if (!paged || !P.sees(t0 + 4 * q4 + v, seen[b])) sc[b][v] = -INFINITY;
            const float mt = fmaxf(fmaxf(sc[b][0], sc[b][1]), fmaxf(sc[b][2], sc[b][3]));
            if (__any(mt > run[b].m + slack)) {
                const float f = run[b].raise(xmax16(xmax32(mt)), a.c);
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int v = 0; v < 4; ++v) acc[b][half][e][v] *= f;
            }
            if (__any(beyond(run[b].off))) {
#pragma unroll
                for (int v = 0; v < 4; ++v) sc[b][v] = run[b].weight_of(sc[b][v], a.c, a.c_lo);
            } else {
#pragma unroll
                for (int v = 0; v < 4; ++v) sc[b][v] = weight32(sc[b][v], a.c, a.c_lo, run[b].off);
            }
            run[b].l += (sc[b][0] + sc[b][1]) + (sc[b][2] + sc[b][3]);
        }
        if (more) wait_loads<L>();
        else wait_loads<0>();
        P.clear_tail(t0, 0, 16, vt);
        bool odd = false;                                  // as Piece's: infinities and NaN among values of masked keys
        if (masked) {
            uint32_t bits = 0;
            for (int i = lane; i < TB / 16; i += 64) {
                const u32x4 w = *reinterpret_cast<const u32x4*>(vt + 16 * i);
#pragma unroll
                for (int k = 0; k < 4; ++k) bits |= w[k] ^ P.finite(w[k]);
            }
            odd = __any(bits != 0);
        }
        // four rows' fragments, the next before the products of these
        auto vfrag = [&](int n) { return *reinterpret_cast<const u32x4*>(vt + (4 * q4 + (n >> 1)) * ROWB + 256 * (n & 1) + 16 * i16); };
        u32x4 f[2] = {vfrag(0)};
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            if (n < 7) f[(n + 1) & 1] = vfrag(n + 1);
            __builtin_amdgcn_sched_barrier(0);
            if (odd)
#pragma unroll
                for (int e = 0; e < 4; ++e) f[n & 1][e] = P.finite(f[n & 1][e]);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    acc[b][n & 1][e] = mfma16(__uint_as_float(f[n & 1][e]), sc[b][n >> 1], acc[b][n & 1][e]);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (odd) {
#pragma unroll 1
            for (int kk = 0; kk < 16; ++kk)
#pragma unroll
                for (int n = 0; n < 8; ++n) {              // dims 64 (n / 4) + 16 q + 4 (n % 4) ..
                    const u32x4 w = *reinterpret_cast<const u32x4*>(vt + kk * ROWB + 256 * (n >> 2) + 64 * q4 + 16 * (n & 3));
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        const bool see = paged && P.sees(t0 + kk, seen[b]);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            acc[b][n >> 2][e][n & 3] += see ? __uint_as_float(w[e] ^ P.finite(w[e])) : 0.f;
                    }
                }
        }
        wait_lds();                                        // the values have been read
        if (more) bring_values(t0 + step);
    }

    float* js = (float*)smem;                              // [NW][16][132] sums
    float* jm = js + NW * 16 * 132;                        // [NW][16][2]
    static_assert(NW * 16 * 134 * 4 <= (int)Form<float>::LDS, "one block at a time");
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const float l = xsum16(xsum32(run[b].l));
        __syncthreads();                                   // every wave is done with what lies there
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                *reinterpret_cast<f32x4*>(js + (wave * 16 + i16) * 132 + 64 * half + 16 * q4 + 4 * v) =
                    f32x4{acc[b][half][0][v], acc[b][half][1][v], acc[b][half][2][v], acc[b][half][3][v]};
        if (q4 == 0) *reinterpret_cast<float2*>(jm + (wave * 16 + i16) * 2) = float2{run[b].m, l};
        __syncthreads();
        const int in = 2 * wave + (lane >> 5), row = 16 * b + in, d0 = 4 * (lane & 31);
        if (row < rows) {
            float M = -INFINITY, Ls = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
            float2 ml[NW];
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                ml[w] = *reinterpret_cast<const float2*>(jm + (w * 16 + in) * 2);
                M = fmaxf(M, ml[w].x);
            }
            const float to = off_of(M, a.c);
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float f = rescale(ml[w].x, M, to, a.c);
                const f32x4 v = *reinterpret_cast<const f32x4*>(js + (w * 16 + in) * 132 + d0);
                Ls = fmaf(f, ml[w].y, Ls);
#pragma unroll
                for (int k = 0; k < 4; ++k) o[k] = fmaf(f, v[k], o[k]);
            }
            if (cut) {
                *reinterpret_cast<f32x4*>(a.rec + (rec_row + row) * D + d0) = f32x4{o[0], o[1], o[2], o[3]};
                if (d0 == 0) *reinterpret_cast<float2*>(a.rec + a.rec_rows * D + (rec_row + row) * 2) = float2{M, Ls};
            } else {
                const float inv = Ls == 0.f ? 0.f : 1.f / Ls;
                float* dst = (float*)a.out + (int64_t)(r.q0 + row / Hg) * a.out_stride + (int64_t)(g * Hg + row % Hg) * D + d0;
                *reinterpret_cast<f32x4*>(dst) = f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
            }
        }
    }
    __syncthreads();                                       // the waves' tiles are free again
}
template <>
__device__ __forceinline__ void few_rows<float>(const Piece<float>& P, uint8_t* smem, int rows, bool cut, int64_t rec_row) {
    if (rows <= 16) few_rows_of<1>(P, smem, rows, cut, rec_row);
    else few_rows_of<2>(P, smem, rows, cut, rec_row);
}

template <>
__device__ __forceinline__ void many_rows<float>(const Piece<float>& P, uint8_t* smem, int32_t row0, int32_t rows, bool cut,
                                                 int64_t rec_row) {
    const AttnArgs& a = P.a;
    Many<float> M(P, smem, row0, rows);
    if (M.stages) M.begin();
    Running run;
    u32x4 qf[1][16];
    f32x16 acc[4];
    int32_t tok, head;
    M.row_of(0, P.l32, tok, head);
    P.query(qf[0], P.r.q0 + tok, head);
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int k = 0; k < 16; ++k) acc[dt][k] = 0.f;
    const auto seen = M.keys_seen(0);
    const float slack = SLACK / a.c;
    for (int j = 0; j < M.stages; ++j) {
        M.arrive(j);
        M.issue(j + 2);
        if (j < M.jf || j >= M.jl) continue;
        f32x16 sc[1];
        P.template scores<1>(M.keys_of(j), qf, sc);
        const bool masked = M.masked(j);
        const int32_t t0 = M.t_first + 32 * j;
        if (masked) P.anew().mask(sc[0], t0, seen, M.gm_of(j));
        const float mt = P.most(sc[0]);
        if (__any(mt > run.m + slack)) {
            const float f = run.raise(mt, a.c);
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                for (int k = 0; k < 16; ++k) acc[dt][k] *= f;
        }
        if (__any(beyond(run.off))) weights32(sc[0], run.l, [&](float x) { return run.weight_of(x, a.c, a.c_lo); });
        else weights32(sc[0], run.l, [&](float x) { return weight32(x, a.c, a.c_lo, run.off); });
        const uint8_t* vt = M.values_of(j);
        const bool odd = masked && P.anew().odd_values(vt);
        P.values(vt, sc[0], acc, odd);
        if (odd)
            P.anew().add_odd(vt, t0, seen, M.gm_of(j), [&](int dt, int i, float x) { acc[i & 3][4 * dt + (i >> 2)] += x; });
    }
    const float l = xsum32(run.l);
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) {
        f32x16 o;
#pragma unroll
        for (int i = 0; i < 16; ++i) o[i] = acc[i & 3][4 * dt + (i >> 2)];
        M.put(0, dt, o, run, l, cut, rec_row, dt == 3);
    }
    M.finish();
}

hipError_t launch_paged_f32(const AttnArgs& a, int groups, hipStream_t st) { return launch_paged<float>(a, groups, st); }

}  // namespace vr
