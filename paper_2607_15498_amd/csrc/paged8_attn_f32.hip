// Attention over pages of e4m3 codes: fp32 queries, 32 rows a wave and two waves a SIMD.  Three bf16 products a fragment and part
// instead of fp32's sixteen times slower ones: 1024 tokens over 16384 of 8 KV heads of 4 take 0.67 ms, 396 TFLOP/s, raw fp32 2.1 ms.
#include "paged8_attn.h"

namespace vr {

template <>
__device__ __forceinline__ void few_rows<Coded<float>>(const Piece<Coded<float>>& P, uint8_t* smem, int rows, bool cut, int64_t rec_row) {
    few_rows8<float>(P, smem, rows, cut, rec_row);
}
// Many rows, one step after another; two parts of the queries stay in registers, the third in shared memory behind the stages.
template <>
__device__ __forceinline__ void many_rows<Coded<float>>(const Piece<Coded<float>>& P, uint8_t* smem, int32_t row0, int32_t rows, bool cut,
                                                        int64_t rec_row) {
    typedef Form<Coded<float>> F;
    const AttnArgs& a = P.a;
    Many<Coded<float>> M(P, smem, row0, rows);
    if (M.stages) M.begin();
    Running run;
    u32x4 qf[2][F::NF];
    u32x4* low = reinterpret_cast<u32x4*>(smem + F::STAGES * 2 * F::SB) + M.wave * F::NF * 64;
    f32x16 acc[4];
    int32_t tok, head;
    M.row_of(0, P.l32, tok, head);
    P.query(qf, low, P.r.q0 + tok, head);
    const auto seen = M.keys_seen(0);
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[dt][i] = 0.f;
    const float slack = SLACK / a.c;
    for (int j = 0; j < F::SPS * M.stages; ++j) {
        if (j % F::SPS == 0) {
            M.arrive(j / F::SPS);
            M.issue(j / F::SPS + 2);
        }
        if (j < M.jf || j >= M.jl) continue;
        f32x16 sc;
        P.scores(M.keys_of(j), M.key_scale(j), qf, low, sc);
        const bool masked = M.masked(j);
        const int32_t t0 = M.t_first + 32 * j;
        if (masked) P.anew().mask(sc, t0, seen, M.gm_of(j));
        const float mt = P.most(sc);
        if (__any(mt > run.m + slack)) {
            const float f = run.raise(mt, a.c);
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[dt][i] *= f;
        }
        weights8<float>(sc, run, a, run.l);
        u32x4 p[3][2];
        parts_of(sc, p);
        const uint8_t* vt = M.values_of(j);
        const bool odd = masked && P.anew().odd_values(vt);
        P.values<3, Piece<Coded<float>>::ODD>(vt, M.value_scale(j), p, acc, odd);
        if (odd) P.anew().add_odd(vt, t0, seen, M.gm_of(j), [&](int dt, int i, float x) { acc[dt][i] += x; });
    }
    const float l = xsum32(run.l);
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) M.put(0, dt, acc[dt], run, l, cut, rec_row, dt == 3);
    M.finish();
}

hipError_t launch_paged8_f32(const AttnArgs& a, int groups, hipStream_t st) { return launch_paged<Coded<float>>(a, groups, st); }

}  // namespace vr
