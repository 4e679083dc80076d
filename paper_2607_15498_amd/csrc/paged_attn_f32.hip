// The fp32 kernel of the paged attention (paged_attn.hip).  Its products take 16 times as long as bf16's, so its
// many-rows form goes one step after another, 32 rows a wave and two waves a SIMD: while one takes exponentials
// or waits for a fragment, the other's products run.
#include "paged_attn.h"

namespace vr {

template <>
__device__ __forceinline__ void many_rows<float>(const Piece<float>& P, uint8_t* smem, int32_t row0, int32_t rows, bool cut,
                                                 int64_t rec_row) {
    const AttnArgs& a = P.a;
    Many<float> M(P, smem, row0, rows);
    if (M.stages) M.begin();
    Running run;
    u32x4 qf[1][16];
    f32x16 acc[1][4];
    int32_t tok, head;
    M.row_of(0, P.l32, tok, head);
    P.query(qf[0], P.r.q0 + tok, head);
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int k = 0; k < 16; ++k) acc[0][dt][k] = 0.f;
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
                for (int k = 0; k < 16; ++k) acc[0][dt][k] *= f;
        }
        weights(sc[0], a.c, run.off, run.l);
        const uint8_t* vt = M.values_of(j);
        if (masked && P.anew().odd_values(vt)) {
            const Piece<float> A = P.anew();
            A.template values<1, true>(vt, sc, acc);
            A.add_odd(vt, t0, seen, M.gm_of(j), [&](int dt, int i, float x) { acc[0][dt][i] += x; });
        } else P.template values<1>(vt, sc, acc);
    }
    const float l = xsum32(run.l);
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) M.put(0, dt, acc[0][dt], run, l, cut, rec_row, dt == 3);
    M.finish();
}

hipError_t launch_paged_f32(const AttnArgs& a, int64_t pieces, hipStream_t st) { return launch_paged<float>(a, pieces, st); }

}  // namespace vr
