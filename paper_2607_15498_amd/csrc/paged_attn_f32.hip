// The fp32 kernel of the paged attention (paged_attn.hip), whose products take 16 times as long as bf16's: one
// step after another keeps the matrix cores busy.
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
    int32_t tok, head, mylo, myhi;
    M.row_of(0, P.l32, tok, head);
    M.keys_seen(0, P.l32, mylo, myhi);
    P.query(qf[0], P.r.q0 + tok, head);
    f32x16 acc[1][4];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int k = 0; k < 16; ++k) acc[0][dt][k] = 0.f;
    const float slack = SLACK / a.c;
    for (int j = 0; j < M.stages; ++j) {
        M.arrive(j);
        M.issue(j + 2);
        if (j < M.jf || j >= M.jl) continue;
        f32x16 sc[1];
        P.template scores<1>(M.keys_of(j), qf, sc);
        const bool masked = M.masked(j);
        if (masked) P.mask(sc[0], M.t_first + 32 * j, mylo, myhi, M.gm_of(j));
        const float mt = P.most(sc[0]);
        if (__any(mt > run.m + slack)) {
            const float f = run.raise(mt, a.c);
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                for (int k = 0; k < 16; ++k) acc[0][dt][k] *= f;
        }
        weights(sc[0], a.c, run.off, run.l);
        if (masked && P.odd_values(M.values_of(j)))
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
                P.values_by_key(M.values_of(j), sc[0], acc[0][dt], dt, M.t_first + 32 * j, mylo, myhi, M.gm_of(j));
        else P.template values<1>(M.values_of(j), sc, acc);
    }
    const float l = xsum32(run.l);
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) M.put(0, dt, acc[0][dt], run, l, cut, rec_row, dt == 3);
    M.finish();
}

hipError_t launch_paged_f32(const AttnArgs& a, int64_t units, int64_t pieces, hipStream_t st) { return launch_paged<float>(a, units, pieces, st); }

}  // namespace vr
