// Attention over pages of e4m3 codes: fp32 queries, 32 rows a wave and two waves a SIMD.  Three bf16 products a fragment and part
// instead of fp32's sixteen times slower ones: 1024 tokens over 16384 of 8 KV heads of 4 take 0.80 ms, 334 TFLOP/s, raw fp32 2.1 ms.
#include "paged8_attn.h"

namespace vr {

template <>
__device__ __forceinline__ void few_rows<Coded<float>>(const Piece<Coded<float>>& P, uint8_t* smem, int rows, bool cut, int64_t rec_row) {
    few_rows8<float>(P, smem, rows, cut, rec_row);
}
template <>
__device__ __forceinline__ void many_rows<Coded<float>>(const Piece<Coded<float>>& P, uint8_t* smem, int32_t row0, int32_t rows, bool cut,
                                                        int64_t rec_row) {
    many_rows8<float>(P, smem, row0, rows, cut, rec_row);
}

hipError_t launch_paged8_f32(const AttnArgs& a, int groups, hipStream_t st) { return launch_paged<Coded<float>>(a, groups, st); }

}  // namespace vr
