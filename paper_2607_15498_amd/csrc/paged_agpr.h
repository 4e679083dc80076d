// Matrix products on registers named in inline assembly: the interleaved many-rows forms of the paged attention.
#pragma once
#include <type_traits>
#include <utility>

#include "paged_attn.h"

namespace vr {

// The many-rows form keeps its value sums and its queries in AGPRs named here, a[16 (4 c + dt)] .. (block c,
// dims 32 dt ..) and a[128 + 4 (8 c + k)] .. (fragment k): left to the compiler, the sums are moved between
// registers at every step.  The sources are compiled with their own products in VGPR form, and the compiler
// places nothing in an AGPR (tests/test_paged_host.py and test_paged8_host.py check the generated code).
#define PA_AGPRS \
    "a0", "a1", "a2", "a3", "a4", "a5", "a6", "a7", "a8", "a9", "a10", "a11", "a12", "a13", "a14", "a15", \
    "a16", "a17", "a18", "a19", "a20", "a21", "a22", "a23", "a24", "a25", "a26", "a27", "a28", "a29", "a30", "a31", \
    "a32", "a33", "a34", "a35", "a36", "a37", "a38", "a39", "a40", "a41", "a42", "a43", "a44", "a45", "a46", "a47", \
    "a48", "a49", "a50", "a51", "a52", "a53", "a54", "a55", "a56", "a57", "a58", "a59", "a60", "a61", "a62", "a63", \
    "a64", "a65", "a66", "a67", "a68", "a69", "a70", "a71", "a72", "a73", "a74", "a75", "a76", "a77", "a78", "a79", \
    "a80", "a81", "a82", "a83", "a84", "a85", "a86", "a87", "a88", "a89", "a90", "a91", "a92", "a93", "a94", "a95", \
    "a96", "a97", "a98", "a99", "a100", "a101", "a102", "a103", "a104", "a105", "a106", "a107", "a108", "a109", "a110", "a111", \
    "a112", "a113", "a114", "a115", "a116", "a117", "a118", "a119", "a120", "a121", "a122", "a123", "a124", "a125", "a126", "a127", \
    "a128", "a129", "a130", "a131", "a132", "a133", "a134", "a135", "a136", "a137", "a138", "a139", "a140", "a141", "a142", "a143", \
    "a144", "a145", "a146", "a147", "a148", "a149", "a150", "a151", "a152", "a153", "a154", "a155", "a156", "a157", "a158", "a159", \
    "a160", "a161", "a162", "a163", "a164", "a165", "a166", "a167", "a168", "a169", "a170", "a171", "a172", "a173", "a174", "a175", \
    "a176", "a177", "a178", "a179", "a180", "a181", "a182", "a183", "a184", "a185", "a186", "a187", "a188", "a189", "a190", "a191"
constexpr int QBASE = 128;

template <int N, typename F, int... I>
__device__ __forceinline__ void static_for_impl(F&& f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>()), ...);
}
template <int N, typename F> __device__ __forceinline__ void static_for(F&& f) {
    static_for_impl<N>(f, std::make_integer_sequence<int, N>());
}
template <int A> __device__ __forceinline__ void agpr_set(uint32_t x) {
    asm volatile("v_accvgpr_write_b32 a[%1], %0" ::"v"(x), "n"(A));
}
template <int A> __device__ __forceinline__ float agpr_get() {
    float x;
    asm volatile("v_accvgpr_read_b32 %0, a[%1]" : "=v"(x) : "n"(A));
    return x;
}
// 19 wait states between the last product into a register and its use by anything else, and 4 before the next
__device__ __forceinline__ void settle() { asm volatile("s_nop 15\n\ts_nop 3" ::: PA_AGPRS); }
// A product may not follow within 2 wait states the vector instruction that wrote one of its operands: they come
// from LDS or from an iteration before (the test of the generated code looks for that).
// s += K Q^T of fragment K, block C; K = 0 starts it
template <int K, int C> __device__ __forceinline__ void score(f32x16& s, const u32x4& f) {
    constexpr int q = QBASE + 4 * (8 * C + K);
    if constexpr (K == 0)
        asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, a[%2:%3], 0" : "=&v"(s) : "v"(f), "n"(q), "n"(q + 3) : PA_AGPRS);
    else
        asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, a[%2:%3], %0" : "+v"(s) : "v"(f), "n"(q), "n"(q + 3) : PA_AGPRS);
}
// sums of block C, dims 32 DT .. += V^T P^T
template <int DT, int C> __device__ __forceinline__ void value(const u32x4& f, const u32x4& p) {
    constexpr int o = 16 * (4 * C + DT);
    asm volatile("v_mfma_f32_32x32x16_bf16 a[%2:%3], %0, %1, a[%2:%3]" ::"v"(f), "v"(p), "n"(o), "n"(o + 15) : PA_AGPRS);
}

}  // namespace vr
