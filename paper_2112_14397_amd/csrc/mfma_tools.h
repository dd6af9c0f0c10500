// What the matrix-core kernels of the expert FFNs share: direct global -> LDS loads and their waits, descriptors for stores and
// loads that end where a tile does, and the fast gelu.  Internal to the library.
#pragma once
#include "common.h"

namespace evomoe {

// gelu(h) = max(h, -4.2) Phi(hc), Phi(hc) = 0.5 + hc Q(hc^2), hc = h clamped to |h| <= 4.2: degree-8 minimax fit of Q, |error of Phi| <
// 1.2e-5 -- below the resolution of the bf16 values it is multiplied into -- and no transcendental; 13 VALU instructions, which GEMM1's
// epilogue is bound by.  Beyond the fitted range the values stay within 2.5e-4 of the true ones for any h: -> h for large h (Phi(4.2) =
// 1 - 1.3e-5), -> -4.2 * 1.3e-5 for very negative ones.  (As max(h, 0) - |h| 2^p(|h|) GEMM1 of 58 330 pairs, d = 768 takes 322 us with p
// of degree four, whose errors are larger in places, and 326 with degree five, whose errors are smaller everywhere, 9.6e-7 at most,
// instead of 336; either rounds other values of A up or down, and with degree five dx at 16 223 pairs had an element at 1.37 times the
// comparison's bound, where 1.35 is allowed for.)
__device__ __forceinline__ float act_fwd_fast(float h, int act) {
    if (act == EVOMOE_RELU) return relu(h);
    const float hc = __builtin_amdgcn_fmed3f(h, -4.2f, 4.2f), u = hc * hc;
    float q = 5.998071484e-11f;
    q = fmaf(q, u, -5.633320033e-09f);
    q = fmaf(q, u, 2.343674907e-07f);
    q = fmaf(q, u, -5.760770819e-06f);
    q = fmaf(q, u, 9.457441047e-05f);
    q = fmaf(q, u, -1.114148065e-03f);
    q = fmaf(q, u, 9.830130264e-03f);
    q = fmaf(q, u, -6.636036932e-02f);
    q = fmaf(q, u, 3.989074528e-01f);
    asm("v_fmaak_f32 %0, %1, %2, 0x3f000000" : "=v"(q) : "v"(hc), "v"(q));     // 0.5 as a literal: half the time of v_fma_f32
    return __builtin_elementwise_maximum(h, -4.2f) * q;      // (a NaN stays one)
}
// 16 bytes per lane, global -> LDS, no registers in between: lane l's data lands at lds + 16*l.
// Written as inline assembly on purpose: the compiler cannot tell which LDS stage a load fills, so with
// its own intrinsic it guards every later LDS read (and every barrier) with s_waitcnt vmcnt(0), which
// serialises the prefetch pipeline.  Here the kernel counts its loads itself (wait_vmcnt below).
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}
// A buffer descriptor of what exists of a tile's rows: lanes beyond it load 0 and store nothing, without a branch around the access.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const void* base, int bytes) {
    const uint64_t b = (uint64_t)(uintptr_t)base;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)b), hi = __builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
    return __builtin_amdgcn_make_buffer_rsrc((void*)(uintptr_t)((uint64_t)hi << 32 | lo), 0,
                                             __builtin_amdgcn_readfirstlane(bytes), 0x27000);
}
// The global address is a wave-uniform base (an SGPR pair) plus a 32-bit unsigned byte offset per lane.
__device__ __forceinline__ void load_to_lds(const unsigned char* base, uint32_t voff, const unsigned char* lds_wave_base) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                 :: "v"(voff), "s"(base), "s"(lds_addr(lds_wave_base)) : "m0", "memory");
}
// 4 bytes per lane in the same way: lane l's data lands at lds + 4*l.
__device__ __forceinline__ void load_dword_to_lds(const int32_t* base, uint32_t voff, const int* lds_wave_base) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1"
                 :: "v"(voff), "s"(base), "s"(lds_addr(lds_wave_base)) : "m0", "memory");
}
// Block barrier that orders LDS traffic only (global loads in flight stay in flight).
__device__ __forceinline__ void block_sync_lds() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
// s_waitcnt vmcnt(n) only (other counters left at their maxima)
template <int N> __device__ __forceinline__ void wait_vmcnt() {
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory");
}

}  // namespace evomoe
