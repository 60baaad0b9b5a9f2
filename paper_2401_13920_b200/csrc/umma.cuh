// Pieces that the kernels on the 5th-generation tensor cores share: tile loads, matrix descriptors, commits, accumulator
// reads, and the GeLU of their epilogues.
#pragma once

#include <cuda.h>

#include "common.cuh"
#include "tensor_map.cuh"

namespace locmoe {

__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void mbar_arrive_n(uint64_t* bar, uint32_t n) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(n) : "memory");
}
// After a wait has been given up: asynchronous work this CTA started (bulk tensor loads that write its shared
// memory and count on its barriers, tcgen05.commit arrivals) may still be in flight, and a CTA must not leave
// while it is.  Nothing tells when the last of it has landed once the barriers' phases are out of step, so the
// CTA simply stays for a millisecond -- hundreds of times the latency of any such operation -- before it goes on
// to free its tensor memory.  Bounded, and only ever executed on the failure path.
__device__ __forceinline__ void quiesce_after_abort(volatile int* abort_word) {
    if (*abort_word) {
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
    }
}

__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int c0, int c1, int c2, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2)
                 : "memory");
}
__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
                 : "memory");
}
// Store of a box, tracked by the issuing thread's bulk async-group; what lies outside the tensor is left out.
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, const void* src, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
                 ::"l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(src)), "r"(c0), "r"(c1), "r"(c2) : "memory");
}

// Shared-memory matrix descriptor of a K-major bf16 tile with 128-byte swizzle: rows of 128 bytes, groups of
// 8 rows 1024 bytes apart (stride byte offset), leading byte offset unused (1), descriptor version 1.
__device__ __forceinline__ uint64_t umma_desc_sw128(uint32_t smem_addr) {
    return (uint64_t)((smem_addr & 0x3ffffu) >> 4) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) |
           (2ull << 61);
}
// Arrives on the mbarrier once all MMAs issued so far by this thread have completed.
__device__ __forceinline__ void umma_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// 32-byte store: one full sector per lane (rows of the output are far apart, so a warp store touches 32 sectors;
// writing each of them whole avoids partial-sector writes in L2).  Needs a 32-byte aligned address.
__device__ __forceinline__ void st_global_v8(void* p, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t a4,
                                             uint32_t a5, uint32_t a6, uint32_t a7) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(a0), "r"(a1), "r"(a2), "r"(a3),
                 "r"(a4), "r"(a5), "r"(a6), "r"(a7) : "memory");
}

__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t (&r)[16]) { tmem_ld16(taddr, r); }
__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t (&r)[32]) { tmem_ld32(taddr, r); }

// GeLU(v) = v * Phi(v) with Phi(v) = 1 - 0.5 erfc(v / sqrt 2).  erfc(x) = P(t) exp(-x^2), t = 1 / (1 + p x), for
// x >= 0 by the five-term rational approximation of Abramowitz & Stegun 7.1.26 (absolute error below 1.5e-7, which is
// less than the bf16 rounding of the result for v > -5); the negative side uses erfc(-x) = 2 - erfc(x) written so that a
// small Phi is not formed by cancellation.  The reciprocal and the exponential are the hardware approximations
// (rcp.approx, ex2.approx: a couple of ulps, far below the bf16 rounding of the result; 2.42 against 2.48 ms for the
// first GEMM of the 65536 x 2560 x 10240 case).  About a third of the instructions of erff().
// Two elements at a time with the two-wide fp32 instructions: the epilogue warps share their schedulers with
// the TMA and MMA warps, so fewer epilogue instructions directly mean fewer bubbles in the MMA stream.
__device__ __forceinline__ float rcp_approx(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float ex2_approx(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float2 gelu_erf2(float2 v) {
    const float2 x = __fmul2_rn(make_float2(fabsf(v.x), fabsf(v.y)), make_float2(0.70710678118654752f, 0.70710678118654752f));
    const float2 den = __ffma2_rn(make_float2(0.3275911f, 0.3275911f), x, make_float2(1.0f, 1.0f));
    const float2 t = make_float2(rcp_approx(den.x), rcp_approx(den.y));
    float2 poly = __ffma2_rn(make_float2(0.5307027145f, 0.5307027145f), t, make_float2(-0.7265760135f, -0.7265760135f));
    poly = __ffma2_rn(poly, t, make_float2(0.7107068705f, 0.7107068705f));
    poly = __ffma2_rn(poly, t, make_float2(-0.142248368f, -0.142248368f));
    poly = __ffma2_rn(poly, t, make_float2(0.127414796f, 0.127414796f));
    const float2 arg = __fmul2_rn(__fmul2_rn(x, x), make_float2(-1.4426950408889634f, -1.4426950408889634f));
    const float2 ex = make_float2(ex2_approx(arg.x), ex2_approx(arg.y));
    const float2 h = __fmul2_rn(__fmul2_rn(poly, t), ex);
    const float2 om = __ffma2_rn(h, make_float2(-1.0f, -1.0f), make_float2(1.0f, 1.0f));
    const float2 phi = make_float2(v.x < 0.0f ? h.x : om.x, v.y < 0.0f ? h.y : om.y);
    return __fmul2_rn(v, phi);
}
// The same for the products on sorted rows, with the digits kept far below zero: that formula's error is an absolute one, and
// Phi(-6) = 1e-9 comes out 0.7 % off, more than a rounding to bf16.  Here erfc(x) / 2 = t P(t) exp(-x^2), t = 1 / (1 + 0.33 x), P a
// polynomial of degree 7 fitted to the relative error for x up to 9.6 (weighted least squares, 8e-8), where the exponential leaves
// the normal numbers; what remains is the rounding of the exponential's argument.  `ex`: exp(-v^2 / 2).
__device__ __forceinline__ float2 normal_cdf2(float2 v, float2& ex) {
    const float2 x = __fmul2_rn(make_float2(fabsf(v.x), fabsf(v.y)), make_float2(0.70710678118654752f, 0.70710678118654752f));
    const float2 den = __ffma2_rn(make_float2(0.33f, 0.33f), x, make_float2(1.0f, 1.0f));
    const float2 t = make_float2(rcp_approx(den.x), rcp_approx(den.y));
    float2 poly = __ffma2_rn(make_float2(-0.067964375f, -0.067964375f), t, make_float2(0.23134398f, 0.23134398f));
    poly = __ffma2_rn(poly, t, make_float2(-0.17771928f, -0.17771928f));
    poly = __ffma2_rn(poly, t, make_float2(0.20627064f, 0.20627064f));
    poly = __ffma2_rn(poly, t, make_float2(0.022505404f, 0.022505404f));
    poly = __ffma2_rn(poly, t, make_float2(0.100961894f, 0.100961894f));
    poly = __ffma2_rn(poly, t, make_float2(0.09141863f, 0.09141863f));
    poly = __ffma2_rn(poly, t, make_float2(0.093183056f, 0.093183056f));
    const float2 arg = __fmul2_rn(__fmul2_rn(x, x), make_float2(-1.4426950408889634f, -1.4426950408889634f));
    ex = make_float2(ex2_approx(arg.x), ex2_approx(arg.y));
    const float2 h = __fmul2_rn(__fmul2_rn(poly, t), ex);
    const float2 om = __ffma2_rn(h, make_float2(-1.0f, -1.0f), make_float2(1.0f, 1.0f));
    return make_float2(v.x < 0.0f ? h.x : om.x, v.y < 0.0f ? h.y : om.y);
}
__device__ __forceinline__ float2 gelu2(float2 v) {
    float2 ex;
    return __fmul2_rn(v, normal_cdf2(v, ex));
}
// Its slope Phi(z) + z phi(z), phi(z) = exp(-z^2 / 2) / sqrt(2 pi): the exponential of erfc serves both terms.
__device__ __forceinline__ float2 gelu_slope2(float2 z) {
    float2 ex;
    const float2 phi = normal_cdf2(z, ex);
    return __ffma2_rn(__fmul2_rn(z, make_float2(0.39894228040143268f, 0.39894228040143268f)), ex, phi);
}

// SiLU(v) = v q, q = 1 / (1 + exp(-v)), and its slope q (1 + v (1 - q)), with the same two approximations.
__device__ __forceinline__ float sigmoid_approx(float v) { return rcp_approx(1.0f + ex2_approx(-1.4426950408889634f * v)); }
__device__ __forceinline__ float2 silu2(float2 v) { return __fmul2_rn(v, make_float2(sigmoid_approx(v.x), sigmoid_approx(v.y))); }
__device__ __forceinline__ float2 silu_slope2(float2 v) {
    const float2 q = make_float2(sigmoid_approx(v.x), sigmoid_approx(v.y));
    const float2 om = __ffma2_rn(q, make_float2(-1.0f, -1.0f), make_float2(1.0f, 1.0f));
    return __fmul2_rn(q, __ffma2_rn(v, om, make_float2(1.0f, 1.0f)));
}

}  // namespace locmoe
