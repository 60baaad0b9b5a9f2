// Expert FFN of the MoE layer (first equation of Sec. 3.2.1):
//   y = W_out . GeLU(W_in . x)   per expert, GeLU(v) = v * Phi(v) (exact erf form),
// on the dispatched buffer in RECV layout, where the rows of one expert are contiguous.
//
// Two grouped GEMMs (all experts in one launch each), both "NT": the activations [rows][K] and the
// weights [E][N][K] are K-major, so both operands are loaded as 128-byte-swizzled K-major tiles.
//   - TMA (cp.async.bulk.tensor, each load into the issuing CTA only) fills a 4-stage ring of 128x64 (A) and 256x64 (B) bf16 tiles,
//   - one elected thread issues tcgen05.mma (128 x 256 x 16 per instruction, fp32 accumulators in TMEM),
//   - two 128x256 accumulators (512 TMEM columns) alternate, so the epilogue of a tile overlaps the MMAs
//     of the next one,
//   - eight epilogue warps read the accumulator with tcgen05.ld (one row per thread, half of the columns per
//     warp), apply GeLU (first GEMM), convert and store.
// Warp roles: warp 0 = TMA producer, warp 1 = MMA issuer, warps 2..9 = epilogue.  Persistent CTAs, one per SM.
// Three kernels share these pieces: ffn_gemm_kernel (one CTA per 128 x 256 tile, as described above),
// ffn_gemm_wide_kernel (one CTA per 256 x 256 tile, both accumulators on it; chosen for long reductions) and
// ffn_gemm2_kernel (a cluster of two CTAs per 256 x 256 tile, tcgen05 cta_group::2; opt-in); the latter two are
// described where they are defined, the choice between them at plan_expert_ffn.
// Every barrier wait is bounded; on a timeout the kernel raises the device diagnostics flag, leaves its
// loops, frees its TMEM and returns.
#include <cuda.h>
#include <math.h>
#include <stdlib.h>

#include <mutex>

#include "common.cuh"
#include "tensor_map.cuh"

namespace locmoe {

namespace {

constexpr int BM = 128, BN = 256, BK = 64, NSTAGE = 4;
constexpr int UMMA_K = 16;
constexpr uint32_t A_BYTES = BM * BK * 2, B_BYTES = BN * BK * 2, STAGE_BYTES = A_BYTES + B_BYTES;
constexpr int kEpiWarps = 8;                       // two warps per TMEM lane quadrant, each takes half of the columns
constexpr int kFfnThreads = 64 + 32 * kEpiWarps;
constexpr uint32_t TMEM_COLS = 512;
constexpr size_t kFfnSmem = (size_t)NSTAGE * STAGE_BYTES + 1024 /*alignment slack*/ + 256 /*barriers*/;

__device__ int g_ffn_flags = 0;  // bit 0: a bounded wait gave up

struct FfnArgs {
    void* out;            // [E * M][N] bf16 or fp32
    int out_f32;          // 0: bf16, 1: fp32
    int gelu;             // apply GeLU in the epilogue
    int E, M, N, K;       // experts, rows per expert, output columns, reduction length
    int m_tiles, n_tiles;
    int split_from;       // wide kernel: tiles from this index on are worked on as two half tiles (see there)
};

__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// Bounded wait that also gives up as soon as another role has raised the abort word.
__device__ __forceinline__ bool wait_or_abort(uint64_t* bar, uint32_t parity, volatile int* abort_word) {
    for (uint32_t i = 0; i < (1u << 22); ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 63u) == 63u && *abort_word) return false;
    }
    *abort_word = 1;
    atomicOr(&g_ffn_flags, 1);
    return false;
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

// Shared-memory matrix descriptor of a K-major bf16 tile with 128-byte swizzle: rows of 128 bytes, groups of
// 8 rows 1024 bytes apart (stride byte offset), leading byte offset unused (1), descriptor version 1.
__device__ __forceinline__ uint64_t umma_desc_sw128(uint32_t smem_addr) {
    return (uint64_t)((smem_addr & 0x3ffffu) >> 4) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) |
           (2ull << 61);
}
// Instruction descriptor: bf16 x bf16 -> fp32, both operands K-major, M = 128, N = 256.
constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(BM >> 4) << 24);

__device__ __forceinline__ void umma_bf16(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(kIdesc), "r"(accumulate) : "memory");
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

// GeLU(v) = v * Phi(v) with Phi(v) = 1 - 0.5 erfc(v / sqrt 2).  erfc(x) = P(t) exp(-x^2), t = 1 / (1 + p x), for
// x >= 0 by the five-term rational approximation of Abramowitz & Stegun 7.1.26 (absolute error below 1.5e-7,
// far under the bf16 rounding of the result); the negative side uses erfc(-x) = 2 - erfc(x) written so that a
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
// Stores 32 consecutive columns of one output row (converted to the output type); static indexing keeps v[] in
// registers.
__device__ __forceinline__ void store_block32(const FfnArgs& a, long long grow, int col0, const float (&v)[32], bool wide_ok) {
    if (col0 + 32 <= a.N && wide_ok) {
        if (a.out_f32) {
            float* dst = static_cast<float*>(a.out) + grow * a.N + col0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                st_global_v8(dst + 8 * i, __float_as_uint(v[8 * i]), __float_as_uint(v[8 * i + 1]),
                             __float_as_uint(v[8 * i + 2]), __float_as_uint(v[8 * i + 3]),
                             __float_as_uint(v[8 * i + 4]), __float_as_uint(v[8 * i + 5]),
                             __float_as_uint(v[8 * i + 6]), __float_as_uint(v[8 * i + 7]));
        } else {
            uint16_t* dst = static_cast<uint16_t*>(a.out) + grow * a.N + col0;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                st_global_v8(dst + 16 * i, cvt_bf16x2(make_float2(v[16 * i], v[16 * i + 1])),
                             cvt_bf16x2(make_float2(v[16 * i + 2], v[16 * i + 3])),
                             cvt_bf16x2(make_float2(v[16 * i + 4], v[16 * i + 5])),
                             cvt_bf16x2(make_float2(v[16 * i + 6], v[16 * i + 7])),
                             cvt_bf16x2(make_float2(v[16 * i + 8], v[16 * i + 9])),
                             cvt_bf16x2(make_float2(v[16 * i + 10], v[16 * i + 11])),
                             cvt_bf16x2(make_float2(v[16 * i + 12], v[16 * i + 13])),
                             cvt_bf16x2(make_float2(v[16 * i + 14], v[16 * i + 15])));
        }
    } else {  // ragged or unaligned column block
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            if (col0 + i < a.N) {
                if (a.out_f32) static_cast<float*>(a.out)[grow * a.N + col0 + i] = v[i];
                else static_cast<uint16_t*>(a.out)[grow * a.N + col0 + i] = (uint16_t)f32_to_bf16_bits(v[i]);
            }
        }
    }
}

// Epilogue of one warp on one accumulator: column blocks [c_begin, c_end) of 32 columns each, one row per lane
// (TMEM lane = row).  taddr = the accumulator's TMEM address at this warp's lane quadrant, column 0.
__device__ __forceinline__ void drain_columns(const FfnArgs& a, uint32_t taddr, long long grow, bool row_ok, int n0,
                                              int c_begin, int c_end, bool wide_ok) {
#pragma unroll 1
    for (int c = c_begin; c < c_end; ++c) {
        __syncwarp();  // tcgen05.ld is warp-collective: reconverge after the masked stores
        uint32_t r[32];
        tmem_ld32(taddr + (uint32_t)(c * 32), r);
        const int col0 = n0 + c * 32;
        if (!row_ok || col0 >= a.N) continue;
        float v[32];
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            float2 pr = make_float2(__uint_as_float(r[i]), __uint_as_float(r[i + 1]));
            if (a.gelu) pr = gelu_erf2(pr);
            v[i] = pr.x; v[i + 1] = pr.y;
        }
        store_block32(a, grow, col0, v, wide_ok);
    }
}

__global__ void __launch_bounds__(kFfnThreads, 1)
ffn_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const FfnArgs a) {
    extern __shared__ unsigned char smraw[];
    // 1024-byte alignment: the 128-byte swizzle pattern repeats every 8 rows of 128 bytes
    unsigned char* base = reinterpret_cast<unsigned char*>(((uintptr_t)smraw + 1023) & ~(uintptr_t)1023);
    uint64_t* bars = reinterpret_cast<uint64_t*>(base + (size_t)NSTAGE * STAGE_BYTES);
    uint64_t* full = bars;                 // [NSTAGE] tile landed in shared memory
    uint64_t* empty = bars + NSTAGE;       // [NSTAGE] MMAs that read the stage are done
    uint64_t* acc_full = bars + 2 * NSTAGE;  // [2] accumulator complete
    uint64_t* acc_empty = acc_full + 2;      // [2] accumulator drained by the epilogue
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
    volatile int* abort_word = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < NSTAGE; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], kEpiWarps); }
        *abort_word = 0;
        mbar_init_fence();
    }
    if (warp == 2) {  // one warp allocates all 512 TMEM columns (one CTA per SM, so this cannot starve)
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    const int tiles_per_expert = a.m_tiles * a.n_tiles;
    const int total_tiles = a.E * tiles_per_expert;
    const int kblocks = (a.K + BK - 1) / BK;

    if (warp == 0) {
        if (lane == 0) {  // ---- TMA producer ----
            int stage = 0; uint32_t phase = 0;
            for (int tile = blockIdx.x; tile < total_tiles; tile += gridDim.x) {
                const int e = tile / tiles_per_expert, rem = tile - e * tiles_per_expert;
                const int nt = rem / a.m_tiles, mt = rem - nt * a.m_tiles;
                const int row0 = e * a.M + mt * BM, n0 = nt * BN;
                bool ok = true;
                for (int kb = 0; kb < kblocks && ok; ++kb) {
                    if (!wait_or_abort(&empty[stage], phase ^ 1u, abort_word)) { ok = false; break; }
                    unsigned char* sa = base + (size_t)stage * STAGE_BYTES;
                    mbar_expect_tx(&full[stage], STAGE_BYTES);
                    tma_load_2d(sa, &tmA, kb * BK, row0, &full[stage]);
                    tma_load_3d(sa + A_BYTES, &tmB, kb * BK, n0, e, &full[stage]);
                    if (++stage == NSTAGE) { stage = 0; phase ^= 1u; }
                }
                if (!ok) break;
            }
            // tail: all asynchronous commits to this CTA's stage barriers have arrived before the CTA leaves
            for (int i = 0; i < NSTAGE; ++i) {
                if (!wait_or_abort(&empty[stage], phase ^ 1u, abort_word)) break;
                if (++stage == NSTAGE) { stage = 0; phase ^= 1u; }
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {  // ---- MMA issuer ----
            int stage = 0; uint32_t phase = 0;
            int acc = 0; uint32_t acc_phase = 0;
            for (int tile = blockIdx.x; tile < total_tiles; tile += gridDim.x) {
                if (!wait_or_abort(&acc_empty[acc], acc_phase ^ 1u, abort_word)) break;
                tc_fence_after();
                const uint32_t tmem_d = tmem_base + (uint32_t)acc * BN;
                bool ok = true;
                for (int kb = 0; kb < kblocks; ++kb) {
                    if (!wait_or_abort(&full[stage], phase, abort_word)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t sa = smem_u32(base + (size_t)stage * STAGE_BYTES);
                    const uint32_t sb = sa + A_BYTES;
#pragma unroll
                    for (int k = 0; k < BK / UMMA_K; ++k)
                        umma_bf16(tmem_d, umma_desc_sw128(sa + k * UMMA_K * 2), umma_desc_sw128(sb + k * UMMA_K * 2),
                                  (kb > 0 || k > 0) ? 1u : 0u);
                    umma_commit(&empty[stage]);
                    if (++stage == NSTAGE) { stage = 0; phase ^= 1u; }
                }
                if (!ok) break;
                umma_commit(&acc_full[acc]);
                if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
            }
        }
    } else {  // ---- epilogue warps 2..9: TMEM lane quadrant = warp % 4, column half = (warp - 2) / 4 ----
        const int q = warp & 3;
        const int half = (warp - 2) >> 2;
        int acc = 0; uint32_t acc_phase = 0;
        for (int tile = blockIdx.x; tile < total_tiles; tile += gridDim.x) {
            const int e = tile / tiles_per_expert, rem = tile - e * tiles_per_expert;
            const int nt = rem / a.m_tiles, mt = rem - nt * a.m_tiles;
            if (!wait_or_abort(&acc_full[acc], acc_phase, abort_word)) break;   // the whole warp polls: one lane polling
                                                                                // alone spins 2.5 times as often
            tc_fence_after();
            const int r_in = mt * BM + q * 32 + lane;        // row inside the expert's block
            const bool row_ok = r_in < a.M;
            const long long grow = (long long)e * a.M + r_in;
            const int n0 = nt * BN;
            const bool wide_ok = (a.N % 16 == 0) && ((uintptr_t)a.out % 32 == 0);
            drain_columns(a, tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * BN), grow, row_ok, n0,
                          half * (BN / 64), (half + 1) * (BN / 64), wide_ok);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&acc_empty[acc]);
            if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
        }
    }
    tc_fence_before();
    __syncthreads();
    quiesce_after_abort(abort_word);
    __syncthreads();
    if (warp == 2) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
    }
}

// =====================================================================================================
// Wide form of the same GEMM: one CTA works on a 256 x 256 output tile as two 128 x 256 halves that share the
// weight tile.  Per k-block 32 KB of activations (256 rows) and 32 KB of weights come in, and eight MMAs use them:
// 64 KB per 1024 tensor-pipe cycles instead of 48 KB per 512, a third less data pulled out of L2 per flop.  The two
// accumulators take all 512 TMEM columns, so a tile's epilogue no longer hides behind the next tile's MMAs except
// for half a tile's worth at either end (each half has its own pair of barriers and the epilogue drains the upper
// half first); that is the better trade where K is long.  Three stages of 64 KB.
constexpr int NSTAGE_W = 3;
// shortest reduction for which the wide kernel is chosen by default, with and without a GeLU in the epilogue (pairs of
// GEMMs on E = 32, M = 2048 back to back: with the GeLU level at K = 6144, 2 % slower at 5120; without it 1.6 % faster
// at 5120, level at 4096)
constexpr int kWideMinK = 6144, kWideMinKPlain = 5120;
constexpr uint32_t AW_BYTES = 2 * A_BYTES, STAGE_W_BYTES = AW_BYTES + B_BYTES;
constexpr size_t kFfnWideSmem = (size_t)NSTAGE_W * STAGE_W_BYTES + 1024 /*alignment slack*/ + 256 /*barriers*/;

// Work item w of the wide kernel: a whole 256 x 256 tile (halves = 3) below split_from, one 128-row half of a tile
// above it.  The last, partly filled wave of tiles is split in this way when its halves fit one wave: 148 CTAs
// then finish after one more 128-row tile instead of one more 256-row tile.
struct WideItem { int tile, halves; };
__device__ __forceinline__ WideItem wide_item(const FfnArgs& a, int w) {
    if (w < a.split_from) return {w, 3};
    const int u = w - a.split_from;
    return {a.split_from + (u >> 1), 1 << (u & 1)};
}

__global__ void __launch_bounds__(kFfnThreads, 1)
ffn_gemm_wide_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const FfnArgs a) {
    extern __shared__ unsigned char smraw[];
    unsigned char* base = reinterpret_cast<unsigned char*>(((uintptr_t)smraw + 1023) & ~(uintptr_t)1023);
    uint64_t* bars = reinterpret_cast<uint64_t*>(base + (size_t)NSTAGE_W * STAGE_W_BYTES);
    uint64_t* full = bars;                     // [NSTAGE_W]
    uint64_t* empty = bars + NSTAGE_W;         // [NSTAGE_W]
    uint64_t* acc_full = bars + 2 * NSTAGE_W;  // [2] one per 128-row half
    uint64_t* acc_empty = acc_full + 2;        // [2]
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
    volatile int* abort_word = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < NSTAGE_W; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], kEpiWarps); }
        *abort_word = 0;
        mbar_init_fence();
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    const int tiles_per_expert = a.m_tiles * a.n_tiles;   // m_tiles counts 256-row tiles here
    const int total_tiles = a.E * tiles_per_expert;
    const int total_items = a.split_from + 2 * (total_tiles - a.split_from);
    const int kblocks = (a.K + BK - 1) / BK;

    if (warp == 0) {
        if (lane == 0) {  // ---- TMA producer: one 256-row box of A and one of B per k-block ----
            int stage = 0; uint32_t phase = 0;
            for (int w = blockIdx.x; w < total_items; w += gridDim.x) {
                const int tile = wide_item(a, w).tile;   // a half-tile item loads the whole boxes all the same
                const int e = tile / tiles_per_expert, rem = tile - e * tiles_per_expert;
                const int nt = rem / a.m_tiles, mt = rem - nt * a.m_tiles;
                const int row0 = e * a.M + mt * 2 * BM, n0 = nt * BN;
                bool ok = true;
                // every other wave sweeps the reduction backwards: an expert whose tiles straddle two waves then
                // finds the end of its operand panels, which the earlier wave read last, still in L2
                const bool rev = ((w / (int)gridDim.x) & 1) != 0;
                for (int kb = 0; kb < kblocks && ok; ++kb) {
                    if (!wait_or_abort(&empty[stage], phase ^ 1u, abort_word)) { ok = false; break; }
                    unsigned char* sa = base + (size_t)stage * STAGE_W_BYTES;
                    const int k0 = (rev ? kblocks - 1 - kb : kb) * BK;
                    mbar_expect_tx(&full[stage], STAGE_W_BYTES);
                    tma_load_2d(sa, &tmA, k0, row0, &full[stage]);
                    tma_load_3d(sa + AW_BYTES, &tmB, k0, n0, e, &full[stage]);
                    if (++stage == NSTAGE_W) { stage = 0; phase ^= 1u; }
                }
                if (!ok) break;
            }
            for (int i = 0; i < NSTAGE_W; ++i) {   // every commit to this CTA's stage barriers has arrived
                if (!wait_or_abort(&empty[stage], phase ^ 1u, abort_word)) break;
                if (++stage == NSTAGE_W) { stage = 0; phase ^= 1u; }
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {  // ---- MMA issuer ----
            int stage = 0; uint32_t phase = 0;
            uint32_t acc_phase = 0;   // bit h: phase of half h's accumulator barriers
            for (int w = blockIdx.x; w < total_items; w += gridDim.x) {
                const int halves = wide_item(a, w).halves;
                bool ok = true;
                for (int kb = 0; kb < kblocks && ok; ++kb) {
                    if (!wait_or_abort(&full[stage], phase, abort_word)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t sa = smem_u32(base + (size_t)stage * STAGE_W_BYTES);
                    const uint32_t sb = sa + AW_BYTES;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (!((halves >> h) & 1)) continue;
                        if (kb == 0) {   // this half's accumulator has been drained
                            if (!wait_or_abort(&acc_empty[h], ((acc_phase >> h) & 1u) ^ 1u, abort_word)) { ok = false; break; }
                            tc_fence_after();
                        }
#pragma unroll
                        for (int k = 0; k < BK / UMMA_K; ++k)
                            umma_bf16(tmem_base + (uint32_t)h * BN, umma_desc_sw128(sa + h * A_BYTES + k * UMMA_K * 2),
                                      umma_desc_sw128(sb + k * UMMA_K * 2), (kb > 0 || k > 0) ? 1u : 0u);
                        if (kb == kblocks - 1) umma_commit(&acc_full[h]);
                    }
                    if (!ok) break;
                    umma_commit(&empty[stage]);
                    if (++stage == NSTAGE_W) { stage = 0; phase ^= 1u; }
                }
                if (!ok) break;
                acc_phase ^= (uint32_t)halves;
            }
        }
    } else {  // ---- epilogue warps 2..9: TMEM lane quadrant = warp % 4, column half = (warp - 2) / 4, both row halves ----
        const int q = warp & 3;
        const int half = (warp - 2) >> 2;
        uint32_t acc_phase = 0;   // bit h: phase of half h's accumulator barriers
        const bool wide_ok = (a.N % 16 == 0) && ((uintptr_t)a.out % 32 == 0);
        for (int w = blockIdx.x; w < total_items; w += gridDim.x) {
            const WideItem it = wide_item(a, w);
            const int tile = it.tile;
            const int e = tile / tiles_per_expert, rem = tile - e * tiles_per_expert;
            const int nt = rem / a.m_tiles, mt = rem - nt * a.m_tiles;
            const int n0 = nt * BN;
            bool ok = true;
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                if (!((it.halves >> h) & 1)) continue;
                if (!wait_or_abort(&acc_full[h], (acc_phase >> h) & 1u, abort_word)) { ok = false; break; }
                tc_fence_after();
                const int r_in = mt * 2 * BM + h * BM + q * 32 + lane;
                const bool row_ok = r_in < a.M;
                const long long grow = (long long)e * a.M + r_in;
                drain_columns(a, tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(h * BN), grow, row_ok, n0,
                              half * (BN / 64), (half + 1) * (BN / 64), wide_ok);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&acc_empty[h]);
                acc_phase ^= 1u << h;
            }
            if (!ok) break;
        }
    }
    tc_fence_before();
    __syncthreads();
    quiesce_after_abort(abort_word);
    __syncthreads();
    if (warp == 2) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
    }
}

// =====================================================================================================
// Two-SM form of the same GEMM: a cluster of two CTAs works on a 256 x 256 output tile.  Each CTA loads its own
// 128 rows of A and only HALF of the B tile (128 of the 256 weight rows); tcgen05.mma.cta_group::2, issued by the
// leader CTA (cluster rank 0), multiplies the 256 x 64 A (both CTAs' shared memory) by the 256 x 64 B (both halves)
// into 128 x 256 accumulators in each CTA's own TMEM.  Per SM and k-block 32 KB instead of 48 KB come out of L2,
// and the ring holds six stages instead of four.
//   full[s]      leader only: both CTAs' TMA loads of stage s have landed (the peer's loads count their bytes on
//                the leader's barrier: cp.async.bulk.tensor ... .cta_group::2, data into the issuing CTA only)
//   empty[s]     MMAs that read stage s are done (tcgen05.commit multicast to both CTAs)
//   acc_full[i]  accumulator i complete (multicast)     acc_empty[i]  leader only: both CTAs' epilogues drained i
// Remote arrives use mapa + mbarrier.arrive.release.cluster; waits that order cross-CTA data use acquire.cluster.
constexpr int NSTAGE2 = 6;
constexpr uint32_t B2_BYTES = (BN / 2) * BK * 2, STAGE2_BYTES = A_BYTES + B2_BYTES;
constexpr size_t kFfn2Smem = (size_t)NSTAGE2 * STAGE2_BYTES + 1024 /*alignment slack*/ + 512 /*barriers*/;
constexpr uint32_t kIdesc2 = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)((2 * BM) >> 4) << 24);

__device__ __forceinline__ uint32_t cluster_ctarank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void mbar_arrive_remote(uint64_t* bar, uint32_t cta) {
    uint32_t ra;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(ra) : "r"(smem_u32(bar)), "r"(cta));
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(ra) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait_cluster(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    return ok != 0;
}
// Raises the abort word of this CTA and of its partner in the pair (a plain store into the partner's shared
// memory through the cluster address), so that both leave their loops together instead of the partner running
// out its own wait against a CTA that has already given up.
__device__ __forceinline__ void raise_abort_pair(volatile int* abort_word) {
    *abort_word = 1;
    uint32_t ra;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(ra) : "r"(smem_u32(const_cast<int*>(abort_word))), "r"(cluster_ctarank() ^ 1u));
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(ra), "r"(1) : "memory");
    atomicOr(&g_ffn_flags, 1);
}
// The two waits of the two-SM kernel: like wait_or_abort, but a give-up is announced to both CTAs of the pair.
__device__ __forceinline__ bool wait_or_abort_pair(uint64_t* bar, uint32_t parity, volatile int* abort_word) {
    for (uint32_t i = 0; i < (1u << 22); ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 63u) == 63u && *abort_word) return false;
    }
    raise_abort_pair(abort_word);
    return false;
}
__device__ __forceinline__ bool wait_or_abort_cluster(uint64_t* bar, uint32_t parity, volatile int* abort_word) {
    for (uint32_t i = 0; i < (1u << 22); ++i) {
        if (mbar_try_wait_cluster(bar, parity)) return true;
        if ((i & 63u) == 63u && *abort_word) return false;
    }
    raise_abort_pair(abort_word);
    return false;
}
__device__ __forceinline__ void umma_bf16_2cta(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(kIdesc2), "r"(accumulate) : "memory");
}
// Arrives on the barrier at this offset in BOTH CTAs of the pair once all MMAs issued so far have completed.
__device__ __forceinline__ void umma_commit_2cta(uint64_t* bar) {
    const uint16_t mask = 3;
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(smem_u32(bar)), "h"(mask) : "memory");
}

// TMA loads of the pair: the data lands in the issuing CTA's shared memory, the bytes are counted on the LEADER's
// barrier (bar_cluster = the shared::cluster address of the leader's barrier).  No multicast.
__device__ __forceinline__ uint32_t leader_addr(const void* p) {
    uint32_t ra;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(ra) : "r"(smem_u32(p)), "r"(0));
    return ra;
}
__device__ __forceinline__ void tma_load_2d_pair(void* dst, const CUtensorMap* map, int c0, int c1, uint32_t bar_cluster) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar_cluster), "r"(c0), "r"(c1)
                 : "memory");
}
__device__ __forceinline__ void tma_load_3d_pair(void* dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar_cluster) {
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar_cluster), "r"(c0), "r"(c1), "r"(c2)
                 : "memory");
}

template <int NACC>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kFfnThreads, 1)
ffn_gemm2_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const FfnArgs a) {
    extern __shared__ unsigned char smraw[];
    unsigned char* base = reinterpret_cast<unsigned char*>(((uintptr_t)smraw + 1023) & ~(uintptr_t)1023);
    uint64_t* bars = reinterpret_cast<uint64_t*>(base + (size_t)NSTAGE2 * STAGE2_BYTES);
    uint64_t* full = bars;
    uint64_t* empty = bars + NSTAGE2;
    uint64_t* acc_full = bars + 2 * NSTAGE2;
    uint64_t* acc_empty = acc_full + 2;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
    volatile int* abort_word = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const bool leader = rank == 0;
    constexpr uint32_t kCols = NACC * BN;
    if (threadIdx.x == 0) {
        for (int s = 0; s < NSTAGE2; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], 2 * kEpiWarps); }
        *abort_word = 0;
        *tmem_slot = 0xffffffffu;
        mbar_init_fence();
    }
    __syncthreads();
    if (warp == 2) {  // one warp of each CTA of the pair takes part in the paired allocation
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();   // both CTAs' barriers are initialised before any remote arrive or multicast commit
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    const int m_tiles2 = (a.M + 2 * BM - 1) / (2 * BM);
    const int tiles_per_expert = m_tiles2 * a.n_tiles;
    const int total_tiles = a.E * tiles_per_expert;
    const int kblocks = (a.K + BK - 1) / BK;
    const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;

    if (warp == 0) {
        if (lane == 0) {  // ---- TMA producer: own rows of A, own half of B ----
            int stage = 0; uint32_t phase = 0;
            for (int tile = pair; tile < total_tiles; tile += npairs) {
                const int e = tile / tiles_per_expert, rem = tile - e * tiles_per_expert;
                const int nt = rem / m_tiles2, mt = rem - nt * m_tiles2;
                const int row0 = e * a.M + mt * 2 * BM + (int)rank * BM, n0 = nt * BN + (int)rank * (BN / 2);
                bool ok = true;
                for (int kb = 0; kb < kblocks && ok; ++kb) {
                    if (!wait_or_abort_pair(&empty[stage], phase ^ 1u, abort_word)) { ok = false; break; }
                    unsigned char* sa = base + (size_t)stage * STAGE2_BYTES;
                    if (leader) mbar_expect_tx(&full[stage], 2 * STAGE2_BYTES);   // both CTAs' bytes are counted here
                    const uint32_t bar = leader_addr(&full[stage]);
                    tma_load_2d_pair(sa, &tmA, kb * BK, row0, bar);
                    tma_load_3d_pair(sa + A_BYTES, &tmB, kb * BK, n0, e, bar);
                    if (++stage == NSTAGE2) { stage = 0; phase ^= 1u; }
                }
                if (!ok) break;
            }
            // tail: every stage has been released, i.e. every commit that targets this CTA's barriers has arrived,
            // before the CTA may leave (the commits are asynchronous and multicast to both CTAs)
            for (int i = 0; i < NSTAGE2; ++i) {
                if (!wait_or_abort_pair(&empty[stage], phase ^ 1u, abort_word)) break;
                if (++stage == NSTAGE2) { stage = 0; phase ^= 1u; }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && leader) {  // ---- MMA issuer (leader CTA) ----
            int stage = 0; uint32_t phase = 0;
            int acc = 0; uint32_t acc_phase = 0;
            for (int tile = pair; tile < total_tiles; tile += npairs) {
                if (!wait_or_abort_cluster(&acc_empty[acc], acc_phase ^ 1u, abort_word)) break;
                tc_fence_after();
                const uint32_t tmem_d = tmem_base + (uint32_t)acc * BN;
                bool ok = true;
                for (int kb = 0; kb < kblocks; ++kb) {
                    if (!wait_or_abort_cluster(&full[stage], phase, abort_word)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t sa = smem_u32(base + (size_t)stage * STAGE2_BYTES);
                    const uint32_t sb = sa + A_BYTES;
#pragma unroll
                    for (int k = 0; k < BK / UMMA_K; ++k)
                        umma_bf16_2cta(tmem_d, umma_desc_sw128(sa + k * UMMA_K * 2), umma_desc_sw128(sb + k * UMMA_K * 2),
                                       (kb > 0 || k > 0) ? 1u : 0u);
                    umma_commit_2cta(&empty[stage]);
                    if (++stage == NSTAGE2) { stage = 0; phase ^= 1u; }
                }
                if (!ok) break;
                umma_commit_2cta(&acc_full[acc]);
                if (++acc == NACC) { acc = 0; acc_phase ^= 1u; }
            }
        }
    } else {  // ---- epilogue warps 2..9 of each CTA on its own 128 rows ----
        const int q = warp & 3;
        const int half = (warp - 2) >> 2;
        int acc = 0; uint32_t acc_phase = 0;
        for (int tile = pair; tile < total_tiles; tile += npairs) {
            const int e = tile / tiles_per_expert, rem = tile - e * tiles_per_expert;
            const int nt = rem / m_tiles2, mt = rem - nt * m_tiles2;
            if (!wait_or_abort_pair(&acc_full[acc], acc_phase, abort_word)) break;
            tc_fence_after();
            const int r_in = mt * 2 * BM + (int)rank * BM + q * 32 + lane;
            const bool row_ok = r_in < a.M;
            const long long grow = (long long)e * a.M + r_in;
            const int n0 = nt * BN;
            const bool wide_ok = (a.N % 16 == 0) && ((uintptr_t)a.out % 32 == 0);
            drain_columns(a, tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * BN), grow, row_ok, n0,
                          half * (BN / 64), (half + 1) * (BN / 64), wide_ok);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_remote(&acc_empty[acc], 0);
            if (++acc == NACC) { acc = 0; acc_phase ^= 1u; }
        }
    }
    tc_fence_before();
    __syncthreads();
    quiesce_after_abort(abort_word);
    __syncthreads();
    cluster_sync_all();   // neither CTA frees its half of the paired allocation while the other may still use it
    if (warp == 2) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kCols) : "memory");
    }
}

// ---- host side: tensor maps through the driver entry point (no link-time dependency on libcuda) ----
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = nullptr;
    static std::mutex m;
    std::lock_guard<std::mutex> lock(m);
    if (!fn) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return nullptr;
        }
        fn = reinterpret_cast<EncodeTiledFn>(p);
    }
    return fn;
}

}  // namespace

// K-major bf16 matrix [outer...][rows][K] with a box of box_rows x 64 elements, 128-byte swizzle.
bool make_map(CUtensorMap* map, const void* ptr, int rank, const uint64_t* dims, uint32_t box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t gdim[3] = {dims[0], dims[1], rank == 3 ? dims[2] : 1};
    cuuint64_t gstr[2] = {dims[0] * 2, dims[0] * dims[1] * 2};
    cuuint32_t box[3] = {(cuuint32_t)BK, box_rows, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(ptr), gdim, gstr, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

namespace {

int launch_gemm(const void* A, const void* W, void* out, int out_f32, int gelu, int E, int M, int N, int K,
                cudaStream_t st) {
    CUtensorMap tmA, tmB;
    const uint64_t da[2] = {(uint64_t)K, (uint64_t)E * M};
    const uint64_t db[3] = {(uint64_t)K, (uint64_t)N, (uint64_t)E};
    if (!make_map(&tmA, A, 2, da, BM) || !make_map(&tmB, W, 3, db, BN)) return LOCMOE_ERR_CUDA;
    FfnArgs a{};
    a.out = out; a.out_f32 = out_f32; a.gelu = gelu; a.E = E; a.M = M; a.N = N; a.K = K;
    a.m_tiles = (M + BM - 1) / BM;
    a.n_tiles = (N + BN - 1) / BN;
    static bool attr_done_dev[64] = {false};   // the attribute is per device
    int attr_dev = 0;
    cudaGetDevice(&attr_dev);
    bool& attr_done = attr_done_dev[attr_dev & 63];
    if (!attr_done) {
        if (cudaFuncSetAttribute(ffn_gemm_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kFfnSmem) != cudaSuccess) {
            cudaGetLastError();
            return LOCMOE_ERR_CUDA;
        }
        attr_done = true;
    }
    long long tiles = (long long)E * a.m_tiles * a.n_tiles;
    int grid = sm_count();
    if (tiles < grid) grid = (int)tiles;
    ffn_gemm_kernel<<<grid, kFfnThreads, kFfnSmem, st>>>(tmA, tmB, a);
    return check_launch();
}

// Wide kernel: 256 x 256 tiles, one CTA each.
int launch_gemm_wide(const void* A, const void* W, void* out, int out_f32, int gelu, int E, int M, int N, int K,
                     cudaStream_t st) {
    CUtensorMap tmA, tmB;
    const uint64_t da[2] = {(uint64_t)K, (uint64_t)E * M};
    const uint64_t db[3] = {(uint64_t)K, (uint64_t)N, (uint64_t)E};
    if (!make_map(&tmA, A, 2, da, 2 * BM) || !make_map(&tmB, W, 3, db, BN)) return LOCMOE_ERR_CUDA;
    FfnArgs a{};
    a.out = out; a.out_f32 = out_f32; a.gelu = gelu; a.E = E; a.M = M; a.N = N; a.K = K;
    a.m_tiles = (M + 2 * BM - 1) / (2 * BM);
    a.n_tiles = (N + BN - 1) / BN;
    static bool attr_done_dev[64] = {false};   // the attribute is per device
    int dev = 0;
    cudaGetDevice(&dev);
    if (!attr_done_dev[dev & 63]) {
        if (cudaFuncSetAttribute(ffn_gemm_wide_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kFfnWideSmem) != cudaSuccess) {
            cudaGetLastError();
            return LOCMOE_ERR_CUDA;
        }
        attr_done_dev[dev & 63] = true;
    }
    const long long tiles = (long long)E * a.m_tiles * a.n_tiles;
    int grid = sm_count();
    const long long tail = tiles % grid;   // tiles of the last, partly filled wave
    a.split_from = (int)(tiles >= grid && tail > 0 && 2 * tail <= grid ? tiles - tail : tiles);
    if (tiles < grid) grid = (int)tiles;
    ffn_gemm_wide_kernel<<<grid, kFfnThreads, kFfnWideSmem, st>>>(tmA, tmB, a);
    return check_launch();
}

// Two-SM kernel.  nacc = 2: two accumulators per CTA (all 512 TMEM columns); nacc = 1: one (256 columns, the
// epilogue does not overlap the next tile's MMAs).
int launch_gemm2(const void* A, const void* W, void* out, int out_f32, int gelu, int E, int M, int N, int K, int nacc,
                 cudaStream_t st) {
    CUtensorMap tmA, tmB;
    const uint64_t da[2] = {(uint64_t)K, (uint64_t)E * M};
    const uint64_t db[3] = {(uint64_t)K, (uint64_t)N, (uint64_t)E};
    if (!make_map(&tmA, A, 2, da, BM) || !make_map(&tmB, W, 3, db, BN / 2)) return LOCMOE_ERR_CUDA;
    FfnArgs a{};
    a.out = out; a.out_f32 = out_f32; a.gelu = gelu; a.E = E; a.M = M; a.N = N; a.K = K;
    a.m_tiles = (M + 2 * BM - 1) / (2 * BM);
    a.n_tiles = (N + BN - 1) / BN;
    static bool attr_done_dev[64] = {false};   // the attribute is per device
    int dev = 0;
    cudaGetDevice(&dev);
    if (!attr_done_dev[dev & 63]) {
        if (cudaFuncSetAttribute(ffn_gemm2_kernel<1>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kFfn2Smem) != cudaSuccess ||
            cudaFuncSetAttribute(ffn_gemm2_kernel<2>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kFfn2Smem) != cudaSuccess) {
            cudaGetLastError();
            return LOCMOE_ERR_CUDA;
        }
        attr_done_dev[dev & 63] = true;
    }
    const long long tiles = (long long)E * a.m_tiles * a.n_tiles;
    long long pairs = sm_count() / 2;
    if (tiles < pairs) pairs = tiles;
    if (pairs < 1) pairs = 1;
    if (nacc == 1) ffn_gemm2_kernel<1><<<(int)pairs * 2, kFfnThreads, kFfn2Smem, st>>>(tmA, tmB, a);
    else ffn_gemm2_kernel<2><<<(int)pairs * 2, kFfnThreads, kFfn2Smem, st>>>(tmA, tmB, a);
    return check_launch();
}

}  // namespace

// Which kernel runs each of the two GEMMs: 0 = 128 x 256 tiles, 1 = wide (256 x 256 tiles), 2 = two-SM, 3 = two-SM with
// one accumulator.  By default the wide kernel where the reduction is long enough for its exposed epilogue not to
// matter, the rows of an expert fill its taller tiles as well as they fill the 128-row ones, and the last wave of its
// twice-as-long tiles does not cost more than the wide tiles save (about 5 %); else the 128 x 256 kernel.
// On E = 32, M = 2048, H = 2560, F = 10240, back to back under the power cap: second GEMM (K = 10240) 2.63
// against 2.77 ms, first GEMM (K = 2560, GeLU) 2.98 against 2.84 ms.
// LOCMOE_FFN (a testing aid) overrides: 1 = 128 x 256 kernel for both, w = wide for both, w1 / w2 = wide for
// the first / second GEMM only, 2 = the two-SM kernel (2s: its single-accumulator form).  The two-SM kernel is
// opt-in only: it passes every test and runs clean in the bench, but launches of it failed under multi-metric
// profiler captures for a reason that reading the code has not shown.
void plan_expert_ffn(const locmoe_shape_t& s, int64_t rows, int F, int kernels[2]) {
    const int E = s.E;
    const int M = (int)(rows / E);
    const char* mode = getenv("LOCMOE_FFN");
    if (mode && mode[0] == '2' && sm_count() >= 2) {
        kernels[0] = kernels[1] = mode[1] == 's' ? 3 : 2;
        return;
    }
    const long long m1 = (M + BM - 1) / BM, m2 = (M + 2 * BM - 1) / (2 * BM), G = sm_count() > 0 ? sm_count() : 1;
    auto pays = [&](int N, int K, bool gelu) {
        const long long n = (N + BN - 1) / BN;
        const long long tw = E * m2 * n, tail = tw % G;
        const long long waves_narrow = (E * m1 * n + G - 1) / G;                      // in 128-row tiles
        const long long waves_wide = tw / G * 2 + (tail == 0 ? 0 : (tw >= G && 2 * tail <= G) ? 1 : 2);   // the same unit
        return K >= (gelu ? kWideMinK : kWideMinKPlain) && m2 * 2 == m1 && waves_wide * 19 <= waves_narrow * 20;
    };
    bool wide1 = pays(F, s.H, true), wide2 = pays(s.H, F, false);
    if (mode && mode[0] == '1') wide1 = wide2 = false;
    if (mode && mode[0] == 'w') { wide1 = mode[1] != '2'; wide2 = mode[1] != '1'; }
    kernels[0] = wide1 ? 1 : 0;
    kernels[1] = wide2 ? 1 : 0;
}

int launch_expert_ffn(const locmoe_shape_t& s, int64_t rows, int F, const void* buf, const void* w_in,
                      const void* w_out, void* h1, void* y, int y_dtype, cudaStream_t st) {
    const int E = s.E;
    const int M = (int)(rows / E);
    const int y_f32 = y_dtype == LOCMOE_F32 ? 1 : 0;
    int kernels[2];
    plan_expert_ffn(s, rows, F, kernels);
    auto run = [&](int kernel, const void* A, const void* W, void* out, int out_f32, int gelu, int N, int K) {
        if (kernel >= 2) return launch_gemm2(A, W, out, out_f32, gelu, E, M, N, K, kernel == 3 ? 1 : 2, st);
        if (kernel == 1) return launch_gemm_wide(A, W, out, out_f32, gelu, E, M, N, K, st);
        return launch_gemm(A, W, out, out_f32, gelu, E, M, N, K, st);
    };
    const int rc = run(kernels[0], buf, w_in, h1, 0, 1, F, s.H);
    if (rc) return rc;
    return run(kernels[1], h1, w_out, y, y_f32, 0, s.H, F);
}

int read_ffn_flags(int* out, cudaStream_t st) {
    if (cudaMemcpyFromSymbolAsync(out, g_ffn_flags, sizeof(int), 0, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaStreamSynchronize(st) != cudaSuccess) {
        cudaGetLastError();
        return LOCMOE_ERR_CUDA;
    }
    return LOCMOE_OK;
}

}  // namespace locmoe
