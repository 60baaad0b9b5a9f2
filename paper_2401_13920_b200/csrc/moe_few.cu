// A whole MoE layer for a few tokens (decoding), in two kernels: gate and first expert product, then second product
// and the gate-weighted sum.
//
//   G_i = ReLU(mean_i x + eps_i),  p = softmax(G),  the K largest;   out_t = sum_c p_{t,c} W_out[e] GeLU(W_in[e] x_t)
//
// Bound by the weights of the experts that the tokens meet (4 F H bytes each), every one of which is read once.  So
// the weights are what moves fast: every warp streams its own tiles of 8 * NB weight rows through a private ring of
// TMA stages.  A task is a block of 8 * NB weight rows of one expert (and, in the second product, one of S slices of
// the reduction); a warp works on its tasks from the first byte to the result with no barrier but its own ring's.
// The products run on mma.sync m16n8k16, tokens as the 16 rows and weight rows as the 8 columns: at a few tokens an
// expert nothing is gained by larger matrix instructions.  The order of k inside a stage is chosen so that a
// thread's fragments of both operands are 16 contiguous bytes of a row (the same permutation on both sides), which
// the tiles' 128-byte swizzle gives without bank conflicts.
// The router is evaluated by every CTA for itself: a few tokens' rows out of L2 cost less than a launch of their own.
#include "common.cuh"
#include "tensor_map.cuh"

namespace locmoe {

namespace {

constexpr int kMaxTokens = LOCMOE_FEW_MAX_TOKENS, kMaxExperts = 1024, kMaxK = 8, kMaxSplit = 8;
constexpr int kBoxK = 64;          // k of one TMA box: 128 bytes of a row

__device__ int g_few_flags = 0;    // bit 0: a bounded wait gave up
constexpr uint32_t kNoRow = 0xffffffffu;

struct FewArgs {
    const uint16_t* x; const float* eps; const uint16_t* w_in; const uint16_t* w_out;
    int32_t* idx_k; float* w_k; uint16_t* out;
    uint16_t* g;        // [2][K * T][F] GeLU(W_in x) as the sum of two bf16 values: the rounded value and what rounding left
    float* part;        // [S][K * T][H] slices of the second product
    int32_t* arrived;   // [row blocks] tasks that have left their slice
    int T, H, E, K, F, max_split, weighted;
};

// A variant: W warps, MT tiles of 16 tokens, NB blocks of 8 weight rows, NBOX boxes of 64 k a stage, D stages a warp;
// the tasks an SM should have at least for an even load, the CTAs for which an SM has room.
template <int W_, int MT_, int NB_, int NBOX_, int D_, int TASKS_, int CTAS_>
struct Variant {
    static constexpr int W = W_, MT = MT_, NB = NB_, NBOX = NBOX_, D = D_, kTasks = TASKS_, kCtas = CTAS_;
    static constexpr int kThreads = 32 * W, kBox = 8 * NB * 128, kStage = NBOX * kBox, kRing = W * D * kStage;
    static constexpr int kStepK = NBOX * kBoxK;
};

struct Smem {   // offsets of the dynamic shared memory, from its first 1024-byte boundary on
    int ring, bars, expert, sorted, score, act, first, chunk, total;
};
__host__ __device__ constexpr int round16(int n) { return (n + 15) / 16 * 16; }
template <class V>
__host__ __device__ inline Smem layout(int TK, int E) {
    Smem s{};
    const int most = TK < E ? TK : E;
    // the router's scratch lies where the ring is later: a strip of E floats per warp, the counters beside it
    const int scratch = (V::W + 2) * E * 4;
    s.ring = 0;
    s.bars = scratch > V::kRing ? round16(scratch) : V::kRing;
    s.expert = s.bars + round16(8 * V::W * V::D);   // int16 [TK]  expert of assignment a = c * T + t
    s.sorted = s.expert + round16(2 * TK);            // int16 [TK]  assignments by expert
    s.score = s.sorted + round16(2 * TK);             // float [TK]
    s.act = s.score + round16(4 * TK);                // int16 [most]      experts met
    s.first = s.act + round16(2 * most);              // int16 [most + 1]  their first entry of `sorted`
    s.chunk = s.first + round16(2 * most + 2);        // int16 [most + 1]  their first chunk of 16 * MT tokens
    s.total = s.chunk + round16(2 * most + 2) + 1024 /* alignment slack */;
    return s;
}

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Sum of `n` consecutive bf16 values from `p`, of which this lane takes every `of`-th piece from `sub` on.
template <int EL>
__device__ __forceinline__ float sum_pieces(const uint16_t* p, int n, int sub, int of) {
    float s0 = 0.0f, s1 = 0.0f;
#pragma unroll 4
    for (int i = sub; i < n / EL; i += of) {
        if constexpr (EL == 8) {
            const uint4 w = __ldg(reinterpret_cast<const uint4*>(p) + i);
            s0 += (bf16_lo(w.x) + bf16_hi(w.x)) + (bf16_lo(w.y) + bf16_hi(w.y));
            s1 += (bf16_lo(w.z) + bf16_hi(w.z)) + (bf16_lo(w.w) + bf16_hi(w.w));
        } else if constexpr (EL == 2) {
            const uint32_t w = __ldg(reinterpret_cast<const uint32_t*>(p) + i);
            s0 += bf16_lo(w); s1 += bf16_hi(w);
        } else {
            s0 += bf16_lo(__ldg(p + i));
        }
    }
    return s0 + s1;
}

// Router for all tokens, one warp per token: fills expert[] and score[].
template <int W>
__device__ __forceinline__ void few_router(const FewArgs& a, int16_t* expert, float* score, float* strip_all) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = a.H / a.E;
    float* G = strip_all + warp * a.E;
    int lanes = 1;                                   // lanes that share one expert's group
    while (lanes * 2 * a.E <= 32) lanes *= 2;
    const int sub = lane % lanes;
    const float inv_g = 1.0f / (float)g;
    for (int t = warp; t < a.T; t += W) {
        const uint16_t* row = a.x + (size_t)t * a.H;
        for (int i0 = 0; i0 < a.E; i0 += 32 / lanes) {
            const int i = i0 + lane / lanes;
            float s = 0.0f;
            if (i < a.E) {
                const uint16_t* p = row + (size_t)i * g;
                s = g % 8 == 0 ? sum_pieces<8>(p, g, sub, lanes) : g % 2 == 0 ? sum_pieces<2>(p, g, sub, lanes) : sum_pieces<1>(p, g, sub, lanes);
            }
            for (int o = 1; o < lanes; o *= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
            if (i < a.E && sub == 0) G[i] = fmaxf(fmaf(s, inv_g, a.eps ? a.eps[i] : 0.0f), 0.0f);   // a NaN logit counts as 0
        }
        __syncwarp();
        float top = 0.0f, z = 0.0f;
        for (int c = 0; c < a.K; ++c) {
            float best = -2.0f;
            int bi = 0x7fffffff;
            for (int i = lane; i < a.E; i += 32)
                if (G[i] > best) { best = G[i]; bi = i; }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {       // the lower index wins a tie
                const float ob = __shfl_xor_sync(0xffffffffu, best, o);
                const int oi = __shfl_xor_sync(0xffffffffu, bi, o);
                if (ob > best || (ob == best && oi < bi)) { best = ob; bi = oi; }
            }
            if (c == 0) {
                top = best;
                for (int i = lane; i < a.E; i += 32) z += expf(G[i] - top);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
            }
            __syncwarp();
            if (lane == 0) {
                G[bi] = -1.0f;                       // below every logit: chosen
                expert[c * a.T + t] = (int16_t)bi;
                score[c * a.T + t] = expf(best - top) / z;
            }
            __syncwarp();
        }
    }
}

// Position in a warp's sequence of tasks: which weight rows and which stages come next.
struct Cursor {
    int task, j;                    // j: index of the task's expert in act[]
    int e, row0, ch, s, rb, step, last;
};

template <class V, bool SECOND>
__global__ void __launch_bounds__(V::kThreads, V::kCtas)
moe_few_kernel(const __grid_constant__ CUtensorMap map, const FewArgs a) {
    constexpr int W = V::W, MT = V::MT, NB = V::NB, NBOX = V::NBOX, D = V::D, kThreads = V::kThreads;
    extern __shared__ unsigned char raw[];
    unsigned char* sm = reinterpret_cast<unsigned char*>(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);   // the swizzle repeats every 1024 bytes
    const int TK = a.T * a.K;
    const Smem L = layout<V>(TK, a.E);
    uint64_t* full = reinterpret_cast<uint64_t*>(sm + L.bars);
    int16_t* expert = reinterpret_cast<int16_t*>(sm + L.expert);
    int16_t* sorted = reinterpret_cast<int16_t*>(sm + L.sorted);
    float* score = reinterpret_cast<float*>(sm + L.score);
    int16_t* act = reinterpret_cast<int16_t*>(sm + L.act);
    int16_t* first = reinterpret_cast<int16_t*>(sm + L.first);
    int16_t* chunk = reinterpret_cast<int16_t*>(sm + L.chunk);
    float* strips = reinterpret_cast<float*>(sm + L.ring);
    int* count = reinterpret_cast<int*>(strips + W * a.E);
    int* place = count + a.E;
    __shared__ int n_act;
    __shared__ volatile int abort_word;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gq = lane >> 2, tq = lane & 3;
    const int N = SECOND ? a.H : a.F, Kd = SECOND ? a.F : a.H;
    const int RB = (N + 8 * NB - 1) / (8 * NB);

    // With few assignments the second kernel evaluates the router again, so that it can fill its ring with weights
    // while the first one is still running; with many it takes the first kernel's choices.
    const bool early = SECOND && TK <= 8;
    if (tid < W * D) mbar_init(&full[tid], 1);
    if (tid == 0) { abort_word = 0; mbar_init_fence(); }
    if (!SECOND) {
        pdl_wait();
        pdl_trigger();
    }
    if (!SECOND || early) {
        few_router<W>(a, expert, score, strips);
    } else {
        pdl_wait();
        pdl_trigger();
        for (int i = tid; i < TK; i += kThreads) { expert[i] = (int16_t)a.idx_k[i]; score[i] = a.w_k[i]; }
    }
    for (int i = tid; i < a.E; i += kThreads) count[i] = 0;
    __syncthreads();
    if (!SECOND && blockIdx.x == 0)
        for (int i = tid; i < TK; i += kThreads) { a.idx_k[i] = expert[i]; a.w_k[i] = score[i]; }
    if (!SECOND) {
        const int blocks = (a.H + 7) / 8;
        for (int i = blockIdx.x * kThreads + tid; i < blocks; i += gridDim.x * kThreads) a.arrived[i] = 0;
    }
    for (int i = tid; i < TK; i += kThreads) atomicAdd(&count[expert[i]], 1);
    __syncthreads();
    if (warp == 0) {
        int na = 0, nf = 0, nc = 0;
        for (int e0 = 0; e0 < a.E; e0 += 32) {
            const int e = e0 + lane, c = e < a.E ? count[e] : 0, ch = (c + 16 * MT - 1) / (16 * MT);
            int sf = c, sc = ch;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int uf = __shfl_up_sync(0xffffffffu, sf, o), uc = __shfl_up_sync(0xffffffffu, sc, o);
                if (lane >= o) { sf += uf; sc += uc; }
            }
            const unsigned met = __ballot_sync(0xffffffffu, c > 0);
            if (e < a.E) place[e] = nf + sf - c;
            if (c > 0) {
                const int j = na + __popc(met & ((1u << lane) - 1u));
                act[j] = (int16_t)e; first[j] = (int16_t)(nf + sf - c); chunk[j] = (int16_t)(nc + sc - ch);
            }
            na += __popc(met);
            nf += __shfl_sync(0xffffffffu, sf, 31);
            nc += __shfl_sync(0xffffffffu, sc, 31);
        }
        if (lane == 0) { n_act = na; first[na] = (int16_t)nf; chunk[na] = (int16_t)nc; }
        __syncwarp();
        // assignments sorted by expert, in ascending order within one: an expert's chunks may fall to different CTAs,
        // which must agree on what is in them
        for (int i0 = 0; i0 < TK; i0 += 32) {
            const int i = i0 + lane;
            const bool in = i < TK;
            const unsigned have = __ballot_sync(0xffffffffu, in);
            if (in) {
                const int e = expert[i];
                const unsigned same = __match_any_sync(have, e);
                const int at = place[e] + __popc(same & ((1u << lane) - 1u));
                sorted[at] = (int16_t)i;
                __syncwarp(have);
                if ((same >> lane) == 1u) place[e] = at + 1;   // the last of them
            }
            __syncwarp();
        }
    }
    fence_async_smem();
    __syncthreads();   // the scratch is free: the ring takes its place

    const int steps = (Kd + V::kStepK - 1) / V::kStepK, chunks = chunk[n_act];
    int S = 1;         // slices of the reduction: enough tasks for an even load, at least four stages each
    if (SECOND)
        while (S < a.max_split && (long long)chunks * RB * S < (long long)V::kTasks * gridDim.x && steps >= 8 * S) S *= 2;
    const long long total = (long long)chunks * RB * S;
    const int t0 = (int)(total * blockIdx.x / gridDim.x) + warp, t1 = (int)(total * (blockIdx.x + 1) / gridDim.x);   // every W-th of these

    auto locate = [&](Cursor& c) {
        while (c.task >= chunk[c.j + 1] * RB * S) ++c.j;
        int r = c.task - chunk[c.j] * RB * S;
        const int nch = chunk[c.j + 1] - chunk[c.j];
        if (nch > 1) { c.ch = r % nch; r /= nch; } else { c.ch = 0; }
        if (S > 1) { c.rb = r % RB; c.s = r / RB; } else { c.rb = r; c.s = 0; }
        c.e = act[c.j];
        c.row0 = c.rb * 8 * NB;
        c.step = steps * c.s / S;
        c.last = steps * (c.s + 1) / S;
    };
    Cursor in{};
    in.task = t0;
    if (t0 < t1) locate(in);
    unsigned char* ring = sm + L.ring + warp * D * V::kStage;
    int in_slot = 0;
    auto issue = [&]() {
        if (in.task < t1) {
            if (lane == 0 && !abort_word) {
                uint64_t* bar = &full[warp * D + in_slot];
                mbar_expect_tx(bar, V::kStage);
#pragma unroll
                for (int b = 0; b < NBOX; ++b)   // beyond the matrix a box is filled with zeros
                    tma_load_2d(ring + in_slot * V::kStage + b * V::kBox, &map, in.step * V::kStepK + b * kBoxK, in.e * N + in.row0, bar);
            }
            if (++in.step == in.last && (in.task += W) < t1) locate(in);
        }
        if (++in_slot == D) in_slot = 0;
    };
#pragma unroll 1
    for (int d = 0; d < D; ++d) issue();

    if (early) {
        pdl_wait();
        pdl_trigger();
    }
    const uint16_t* A = SECOND ? a.g : a.x;
    int slot = 0;
    uint32_t phase = 0;
    Cursor c{};
    for (int task = t0; task < t1; task += W) {
        c.task = task;
        locate(c);
        const int base = first[c.j] + c.ch * 16 * MT, m_here = min(16 * MT, first[c.j + 1] - base);
        // The second product takes the intermediate as high + low part.  While its tokens fill no more than half of
        // the tile's rows, the low parts are the other half; beyond that they take products of their own.
        constexpr int half = 8 * MT;
        const bool packed = SECOND && m_here <= half, two_pass = SECOND && !packed;
        const int rows_used = packed ? half + m_here : m_here;
        const uint32_t low = (uint32_t)TK * (uint32_t)Kd;
        uint32_t off[2 * MT];   // element offset of the row in A; kNoRow: a row of zeros
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i) {
            const int m = i * 8 + gq;
            const bool lower = packed && i >= MT;
            const int mm = lower ? m - half : m;
            const int as = mm < m_here ? sorted[base + mm] : -1;
            off[i] = as < 0 ? kNoRow : (uint32_t)(SECOND ? as : as % a.T) * (uint32_t)Kd + (lower ? low : 0u);
        }
        constexpr int P = 2 * NBOX;   // 16-byte pieces of a row that one thread holds of a stage
        float acc[MT][NB][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][n][i] = 0.0f;
#pragma unroll 1
        for (; c.step < c.last; ++c.step) {
            const int k0 = c.step * V::kStepK + tq * 16;
            uint4 av[P][2 * MT], al[SECOND && NB > 1 ? P : 1][2 * MT];
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int k = k0 + (p >> 1) * kBoxK + (p & 1) * 8;
#pragma unroll
                for (int i = 0; i < 2 * MT; ++i) {
                    av[p][i] = make_uint4(0, 0, 0, 0);
                    if (off[i] != kNoRow && k < Kd) av[p][i] = *reinterpret_cast<const uint4*>(A + off[i] + k);
                }
            }
            if constexpr (SECOND && NB > 1) {   // at most 8 assignments (NB = 1) are always packed
                if (two_pass) {
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        const int k = k0 + (p >> 1) * kBoxK + (p & 1) * 8;
#pragma unroll
                        for (int i = 0; i < 2 * MT; ++i) {
                            al[p][i] = make_uint4(0, 0, 0, 0);
                            if (off[i] != kNoRow && k < Kd) al[p][i] = *reinterpret_cast<const uint4*>(A + off[i] + low + k);
                        }
                    }
                }
            }
            if (!abort_word && !mbar_wait_bounded(&full[warp * D + slot], phase)) {
                abort_word = 1;
                atomicOr(&g_few_flags, 1);
            }
#pragma unroll
            for (int p = 0; p < P; ++p) {
                uint4 wv[NB];
#pragma unroll
                for (int n = 0; n < NB; ++n)
                    wv[n] = *reinterpret_cast<const uint4*>(ring + slot * V::kStage + (p >> 1) * V::kBox + (n * 8 + gq) * 128 +
                                                            (((2 * tq + (p & 1)) ^ gq) * 16));
                auto products = [&](const uint4 (&v)[2 * MT]) {
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        if (m > 0 && m * 16 >= rows_used) break;
#pragma unroll
                        for (int n = 0; n < NB; ++n) mma16816(acc[m][n], v[2 * m].x, v[2 * m + 1].x, v[2 * m].y, v[2 * m + 1].y, wv[n].x, wv[n].y);
#pragma unroll
                        for (int n = 0; n < NB; ++n) mma16816(acc[m][n], v[2 * m].z, v[2 * m + 1].z, v[2 * m].w, v[2 * m + 1].w, wv[n].z, wv[n].w);
                    }
                };
                products(av[p]);
                if constexpr (SECOND && NB > 1) {
                    if (two_pass) products(al[p]);
                }
            }
            __syncwarp();   // the stage has been read by the whole warp
            issue();
            if (++slot == D) { slot = 0; phase ^= 1u; }
        }
        // Results straight from the accumulators: thread (gq, tq) has weight rows 2 tq and 2 tq + 1 of each block and
        // the tokens gq of each group of eight; the low parts' shares lie in the same thread.
        const bool direct = SECOND && S == 1 && a.K == 1;
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i) {
            const int m = i * 8 + gq;
            if (m >= m_here) continue;
            const int as = sorted[base + m];
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const int row = c.row0 + n * 8 + tq * 2;
                if (row >= N) continue;
                float2 v = make_float2(acc[i >> 1][n][(i & 1) * 2], acc[i >> 1][n][(i & 1) * 2 + 1]);
                if (packed && i < MT) {
                    v.x += acc[(i + MT) >> 1][n][((i + MT) & 1) * 2];
                    v.y += acc[(i + MT) >> 1][n][((i + MT) & 1) * 2 + 1];
                }
                if (!SECOND) {
                    v.x = 0.5f * v.x * erfcf(-0.70710678118654752f * v.x);
                    v.y = 0.5f * v.y * erfcf(-0.70710678118654752f * v.y);
                    const uint32_t hi = cvt_bf16x2(v);
                    uint16_t* g = a.g + (size_t)as * a.F + row;
                    *reinterpret_cast<uint32_t*>(g) = hi;
                    *reinterpret_cast<uint32_t*>(g + (size_t)TK * a.F) = cvt_bf16x2(make_float2(v.x - bf16_lo(hi), v.y - bf16_hi(hi)));
                } else if (direct) {
                    const float f = a.weighted ? score[as] : 1.0f;
                    *reinterpret_cast<uint32_t*>(a.out + (size_t)as * a.H + row) = cvt_bf16x2(make_float2(v.x * f, v.y * f));
                } else {
                    *reinterpret_cast<float2*>(a.part + ((size_t)c.s * TK + as) * a.H + row) = v;
                }
            }
        }
        if (SECOND && !direct) {   // the last task of these columns to arrive adds them all up, in a fixed order
            __threadfence();
            __syncwarp();
            int last = 0;
            if (lane == 0) last = atomicAdd(&a.arrived[c.rb], 1) == chunks * S - 1;
            if (__shfl_sync(0xffffffffu, last, 0)) {
                __threadfence();
                constexpr int Q = 2 * NB;   // lanes that share a token's 8 * NB columns
                const int row = c.row0 + (lane % Q) * 4;
                if (row < N) {
                    for (int t = lane / Q; t < a.T; t += 32 / Q) {
                        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                        for (int k = 0; k < a.K; ++k) {
                            const float* p = a.part + ((size_t)k * a.T + t) * a.H + row;
                            float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
                            for (int s = 0; s < S; ++s) {
                                const float4 z = __ldcg(reinterpret_cast<const float4*>(p + (size_t)s * TK * a.H));
                                y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
                            }
                            const float f = a.weighted ? score[k * a.T + t] : 1.0f;
                            v.x = fmaf(f, y.x, v.x); v.y = fmaf(f, y.y, v.y); v.z = fmaf(f, y.z, v.z); v.w = fmaf(f, y.w, v.w);
                        }
                        *reinterpret_cast<uint2*>(a.out + (size_t)t * a.H + row) =
                            make_uint2(cvt_bf16x2(make_float2(v.x, v.y)), cvt_bf16x2(make_float2(v.z, v.w)));
                    }
                }
                __syncwarp();
            }
        }
    }
    // After a wait that was given up copies may still be on their way into this CTA's shared memory: it stays for a
    // millisecond, hundreds of times their latency, before it leaves.
    __syncthreads();
    if (abort_word)
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
}

struct FewPlan { size_t off_g, off_part, off_arrived, total; int max_split; };
FewPlan plan_few(const locmoe_shape_t& s, int F, int K) {
    FewPlan p{};
    const size_t TK = (size_t)s.T * K;
    // slices only pay while there are few tasks, that is few assignments: at most 512 rows of partial sums for them
    p.max_split = 1;
    while (p.max_split < kMaxSplit && TK * p.max_split * 2 <= 512) p.max_split *= 2;
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    p.off_g = 0;
    p.off_part = up(2 * TK * F * 2);
    p.off_arrived = p.off_part + up(p.max_split * TK * s.H * 4);
    p.total = p.off_arrived + up((size_t)(s.H + 7) / 8 * 4);
    return p;
}

template <class V>
int run_few(const FewArgs& a, cudaStream_t st) {
    const Smem L = layout<V>(a.T * a.K, a.E);
    static bool done_dev[64] = {false};   // the attribute is per device
    int dev = 0;
    cudaGetDevice(&dev);
    if (!done_dev[dev & 63]) {
        const int most = layout<V>(kMaxTokens * kMaxK, kMaxExperts).total;
        if (cudaFuncSetAttribute(moe_few_kernel<V, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) != cudaSuccess ||
            cudaFuncSetAttribute(moe_few_kernel<V, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) != cudaSuccess) {
            cudaGetLastError();
            return LOCMOE_ERR_CUDA;
        }
        done_dev[dev & 63] = true;
    }
    CUtensorMap m1, m2;
    const uint64_t d1[2] = {(uint64_t)a.H, (uint64_t)a.E * a.F}, d2[2] = {(uint64_t)a.F, (uint64_t)a.E * a.H};
    if (!make_map(&m1, a.w_in, 2, d1, 8 * V::NB) || !make_map(&m2, a.w_out, 2, d2, 8 * V::NB)) return LOCMOE_ERR_CUDA;
    const dim3 grid(sm_count());
    const int rc = launch_pdl(moe_few_kernel<V, false>, grid, dim3(V::kThreads), L.total, st, m1, a);
    if (rc) return rc;
    return launch_pdl(moe_few_kernel<V, true>, grid, dim3(V::kThreads), L.total, st, m2, a);
}

}  // namespace

size_t few_ws_bytes(const locmoe_shape_t& s, int F, int K) { return plan_few(s, F, K).total; }

int launch_moe_few(const locmoe_shape_t& s, const void* x, const float* eps, int K, int F, const void* w_in, const void* w_out,
                   int weighted, int32_t* idx_k, float* w_k, void* out, void* ws, cudaStream_t st) {
    const FewPlan p = plan_few(s, F, K);
    unsigned char* base = static_cast<unsigned char*>(ws);
    const FewArgs a{static_cast<const uint16_t*>(x), eps, static_cast<const uint16_t*>(w_in), static_cast<const uint16_t*>(w_out), idx_k,
                    w_k, static_cast<uint16_t*>(out), reinterpret_cast<uint16_t*>(base + p.off_g),
                    reinterpret_cast<float*>(base + p.off_part), reinterpret_cast<int32_t*>(base + p.off_arrived), s.T, s.H, s.E, K, F,
                    p.max_split, weighted};
    if (s.T * K <= 8) return run_few<Variant<16, 1, 1, 2, 3, 8, 2>>(a, st);
    if (s.T <= 16) return run_few<Variant<12, 1, 2, 2, 4, 48, 1>>(a, st);
    return run_few<Variant<12, 2, 4, 1, 4, 48, 1>>(a, st);
}

int read_few_flags(int* out, cudaStream_t st) {
    if (cudaMemcpyFromSymbolAsync(out, g_few_flags, sizeof(int), 0, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaStreamSynchronize(st) != cudaSuccess) {
        cudaGetLastError();
        return LOCMOE_ERR_CUDA;
    }
    return LOCMOE_OK;
}

}  // namespace locmoe
