// A whole MoE layer for a few tokens (decoding): the router and the first product of the experts, then the second
// product and the gate-weighted sum.  Two launches up to 8 tokens; beyond that the router has one of its own.
//
//   G_i = ReLU(mean_i x + eps_i),  p = softmax(G),  the K largest;   out_t = sum_c p_{t,c} W_out[e] GeLU(W_in[e] x_t)
//
// Bound by the weights of the experts that the tokens meet (4 F H bytes each), every one of which is read once.  A task
// is a block of R weight rows of one expert (and, in the second product, one of S slices of the reduction).  A CTA has
// independent groups, each with its own ring of stages that a producer warp fills with a TMA box of weights and the
// tokens' pieces of the same k (bulk copies, one a row) without a pause between tasks; the other warps multiply.
// The tokens travel with the weights because a load that a multiplying warp issues itself queues behind the ring's
// own (4000 cycles at a full ring: 2.9 against 6.5 TB/s on a stream of rows of 10240).
// Both launches are programmatic: the CTAs of one take the SMs over as those of the one before leave them.  (One
// cooperative kernel with a wait of the grid in between, behind a router launch of its own, took 37 us for one token where
// two launches with the router inside took 36; without the router launch it was not tried.)
// The products run on mma.sync m16n8k16, tokens as the 16 rows and weight rows as the 8 columns: at a few tokens an
// expert nothing is gained by larger matrix instructions.  The order of k inside a stage is chosen so that a thread's
// fragments of both operands are 16 contiguous bytes of a row (the same permutation on both sides), which the weight
// tiles' 128-byte swizzle and the token rows' pitch give without bank conflicts.
#include "common.cuh"
#include "tensor_map.cuh"

namespace locmoe {

namespace {

constexpr int kMaxTokens = LOCMOE_FEW_MAX_TOKENS, kMaxExperts = 1024, kMaxK = 8, kMaxSplit = 8;
constexpr int kMostSmem = 226 << 10;   // of the 227 KB that a CTA can have
// Up to here every CTA routes all tokens itself, beyond that a kernel of its own does (H = 2560, F = 10240, E = 32: one token
// 35.2 us against 35.9, 8 tokens 129.2 / 131.6, 9 tokens 147.4 / 147.5, 16 tokens 220.5 / 217.2).
constexpr int kInlineTokens = 8;
constexpr int kBoxK = 64;          // k of one TMA box: 128 bytes of a row

__device__ int g_few_flags = 0;    // bit 0: a bounded wait gave up

struct FewArgs {
    const uint16_t* x; const float* eps; const uint16_t* w_in; const uint16_t* w_out;
    int32_t* idx_k; float* w_k; uint16_t* out;
    uint16_t* g;        // [2][K * T][F] GeLU(W_in x) as the sum of two bf16 values: the rounded value and what rounding left
    float* part;        // [S][K * T][H] slices of the second product
    int32_t* arrived;   // [H / 8] tasks of the second product that have left their slice, by column block
    int T, H, E, K, F, max_split, weighted, inline_router;
};

// A variant: GR groups, each with a ring, a producer warp and multiplying warps, WR along the weight rows and WK along
// k; NB blocks of 8 weight rows a warp, BW boxes of 64 k a warp and stage, MT tiles of 16 tokens; the shared memory of
// a CTA; the tasks an SM that the second product's reduction is sliced for.  A group works on every GR-th task by itself,
// so that one group's sums and stores run beside the others' products.
constexpr int kMaxStages = 8;   // of a group's ring
template <int GR_, int WR_, int WK_, int NB_, int BW_, int MT_, int SMEM_, int WANT_>
struct Variant {
    static constexpr int GR = GR_, WR = WR_, WK = WK_, NB = NB_, BW = BW_, MT = MT_, kSmem = SMEM_, kWant = WANT_;
    static constexpr int kMulWarps = WR * WK, kThreads = 32 * GR * (kMulWarps + 1);
    static constexpr int kBoxes = WK * BW;
    static constexpr int R = 8 * NB * WR, kStepK = kBoxK * kBoxes;      // weight rows of a task, k of a stage
    static constexpr int kBox = R * 128, kWeights = kBoxes * kBox;      // bytes of one box and of a stage's weights
    static constexpr int kPitch = kStepK * 2 + 16;                      // of a token's row: an odd number of 16-byte banks
    static constexpr int kRed = WK > 1 ? WK * 16 * MT * R : 0;          // floats of a group's strip of partial sums
};

struct Smem {   // offsets of the dynamic shared memory, from its first 1024-byte boundary on
    int ring, red, full, empty, expert, sorted, score, act, first, chunk, total;
    int stage, stages;   // bytes of a stage, stages of a group's ring
};
__host__ __device__ constexpr int round_up(int n, int to) { return (n + to - 1) / to * to; }
// rows: token rows of a stage at most.  The ring takes what the rest leaves.
template <class V>
__host__ __device__ inline Smem layout(int TK, int E, int rows) {
    Smem s{};
    const int most = TK < E ? TK : E, red = V::GR * V::kRed * 4;
    s.stage = round_up(V::kWeights + rows * V::kPitch, 1024);
    const int tail = red + 16 * V::GR * kMaxStages + round_up(2 * TK, 16) * 2 + round_up(4 * TK, 16) + round_up(2 * most, 16) +
                     2 * round_up(2 * most + 2, 16) + 1024 /* alignment slack */;
    s.stages = (V::kSmem - tail) / s.stage / V::GR;
    if (s.stages > kMaxStages) s.stages = kMaxStages;
    // the counters of the sort (2 E ints) lie where the ring is later
    s.ring = 0;
    s.red = round_up(V::GR * s.stages * s.stage > 2 * E * 4 ? V::GR * s.stages * s.stage : 2 * E * 4, 16);
    s.full = s.red + red;
    s.empty = s.full + 8 * V::GR * kMaxStages;
    s.expert = s.empty + 8 * V::GR * kMaxStages;              // int16 [TK]  expert of assignment a = c * T + t
    s.sorted = s.expert + round_up(2 * TK, 16);       // int16 [TK]  assignments by expert
    s.score = s.sorted + round_up(2 * TK, 16);        // float [TK]
    s.act = s.score + round_up(4 * TK, 16);           // int16 [most]      experts met
    s.first = s.act + round_up(2 * most, 16);         // int16 [most + 1]  their first entry of `sorted`
    s.chunk = s.first + round_up(2 * most + 2, 16);   // int16 [most + 1]  their first chunk of 16 * MT tokens
    s.total = s.chunk + round_up(2 * most + 2, 16) + 1024;
    return s;
}

__device__ __forceinline__ uint4 ld_shared(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Sum of `n` consecutive bf16 values from `p`, of which this lane takes every `of`-th piece of EL from `sub` on.
template <int EL>
__device__ __forceinline__ float sum_pieces(const uint16_t* p, int n, int sub, int of) {
    float s0 = 0.0f, s1 = 0.0f;
#pragma unroll 10
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

__device__ __forceinline__ int add_acq_rel(int* p) {
    int old;
    asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(old) : "l"(p) : "memory");
    return old;
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// global -> shared bulk copy by shared-memory address (16-byte aligned, a multiple of 16 bytes)
__device__ __forceinline__ void bulk_row(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// Bounded wait that also ends once another warp has given up.
__device__ __forceinline__ bool wait_or_abort(uint32_t bar, uint32_t parity, volatile int* abort_word) {
    for (uint32_t i = 0; i < (1u << 17); ++i) {   // about half a second
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 15u) == 15u && *abort_word) return false;
    }
    *abort_word = 1;
    atomicOr(&g_few_flags, 1);
    return false;
}
// Router for `nt` tokens from `b0` on, by a CTA of W warps; G: room for their logits.  The threads share out the (token,
// expert) pairs, several lanes a pair while there are threads for that; then a warp a token takes the softmax and the
// K largest and hands each choice to `put(c, t, expert, score)`.
template <int W, typename Put>
__device__ __forceinline__ void route_tokens(const FewArgs& a, int b0, int nt, float* logits, Put put) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = a.H / a.E, el = g % 8 == 0 ? 8 : g % 2 == 0 ? 2 : 1, pairs = nt * a.E;
    const float inv_g = 1.0f / (float)g;
    int lanes = 1;
    while (lanes < 32 && lanes * 2 * pairs <= 32 * W && lanes * 2 * el <= g) lanes *= 2;
    const int sub = lane & (lanes - 1);
    for (int p0 = 0; p0 < pairs; p0 += 32 * W / lanes) {   // a round is the same for all lanes: the sums are shuffled
        const int p = p0 + threadIdx.x / lanes;
        const int t = p / a.E, i = p - t * a.E;
        float s = 0.0f;
        if (p < pairs) {
            const uint16_t* from = a.x + (size_t)(b0 + t) * a.H + (size_t)i * g;
            s = el == 8 ? sum_pieces<8>(from, g, sub, lanes) : el == 2 ? sum_pieces<2>(from, g, sub, lanes) : sum_pieces<1>(from, g, sub, lanes);
        }
        for (int o = 1; o < lanes; o *= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (p < pairs && sub == 0) logits[p] = fmaxf(fmaf(s, inv_g, a.eps ? a.eps[i] : 0.0f), 0.0f);   // a NaN logit counts as 0
    }
    __syncthreads();
    for (int t = warp; t < nt; t += W) {
        float* G = logits + t * a.E;
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
                put(c, b0 + t, bi, expf(best - top) / z);
            }
            __syncwarp();
        }
    }
}

constexpr int kRouterThreads = 256;
__global__ void __launch_bounds__(kRouterThreads) few_router_kernel(const FewArgs a) {   // a CTA a token
    __shared__ float G[kMaxExperts];
    pdl_wait();
    pdl_trigger();
    route_tokens<kRouterThreads / 32>(a, blockIdx.x, 1, G, [&](int c, int t, int e, float w) {
        a.idx_k[c * a.T + t] = e;
        a.w_k[c * a.T + t] = w;
    });
}

// What one product is about: weight rows, reduction length, and how its tasks are cut.
struct Product { int N, Kd, RB, S, stages, t0, t1; };
__device__ __forceinline__ int token_of(int as, int T) {   // as mod T, for as < 8 T
    while (as >= T) as -= T;
    return as;
}
struct Task { int row0, rb, s, base, m, step; };

template <class V>
__global__ void __launch_bounds__(V::kThreads, 1)
moe_few_kernel(const __grid_constant__ CUtensorMap map, const FewArgs a, const int second) {
    constexpr int NB = V::NB, MT = V::MT, WK = V::WK, BW = V::BW, R = V::R, GR = V::GR, kThreads = V::kThreads;
    extern __shared__ unsigned char raw[];
    unsigned char* sm = reinterpret_cast<unsigned char*>(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);   // the swizzle repeats every 1024 bytes
    const int TK = a.T * a.K;
    const Smem L = layout<V>(TK, a.E, 2 * min(a.T, 16 * MT));
    int16_t* expert = reinterpret_cast<int16_t*>(sm + L.expert);
    int16_t* sorted = reinterpret_cast<int16_t*>(sm + L.sorted);
    float* score = reinterpret_cast<float*>(sm + L.score);
    int16_t* act = reinterpret_cast<int16_t*>(sm + L.act);
    int16_t* first = reinterpret_cast<int16_t*>(sm + L.first);
    int16_t* chunk = reinterpret_cast<int16_t*>(sm + L.chunk);
    int* count = reinterpret_cast<int*>(sm + L.ring);
    int* place = count + a.E;
    __shared__ int n_act;
    __shared__ volatile int abort_word;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid < GR * L.stages) {
        mbar_init(reinterpret_cast<uint64_t*>(sm + L.full) + tid, 1);
        mbar_init(reinterpret_cast<uint64_t*>(sm + L.empty) + tid, V::kMulWarps);
    }
    if (tid == 0) abort_word = 0;
    mbar_init_fence();
    if (tid == 0) prefetch_map(&map);
    pdl_wait();
    pdl_trigger();
    if (!second) {
        for (int i = blockIdx.x * kThreads + tid; i < (a.H + 7) / 8; i += gridDim.x * kThreads) a.arrived[i] = 0;
    }
    // A handful of tokens every CTA routes for itself: their rows out of L2 cost less than a launch of their own.
    if (a.inline_router && !second) {
        route_tokens<kThreads / 32>(a, 0, a.T, reinterpret_cast<float*>(sm + L.ring), [&](int c, int t, int e, float w) {
            expert[c * a.T + t] = (int16_t)e;
            score[c * a.T + t] = w;
            if (blockIdx.x == 0) { a.idx_k[c * a.T + t] = e; a.w_k[c * a.T + t] = w; }
        });
    } else {
        for (int i = tid; i < TK; i += kThreads) { expert[i] = (int16_t)a.idx_k[i]; score[i] = a.w_k[i]; }
    }
    __syncthreads();
    // The assignments sorted by expert, in ascending order within one: an expert's chunks of 16 * MT tokens may fall to
    // different CTAs, which must agree on what is in them.
    if (TK <= 32 && a.T <= 16 * MT) {   // one assignment a lane, one chunk an expert; every warp does it for itself and writes the same
        const int e = lane < TK ? expert[lane] : 0x7fff;
        const unsigned same = __match_any_sync(0xffffffffu, e), below = (1u << lane) - 1u;
        const unsigned heads = __ballot_sync(0xffffffffu, lane < TK && (same & below) == 0);
        int less = 0, j = 0;   // assignments and experts met with a lower expert index
        for (int i = 0; i < TK; ++i) {
            const int o = __shfl_sync(0xffffffffu, e, i);
            less += o < e;
            j += o < e && ((heads >> i) & 1u);
        }
        if (lane < TK) {
            sorted[less + __popc(same & below)] = (int16_t)lane;
            if ((same & below) == 0) { act[j] = (int16_t)e; first[j] = (int16_t)less; chunk[j] = (int16_t)j; }
        }
        if (lane == 0) { n_act = __popc(heads); first[n_act] = (int16_t)TK; chunk[n_act] = (int16_t)n_act; }
        fence_async_smem();
        __syncthreads();
    } else {
        for (int i = tid; i < a.E; i += kThreads) count[i] = 0;
        __syncthreads();
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
    }

    const int chunks = chunk[n_act];
    Product p;
    p.N = second ? a.H : a.F;
    p.Kd = second ? a.F : a.H;
    p.RB = (p.N + R - 1) / R;
    const int steps = (p.Kd + V::kStepK - 1) / V::kStepK;
    p.S = 1;                // slices of the reduction: enough tasks for an even load, at least four stages each
    if (second)
        while (p.S < a.max_split && chunks * p.RB * p.S < V::kWant * (int)gridDim.x && steps >= 8 * p.S) p.S *= 2;
    p.stages = (steps + p.S - 1) / p.S;   // of a task; those beyond K are zeros
    const int total = chunks * p.RB * p.S, share = total / (int)gridDim.x, more = total - share * (int)gridDim.x;
    p.t0 = blockIdx.x * share + min((int)blockIdx.x, more);
    p.t1 = p.t0 + share + ((int)blockIdx.x < more ? 1 : 0);

    int j = 0;              // tasks come by expert, slice, row block and chunk: the chunks of a row block follow each other
    auto locate = [&](int task) {
        while (task >= chunk[j + 1] * p.RB * p.S) ++j;
        int r = task - chunk[j] * p.RB * p.S, ch = 0;
        const int nch = chunk[j + 1] - chunk[j];
        Task t;
        if (nch > 1) { ch = r % nch; r /= nch; }
        t.rb = r; t.s = 0;
        if (p.S > 1) { t.rb = r % p.RB; t.s = r / p.RB; }
        t.row0 = t.rb * R;
        t.base = first[j] + ch * 16 * MT;
        t.m = min(16 * MT, first[j + 1] - t.base);
        t.step = t.s * p.stages;
        return t;
    };
    const int group = warp / (V::kMulWarps + 1), gw = warp - group * (V::kMulWarps + 1);
    const uint32_t ring = smem_u32(sm + L.ring) + group * L.stages * L.stage;
    const uint32_t full = smem_u32(sm + L.full) + group * L.stages * 8, empty = smem_u32(sm + L.empty) + group * L.stages * 8;
    int slot = 0;
    uint32_t phase = 0;
    bool alive = true;      // no wait has been given up
    auto next_slot = [&]() {
        if (++slot == L.stages) { slot = 0; phase ^= 1u; }
    };

    if (second) asm volatile("fence.proxy.async;" ::: "memory");   // the first product's stores, read by bulk copies here
    if (gw == V::kMulWarps) {   // ---- producer: a lane a box of weights, a lane a token row ----
        constexpr int kMine = (32 * MT + 31) / 32;   // token rows of a lane: at most 2 * 16 * MT in all
        const uint16_t* src[kMine];
        int w_row = 0, rows = 0;
        auto enter = [&](const Task& t) {   // what stays the same over a task's stages
            w_row = act[j] * p.N + t.row0;
            rows = second ? 2 * t.m : t.m;
#pragma unroll
            for (int q = 0; q < kMine; ++q) {
                const int i = lane + 32 * q;
                if (i < rows) {
                    const bool lower = i >= t.m;
                    const int as = sorted[t.base + (lower ? i - t.m : i)];
                    src[q] = (second ? a.g + (size_t)(as + (lower ? TK : 0)) * p.Kd : a.x + (size_t)token_of(as, a.T) * p.Kd) + t.step * V::kStepK;
                }
            }
        };
        for (int task = p.t0 + group; task < p.t1 && alive; task += GR) {
            const Task t = locate(task);
            enter(t);
            int k = t.step * V::kStepK;
#pragma unroll 1
            for (int i = 0; i < p.stages; ++i, k += V::kStepK) {
                if (!wait_or_abort(empty + slot * 8, phase ^ 1u, &abort_word)) { alive = false; break; }
                const uint32_t dst = ring + slot * L.stage, bar = full + slot * 8, bytes = 2 * max(0, min(V::kStepK, p.Kd - k));
                if (lane == 0) mbar_expect_tx(bar, V::kWeights + rows * bytes);
                __syncwarp();
                if (lane < V::kBoxes) tma_load_2d(dst + lane * V::kBox, &map, k + lane * kBoxK, w_row, bar);   // beyond the matrix: zeros
#pragma unroll
                for (int q = 0; q < kMine; ++q) {
                    if (lane + 32 * q < rows && bytes) bulk_row(dst + V::kWeights + (lane + 32 * q) * V::kPitch, src[q], bytes, bar);
                    src[q] += V::kStepK;
                }
                next_slot();
            }
        }
    } else {                    // ---- the other warps of the group multiply ----
        const int gt = gw * 32 + lane, gq = lane >> 2, tq = lane & 3, wk = gw % WK, wr = gw / WK;
        auto group_sync = [&]() { asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(V::kMulWarps * 32) : "memory"); };
        // this thread's bytes of a stage: weight row gq of each block, 16-byte pieces 2 tq and 2 tq + 1
        const uint32_t wrow = wk * BW * V::kBox + (wr * 8 * NB + gq) * 128, even = wrow + ((2 * tq) ^ gq) * 16, odd = wrow + ((2 * tq + 1) ^ gq) * 16;
        const bool direct = second && p.S == 1 && a.K == 1;
        int turn = 0;
        for (int task = p.t0 + group; task < p.t1; task += GR) {
            const Task t = locate(task);
            // The second product takes the intermediate as high + low part.  While its tokens fill no more than half
            // of the tile's rows, the low parts are the other half; beyond that they take products of their own.
            constexpr int half = 8 * MT;
            const bool packed = second && t.m <= half, two_pass = second && !packed;
            const int rows_used = packed ? half + t.m : t.m;
            // Rows of the tile beyond the tokens repeat a token: a row enters no other row's results.
            uint32_t at[2 * MT];
#pragma unroll
            for (int i = 0; i < 2 * MT; ++i) {
                const bool lower = packed && i >= MT;
                const int row = min((lower ? i - MT : i) * 8 + gq, t.m - 1) + (lower ? t.m : 0);
                at[i] = V::kWeights + row * V::kPitch + wk * BW * 128 + tq * 32;
            }
            float acc[MT][NB][4];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[m][n][i] = 0.0f;
            int left = p.Kd - t.step * V::kStepK - wk * BW * kBoxK - tq * 16;   // from this thread's first k to the end of the rows
#pragma unroll 1
            for (int i = 0; i < p.stages; ++i) {
                if (alive) alive = wait_or_abort(full + slot * 8, phase, &abort_word);
                const uint32_t stage = ring + slot * L.stage;
#pragma unroll
                for (int c = 0; c < 2 * BW; ++c) {
                    uint4 wv[NB], av[2 * MT];
#pragma unroll
                    for (int n = 0; n < NB; ++n) wv[n] = ld_shared(stage + (c >> 1) * V::kBox + n * 1024 + ((c & 1) ? odd : even));
                    auto tokens = [&](uint32_t more) {   // beyond K zeros: the weights' zeros alone would keep a NaN
#pragma unroll
                        for (int q = 0; q < 2 * MT; ++q) {
                            av[q] = ld_shared(stage + at[q] + more + (c >> 1) * 128 + (c & 1) * 16);
                            if ((c >> 1) * kBoxK + (c & 1) * 8 >= left) av[q] = make_uint4(0, 0, 0, 0);
                        }
                    };
                    auto products = [&]() {
#pragma unroll
                        for (int m = 0; m < MT; ++m) {
                            if (m > 0 && m * 16 >= rows_used) break;
#pragma unroll
                            for (int n = 0; n < NB; ++n) mma16816(acc[m][n], av[2 * m].x, av[2 * m + 1].x, av[2 * m].y, av[2 * m + 1].y, wv[n].x, wv[n].y);
#pragma unroll
                            for (int n = 0; n < NB; ++n) mma16816(acc[m][n], av[2 * m].z, av[2 * m + 1].z, av[2 * m].w, av[2 * m + 1].w, wv[n].z, wv[n].w);
                        }
                    };
                    tokens(0);
                    products();
                    if (two_pass) {
                        tokens(t.m * V::kPitch);
                        products();
                    }
                }
                __syncwarp();   // the stage has been read by the whole warp
                if (lane == 0) mbar_arrive(empty + slot * 8);
                left -= V::kStepK;
                next_slot();
            }
            // A result pair: weight rows `row` and `row` + 1 of token m of the chunk.
            auto emit = [&](int m, int row, float2 v) {
                const int as = sorted[t.base + m];
                if (!second) {
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
                    *reinterpret_cast<float2*>(a.part + ((size_t)t.s * TK + as) * a.H + row) = v;
                }
            };
            if constexpr (WK > 1) {   // the shares of the warps along k, added in warp order; then the low parts' rows
                float* red = reinterpret_cast<float*>(sm + L.red) + group * V::kRed;
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int n = 0; n < NB; ++n) {
                        float* r = red + ((wk * 16 * MT) + m * 16 + gq) * R + (wr * NB + n) * 8 + tq * 2;
                        *reinterpret_cast<float2*>(r) = make_float2(acc[m][n][0], acc[m][n][1]);
                        *reinterpret_cast<float2*>(r + 8 * R) = make_float2(acc[m][n][2], acc[m][n][3]);
                    }
                group_sync();
                for (int o = gt; o < t.m * (R / 2); o += V::kMulWarps * 32) {
                    const int m = o / (R / 2), r = o % (R / 2) * 2;
                    if (t.row0 + r >= p.N) continue;
                    float2 v = make_float2(0.0f, 0.0f), l = v;
#pragma unroll
                    for (int w = 0; w < WK; ++w) {
                        const float2 z = *reinterpret_cast<const float2*>(red + (w * 16 * MT + m) * R + r);
                        v.x += z.x; v.y += z.y;
                        if (packed) {
                            const float2 y = *reinterpret_cast<const float2*>(red + (w * 16 * MT + half + m) * R + r);
                            l.x += y.x; l.y += y.y;
                        }
                    }
                    emit(m, t.row0 + r, make_float2(v.x + l.x, v.y + l.y));
                }
                group_sync();   // also: the strip may be written again
            } else {          // thread (gq, tq) has the tokens gq of each eight and weight rows 2 tq, 2 tq + 1 of each block
#pragma unroll
                for (int i = 0; i < 2 * MT; ++i) {
                    const int m = i * 8 + gq;
                    if (m >= t.m) continue;
#pragma unroll
                    for (int n = 0; n < NB; ++n) {
                        const int row = t.row0 + (wr * NB + n) * 8 + tq * 2;
                        if (row >= p.N) continue;
                        float2 v = make_float2(acc[i >> 1][n][(i & 1) * 2], acc[i >> 1][n][(i & 1) * 2 + 1]);
                        if (packed && i < MT) {
                            v.x += acc[(i + MT) >> 1][n][((i + MT) & 1) * 2];
                            v.y += acc[(i + MT) >> 1][n][((i + MT) & 1) * 2 + 1];
                        }
                        emit(m, row, v);
                    }
                }
            }
            // The last task to arrive at a warp's columns adds them all up, in a fixed order.  One lane's acquire-release
            // addition orders the group's stores before it (they are behind a barrier) and the sums after it; the warps
            // along k take turns, since it costs the one that does it a round trip to L2.
            if (second && !direct && (WK == 1 || wk == turn)) {
                __syncwarp();
                int last = 0;
                if (lane == 0) last = add_acq_rel(&a.arrived[t.rb * V::WR + wr]) == chunks * p.S - 1;
                last = __shfl_sync(0xffffffffu, last, 0);
                __syncwarp();   // a shuffle orders no memory: what lane 0 has acquired, the other lanes read behind this
                if (last) {
                    constexpr int Q = 2 * NB;   // lanes that share a token's 8 * NB columns
                    const int row = t.row0 + wr * 8 * NB + (lane % Q) * 4;
                    if (row < p.N) {
                        for (int tok = lane / Q; tok < a.T; tok += 32 / Q) {
                            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                            for (int k = 0; k < a.K; ++k) {
                                const float* from = a.part + ((size_t)k * a.T + tok) * a.H + row;
                                float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
                                for (int s = 0; s < p.S; ++s) {
                                    const float4 z = __ldcg(reinterpret_cast<const float4*>(from + (size_t)s * TK * a.H));
                                    y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
                                }
                                const float f = a.weighted ? score[k * a.T + tok] : 1.0f;
                                v.x = fmaf(f, y.x, v.x); v.y = fmaf(f, y.y, v.y); v.z = fmaf(f, y.z, v.z); v.w = fmaf(f, y.w, v.w);
                            }
                            *reinterpret_cast<uint2*>(a.out + (size_t)tok * a.H + row) =
                                make_uint2(cvt_bf16x2(make_float2(v.x, v.y)), cvt_bf16x2(make_float2(v.z, v.w)));
                        }
                    }
                    __syncwarp();
                }
            }
            turn = turn + 1 == WK ? 0 : turn + 1;
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
    // at most 512 rows of partial sums for the slices: with many assignments there are tasks enough, and the sums would
    // be a workspace of many times the tokens (H = 1024, F = 1024, E = 4, T = 128, K = 2 would take 57 us instead of 66)
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
    static bool done_dev[64] = {false};   // the attribute is per device
    int dev = 0;
    cudaGetDevice(&dev);
    if (!done_dev[dev & 63]) {
        if (cudaFuncSetAttribute(moe_few_kernel<V>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem) != cudaSuccess) {
            cudaGetLastError();
            return LOCMOE_ERR_CUDA;
        }
        done_dev[dev & 63] = true;
    }
    CUtensorMap m1, m2;
    const uint64_t d1[2] = {(uint64_t)a.H, (uint64_t)a.E * a.F}, d2[2] = {(uint64_t)a.F, (uint64_t)a.E * a.H};
    if (!make_map(&m1, a.w_in, 2, d1, V::R) || !make_map(&m2, a.w_out, 2, d2, V::R)) return LOCMOE_ERR_CUDA;
    int rc = LOCMOE_OK;
    if (!a.inline_router && (rc = launch_pdl(few_router_kernel, dim3(a.T), dim3(kRouterThreads), 0, st, a))) return rc;
    const dim3 grid(sm_count()), block(V::kThreads);
    const int smem = layout<V>(a.T * a.K, a.E, 2 * (a.T < 16 * V::MT ? a.T : 16 * V::MT)).total;
    if ((rc = launch_pdl(moe_few_kernel<V>, grid, block, smem, st, m1, a, 0))) return rc;
    return launch_pdl(moe_few_kernel<V>, grid, block, smem, st, m2, a, 1);
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
                    p.max_split, weighted, s.T <= kInlineTokens};
    // Which variant: measured on H = 2560, F = 10240, E = 32 (us), beside H = 1024, F = 1024, E = 4 where it says so.
    // - Up to 8 assignments a task of 16 weight rows, its reduction shared out over four warps: few tasks, so a short way
    //   through each counts (T = 1, K = 1: 31.4; tasks of 64 rows 31.9, of 128 rows 40.5.  T = 4, K = 2: 133 / 141 / 142).
    //   Beyond, each warp has rows of its own and no sums to meet for (T = 16, K = 1: 260 / 217 / 231).
    // - Tiles of 32 tokens and 128 rows where experts with more than 16 tokens are common and the tasks are still many:
    //   T = 128, K = 2 684 against 849 with tiles of 16 and 64 rows, whose second chunk of tokens takes the weights
    //   through shared memory again; T = 64, K = 2 577 / 629.  With fewer tokens an expert (T = 64, K = 1: 495 / 470) or
    //   fewer tasks (the small layer at T = 128, K = 2: 112 / 66) the smaller tiles win.
    // The slices of the second product (tasks an SM: 1, 2 or 8): each is a pass over the partial sums more, but evens the
    // load out.  A few assignments: 1 (H = 2048, F = 5632, E = 8, one token 18.5 us, with 2 21.2; H = 1560, F = 4104, E = 24,
    // K = 3, one token 26.6 / 31.9).  Tiles of 16 tokens: 2 (13 of those tokens 104 us, with 8 115; 16 tokens of the former
    // 71, with 1 81, with 8 79).  Tiles of 32 tokens differ most in their work: 8 (T = 128, K = 2 680 us, with 2 763).
    if (s.T * K <= 8) return run_few<Variant<3, 1, 4, 2, 1, 1, 220 << 10, 1>>(a, st);
    if (s.T > 16 && (long long)s.T * K >= 4ll * s.E && (long long)s.E * ((F + 127) / 128) >= 4 * sm_count())
        return run_few<Variant<3, 4, 1, 4, 1, 2, 220 << 10, 8>>(a, st);
    return run_few<Variant<4, 4, 1, 2, 1, 1, 220 << 10, 2>>(a, st);
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
