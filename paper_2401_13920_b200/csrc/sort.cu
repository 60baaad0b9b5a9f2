// Tokens sorted by expert and back, without a capacity: the order (stable, by expert), the rows in it, the weighted sum back
// in token order, and the gradients of both, the router's among them.
//
// An assignment v = c * T + t is choice c of token t.  slot[v] is its row: the number of assignments with a lower expert plus
// those of the same expert with a lower v; inv is the inverse.  All kernels but the first move rows and are bound by HBM:
// a warp works on a token (or, with short rows, on several), reads each row it needs once with 16-byte streaming loads and
// writes whole rows; rows that are no multiple of 16 bytes go by two bf16 or one element, more of them in flight (65536 tokens
// of 2560 bf16, two choices, their gradient 259 us, of 2562 338, of 2559 470; of 2560 floats 514, of 2559 657).
#include <initializer_list>

#include "common.cuh"

namespace locmoe {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

// ---- the order: one cluster, counts in shared memory ----
// A warp owns a contiguous run of assignments, a CTA the runs of its 32 warps, the cluster all of them.  Pass 1 ranks each
// assignment among its warp's of the same expert and counts them, without atomics: lanes with the same expert find each
// other by a ballot a bit, the lowest adds.  The counts become first rows by sums over experts, CTAs (through distributed
// shared memory) and warps; pass 2 adds them to the ranks.  131072 assignments by 16 CTAs in 13 us (28 with 8 and match.any, of
// which an SM does one in 60 cycles, in both passes).
constexpr int kPlanThreads = 1024, kPlanWarps = kPlanThreads / 32, kPlanBatch = 8;
constexpr int kPlanRun = 1024;           // assignments a CTA before another is taken, up to 16 (8 where the device has no more)
constexpr size_t plan_smem(int E) { return ((size_t)(kPlanWarps + 2) * E + 32) * sizeof(int); }

__device__ __forceinline__ int ld_cluster(const int* p, int cta) {
    uint32_t ra;
    int v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(ra) : "r"(smem_u32(p)), "r"(cta));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(ra) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Lanes that hold the same key of BITS bits.
template <int BITS>
__device__ __forceinline__ unsigned same_key(int key) {
    unsigned same = 0xffffffffu;
#pragma unroll
    for (int i = 0; i < BITS; ++i) {
        const bool on = (key >> i) & 1;
        const unsigned b = __ballot_sync(0xffffffffu, on);
        same &= on ? b : ~b;
    }
    return same;
}

template <int BITS>
__global__ void __launch_bounds__(kPlanThreads) sort_plan_kernel(const int32_t* __restrict__ idx, int V, int T, int E, int32_t* __restrict__ offsets,
                                                                 int32_t* __restrict__ slot, int32_t* __restrict__ inv, int with_inv,
                                                                 int32_t* __restrict__ load) {
    extern __shared__ int sm[];
    int* tot = sm;              // [E] assignments of this CTA
    int* first = tot + E;       // [E] assignments of this CTA's first choices
    int* scan = first + E;      // [32]
    int* cnt = scan + 32;       // [32][E] by warp: counts, then next row
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, nc = gridDim.x, rank = blockIdx.x;   // the grid is one cluster
    for (int i = threadIdx.x; i < 2 * E + 32 + kPlanWarps * E; i += kPlanThreads) sm[i] = 0;
    __syncthreads();
    pdl_wait();
    pdl_trigger();
    const long long per = (((long long)V + (long long)nc * kPlanWarps - 1) / (nc * kPlanWarps) + 31) & ~31ll;
    const long long lo = min((long long)V, ((long long)rank * kPlanWarps + warp) * per), hi = min((long long)V, lo + per);
    int* mine = cnt + warp * E;
    for (long long b = lo; b < hi; b += 32 * kPlanBatch) {
        int key[kPlanBatch];
#pragma unroll
        for (int i = 0; i < kPlanBatch; ++i) {
            const long long v = b + 32 * i + lane;
            key[i] = v < hi ? __ldg(idx + v) : -1;
        }
#pragma unroll
        for (int i = 0; i < kPlanBatch; ++i) {
            const long long v = b + 32 * i + lane;
            if (b + 32 * i >= hi) break;
            const bool ok = key[i] >= 0 && key[i] < E;
            const unsigned same = same_key<BITS>(ok ? key[i] : E), below = same & ((1u << lane) - 1u);
            const int before = ok ? mine[key[i]] : 0;
            __syncwarp();
            if (ok && below == 0) mine[key[i]] = before + __popc(same);
            if (load && ok && v < T) atomicAdd(first + key[i], 1);
            if (v < hi) slot[v] = before + __popc(below);       // among this warp's
            __syncwarp();
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += kPlanThreads) {
        int sum = 0;
#pragma unroll 16
        for (int w = 0; w < kPlanWarps; ++w) sum += cnt[w * E + e];
        tot[e] = sum;
    }
    cluster_barrier();
    const int e = threadIdx.x;     // E <= 1024
    int before = 0, all = 0;
    if (e < E) {
        for (int r = 0; r < nc; ++r) {
            const int n = ld_cluster(tot + e, r);
            if (r < rank) before += n;
            all += n;
        }
        if (load && rank == 0) {
            int n = 0;
            for (int r = 0; r < nc; ++r) n += ld_cluster(first + e, r);
            load[e] = n;
        }
    }
    int up = all;                  // inclusive sum over the experts
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int n = __shfl_up_sync(0xffffffffu, up, d);
        if (lane >= d) up += n;
    }
    if (lane == 31) scan[warp] = up;
    cluster_barrier();             // the other CTAs' counts have been read, and scan is complete
    int lower = 0, kept = 0;
#pragma unroll
    for (int w = 0; w < 32; ++w) {
        const int n = scan[w];
        if (w < warp) lower += n;
        kept += n;
    }
    if (e < E) {
        int row = lower + up - all;
        if (rank == 0) {
            offsets[e] = row;
            if (e == E - 1) offsets[E] = row + all;
        }
        row += before;
#pragma unroll 8
        for (int w = 0; w < kPlanWarps; ++w) {
            const int n = cnt[w * E + e];
            cnt[w * E + e] = row;
            row += n;
        }
    }
    __syncthreads();
    for (long long b = lo; b < hi; b += 32 * kPlanBatch) {
        int key[kPlanBatch], row[kPlanBatch];
#pragma unroll
        for (int i = 0; i < kPlanBatch; ++i) {
            const long long v = b + 32 * i + lane;
            key[i] = v < hi ? __ldg(idx + v) : -1;
            row[i] = v < hi ? slot[v] : 0;
        }
#pragma unroll
        for (int i = 0; i < kPlanBatch; ++i) {
            const long long v = b + 32 * i + lane;
            const bool ok = key[i] >= 0 && key[i] < E;
            row[i] = ok ? row[i] + mine[key[i]] : -1;
            if (v < hi) slot[v] = row[i];
            if (ok && with_inv) inv[row[i]] = (int)v;
        }
    }
    for (long long r = (long long)kept + rank * kPlanThreads + threadIdx.x; r < V; r += (long long)nc * kPlanThreads) inv[r] = -1;
}

// ---- rows ----
// A row in units: 16 bytes of elements (WIDE), where rows or arrays do not allow that two bf16 (PAIR), else one element (ONE).
enum { ONE = 0, PAIR = 1, WIDE = 2 };
template <int DT, int CLS> struct Unit;
template <> struct Unit<LOCMOE_BF16, WIDE> {
    static constexpr int N = 8, CH = 2;      // elements, units in flight a lane and row
    typedef uint4 Raw;
    static __device__ __forceinline__ Raw load(const void* p, long long i) { return ld_stream(static_cast<const uint4*>(p) + i); }
    static __device__ __forceinline__ void widen(const Raw& r, float (&f)[N]) {
        f[0] = bf16_lo(r.x); f[1] = bf16_hi(r.x); f[2] = bf16_lo(r.y); f[3] = bf16_hi(r.y);
        f[4] = bf16_lo(r.z); f[5] = bf16_hi(r.z); f[6] = bf16_lo(r.w); f[7] = bf16_hi(r.w);
    }
    static __device__ __forceinline__ Raw narrow(const float (&f)[N]) {
        return make_uint4(cvt_bf16x2(make_float2(f[0], f[1])), cvt_bf16x2(make_float2(f[2], f[3])), cvt_bf16x2(make_float2(f[4], f[5])),
                          cvt_bf16x2(make_float2(f[6], f[7])));
    }
    static __device__ __forceinline__ void store(void* p, long long i, const Raw& r) { st_stream(static_cast<uint4*>(p) + i, r); }
    static __device__ __forceinline__ Raw zero() { return make_uint4(0, 0, 0, 0); }
};
template <> struct Unit<LOCMOE_F32, WIDE> {
    static constexpr int N = 4, CH = 2;
    typedef uint4 Raw;
    static __device__ __forceinline__ Raw load(const void* p, long long i) { return ld_stream(static_cast<const uint4*>(p) + i); }
    static __device__ __forceinline__ void widen(const Raw& r, float (&f)[N]) {
        f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y); f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
    }
    static __device__ __forceinline__ Raw narrow(const float (&f)[N]) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    static __device__ __forceinline__ void store(void* p, long long i, const Raw& r) { st_stream(static_cast<uint4*>(p) + i, r); }
    static __device__ __forceinline__ Raw zero() { return make_uint4(0, 0, 0, 0); }
};
template <> struct Unit<LOCMOE_BF16, ONE> {
    static constexpr int N = 1, CH = 8;
    typedef uint16_t Raw;
    static __device__ __forceinline__ Raw load(const void* p, long long i) { return __ldcs(static_cast<const unsigned short*>(p) + i); }
    static __device__ __forceinline__ void widen(const Raw& r, float (&f)[N]) { f[0] = bf16_lo(r); }
    static __device__ __forceinline__ Raw narrow(const float (&f)[N]) { return (Raw)cvt_bf16x2(make_float2(f[0], f[0])); }
    static __device__ __forceinline__ void store(void* p, long long i, const Raw& r) { static_cast<uint16_t*>(p)[i] = r; }
    static __device__ __forceinline__ Raw zero() { return 0; }
};
template <> struct Unit<LOCMOE_BF16, PAIR> {
    static constexpr int N = 2, CH = 8;
    typedef uint32_t Raw;
    static __device__ __forceinline__ Raw load(const void* p, long long i) { return __ldcs(static_cast<const unsigned int*>(p) + i); }
    static __device__ __forceinline__ void widen(const Raw& r, float (&f)[N]) { f[0] = bf16_lo(r); f[1] = bf16_hi(r); }
    static __device__ __forceinline__ Raw narrow(const float (&f)[N]) { return cvt_bf16x2(make_float2(f[0], f[1])); }
    static __device__ __forceinline__ void store(void* p, long long i, const Raw& r) { static_cast<uint32_t*>(p)[i] = r; }
    static __device__ __forceinline__ Raw zero() { return 0u; }
};
template <> struct Unit<LOCMOE_F32, ONE> {
    static constexpr int N = 1, CH = 8;
    typedef uint32_t Raw;
    static __device__ __forceinline__ Raw load(const void* p, long long i) { return __ldcs(static_cast<const unsigned int*>(p) + i); }
    static __device__ __forceinline__ void widen(const Raw& r, float (&f)[N]) { f[0] = __uint_as_float(r); }
    static __device__ __forceinline__ Raw narrow(const float (&f)[N]) { return __float_as_uint(f[0]); }
    static __device__ __forceinline__ void store(void* p, long long i, const Raw& r) { static_cast<uint32_t*>(p)[i] = r; }
    static __device__ __forceinline__ Raw zero() { return 0u; }
};

// Order and rows of a few assignments in one launch: CTA v finds the row of assignment v by counting the assignments that come
// before it, and copies the token there; the assignments that are not routed take the rows behind the last group, in
// order, as rows of zeros.  The CTAs after those count for the offsets.  V^2 reads of the index array out of L2 and L1: up to
// kFewMax assignments that is less than two launches (8 tokens x 2 choices 12.9 against 15.6 us a call, 2048 assignments with
// their rows 7.7 against 9.7 us on the device, 4096 already 14.7 against 9.4).
constexpr int kFewThreads = 128, kFewMax = 2048;
template <typename R>
__global__ void __launch_bounds__(kFewThreads) sort_few_kernel(const int32_t* __restrict__ idx, int V, int T, int E, const R* __restrict__ x, int U,
                                                               int32_t* __restrict__ offsets, int32_t* __restrict__ slot, int32_t* __restrict__ inv,
                                                               int32_t* __restrict__ load, R* __restrict__ xs) {
    pdl_wait();
    pdl_trigger();
    if ((int)blockIdx.x >= V) {             // a warp an offset
        const int e = ((int)blockIdx.x - V) * (kFewThreads / 32) + (threadIdx.x >> 5);
        if (e > E) return;
        int below = 0, first = 0;
#pragma unroll 4
        for (int u = threadIdx.x & 31; u < V; u += 32) {
            const int k = __ldg(idx + u);
            below += k >= 0 && k < e;
            first += u < T && k == e;
        }
        below = __reduce_add_sync(0xffffffffu, below);
        first = __reduce_add_sync(0xffffffffu, first);
        if ((threadIdx.x & 31) == 0) {
            offsets[e] = below;
            if (load && e < E) load[e] = first;
        }
        return;
    }
    const int v = blockIdx.x, key = __ldg(idx + v), t = v % T;
    const bool ok = key >= 0 && key < E;
    constexpr int CH = sizeof(R) == 16 ? 4 : 8;
    R r[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i)
        if (ok && (int)threadIdx.x + i * kFewThreads < U) r[i] = x[(size_t)t * U + threadIdx.x + i * kFewThreads];
    int row = 0;
#pragma unroll 4
    for (int u = threadIdx.x; u < V; u += kFewThreads) {
        const int k = __ldg(idx + u);
        const bool routed = k >= 0 && k < E;
        row += ok ? routed && (k < key || (k == key && u < v)) : routed || u < v;
    }
    row = __reduce_add_sync(0xffffffffu, row);
    __shared__ int part[kFewThreads / 32];
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = row;
    __syncthreads();
    row = part[0] + part[1] + part[2] + part[3];
    if (threadIdx.x == 0) {
        slot[v] = ok ? row : -1;
        inv[row] = ok ? v : -1;
    }
    for (int u0 = threadIdx.x; u0 < U; u0 += CH * kFewThreads) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int u = u0 + i * kFewThreads;
            if (u >= U) break;
            if (u0 != (int)threadIdx.x && ok) r[i] = x[(size_t)t * U + u];
            xs[(size_t)row * U + u] = ok ? r[i] : R{};
        }
    }
}

// What a row kernel works on.  `width` threads (a power of two, up to a CTA) share a token; a CTA owns `tpc` consecutive tokens.
struct RowArgs {
    int T, U, K, E;             // tokens, units a row, choices, experts
    long long rows;             // K * T
    int width, tpc;
};

// Rows [offsets[E], rows) hold no assignment: zeros.
template <typename U>
__device__ __forceinline__ void zero_tail(const RowArgs& a, const int32_t* __restrict__ offsets, void* __restrict__ out) {
    const long long kept = max(0, __ldg(offsets + a.E));
    const long long n = (a.rows - kept) * a.U;
    for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < n; i += (long long)gridDim.x * kThreads)
        U::store(out, kept * a.U + i, U::zero());
}

// xs[slot[c][t]] = x[t]: a token's row is read once and written K times; inv along with it.
template <int DT, int CLS>
__global__ void __launch_bounds__(kThreads) sort_rows_kernel(const RowArgs a, const void* __restrict__ x, const int32_t* __restrict__ offsets,
                                                             const int32_t* __restrict__ slot, int32_t* __restrict__ inv, void* __restrict__ xs) {
    typedef Unit<DT, CLS> U;
    constexpr int CH = 2 * U::CH;
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x % a.width, step = kThreads / a.width;
    const long long lo = (long long)blockIdx.x * a.tpc, hi = min((long long)a.T, lo + a.tpc);
    for (long long t = lo + threadIdx.x / a.width; t < hi; t += step) {
        bool any = false;
        for (int c = 0; c < a.K; ++c) any |= __ldg(slot + (long long)c * a.T + t) >= 0;
        if (!any) continue;
        for (int u0 = lane; u0 < a.U; u0 += CH * a.width) {
            typename U::Raw r[CH];
#pragma unroll
            for (int i = 0; i < CH; ++i)
                if (u0 + i * a.width < a.U) r[i] = U::load(x, t * a.U + u0 + i * a.width);
            for (int c = 0; c < a.K; ++c) {
                const int s = __ldg(slot + (long long)c * a.T + t);
                if (s < 0 || s >= a.rows) continue;
                if (u0 == 0) inv[s] = (int)((long long)c * a.T + t);
#pragma unroll
                for (int i = 0; i < CH; ++i)
                    if (u0 + i * a.width < a.U) U::store(xs, (long long)s * a.U + u0 + i * a.width, r[i]);
            }
        }
    }
    zero_tail<U>(a, offsets, xs);
}

// out[t] = residual[t] + sum_c w[c][t] * y[slot[c][t]], choices without a row left out.
template <int DT, int CLS, int KM>
__global__ void __launch_bounds__(kThreads) unsort_rows_kernel(const RowArgs a, const void* __restrict__ y, const int32_t* __restrict__ slot,
                                                               const float* __restrict__ w, const void* __restrict__ residual, void* __restrict__ out) {
    typedef Unit<DT, CLS> U;
    constexpr int CH = KM <= 2 ? U::CH : U::CH / 2;
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x % a.width, step = kThreads / a.width;
    const long long lo = (long long)blockIdx.x * a.tpc, hi = min((long long)a.T, lo + a.tpc);
    for (long long t = lo + threadIdx.x / a.width; t < hi; t += step) {
        int s[KM];
        float g[KM];
#pragma unroll
        for (int c = 0; c < KM; ++c) {
            s[c] = c < a.K ? __ldg(slot + (long long)c * a.T + t) : -1;
            g[c] = w && c < a.K ? __ldg(w + (long long)c * a.T + t) : 1.0f;
            if (s[c] >= a.rows) s[c] = -1;
        }
        for (int u0 = lane; u0 < a.U; u0 += CH * a.width) {
            typename U::Raw r[CH][KM], h[CH];
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int u = u0 + i * a.width;
                if (u >= a.U) break;
                if (residual) h[i] = U::load(residual, t * a.U + u);
#pragma unroll
                for (int c = 0; c < KM; ++c)
                    if (s[c] >= 0) r[i][c] = U::load(y, (long long)s[c] * a.U + u);
            }
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int u = u0 + i * a.width;
                if (u >= a.U) break;
                float acc[U::N], v[U::N];
                if (residual) U::widen(h[i], acc);
                else {
#pragma unroll
                    for (int k = 0; k < U::N; ++k) acc[k] = 0.0f;
                }
#pragma unroll
                for (int c = 0; c < KM; ++c) {
                    if (s[c] < 0) continue;
                    U::widen(r[i][c], v);
#pragma unroll
                    for (int k = 0; k < U::N; ++k) acc[k] = __fmaf_rn(g[c], v[k], acc[k]);
                }
                U::store(out, t * a.U + u, U::narrow(acc));
            }
        }
    }
}

// dy[slot[c][t]] = w[c][t] * dout[t],  dw[c][t] = <dout[t], y[slot[c][t]]>; a token's dout is read once.
template <int DT, int CLS, int KM>
__global__ void __launch_bounds__(kThreads) unsort_grad_kernel(const RowArgs a, const void* __restrict__ dout, const void* __restrict__ y,
                                                               const int32_t* __restrict__ offsets, const int32_t* __restrict__ slot,
                                                               const float* __restrict__ w, void* __restrict__ dy, float* __restrict__ dw) {
    __shared__ float sums[kWarps][KM];
    typedef Unit<DT, CLS> U;
    constexpr int CH = KM <= 2 ? U::CH : U::CH / 2;
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x % a.width, step = kThreads / a.width;
    const long long lo = (long long)blockIdx.x * a.tpc, hi = min((long long)a.T, lo + a.tpc);
    for (long long t0 = lo; t0 < hi; t0 += step) {          // the CTA stays together: the sums are shuffled and shared
        const long long t = t0 + threadIdx.x / a.width;
        int s[KM];
        float g[KM], dot[KM];
        bool any = false;
#pragma unroll
        for (int c = 0; c < KM; ++c) {
            s[c] = c < a.K && t < hi ? __ldg(slot + (long long)c * a.T + t) : -1;
            if (s[c] >= a.rows) s[c] = -1;
            g[c] = w && s[c] >= 0 ? __ldg(w + (long long)c * a.T + t) : 1.0f;
            dot[c] = 0.0f;
            any |= s[c] >= 0;
        }
        if (any) {
            for (int u0 = lane; u0 < a.U; u0 += CH * a.width) {
                typename U::Raw r[CH][KM], d[CH];
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    const int u = u0 + i * a.width;
                    if (u >= a.U) break;
                    d[i] = U::load(dout, t * a.U + u);
                    if (dw) {
#pragma unroll
                        for (int c = 0; c < KM; ++c)
                            if (s[c] >= 0) r[i][c] = U::load(y, (long long)s[c] * a.U + u);
                    }
                }
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    const int u = u0 + i * a.width;
                    if (u >= a.U) break;
                    float f[U::N], v[U::N];
                    U::widen(d[i], f);
#pragma unroll
                    for (int c = 0; c < KM; ++c) {
                        if (s[c] < 0) continue;
                        if (dw) {
                            U::widen(r[i][c], v);
#pragma unroll
                            for (int k = 0; k < U::N; ++k) dot[c] = __fmaf_rn(f[k], v[k], dot[c]);
                        }
                        if (dy) {
#pragma unroll
                            for (int k = 0; k < U::N; ++k) v[k] = __fmul_rn(g[c], f[k]);
                            U::store(dy, (long long)s[c] * a.U + u, U::narrow(v));
                        }
                    }
                }
            }
        }
        if (dw) {
#pragma unroll
            for (int c = 0; c < KM; ++c)
                for (int o = min(a.width, 32) >> 1; o; o >>= 1) dot[c] += __shfl_xor_sync(0xffffffffu, dot[c], o);
            if (a.width > 32) {             // several warps a token: their sums in order
                if ((threadIdx.x & 31) == 0) {
#pragma unroll
                    for (int c = 0; c < KM; ++c) sums[threadIdx.x >> 5][c] = dot[c];
                }
                __syncthreads();
                if (lane == 0) {
                    for (int w = 1; w < a.width / 32; ++w) {
#pragma unroll
                        for (int c = 0; c < KM; ++c) dot[c] += sums[(threadIdx.x >> 5) + w][c];
                    }
                }
                __syncthreads();
            }
#pragma unroll
            for (int c = 0; c < KM; ++c)
                if (lane == 0 && t < hi && c < a.K) dw[(long long)c * a.T + t] = dot[c];
        }
    }
    if (dy) zero_tail<U>(a, offsets, dy);
}

// Gradient of the sorted rows towards the tokens, the router's gradient added:
//   dx[t][j] = sum_c dxs[slot[c][t]][j] + dG[t][j / g] / g,   dG_i = [G_i > 0] p_i (q_i - sum_j p_j q_j),
//   G = group means of x[t] + eps, p = softmax(ReLU(G)), q_i = dp_i + sum_c [idx[c][t] = i] dw[c][t].
// G, p and dG are formed anew from the row, which costs the read of x; keeping p would cost E floats a token instead but leave
// the sign of G open, which the ReLU needs.  A team of 8 lanes or 1 to 8 warps works on a token: the sums of the row's units go
// through shared memory, where a few lanes each add up a group's; a unit that two groups meet in (MIXED) leaves two sums.  The
// softmax is every warp's, to save barriers.  deps: the team's sums in shared memory, then the CTA's in `part`.  One warp a
// token is best where there are many tokens and their sums leave room for them (65536 x 5120: 331 us, 566 with eight), more
// where a row is long or the tokens few (10737 rows of 5912 floats in 4 groups: 708 us with one, 197 with eight; 4 rows of 3216
// 20.7 against 5.9 us), eight lanes where rows are short and a token is latencies (29585 rows of 72 floats 28 us with a warp,
// 12 so; 65536 x 256 in 32 groups 58 against 33; 3751 x 168 10.4 against 12.5).  Five to eight choices spill at four CTAs an SM (65536
// x 2560 in bf16: eight 663 us, 512 at the copy rate; four 343 and 307).
struct RouterArgs {
    const void* x; const float* eps; const int32_t* idx; const float* dw; const float* dp; float* part;
    int g;                      // elements a group
    unsigned rcp_g;             // floor((2^32 - 1) / g)
    float inv_g;
    int team;                   // threads: 8, or 1, 2, 4, 8 warps
    int lanes;                  // that share a group's sum, a power of two up to 32
    size_t floats;              // of shared memory a team
};

// n / g: the product with the reciprocal falls short by one at most (34735 rows of 4830 in pairs 283 us with a division, 269 so).
__device__ __forceinline__ int group_at(const RouterArgs& b, int n) {
    const int e = (int)__umulhi((unsigned)n, b.rcp_g);
    return n - e * b.g >= b.g ? e + 1 : e;
}

// W: lanes of a warp that work on one token, 32 (and more warps with them) or 8.
template <int DT, int CLS, bool MIXED, int KM, int W>
__global__ void __launch_bounds__(kThreads, 4) sort_grad_router_kernel(const RowArgs a, const RouterArgs b, const void* __restrict__ dxs,
                                                                    const int32_t* __restrict__ slot, void* __restrict__ dx) {
    typedef Unit<DT, CLS> U;
    // units in flight a lane and row: registers for four CTAs an SM, which spills cost more than loads in flight gain
    constexpr int CH = CLS == WIDE ? (KM <= 2 ? 2 : 1) : KM <= 2 ? 8 / KM : 16 / KM, XCH = CLS == WIDE ? 4 : 8;
    extern __shared__ float smf[];
    const int nt = W < 32 ? W : b.team, team = threadIdx.x / nt, teams = kThreads / nt, tid = threadIdx.x - team * nt, lane = tid & 31, E = a.E;
    auto meet = [&] {               // the team, or the teams of a warp
        if (W < 32 || nt == 32) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(nt) : "memory");
    };
    float* lo = smf + team * b.floats;                            // [U] sum of a unit's elements in the group of its first
    float* hi = lo + a.U;                       // [U] and of the others (MIXED)
    float* G = hi + (MIXED ? a.U : 0);          // [E]
    float* dG = G + E;                          // [E] dG / g
    float* deps = dG + E;                       // [E] sums over this team's tokens
    for (int e = tid; e < E; e += nt) deps[e] = 0.0f;
    pdl_wait();
    pdl_trigger();
    const long long first = (long long)blockIdx.x * a.tpc, last = min((long long)a.T, first + a.tpc);
    for (long long t0 = first; t0 < last; t0 += teams) {
        const long long t = t0 + team;
        const bool on = W == 32 || t < last;    // the teams of a warp stay together
        if (W == 32 && t >= last) break;
        const int units = on ? a.U : 0;
        int s[KM];
#pragma unroll
        for (int c = 0; c < KM; ++c) {
            s[c] = on && dxs && c < a.K ? __ldg(slot + (long long)c * a.T + t) : -1;
            if (s[c] >= a.rows) s[c] = -1;
        }
        for (int u0 = tid; u0 < units; u0 += XCH * nt) {
            typename U::Raw r[XCH];
#pragma unroll
            for (int i = 0; i < XCH; ++i)
                if (u0 + nt * i < a.U) r[i] = U::load(b.x, t * a.U + u0 + nt * i);
#pragma unroll
            for (int i = 0; i < XCH; ++i) {
                const int u = u0 + nt * i;
                if (u >= a.U) break;
                float f[U::N];
                U::widen(r[i], f);
                if (MIXED) {
                    const int left = (group_at(b, u * U::N) + 1) * b.g - u * U::N;     // elements to the group's end
                    float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
                    for (int k = 0; k < U::N; ++k) {
                        if (k < left) s0 += f[k];
                        else s1 += f[k];
                    }
                    lo[u] = s0;
                    hi[u] = s1;
                } else {
                    float sum = f[0];
#pragma unroll
                    for (int k = 1; k < U::N; ++k) sum += f[k];
                    lo[u] = sum;
                }
            }
        }
        meet();
        {
            const int j = tid & (b.lanes - 1), per = nt / b.lanes;
            for (int e0 = 0; e0 < E; e0 += per) {
                const int e = e0 + tid / b.lanes;
                float sum = 0.0f;
                if (e < E) {
                    const int begin = e * b.g, end = begin + b.g - 1;      // first and last element
                    const int ub = begin / U::N, ue = end / U::N;
                    for (int u = ub + j; u <= ue; u += b.lanes) sum += MIXED && u == ub && begin % U::N != 0 ? hi[u] : lo[u];
                }
                for (int o = b.lanes >> 1; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                if (e < E && j == 0) G[e] = sum * b.inv_g + (b.eps ? __ldg(b.eps + e) : 0.0f);
            }
        }
        int id[KM];
        float dw[KM];
#pragma unroll
        for (int c = 0; c < KM; ++c) {
            id[c] = on && c < a.K && b.dw ? __ldg(b.idx + (long long)c * a.T + t) : -1;
            dw[c] = on && c < a.K && b.dw ? __ldg(b.dw + (long long)c * a.T + t) : 0.0f;
        }
        meet();
        float top = 0.0f, z = 0.0f, m = 0.0f;
        for (int e = lane; e < E; e += W) top = fmaxf(top, G[e]);
#pragma unroll
        for (int o = W / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        for (int e = lane; e < E; e += W) {
            const float v = expf(fmaxf(G[e], 0.0f) - top);                  // a mean that is NaN counts as 0, as in the forward pass
            float q = b.dp ? __ldg(b.dp + e) : 0.0f;
#pragma unroll
            for (int c = 0; c < KM; ++c) q += id[c] == e ? dw[c] : 0.0f;
            z += v;
            m = __fmaf_rn(v, q, m);
        }
#pragma unroll
        for (int o = W / 2; o; o >>= 1) { z += __shfl_xor_sync(0xffffffffu, z, o); m += __shfl_xor_sync(0xffffffffu, m, o); }
        const float rz = 1.0f / z;
        m *= rz;
        if (on && tid < 32) {
            for (int e = lane; e < E; e += W) {
                float q = b.dp ? __ldg(b.dp + e) : 0.0f;
#pragma unroll
                for (int c = 0; c < KM; ++c) q += id[c] == e ? dw[c] : 0.0f;
                const float v = expf(fmaxf(G[e], 0.0f) - top) * rz;
                const float d = G[e] > 0.0f ? v * (q - m) : 0.0f * v;       // what leaves through the ReLU
                deps[e] += d;
                dG[e] = d * b.inv_g;
            }
        }
        meet();
        for (int u0 = tid; u0 < units; u0 += CH * nt) {
            typename U::Raw r[CH][KM];
#pragma unroll
            for (int i = 0; i < CH; ++i) {
#pragma unroll
                for (int c = 0; c < KM; ++c) {
                    if (u0 + nt * i < a.U && s[c] >= 0) r[i][c] = U::load(dxs, (long long)s[c] * a.U + u0 + nt * i);
                }
            }
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int u = u0 + nt * i;
                if (u >= a.U) break;
                const int e = group_at(b, u * U::N);
                float acc[U::N], v[U::N];
                const float d = dG[e];
                if (MIXED) {
                    const int left = (e + 1) * b.g - u * U::N;
                    const float d1 = left < U::N ? dG[e + 1] : 0.0f;
#pragma unroll
                    for (int k = 0; k < U::N; ++k) acc[k] = k < left ? d : d1;
                } else {
#pragma unroll
                    for (int k = 0; k < U::N; ++k) acc[k] = d;
                }
#pragma unroll
                for (int c = 0; c < KM; ++c) {
                    if (s[c] < 0) continue;
                    U::widen(r[i][c], v);
#pragma unroll
                    for (int k = 0; k < U::N; ++k) acc[k] += v[k];
                }
                U::store(dx, t * a.U + u, U::narrow(acc));
            }
        }
    }
    if (!b.part) return;
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += kThreads) {
        float sum = 0.0f;
        for (int w = 0; w < teams; ++w) sum += smf[w * b.floats + (deps - lo) + e];
        b.part[(size_t)blockIdx.x * E + e] = sum;
    }
}

// deps[e] = sum of the CTAs' sums, in a fixed order: 32 experts a CTA, the rows dealt to 32 warps, eight loads in flight.
constexpr int kFinishThreads = 1024;
__global__ void __launch_bounds__(kFinishThreads) deps_finish_kernel(const float* __restrict__ part, int n, int E, float* __restrict__ deps) {
    __shared__ float sm[32][33];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = blockIdx.x * 32 + lane;
    float sum = 0.0f;
    if (e < E)
        for (int r = warp; r < n; r += 32 * 8) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = r + 32 * i < n ? __ldcg(part + (size_t)(r + 32 * i) * E + e) : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += v[i];
        }
    sm[warp][lane] = sum;
    __syncthreads();
    sum = sm[lane][warp];           // expert `warp` of the CTA's 32
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0 && blockIdx.x * 32 + warp < E) deps[blockIdx.x * 32 + warp] = sum;
}

// Tokens a CTA and threads a token of a row kernel.
RowArgs row_args(const locmoe_shape_t& s, int K, int U, int* grid) {
    RowArgs a{s.T, U, K, s.E, (long long)K * s.T, 32, 1};
    while (a.width > 1 && a.width / 2 >= U) a.width /= 2;
    // few tokens with long rows: more threads a token (48 tokens of 7928, three choices, their gradient 19.6 against 5.3 us)
    while (a.width >= 32 && a.width < kThreads && a.width < U && 2ll * s.T * a.width <= 1024ll * sm_count()) a.width *= 2;
    const long long step = kThreads / a.width;
    const long long want = (s.T + step - 1) / step, cap = 1024ll * sm_count();     // many short CTAs, in ascending token order
    const long long g = want < cap ? want : cap;
    a.tpc = (int)((s.T + g - 1) / g);
    a.tpc = (int)((a.tpc + step - 1) / step * step);
    *grid = (int)((s.T + a.tpc - 1) / a.tpc);
    return a;
}

// The widest unit that rows of H elements in these arrays (absent ones are no obstacle) are made of.
int unit_of(const locmoe_shape_t& s, std::initializer_list<const void*> arrays) {
    const int esz = s.x_dtype == LOCMOE_F32 ? 4 : 2;
    uintptr_t any = (uintptr_t)s.H * esz;
    for (const void* p : arrays) any |= (uintptr_t)p;
    return any % 16 == 0 ? WIDE : esz == 2 && any % 4 == 0 ? PAIR : ONE;
}
int unit_elements(const locmoe_shape_t& s, int cls) { return cls == WIDE ? (s.x_dtype == LOCMOE_F32 ? 4 : 8) : cls == PAIR ? 2 : 1; }

constexpr int kLanes = 8;                // that share a token whose row is short
constexpr size_t kRouterSmem = 200 * 1024;
// How a row is cut for the router's gradient: units that meet two groups at most, whole in one or of 16 bytes (MIXED).
struct RouterPlan { int cls; bool mixed; int U; size_t smem; };
RouterPlan router_plan(const locmoe_shape_t& s, int cls) {
    const int g = s.H / s.E;
    RouterPlan p;
    p.cls = cls == WIDE && g < unit_elements(s, WIDE) ? PAIR : cls;
    if (p.cls == PAIR && (s.x_dtype == LOCMOE_F32 || g % 2 != 0)) p.cls = ONE;
    p.mixed = p.cls == WIDE && g % unit_elements(s, WIDE) != 0;
    p.U = s.H / unit_elements(s, p.cls);
    p.smem = ((size_t)p.U * (p.mixed ? 2 : 1) + 3 * (size_t)s.E) * sizeof(float);
    return p;
}
int router_grid_cap() { return 4 * sm_count(); }        // what is resident

#define LOCMOE_BY_UNIT(DTYPE, CLS, F, ...)                                                       \
    ((DTYPE) == LOCMOE_F32 ? ((CLS) == WIDE ? F<LOCMOE_F32, WIDE>(__VA_ARGS__) : F<LOCMOE_F32, ONE>(__VA_ARGS__)) \
     : (CLS) == WIDE ? F<LOCMOE_BF16, WIDE>(__VA_ARGS__)                                         \
     : (CLS) == PAIR ? F<LOCMOE_BF16, PAIR>(__VA_ARGS__) : F<LOCMOE_BF16, ONE>(__VA_ARGS__))

template <int DT, int CLS>
int sort_rows_dt(int grid, const RowArgs& a, const void* x, const int32_t* offsets, const int32_t* slot, int32_t* inv, void* xs, cudaStream_t st) {
    return launch_pdl(sort_rows_kernel<DT, CLS>, dim3(grid), dim3(kThreads), 0, st, a, x, offsets, slot, inv, xs);
}
template <int DT, int CLS>
int unsort_rows_dt(int grid, const RowArgs& a, const void* y, const int32_t* slot, const float* w, const void* residual, void* out, cudaStream_t st) {
    auto* k = a.K == 1 ? unsort_rows_kernel<DT, CLS, 1> : a.K == 2 ? unsort_rows_kernel<DT, CLS, 2>
            : a.K <= 4 ? unsort_rows_kernel<DT, CLS, 4> : unsort_rows_kernel<DT, CLS, 8>;
    return launch_pdl(k, dim3(grid), dim3(kThreads), 0, st, a, y, slot, w, residual, out);
}
template <int DT, int CLS>
int unsort_grad_dt(int grid, const RowArgs& a, const void* dout, const void* y, const int32_t* offsets, const int32_t* slot, const float* w,
                   void* dy, float* dw, cudaStream_t st) {
    auto* k = a.K == 1 ? unsort_grad_kernel<DT, CLS, 1> : a.K == 2 ? unsort_grad_kernel<DT, CLS, 2>
            : a.K <= 4 ? unsort_grad_kernel<DT, CLS, 4> : unsort_grad_kernel<DT, CLS, 8>;
    return launch_pdl(k, dim3(grid), dim3(kThreads), 0, st, a, dout, y, offsets, slot, w, dy, dw);
}
template <int DT, int CLS>
int sort_grad_router_dt(int grid, const RouterPlan& p, const RowArgs& a, const RouterArgs& b, const void* dxs, const int32_t* slot, void* dx,
                        cudaStream_t st) {
#define LOCMOE_BY_CHOICES(MIXED, W)                                                                                                 \
    (a.K == 1 ? sort_grad_router_kernel<DT, CLS, MIXED, 1, W> : a.K == 2 ? sort_grad_router_kernel<DT, CLS, MIXED, 2, W>             \
     : a.K <= 4 ? sort_grad_router_kernel<DT, CLS, MIXED, 4, W> : sort_grad_router_kernel<DT, CLS, MIXED, 8, W>)
#define LOCMOE_BY_TEAM(MIXED) (b.team < 32 ? LOCMOE_BY_CHOICES(MIXED, kLanes) : LOCMOE_BY_CHOICES(MIXED, 32))
    auto* k = CLS == WIDE && p.mixed ? LOCMOE_BY_TEAM(CLS == WIDE) : LOCMOE_BY_TEAM(false);
#undef LOCMOE_BY_TEAM
#undef LOCMOE_BY_CHOICES
    const size_t smem = p.smem * (kThreads / b.team);
    if (smem > 48 * 1024 && cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRouterSmem) != cudaSuccess) {
        cudaGetLastError();
        return LOCMOE_ERR_CUDA;
    }
    return launch_pdl(k, dim3(grid), dim3(kThreads), smem, st, a, b, dxs, slot, dx);
}

}  // namespace

// `with_inv` = 0: the rows' kernel, which follows, writes inv's part with assignments.
int launch_sort_plan(int T, int K, int E, const int32_t* idx, int32_t* offsets, int32_t* slot, int32_t* inv, int with_inv, int32_t* load, cudaStream_t st) {
    const long long V = (long long)K * T;
    const size_t smem = plan_smem(E);
    auto* kernel = E < 16 ? sort_plan_kernel<4> : E < 64 ? sort_plan_kernel<6> : E < 256 ? sort_plan_kernel<8> : sort_plan_kernel<11>;    // keys 0 to E
    // always the most that any call needs: the limit is the kernel's, and another host thread's smaller one would refuse this launch
    if ((smem > 48 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)plan_smem(1024)) != cudaSuccess) ||
        (V > 8ll * kPlanRun && cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)) {
        cudaGetLastError();
        return LOCMOE_ERR_CUDA;
    }
    cudaLaunchConfig_t cfg = {};
    int nc = 1;
    while (nc < 16 && V > (long long)nc * kPlanRun) nc *= 2;
    cfg.gridDim = dim3(nc); cfg.blockDim = dim3(kPlanThreads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = nc; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    cfg.attrs = attr; cfg.numAttrs = 2;
    int fit = 1;
    if (nc == 16 && (cudaOccupancyMaxActiveClusters(&fit, kernel, &cfg) != cudaSuccess || fit < 1)) {
        cudaGetLastError();
        nc = 8;
        cfg.gridDim = dim3(nc);
        attr[0].val.clusterDim.x = nc;
    }
    if (cudaLaunchKernelEx(&cfg, kernel, idx, (int)V, T, E, offsets, slot, inv, with_inv, load) != cudaSuccess) {
        cudaGetLastError();
        return LOCMOE_ERR_CUDA;
    }
    return check_launch();
}

// Whether locmoe_sort is one launch.
bool sort_is_few(int T, int K) { return (long long)K * T <= kFewMax; }

int launch_sort_few(const locmoe_shape_t& s, int K, const int32_t* idx, const void* x, int32_t* offsets, int32_t* slot, int32_t* inv, int32_t* load,
                    void* xs, cudaStream_t st) {
    const int V = K * s.T, esz = s.x_dtype == LOCMOE_F32 ? 4 : 2;
    const long long bytes = (long long)s.H * esz;
    const dim3 grid(V + (s.E + kFewThreads / 32) / (kFewThreads / 32)), block(kFewThreads);      // E + 1 offsets
    int rc;
    const int cls = unit_of(s, {x, xs});
    if (cls == WIDE)
        rc = launch_pdl(sort_few_kernel<uint4>, grid, block, 0, st, idx, V, (int)s.T, (int)s.E, (const uint4*)x, (int)(bytes / 16), offsets, slot, inv, load, (uint4*)xs);
    else if (cls == PAIR || esz == 4)
        rc = launch_pdl(sort_few_kernel<uint32_t>, grid, block, 0, st, idx, V, (int)s.T, (int)s.E, (const uint32_t*)x, (int)(bytes / 4), offsets, slot, inv, load, (uint32_t*)xs);
    else
        rc = launch_pdl(sort_few_kernel<uint16_t>, grid, block, 0, st, idx, V, (int)s.T, (int)s.E, (const uint16_t*)x, (int)s.H, offsets, slot, inv, load, (uint16_t*)xs);
    return rc ? rc : check_launch();
}

int launch_sort_rows(const locmoe_shape_t& s, int K, const void* x, const int32_t* offsets, const int32_t* slot, int32_t* inv, void* xs, cudaStream_t st) {
    const int cls = unit_of(s, {x, xs});
    int grid;
    const RowArgs a = row_args(s, K, s.H / unit_elements(s, cls), &grid);
    const int rc = LOCMOE_BY_UNIT(s.x_dtype, cls, sort_rows_dt, grid, a, x, offsets, slot, inv, xs, st);
    return rc ? rc : check_launch();
}

int launch_unsort_rows(const locmoe_shape_t& s, int K, const void* y, const int32_t* slot, const float* w, const void* residual, void* out,
                       cudaStream_t st) {
    const int cls = unit_of(s, {y, residual, out});
    int grid;
    const RowArgs a = row_args(s, K, s.H / unit_elements(s, cls), &grid);
    const int rc = LOCMOE_BY_UNIT(s.x_dtype, cls, unsort_rows_dt, grid, a, y, slot, w, residual, out, st);
    return rc ? rc : check_launch();
}

int launch_unsort_grad(const locmoe_shape_t& s, int K, const void* dout, const void* y, const int32_t* offsets, const int32_t* slot,
                       const float* w, void* dy, float* dw, cudaStream_t st) {
    const int cls = unit_of(s, {dout, y, dy});
    int grid;
    const RowArgs a = row_args(s, K, s.H / unit_elements(s, cls), &grid);
    const int rc = LOCMOE_BY_UNIT(s.x_dtype, cls, unsort_grad_dt, grid, a, dout, y, offsets, slot, w, dy, dw, st);
    return rc ? rc : check_launch();
}

// A row's sums have to fit the shared memory of a CTA.
bool sort_grad_fits(const locmoe_shape_t& s) { return router_plan(s, unit_of(s, {})).smem <= kRouterSmem; }
size_t sort_grad_ws_bytes(const locmoe_shape_t& s) { return ((size_t)router_grid_cap() * s.E * sizeof(float) + 255) & ~(size_t)255; }

int launch_sort_grad(const locmoe_shape_t& s, int K, const locmoe_sort_grad_t& g, void* ws, cudaStream_t st) {
    if (!g.x) return launch_unsort_rows(s, K, g.dxs, g.slot, nullptr, nullptr, g.dx, st);
    const RouterPlan p = router_plan(s, unit_of(s, {g.x, g.dxs, g.dx}));
    if (p.smem > kRouterSmem) return LOCMOE_ERR_ALIGN;      // arrays that are not 16-byte aligned take more room
    // warps a token: so many that four CTAs' sums fit an SM, and while all tokens are still at work at once
    int team = 32;
    while (team < kThreads && ((kThreads / team) * p.smem > 50 * 1024 || 2ll * team * s.T <= (long long)router_grid_cap() * kThreads)) team *= 2;
    // eight lanes a token: short rows, and a third of the lanes that fit at work at least
    if (team == 32 && p.U <= (p.cls == WIDE ? 12 : 24) * kLanes && 3ll * kLanes * s.T >= (long long)router_grid_cap() * kThreads &&
        (kThreads / kLanes) * p.smem <= 50 * 1024)
        team = kLanes;
    int lanes = min(team, 32);
    while (lanes > 1 && (long long)lanes * s.E > team) lanes /= 2;
    const int teams = kThreads / team;
    RowArgs a{s.T, p.U, K, s.E, (long long)K * s.T, 32, 1};
    long long grid = ((long long)s.T + teams - 1) / teams;
    if (grid > router_grid_cap()) grid = router_grid_cap();
    a.tpc = (int)((s.T + grid - 1) / grid);
    grid = (s.T + a.tpc - 1) / a.tpc;
    const RouterArgs b{g.x, g.eps, g.idx_k, g.dw, g.dp, g.deps ? static_cast<float*>(ws) : nullptr, s.H / s.E, 0xffffffffu / (unsigned)(s.H / s.E), 1.0f / (float)(s.H / s.E), team, lanes,
                       p.smem / sizeof(float)};
    int rc = LOCMOE_BY_UNIT(s.x_dtype, p.cls, sort_grad_router_dt, (int)grid, p, a, b, g.dxs, g.slot, g.dx, st);
    if (rc == LOCMOE_OK && g.deps)
        rc = launch_pdl(deps_finish_kernel, dim3((s.E + 31) / 32), dim3(kFinishThreads), 0, st, (const float*)ws, (int)grid, s.E, g.deps);
    return rc ? rc : check_launch();
}

}  // namespace locmoe
