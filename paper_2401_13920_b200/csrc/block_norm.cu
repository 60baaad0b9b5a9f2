// The norms around one MoE block, fused with its gate and its residual, and their gradient.
//
//   forward    v = y[slot[t]] (0 for a dropped token),  u = v r,  r = (mean v^2 + eps)^-1/2
//              h' = a h + R_t w_post u,                 x = h' q, q = (mean h'^2 + eps)^-1/2,   n = x w_pre
//   gradient   D  = dh' + q (dn w_pre - x mean(dn w_pre x)),   dh = a D
//              k  = sum_j D w_post u,   dR = k,   dv = r (R w_post D - u R k / H)
//              dw_pre = sum_t dn x,     dw_post = sum_t R D u
//
// A row is worked on by a group of kWarp-multiple threads that keep it in registers between its two sums, so every
// element is read and written once.  Sums are fp32 in a fixed order; outputs are rounded once.
// With checkpoints the forward also leaves u and x in E4M3: a normalised row has mean square <= 1 and so no element
// above sqrt(H), which the format's 448 covers for every H the library takes here; r and q carry the scale.
#include <cuda_fp8.h>

#include "common.cuh"

namespace locmoe {

namespace {

constexpr int kMaxGroups = 15;   // row groups of a CTA: one named barrier each (barrier 0 is the whole CTA's)

struct NormArgs {
    const void* h; const void* y; const int32_t* slot; const float* gate; const float* w_post; const float* w_pre;
    float res_scale, eps;
    void* h_out; void* n_out; uint8_t* u8; uint8_t* x8; float* r_post; float* r_pre;
    long long rows;
    int T, H, tpr, groups;
};

struct NormGradArgs {
    const void* dh_out; const void* dn; const void* h_out; const void* y; const uint8_t* x8; const uint8_t* u8;
    const float* r_pre; const float* r_post;
    const int32_t* slot; const int32_t* inv; const float* gate; const float* w_post; const float* w_pre;
    float res_scale, eps;
    void* dh; void* dy; float* dgate; float* part_post; float* part_pre;   // parts: [grid][H]
    long long rows;
    int T, H, tpr, groups;
};

// ---- one unit of a row: VEC = 8 elements by 16-byte accesses, VEC = 1 a single element ----
template <typename X, int VEC> struct Unit;
template <> struct Unit<uint16_t, 8> {
    static __device__ __forceinline__ void load(const void* base, size_t at, float* f) {
        const uint4 w = ld_stream(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + at));
        f[0] = bf16_lo(w.x); f[1] = bf16_hi(w.x); f[2] = bf16_lo(w.y); f[3] = bf16_hi(w.y);
        f[4] = bf16_lo(w.z); f[5] = bf16_hi(w.z); f[6] = bf16_lo(w.w); f[7] = bf16_hi(w.w);
    }
    static __device__ __forceinline__ void store(void* base, size_t at, const float* f) {
        const uint4 w = make_uint4(cvt_bf16x2(make_float2(f[0], f[1])), cvt_bf16x2(make_float2(f[2], f[3])),
                                   cvt_bf16x2(make_float2(f[4], f[5])), cvt_bf16x2(make_float2(f[6], f[7])));
        st_stream(reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + at), w);
    }
};
template <> struct Unit<float, 8> {
    static __device__ __forceinline__ void load(const void* base, size_t at, float* f) {
        const uint4* p = reinterpret_cast<const uint4*>(static_cast<const float*>(base) + at);
        const uint4 a = ld_stream(p), b = ld_stream(p + 1);
        f[0] = __uint_as_float(a.x); f[1] = __uint_as_float(a.y); f[2] = __uint_as_float(a.z); f[3] = __uint_as_float(a.w);
        f[4] = __uint_as_float(b.x); f[5] = __uint_as_float(b.y); f[6] = __uint_as_float(b.z); f[7] = __uint_as_float(b.w);
    }
    static __device__ __forceinline__ void store(void* base, size_t at, const float* f) {
        uint4* p = reinterpret_cast<uint4*>(static_cast<float*>(base) + at);
        st_stream(p, make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
        st_stream(p + 1, make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])));
    }
};
template <> struct Unit<uint16_t, 1> {
    static __device__ __forceinline__ void load(const void* base, size_t at, float* f) {
        f[0] = bf16_lo(static_cast<const uint16_t*>(base)[at]);
    }
    static __device__ __forceinline__ void store(void* base, size_t at, const float* f) {
        static_cast<uint16_t*>(base)[at] = (uint16_t)f32_to_bf16_bits(f[0]);
    }
};
template <> struct Unit<float, 1> {
    static __device__ __forceinline__ void load(const void* base, size_t at, float* f) { f[0] = static_cast<const float*>(base)[at]; }
    static __device__ __forceinline__ void store(void* base, size_t at, const float* f) { static_cast<float*>(base)[at] = f[0]; }
};

template <int VEC>
__device__ __forceinline__ void load_weight(const float* w, int at, float* f) {   // a NULL weight is 1
    if constexpr (VEC == 8) {
        if (w) {
            const float4 a = __ldg(reinterpret_cast<const float4*>(w + at)), b = __ldg(reinterpret_cast<const float4*>(w + at) + 1);
            f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = 1.0f;
        }
    } else {
        f[0] = w ? __ldg(w + at) : 1.0f;
    }
}

template <int VEC>
__device__ __forceinline__ void store_e4m3(uint8_t* base, size_t at, const float* f) {   // round to nearest even, NaN kept
    if constexpr (VEC == 8) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __nv_cvt_float2_to_fp8x2(make_float2(f[2 * i], f[2 * i + 1]), __NV_SATFINITE, __NV_E4M3);
        *reinterpret_cast<uint2*>(base + at) = make_uint2(w[0] | (w[1] << 16), w[2] | (w[3] << 16));
    } else {
        base[at] = __nv_cvt_float_to_fp8(f[0], __NV_SATFINITE, __NV_E4M3);
    }
}
__device__ __forceinline__ float2 e4m3x2_to_float2(uint32_t two) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
    return __half22float2(__half2(h));
}
template <int VEC>
__device__ __forceinline__ void load_e4m3(const uint8_t* base, size_t at, float* f) {
    if constexpr (VEC == 8) {
        const uint2 w = __ldcs(reinterpret_cast<const uint2*>(base + at));
        const float2 a = e4m3x2_to_float2(w.x & 0xffffu), b = e4m3x2_to_float2(w.x >> 16);
        const float2 c = e4m3x2_to_float2(w.y & 0xffffu), d = e4m3x2_to_float2(w.y >> 16);
        f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y; f[4] = c.x; f[5] = c.y; f[6] = d.x; f[7] = d.y;
    } else {
        f[0] = e4m3x2_to_float2(base[at]).x;
    }
}

constexpr int kRedFloats = 2 * 32 * 3;   // per group: two strips of 32 warps x up to 3 values
// Sum of N values over the threads of a row group, the same bits in every thread.  red: the group's own two
// shared strips, used alternately, so that one barrier per sum is enough.
template <int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float* red, int& parity, int group, int tpr) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if (tpr == kWarp) return;
    const int warps = tpr / kWarp, w = (threadIdx.x % tpr) / kWarp;
    float* strip = red + parity * (kRedFloats / 2);
    parity ^= 1;
    if (threadIdx.x % kWarp == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) strip[w * N + i] = v[i];
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(tpr) : "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.0f;
    for (int k = 0; k < warps; ++k)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += strip[k * N + i];
}

// NV > 0: the row stays in registers (NV units a thread).  NV == 0: any length; the row is read again after each sum.
template <typename X, int VEC, int NV>
__global__ void __launch_bounds__(1024) block_norm_kernel(const NormArgs a) {
    __shared__ float red_all[kMaxGroups * kRedFloats];
    pdl_wait();
    pdl_trigger();
    const int tpr = a.tpr, group = threadIdx.x / tpr, lane = threadIdx.x - group * tpr;
    float* red = red_all + group * kRedFloats;
    int parity = 0;
    const float inv_h = 1.0f / (float)a.H;
    const int units = a.H / VEC;
    const bool want_pre = a.n_out || a.x8 || a.r_pre;
    constexpr int R = (NV > 0 ? NV : 1) * VEC;
    for (long long t = (long long)blockIdx.x * a.groups + group; t < a.T; t += (long long)gridDim.x * a.groups) {
        long long s = !a.y ? -1 : a.slot ? (long long)a.slot[t] : t;
        if (s >= a.rows) s = -1;   // no row of the buffer
        const size_t at_t = (size_t)t * a.H, at_s = s < 0 ? 0 : (size_t)s * a.H;
        const float gate = a.gate ? a.gate[t] : 1.0f;
        float v[R], h[R];
        float sum[1] = {0.0f};
        if constexpr (NV > 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int un = lane + i * tpr;
                if (un < units) {
                    Unit<X, VEC>::load(a.h, at_t + (size_t)un * VEC, h + i * VEC);
                    if (s >= 0) Unit<X, VEC>::load(a.y, at_s + (size_t)un * VEC, v + i * VEC);
                }
                if (un >= units || s < 0)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) v[i * VEC + j] = 0.0f;
                if (un >= units)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) h[i * VEC + j] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < R; ++i) sum[0] = fmaf(v[i], v[i], sum[0]);
        } else if (s >= 0) {
            for (int un = lane; un < units; un += tpr) {
                Unit<X, VEC>::load(a.y, at_s + (size_t)un * VEC, v);
#pragma unroll
                for (int j = 0; j < VEC; ++j) sum[0] = fmaf(v[j], v[j], sum[0]);
            }
        }
        if (a.y) group_sum(sum, red, parity, group, tpr);
        const float r = 1.0f / sqrtf(fmaf(sum[0], inv_h, a.eps));
        if (a.r_post && lane == 0) a.r_post[t] = r;
        const float gr = gate;
        // h' of unit `un` into h[], u into v[]
        auto mix = [&](int un, float* hv, float* vv) {
            float w[VEC];
            load_weight<VEC>(a.w_post, un * VEC, w);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                vv[j] *= r;
                hv[j] = fmaf(gr * w[j], vv[j], a.res_scale * hv[j]);
            }
        };
        auto finish = [&](int un, float* hv, float q) {   // hv holds h'
            float w[VEC];
            load_weight<VEC>(a.w_pre, un * VEC, w);
#pragma unroll
            for (int j = 0; j < VEC; ++j) hv[j] *= q;
            if (a.x8) store_e4m3<VEC>(a.x8, at_t + (size_t)un * VEC, hv);
#pragma unroll
            for (int j = 0; j < VEC; ++j) w[j] *= hv[j];
            if (a.n_out) Unit<X, VEC>::store(a.n_out, at_t + (size_t)un * VEC, w);
        };
        float ss[1] = {0.0f};
        if constexpr (NV > 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int un = lane + i * tpr;
                if (un < units) {
                    mix(un, h + i * VEC, v + i * VEC);
                    if (a.h_out) Unit<X, VEC>::store(a.h_out, at_t + (size_t)un * VEC, h + i * VEC);
                    if (a.u8) store_e4m3<VEC>(a.u8, at_t + (size_t)un * VEC, v + i * VEC);
                }
            }
#pragma unroll
            for (int i = 0; i < R; ++i) ss[0] = fmaf(h[i], h[i], ss[0]);
        } else {
            for (int un = lane; un < units; un += tpr) {
                Unit<X, VEC>::load(a.h, at_t + (size_t)un * VEC, h);
#pragma unroll
                for (int j = 0; j < VEC; ++j) v[j] = 0.0f;
                if (s >= 0) Unit<X, VEC>::load(a.y, at_s + (size_t)un * VEC, v);
                mix(un, h, v);
                if (a.u8) store_e4m3<VEC>(a.u8, at_t + (size_t)un * VEC, v);
#pragma unroll
                for (int j = 0; j < VEC; ++j) ss[0] = fmaf(h[j], h[j], ss[0]);
                if (a.h_out && !want_pre) Unit<X, VEC>::store(a.h_out, at_t + (size_t)un * VEC, h);
            }
        }
        if (want_pre) {
            group_sum(ss, red, parity, group, tpr);
            const float q = 1.0f / sqrtf(fmaf(ss[0], inv_h, a.eps));
            if (a.r_pre && lane == 0) a.r_pre[t] = q;
            if constexpr (NV > 0) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int un = lane + i * tpr;
                    if (un < units) finish(un, h + i * VEC, q);
                }
            } else {   // h' is formed again from h and y; h_out may be h itself, so it is stored only now
                for (int un = lane; un < units; un += tpr) {
                    Unit<X, VEC>::load(a.h, at_t + (size_t)un * VEC, h);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) v[j] = 0.0f;
                    if (s >= 0) Unit<X, VEC>::load(a.y, at_s + (size_t)un * VEC, v);
                    mix(un, h, v);
                    if (a.h_out) Unit<X, VEC>::store(a.h_out, at_t + (size_t)un * VEC, h);
                    finish(un, h, q);
                }
            }
        }
    }
}

// Gradient.  CK: normalised rows from E4M3 and their reciprocal norms, else h' and y as stored.
template <typename X, int VEC, int NV, bool CK>
__global__ void __launch_bounds__(512) block_norm_grad_kernel(const NormGradArgs a) {
    __shared__ float red_all[kMaxGroups * kRedFloats];
    extern __shared__ float cols[];   // [2][H]: the groups' column sums, joined in group order (NV > 0, several groups)
    pdl_wait();
    pdl_trigger();
    const int tpr = a.tpr, group = threadIdx.x / tpr, lane = threadIdx.x - group * tpr;
    float* red = red_all + group * kRedFloats;
    int parity = 0;
    const float inv_h = 1.0f / (float)a.H;
    const int units = a.H / VEC;
    constexpr int R = (NV > 0 ? NV : 1) * VEC;
    const bool branch = CK ? a.u8 != nullptr : a.y != nullptr;
    const bool need_k = branch && (a.dgate || a.dy);
    float acc_post[R], acc_pre[R];
#pragma unroll
    for (int i = 0; i < R; ++i) { acc_post[i] = 0.0f; acc_pre[i] = 0.0f; }
    float* mine_post = a.part_post ? a.part_post + (size_t)blockIdx.x * a.H : nullptr;
    float* mine_pre = a.part_pre ? a.part_pre + (size_t)blockIdx.x * a.H : nullptr;
    if constexpr (NV == 0) {   // column sums live in the CTA's own row of the workspace; a thread owns its columns
        for (int un = lane; un < units; un += tpr)
            for (int j = 0; j < VEC; ++j) {
                if (mine_post) mine_post[un * VEC + j] = 0.0f;
                if (mine_pre) mine_pre[un * VEC + j] = 0.0f;
            }
    }
    for (long long t = (long long)blockIdx.x * a.groups + group; t < a.T; t += (long long)gridDim.x * a.groups) {
        long long s = !branch ? -1 : a.slot ? (long long)a.slot[t] : t;
        if (s >= a.rows) s = -1;   // no row of the buffer
        const size_t at_t = (size_t)t * a.H, at_s = s < 0 ? 0 : (size_t)s * a.H;
        const float gate = a.gate ? a.gate[t] : 1.0f;
        float x[R], u[R], dn[R], D[R];
        // one unit of the four inputs; x / u are h' / v (or the normalised values with CK), missing ones zero
        auto load = [&](int un, float* xv, float* uv, float* nv, float* dv) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) { xv[j] = 0.0f; uv[j] = 0.0f; nv[j] = 0.0f; dv[j] = 0.0f; }
            if (un >= units) return;
            if (a.dh_out) Unit<X, VEC>::load(a.dh_out, at_t + (size_t)un * VEC, dv);
            if (a.dn) {
                Unit<X, VEC>::load(a.dn, at_t + (size_t)un * VEC, nv);
                if constexpr (CK) load_e4m3<VEC>(a.x8, at_t + (size_t)un * VEC, xv);
                else Unit<X, VEC>::load(a.h_out, at_t + (size_t)un * VEC, xv);
            }
            if (s >= 0) {
                if constexpr (CK) load_e4m3<VEC>(a.u8, at_t + (size_t)un * VEC, uv);
                else Unit<X, VEC>::load(a.y, at_s + (size_t)un * VEC, uv);
            }
        };
        float sum[3] = {0.0f, 0.0f, 0.0f};   // x^2, u^2, dn w_pre x
        auto gather = [&](int un, const float* xv, const float* uv, const float* nv) {
            if (un >= units) return;
            float w[VEC];
            load_weight<VEC>(a.w_pre, un * VEC, w);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                sum[0] = fmaf(xv[j], xv[j], sum[0]);
                sum[1] = fmaf(uv[j], uv[j], sum[1]);
                sum[2] = fmaf(nv[j] * w[j], xv[j], sum[2]);
            }
        };
        if constexpr (NV > 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i) load(lane + i * tpr, x + i * VEC, u + i * VEC, dn + i * VEC, D + i * VEC);
#pragma unroll
            for (int i = 0; i < NV; ++i) gather(lane + i * tpr, x + i * VEC, u + i * VEC, dn + i * VEC);
        } else {
            for (int un = lane; un < units; un += tpr) { load(un, x, u, dn, D); gather(un, x, u, dn); }
        }
        group_sum(sum, red, parity, group, tpr);
        float q, r;
        if constexpr (CK) {
            q = a.dn ? a.r_pre[t] : 0.0f;
            r = branch ? a.r_post[t] : 0.0f;
        } else {
            q = 1.0f / sqrtf(fmaf(sum[0], inv_h, a.eps));
            r = 1.0f / sqrtf(fmaf(sum[1], inv_h, a.eps));
        }
        const float xs = CK ? 1.0f : q, us = CK ? 1.0f : r;   // what turns x, u into normalised values
        const float c1 = sum[2] * xs * inv_h;
        // D of one unit; x, u become normalised
        auto upstream = [&](int un, float* xv, float* uv, const float* nv, float* dv) {
            float w[VEC];
            load_weight<VEC>(a.w_pre, un * VEC, w);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                xv[j] *= xs; uv[j] *= us;
                dv[j] = fmaf(q, fmaf(nv[j], w[j], -xv[j] * c1), dv[j]);
            }
        };
        float k[1] = {0.0f};
        auto add_k = [&](int un, const float* uv, const float* dv) {
            float w[VEC];
            load_weight<VEC>(a.w_post, un * VEC, w);
#pragma unroll
            for (int j = 0; j < VEC; ++j) k[0] = fmaf(dv[j] * w[j], uv[j], k[0]);
        };
        if constexpr (NV > 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int un = lane + i * tpr;
                if (un < units) {
                    if (a.dn) upstream(un, x + i * VEC, u + i * VEC, dn + i * VEC, D + i * VEC);
                    else
#pragma unroll
                        for (int j = 0; j < VEC; ++j) u[i * VEC + j] *= us;
                    if (need_k) add_k(un, u + i * VEC, D + i * VEC);
                }
            }
        } else if (need_k) {
            for (int un = lane; un < units; un += tpr) {
                load(un, x, u, dn, D);
                if (a.dn) upstream(un, x, u, dn, D);
                else
#pragma unroll
                    for (int j = 0; j < VEC; ++j) u[j] *= us;
                add_k(un, u, D);
            }
        }
        if (need_k) {
            group_sum(k, red, parity, group, tpr);
            if (a.dgate && lane == 0) a.dgate[t] = k[0];
        } else if (a.dgate && lane == 0) {
            a.dgate[t] = 0.0f;
        }
        const float rg = r * gate, kh = k[0] * inv_h;
        auto emit = [&](int un, const float* xv, const float* uv, const float* nv, const float* dv, float* ap, float* an) {
            float w[VEC], o[VEC];
            load_weight<VEC>(a.w_post, un * VEC, w);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                ap[j] = fmaf(gate * dv[j], uv[j], ap[j]);
                an[j] = fmaf(nv[j], xv[j], an[j]);
            }
            if (a.dy && s >= 0) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) o[j] = rg * fmaf(dv[j], w[j], -uv[j] * kh);
                Unit<X, VEC>::store(a.dy, at_s + (size_t)un * VEC, o);
            }
            if (a.dh) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) o[j] = a.res_scale * dv[j];
                Unit<X, VEC>::store(a.dh, at_t + (size_t)un * VEC, o);
            }
        };
        if constexpr (NV > 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int un = lane + i * tpr;
                if (un < units) emit(un, x + i * VEC, u + i * VEC, dn + i * VEC, D + i * VEC, acc_post + i * VEC, acc_pre + i * VEC);
            }
        } else {
            for (int un = lane; un < units; un += tpr) {
                load(un, x, u, dn, D);
                if (a.dn) upstream(un, x, u, dn, D);
                else
#pragma unroll
                    for (int j = 0; j < VEC; ++j) u[j] *= us;
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    acc_post[j] = mine_post ? mine_post[un * VEC + j] : 0.0f;
                    acc_pre[j] = mine_pre ? mine_pre[un * VEC + j] : 0.0f;
                }
                emit(un, x, u, dn, D, acc_post, acc_pre);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    if (mine_post) mine_post[un * VEC + j] = acc_post[j];
                    if (mine_pre) mine_pre[un * VEC + j] = acc_pre[j];
                }
            }
        }
    }
    if constexpr (NV > 0) {
        if (mine_post || mine_pre) {
            for (int g = 0; g < a.groups; ++g) {   // groups add their columns one after the other: a fixed order
                if (group == g) {
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        const int un = lane + i * tpr;
                        if (un < units)
#pragma unroll
                            for (int j = 0; j < VEC; ++j) {
                                const int c = un * VEC + j;
                                const float p = acc_post[i * VEC + j] + (g ? cols[c] : 0.0f);
                                const float n = acc_pre[i * VEC + j] + (g ? cols[a.H + c] : 0.0f);
                                if (g + 1 < a.groups) { cols[c] = p; cols[a.H + c] = n; }
                                else {
                                    if (mine_post) mine_post[c] = p;
                                    if (mine_pre) mine_pre[c] = n;
                                }
                            }
                    }
                }
                __syncthreads();
            }
        }
    }
    // rows of the slot buffer that no token owns have a zero gradient
    if (a.dy && a.inv) {
        float z[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) z[j] = 0.0f;
        for (long long row = (long long)blockIdx.x * a.groups + group; row < a.rows; row += (long long)gridDim.x * a.groups) {
            if (a.inv[row] >= 0) continue;
            for (int un = lane; un < units; un += tpr) Unit<X, VEC>::store(a.dy, (size_t)row * a.H + (size_t)un * VEC, z);
        }
    }
}

// Column sums: the CTAs' rows of the workspace added in index order (fp32, 8 interleaved chains joined in order).
constexpr int kColThreads = 256, kColChains = 8;
__global__ void __launch_bounds__(kColThreads) block_norm_cols_kernel(const float* part_post, const float* part_pre, int parts, int H,
                                                                      float* dw_post, float* dw_pre) {
    __shared__ float strip[kColChains][32];
    pdl_wait();
    pdl_trigger();
    const float* part = blockIdx.y ? part_pre : part_post;
    float* dw = blockIdx.y ? dw_pre : dw_post;
    if (!dw) return;
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), chain = threadIdx.x >> 5;
    float s = 0.0f;
    if (c < H)
        for (int p = chain; p < parts; p += kColChains) s += part[(size_t)p * H + c];
    strip[chain][threadIdx.x & 31] = s;
    __syncthreads();
    if (chain == 0 && c < H) {
        for (int i = 1; i < kColChains; ++i) s += strip[i][threadIdx.x];
        dw[c] = s;
    }
}

// Threads of a row group and the number of groups of a CTA for `units` units of which a thread keeps nv.
struct RowPlan { int tpr, groups; };
RowPlan plan_rows(int units, int nv, int threads) {
    int tpr = nv > 0 ? (units + nv - 1) / nv : threads;
    tpr = (tpr + kWarp - 1) / kWarp * kWarp;
    if (tpr > 1024) tpr = 1024;
    int groups = nv > 0 ? threads / tpr : 1;
    if (groups < 1) groups = 1;
    if (groups > kMaxGroups) groups = kMaxGroups;
    return {tpr, groups};
}

constexpr int kGradCtasPerSm = 2;

bool aligned(const void* p, int n) { return (uintptr_t)p % n == 0; }

template <typename X>
int forward(NormArgs& a, cudaStream_t st) {
    const bool wide = a.H % 8 == 0 && aligned(a.h, 16) && aligned(a.y, 16) && aligned(a.h_out, 16) && aligned(a.n_out, 16) &&
                      aligned(a.w_post, 16) && aligned(a.w_pre, 16) && aligned(a.u8, 8) && aligned(a.x8, 8);
    const int units = wide ? a.H / 8 : a.H;
    const int nv = wide ? (units <= 1024 * 2 ? 2 : 0) : (units <= 1024 * 8 ? 8 : 0);
    const RowPlan p = plan_rows(units, nv, 256);
    a.tpr = p.tpr; a.groups = p.groups;
    const int threads = p.tpr * p.groups;
    long long grid = (a.T + p.groups - 1) / p.groups;
    const long long most = (long long)sm_count() * (2048 / threads > 0 ? 2048 / threads : 1);
    if (grid > most) grid = most;
    auto run = [&](auto kernel) { return launch_pdl(kernel, dim3((unsigned)grid), dim3(threads), 0, st, a); };
    if (wide) return nv ? run(block_norm_kernel<X, 8, 2>) : run(block_norm_kernel<X, 8, 0>);
    return nv ? run(block_norm_kernel<X, 1, 8>) : run(block_norm_kernel<X, 1, 0>);
}

template <typename X, bool CK>
int backward(NormGradArgs& a, float* dw_post, float* dw_pre, cudaStream_t st) {
    const bool wide = a.H % 8 == 0 && aligned(a.dh_out, 16) && aligned(a.dn, 16) && aligned(a.h_out, 16) && aligned(a.y, 16) &&
                      aligned(a.x8, 8) && aligned(a.u8, 8) && aligned(a.w_post, 16) && aligned(a.w_pre, 16) && aligned(a.dh, 16) &&
                      aligned(a.dy, 16);
    const int units = wide ? a.H / 8 : a.H;
    const int nv = wide ? (units <= 512 ? 1 : 0) : (units <= 512 * 8 ? 8 : 0);
    const RowPlan p = plan_rows(units, nv, 512);
    a.tpr = p.tpr; a.groups = p.groups;
    const int threads = p.tpr * p.groups;
    long long grid = (a.T + p.groups - 1) / p.groups;
    const long long most = (long long)sm_count() * kGradCtasPerSm;
    if (grid > most) grid = most;
    const size_t smem = nv && p.groups > 1 ? (size_t)a.H * 8 : 0;
    auto run = [&](auto kernel) { return launch_pdl(kernel, dim3((unsigned)grid), dim3(threads), smem, st, a); };
    int rc;
    if (wide) rc = nv ? run(block_norm_grad_kernel<X, 8, 1, CK>) : run(block_norm_grad_kernel<X, 8, 0, CK>);
    else rc = nv ? run(block_norm_grad_kernel<X, 1, 8, CK>) : run(block_norm_grad_kernel<X, 1, 0, CK>);
    if (rc || (!dw_post && !dw_pre)) return rc;
    return launch_pdl(block_norm_cols_kernel, dim3((a.H + 31) / 32, 2), dim3(kColThreads), 0, st, a.part_post, a.part_pre, (int)grid,
                      a.H, dw_post, dw_pre);
}

}  // namespace

// Workspace of the gradient: one row of column sums per CTA and weight.
size_t block_norm_grad_ws_bytes(const locmoe_shape_t& s) {
    const size_t b = (size_t)sm_count() * kGradCtasPerSm * s.H * 4 * 2;
    return (b + 255) / 256 * 256;
}

int launch_block_norm(const locmoe_shape_t& s, long long rows, const locmoe_block_norm_t& b, cudaStream_t st) {
    NormArgs a{b.h, b.y, b.slot, b.gate_w, b.w_post, b.w_pre, b.res_scale, b.eps, b.h_out, b.n_out, b.u8, b.x8, b.r_post, b.r_pre,
               rows, s.T, s.H, 0, 0};
    return s.x_dtype == LOCMOE_F32 ? forward<float>(a, st) : forward<uint16_t>(a, st);
}

int launch_block_norm_grad(const locmoe_shape_t& s, long long rows, const locmoe_block_norm_grad_t& b, void* ws, cudaStream_t st) {
    float* part = static_cast<float*>(ws);
    NormGradArgs a{b.dh_out, b.dn, b.h_out, b.y, b.x8, b.u8, b.r_pre, b.r_post, b.slot, b.slot ? b.inv : nullptr, b.gate_w, b.w_post,
                   b.w_pre, b.res_scale, b.eps, b.dh, b.dy, b.dgate, b.dw_post ? part : nullptr,
                   b.dw_pre ? part + (size_t)sm_count() * kGradCtasPerSm * s.H : nullptr, rows, s.T, s.H, 0, 0};
    const bool ck = b.x8 || b.u8;
    if (s.x_dtype == LOCMOE_F32)
        return ck ? backward<float, true>(a, b.dw_post, b.dw_pre, st) : backward<float, false>(a, b.dw_post, b.dw_pre, st);
    return ck ? backward<uint16_t, true>(a, b.dw_post, b.dw_pre, st) : backward<uint16_t, false>(a, b.dw_post, b.dw_pre, st);
}

}  // namespace locmoe
