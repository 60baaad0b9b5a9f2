// The norms around one MoE block, fused with its gate and its residual, and their gradient.
//
//   forward    v = y[slot[t]] (0 for a dropped token),  u = v r,  r = (mean v^2 + eps)^-1/2
//              h' = a h + R_t w_post u,                 x = h' q, q = (mean h'^2 + eps)^-1/2,   n = x w_pre
//   gradient   D  = dh' + q (dn w_pre - x mean(dn w_pre x)),   dh = a D
//              k  = sum_j D w_post u,   dR = k,   dv = r (R w_post D - u R k / H)
//              dw_pre = sum_t dn x,     dw_post = sum_t R D u
//
// Bound by memory: 8 bytes an element forward and 12 backward in bf16, 10 with checkpoints.  A row is worked on by a
// group of kWarp-multiple threads that keep it in registers between its two sums, so every element is read and written
// once.  The two sums of a row are two round trips through the group, during which a kernel that loads its rows itself
// asks memory for nothing (65536 x 5120 in bf16: 699 us forward, 58 % of the copy bandwidth); so each group has a ring
// of rows in shared memory that bulk copies fill D rows ahead, a thread asking for an array of the row D on as soon as a
// sum's barrier shows that the group has taken a row out of its place (forward 415-435 us, 92-97 % of the copy bandwidth;
// with checkpoints at 65536 x 2560 478 -> 277-295 us, 86-91 %).
// Sums are fp32 in a fixed order; outputs are rounded once.
// With checkpoints the forward also leaves u and x in E4M3: a normalised row has mean square <= 1 and so no element
// above sqrt(H), which the format's 448 covers for every H the library takes here; r and q carry the scale.
#include <cuda_fp8.h>

#include "common.cuh"

namespace locmoe {

namespace {

constexpr int kMaxGroups = 15;      // row groups of a CTA: one named barrier each (barrier 0 is the whole CTA's)

struct NormArgs {
    const void* h; const void* y; const int32_t* slot; const float* gate; const float* w_post; const float* w_pre;
    float res_scale, eps;
    void* h_out; void* n_out; uint8_t* u8; uint8_t* x8; float* r_post; float* r_pre;
    long long rows;
    int T, H, tpr, groups, depth;   // depth: rows of a group's ring
};

struct NormGradArgs {
    const void* dh_out; const void* dn; const void* h_out; const void* y; const uint8_t* x8; const uint8_t* u8;
    const float* r_pre; const float* r_post;
    const int32_t* slot; const int32_t* inv; const float* gate; const float* w_post; const float* w_pre;
    float res_scale, eps;
    void* dh; void* dy; float* dgate; float* part_post; float* part_pre;   // parts: [grid][H]
    long long rows;
    int T, H, tpr, groups, depth;
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

// ---- the ring kernels work on pairs: two-wide fp32 instructions, four pairs a unit ----
struct Unit8 { float2 p[4]; };
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
template <typename X>
__device__ __forceinline__ Unit8 load_pairs(const unsigned char* at) {   // out of shared memory
    Unit8 f;
    if constexpr (sizeof(X) == 2) {
        const uint4 w = *reinterpret_cast<const uint4*>(at);
        f.p[0] = make_float2(bf16_lo(w.x), bf16_hi(w.x)); f.p[1] = make_float2(bf16_lo(w.y), bf16_hi(w.y));
        f.p[2] = make_float2(bf16_lo(w.z), bf16_hi(w.z)); f.p[3] = make_float2(bf16_lo(w.w), bf16_hi(w.w));
    } else {
        const float4 a = *reinterpret_cast<const float4*>(at), b = *reinterpret_cast<const float4*>(at + 16);
        f.p[0] = make_float2(a.x, a.y); f.p[1] = make_float2(a.z, a.w); f.p[2] = make_float2(b.x, b.y); f.p[3] = make_float2(b.z, b.w);
    }
    return f;
}
template <typename X>
__device__ __forceinline__ void store_pairs(unsigned char* at, const Unit8& f) {
    uint4* to = reinterpret_cast<uint4*>(at);
    if constexpr (sizeof(X) == 2) {
        st_stream(to, make_uint4(cvt_bf16x2(f.p[0]), cvt_bf16x2(f.p[1]), cvt_bf16x2(f.p[2]), cvt_bf16x2(f.p[3])));
    } else {
        st_stream(to, make_uint4(__float_as_uint(f.p[0].x), __float_as_uint(f.p[0].y), __float_as_uint(f.p[1].x), __float_as_uint(f.p[1].y)));
        st_stream(to + 1, make_uint4(__float_as_uint(f.p[2].x), __float_as_uint(f.p[2].y), __float_as_uint(f.p[3].x), __float_as_uint(f.p[3].y)));
    }
}
__device__ __forceinline__ void clear(Unit8& f) {
#pragma unroll
    for (int j = 0; j < 4; ++j) f.p[j] = make_float2(0.0f, 0.0f);
}
__device__ __forceinline__ Unit8 load_weight_pairs(const float* w, int un) {   // a NULL weight is 1
    Unit8 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) f.p[i] = both(1.0f);
    if (w) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(w) + 2 * un), b = __ldg(reinterpret_cast<const float4*>(w) + 2 * un + 1);
        f.p[0] = make_float2(a.x, a.y); f.p[1] = make_float2(a.z, a.w); f.p[2] = make_float2(b.x, b.y); f.p[3] = make_float2(b.z, b.w);
    }
    return f;
}

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
__device__ __forceinline__ void widen_e4m3(const uint2& w, float* f) {
    const float2 a = e4m3x2_to_float2(w.x & 0xffffu), b = e4m3x2_to_float2(w.x >> 16);
    const float2 c = e4m3x2_to_float2(w.y & 0xffffu), d = e4m3x2_to_float2(w.y >> 16);
    f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y; f[4] = c.x; f[5] = c.y; f[6] = d.x; f[7] = d.y;
}
template <int VEC>
__device__ __forceinline__ void load_e4m3(const uint8_t* base, size_t at, float* f) {
    if constexpr (VEC == 8) {
        widen_e4m3(__ldcs(reinterpret_cast<const uint2*>(base + at)), f);
    } else {
        f[0] = e4m3x2_to_float2(base[at]).x;
    }
}

constexpr int kRedFloats = 2 * 32 * 4;   // per group: two strips of up to 4 values x 32 warps
// A unit of activations as it lies in memory: bf16, fp32 or codes.
struct alignas(16) RawF32 { float4 a, b; };
template <typename X, bool CK> struct RawUnit { using type = uint2; };
template <> struct RawUnit<uint16_t, false> { using type = uint4; };
template <> struct RawUnit<float, false> { using type = RawF32; };
template <typename X>
__device__ __forceinline__ Unit8 widen(const uint4& w) {
    return {{make_float2(bf16_lo(w.x), bf16_hi(w.x)), make_float2(bf16_lo(w.y), bf16_hi(w.y)), make_float2(bf16_lo(w.z), bf16_hi(w.z)),
             make_float2(bf16_lo(w.w), bf16_hi(w.w))}};
}
template <typename X>
__device__ __forceinline__ Unit8 widen(const RawF32& w) {
    return {{make_float2(w.a.x, w.a.y), make_float2(w.a.z, w.a.w), make_float2(w.b.x, w.b.y), make_float2(w.b.z, w.b.w)}};
}
template <typename X>
__device__ __forceinline__ Unit8 widen(const uint2& w) {
    Unit8 f;
    f.p[0] = e4m3x2_to_float2(w.x & 0xffffu); f.p[1] = e4m3x2_to_float2(w.x >> 16);
    f.p[2] = e4m3x2_to_float2(w.y & 0xffffu); f.p[3] = e4m3x2_to_float2(w.y >> 16);
    return f;
}
__device__ __forceinline__ void store_codes(uint8_t* at, const Unit8& f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __nv_cvt_float2_to_fp8x2(f.p[i], __NV_SATFINITE, __NV_E4M3);
    *reinterpret_cast<uint2*>(at) = make_uint2(w[0] | (w[1] << 16), w[2] | (w[3] << 16));
}

// ---- rows whose length is no multiple of 16 bytes (ODD): bulk copies bring the 16-byte pieces that hold the row, which
// then begins `mis` bytes into its place, and a unit is eight single elements, tpr apart, instead of eight in a row ----
struct Piece { size_t from; uint32_t bytes, tail; };   // copy `bytes` from `from` on; then `tail` bytes by hand
__device__ __forceinline__ Piece piece_of(size_t off, uint32_t len, size_t total) {   // of an array of `total` bytes, 16-byte aligned
    const size_t end = off + len, whole = total & ~(size_t)15, from = off & ~(size_t)15;
    size_t stop = (end + 15) & ~(size_t)15;
    if (stop > whole) stop = whole;          // the array's last bytes: nothing beyond them is read
    if (stop < from) stop = from;
    return {from, (uint32_t)(stop - from), end > stop ? (uint32_t)(end - stop) : 0u};
}
__device__ __forceinline__ void tail_of(unsigned char* to, const unsigned char* base, const Piece& p) {
    for (uint32_t i = 0; i < p.tail; ++i) to[p.bytes + i] = base[p.from + p.bytes + i];
}
template <typename X, bool CODE, bool ODD>
__device__ __forceinline__ typename RawUnit<X, CODE>::type load_raw(const unsigned char* row, uint32_t off, int first, int step, int H) {
    using Raw = typename RawUnit<X, CODE>::type;
    if constexpr (!ODD) {
        return *reinterpret_cast<const Raw*>(row + off);
    } else if constexpr (CODE) {
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = first + j * step < H ? row[first + j * step] : 0u;
        return make_uint2(w[0] | (w[1] << 8) | (w[2] << 16) | (w[3] << 24), w[4] | (w[5] << 8) | (w[6] << 16) | (w[7] << 24));
    } else if constexpr (sizeof(X) == 2) {
        const uint16_t* r = reinterpret_cast<const uint16_t*>(row);
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = first + j * step < H ? r[first + j * step] : 0u;
        return make_uint4(w[0] | (w[1] << 16), w[2] | (w[3] << 16), w[4] | (w[5] << 16), w[6] | (w[7] << 16));
    } else {
        const float* r = reinterpret_cast<const float*>(row);
        float w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = first + j * step < H ? r[first + j * step] : 0.0f;
        return {make_float4(w[0], w[1], w[2], w[3]), make_float4(w[4], w[5], w[6], w[7])};
    }
}
template <typename X, bool ODD>
__device__ __forceinline__ void store_unit(unsigned char* row, uint32_t off, int first, int step, int H, const Unit8& f) {
    if constexpr (!ODD) {
        store_pairs<X>(row + off, f);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int a = first + 2 * j * step, b = a + step;
            if constexpr (sizeof(X) == 2) {
                const uint32_t w = cvt_bf16x2(f.p[j]);
                if (a < H) reinterpret_cast<uint16_t*>(row)[a] = (uint16_t)w;
                if (b < H) reinterpret_cast<uint16_t*>(row)[b] = (uint16_t)(w >> 16);
            } else {
                if (a < H) reinterpret_cast<float*>(row)[a] = f.p[j].x;
                if (b < H) reinterpret_cast<float*>(row)[b] = f.p[j].y;
            }
        }
    }
}
template <bool ODD>
__device__ __forceinline__ void store_unit_codes(uint8_t* row, uint32_t off, int first, int step, int H, const Unit8& f) {
    if constexpr (!ODD) {
        store_codes(row + off, f);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t w = __nv_cvt_float2_to_fp8x2(f.p[j], __NV_SATFINITE, __NV_E4M3);
            const int a = first + 2 * j * step, b = a + step;
            if (a < H) row[a] = (uint8_t)w;
            if (b < H) row[b] = (uint8_t)(w >> 8);
        }
    }
}
template <bool ODD>
__device__ __forceinline__ Unit8 weight_unit(const float* w, int un, int first, int step, int H) {   // from global memory; a NULL weight is 1
    if constexpr (!ODD) {
        return load_weight_pairs(w, un);
    } else {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = !w ? 1.0f : first + j * step < H ? __ldg(w + first + j * step) : 0.0f;
        return {{make_float2(f[0], f[1]), make_float2(f[2], f[3]), make_float2(f[4], f[5]), make_float2(f[6], f[7])}};
    }
}

// Sums over the threads of a row group, the same bits in every thread.  Each warp adds up its lanes, the warps' partials
// meet in one of two shared strips used alternately, so that one barrier per sum is enough.
struct GroupSum {
    float* strip;      // the next of the two
    int other;         // from it to the other one, in floats
    int barrier, tpr, warps, warp, lane;
    __device__ __forceinline__ GroupSum(float* red, int group, int tpr_) {
        strip = red; other = kRedFloats / 2; barrier = group + 1; tpr = tpr_; warps = tpr / kWarp;
        warp = (threadIdx.x - group * tpr) / kWarp; lane = threadIdx.x % kWarp;
    }
    __device__ __forceinline__ void meet() { asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(tpr) : "memory"); }
    __device__ __forceinline__ void turn() { strip += other; other = -other; }
    __device__ __forceinline__ float butterfly(float v, int from) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            if (o <= from) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    }
    __device__ __forceinline__ float one(float v) {
        v = butterfly(v, 16);
        if (warps == 1) return v;
        if (lane == 0) strip[warp] = v;
        meet();
        v = butterfly(lane < warps ? strip[lane] : 0.0f, 16);
        turn();
        return v;
    }
    // Three values with a third of the shuffles: lanes first trade values, so that each goes on with one; later a quarter
    // of the lanes adds up each value's partials.
    __device__ __forceinline__ void three(float& x, float& y, float& z) {
        constexpr unsigned full = 0xffffffffu;
        const bool upper = lane & 16, second = lane & 8;
        const float a = (upper ? z : x) + __shfl_xor_sync(full, upper ? x : z, 16);
        const float b = (upper ? 0.0f : y) + __shfl_xor_sync(full, upper ? y : 0.0f, 16);
        float s = (second ? b : a) + __shfl_xor_sync(full, second ? a : b, 8);
        s = butterfly(s, 4);   // lanes 0..7: x, 8..15: y, 16..23: z
        if (warps > 1) {
            if ((lane & 7) == 0) strip[(lane >> 3) * kWarp + warp] = s;
            meet();
            const float* p = strip + (lane >> 3) * kWarp;
            s = 0.0f;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if ((lane & 7) + 8 * k < warps) s += p[(lane & 7) + 8 * k];
            s = butterfly(s, 4);
            turn();
        }
        x = __shfl_sync(full, s, 0); y = __shfl_sync(full, s, 8); z = __shfl_sync(full, s, 16);
    }
    __device__ __forceinline__ void four(float& x, float& y, float& z, float& w) {
        constexpr unsigned full = 0xffffffffu;
        const bool upper = lane & 16, second = lane & 8;
        const float a = (upper ? z : x) + __shfl_xor_sync(full, upper ? x : z, 16);
        const float b = (upper ? w : y) + __shfl_xor_sync(full, upper ? y : w, 16);
        float s = (second ? b : a) + __shfl_xor_sync(full, second ? a : b, 8);
        s = butterfly(s, 4);   // lanes 0..7: x, 8..15: y, 16..23: z, 24..31: w
        if (warps > 1) {
            float* p = strip + (lane >> 3) * kWarp;
            if ((lane & 7) == 0) p[warp] = s;
            meet();
            s = 0.0f;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if ((lane & 7) + 8 * k < warps) s += p[(lane & 7) + 8 * k];
            s = butterfly(s, 4);
            turn();
        }
        x = __shfl_sync(full, s, 0); y = __shfl_sync(full, s, 8); z = __shfl_sync(full, s, 16); w = __shfl_sync(full, s, 24);
    }
};

__device__ int g_norm_flags = 0;   // bit 0: a bounded wait for a row gave up

// One group's ring: D places of `stage` bytes, a barrier each.
struct RowRing {
    unsigned char* base;
    uint64_t* bars;
    int stage, depth, place;
    uint32_t phase;
    bool dead;   // a wait (half a second) was given up: nothing is waited for any more
    __device__ __forceinline__ unsigned char* wait() {   // the place whose row is next, once it is there
        if (!dead && !mbar_wait_bounded(bars + place, phase, 1u << 17)) { dead = true; atomicOr(&g_norm_flags, 1); }
        return base + (size_t)place * stage;
    }
    __device__ __forceinline__ void leave() {   // copies that were not waited for may still be on their way: hundreds of times their latency
        if (dead)
            for (int i = 0; i < 1000; ++i) __nanosleep(1000);
    }
    __device__ __forceinline__ void next() {
        if (++place == depth) { place = 0; phase ^= 1u; }
    }
};
// What a row needs besides its elements (s: its row of the block's output, -1: none); a group's table holds 64 rows of
// them, by the row's number within the group.
struct alignas(16) RowInfo { int s; float gate, q, r; };
constexpr int kTable = 64;
__device__ __forceinline__ int output_row(const int32_t* slot, bool branch, long long rows, int T, long long t) {
    if (!branch || t >= T) return -1;
    const long long s = slot ? (long long)slot[t] : t;
    return s >= rows ? -1 : (int)s;
}
__device__ __forceinline__ RowInfo info_of(const NormArgs& a, long long t) {
    return {output_row(a.slot, a.y != nullptr, a.rows, a.T, t), t < a.T && a.gate ? a.gate[t] : 1.0f, 0.0f, 0.0f};
}
template <bool CK>
__device__ __forceinline__ RowInfo info_of(const NormGradArgs& a, bool branch, long long t) {
    RowInfo f{output_row(a.slot, branch, a.rows, a.T, t), 1.0f, 0.0f, 0.0f};
    if (t >= a.T) return f;
    if (a.gate) f.gate = a.gate[t];
    if constexpr (CK) {
        if (a.dn) f.q = a.r_pre[t];
        if (branch) f.r = a.r_post[t];
    }
    return f;
}

// Rings of all groups lie one after the other, then their barriers (16 bytes a place are kept, so that what follows is aligned).
__device__ __forceinline__ RowRing ring_of(unsigned char* smem, int group, int groups, int depth, int stage, int askers) {
    RowRing r{smem + (size_t)group * depth * stage, reinterpret_cast<uint64_t*>(smem + (size_t)groups * depth * stage) + group * depth, stage,
              depth, 0, 0u, false};
    for (int i = threadIdx.x; i < groups * depth; i += blockDim.x) mbar_init(reinterpret_cast<uint64_t*>(smem + (size_t)groups * depth * stage) + i, askers);
    mbar_init_fence();
    __syncthreads();
    return r;
}

// Rows that bulk copies cannot move (or too long for a ring).  NV > 0: the row stays in registers (NV units a thread).
// NV == 0: any length; the row is read again after each sum.
template <typename X, int VEC, int NV>
__global__ void __launch_bounds__(1024) block_norm_kernel(const NormArgs a) {
    __shared__ float red_all[kMaxGroups * kRedFloats];
    pdl_wait();
    pdl_trigger();
    const int tpr = a.tpr, group = threadIdx.x / tpr, lane = threadIdx.x - group * tpr;
    GroupSum total(red_all + group * kRedFloats, group, tpr);
    const float inv_h = 1.0f / (float)a.H;
    const int units = a.H / VEC;
    const bool want_pre = a.n_out || a.x8 || a.r_pre;
    constexpr int R = (NV > 0 ? NV : 1) * VEC;
    const long long t_step = (long long)gridDim.x * a.groups;
    for (long long t = (long long)blockIdx.x * a.groups + group; t < a.T; t += t_step) {
        const RowInfo f = info_of(a, t);
        const long long s = f.s;
        const size_t at_t = (size_t)t * a.H, at_s = s < 0 ? 0 : (size_t)s * a.H;
        const float gate = f.gate;
        float v[R], h[R];
        float sum[1] = {0.0f};
        if constexpr (NV > 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int un = min(lane + i * tpr, units - 1);   // loads without branches: all of them in flight together
                Unit<X, VEC>::load(a.h, at_t + (size_t)un * VEC, h + i * VEC);
                if (a.y) Unit<X, VEC>::load(a.y, at_s + (size_t)un * VEC, v + i * VEC);
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const bool none = lane + i * tpr >= units;
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    if (none) h[i * VEC + j] = 0.0f;
                    if (none || s < 0) v[i * VEC + j] = 0.0f;
                }
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
        if (a.y) sum[0] = total.one(sum[0]);
        const float r = rsqrtf(fmaf(sum[0], inv_h, a.eps));
        if (a.r_post && lane == 0) a.r_post[t] = r;
        const float gr = gate;
        // h' of unit `un` into h[], u into v[]
        auto mix = [&](int un, float* hv, float* vv) {
            float w[VEC];
            load_weight<VEC>(a.w_post, un * VEC, w);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                vv[j] *= s < 0 ? 0.0f : r;   // nothing stays 0 where eps is 0 and r infinite
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
            ss[0] = total.one(ss[0]);
            const float q = rsqrtf(fmaf(ss[0], inv_h, a.eps));
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

// Its gradient.  CK: normalised rows from E4M3 and their reciprocal norms, else h' and y as stored.
template <typename X, int VEC, int NV, bool CK>
__global__ void __launch_bounds__(512) block_norm_grad_kernel(const NormGradArgs a) {
    __shared__ float red_all[kMaxGroups * kRedFloats];
    extern __shared__ float cols[];   // [2][H]: the groups' column sums, joined in group order at the end
    pdl_wait();
    pdl_trigger();
    const int tpr = a.tpr, group = threadIdx.x / tpr, lane = threadIdx.x - group * tpr;
    GroupSum total(red_all + group * kRedFloats, group, tpr);
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
    const long long t_step = (long long)gridDim.x * a.groups;
    for (long long t = (long long)blockIdx.x * a.groups + group; t < a.T; t += t_step) {
        const RowInfo f = info_of<CK>(a, branch, t);
        const long long s = f.s;
        const size_t at_t = (size_t)t * a.H, at_s = s < 0 ? 0 : (size_t)s * a.H;
        const float gate = f.gate;
        float q = f.q, r = f.r;
        float x[R], u[R], dn[R], D[R];
        // one unit of the four inputs; x / u are h' / v (or the normalised values with CK), missing ones zero
        auto load = [&](int un, float* xv, float* uv, float* nv, float* dv) {
            const size_t c = (size_t)min(un, units - 1) * VEC;   // loads without branches: all of them in flight together
            const bool none = un >= units;
            if (a.dh_out) Unit<X, VEC>::load(a.dh_out, at_t + c, dv);
            if (a.dn) {
                Unit<X, VEC>::load(a.dn, at_t + c, nv);
                if constexpr (CK) load_e4m3<VEC>(a.x8, at_t + c, xv);
                else Unit<X, VEC>::load(a.h_out, at_t + c, xv);
            }
            if (branch) {
                if constexpr (CK) load_e4m3<VEC>(a.u8, at_t + c, uv);
                else Unit<X, VEC>::load(a.y, at_s + c, uv);
            }
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                if (none || !a.dh_out) dv[j] = 0.0f;
                if (none || !a.dn) { nv[j] = 0.0f; xv[j] = 0.0f; }
                if (none || s < 0) uv[j] = 0.0f;
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
        total.three(sum[0], sum[1], sum[2]);
        if constexpr (!CK) {
            q = rsqrtf(fmaf(sum[0], inv_h, a.eps));
            r = rsqrtf(fmaf(sum[1], inv_h, a.eps));
        }
        const float xs = CK ? 1.0f : q, us = CK ? 1.0f : s < 0 ? 0.0f : r;   // what turns x, u into normalised values (no row: r may be infinite)
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
            k[0] = total.one(k[0]);
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

// ---- ring kernels: two units a thread ----
constexpr int kRingThreads = 640;   // of a CTA, which has an SM to itself: 102 registers a thread

// ODD rows need more registers: fp32 rows without checkpoints do better with fewer threads that have them (32768 x 2561 211 us
// against 263, x 4097 389 / 416), bf16 rows and checkpoints with more groups (2561 in bf16 248 / 233, 4097 490 / 358).
constexpr int kOddThreads = 512;

// FULL: every thread has two units.  CKPT: checkpoints are left.  ODD: see above.  TH: threads at most.
template <typename X, bool FULL, bool CKPT, bool ODD, int TH = kRingThreads>
__global__ void __launch_bounds__(TH) block_norm_ring_kernel(const NormArgs a) {
    __shared__ float red_all[kMaxGroups * kRedFloats];
    extern __shared__ __align__(128) unsigned char ring_mem[];
    pdl_wait();
    pdl_trigger();
    constexpr int UB = 8 * sizeof(X);   // bytes of a unit
    const int tpr = a.tpr, group = threadIdx.x / tpr, lane = threadIdx.x - group * tpr;
    GroupSum total(red_all + group * kRedFloats, group, tpr);
    const float inv_h = 1.0f / (float)a.H;
    const int units = (a.H + 7) / 8;
    const bool want_pre = a.n_out || (CKPT && a.x8);
    const int t_first = (int)(blockIdx.x * a.groups + group), t_step = (int)(gridDim.x * a.groups);
    const uint32_t row_bytes = (uint32_t)(a.H * sizeof(X)), pitch = ODD ? (row_bytes + 30) / 16 * 16 : row_bytes;   // of an array in a place
    RowInfo* table = reinterpret_cast<RowInfo*>(ring_mem + (size_t)a.groups * a.depth * (2 * pitch + 16)) + group * kTable;
    for (int i = lane; i < kTable; i += tpr) table[i] = info_of(a, t_first + (long long)i * t_step);
    const bool have[2] = {FULL || lane < units, FULL || lane + tpr < units};
    const uint32_t off[2] = {(uint32_t)(lane * UB), (uint32_t)((lane + tpr) * UB)};
    const int first[2] = {lane, lane + 8 * tpr};   // ODD: this thread's elements are first + j * tpr
    Unit8 wp[2], wn[2];   // this thread's columns of the weights
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (ODD || have[i]) {
            wp[i] = weight_unit<ODD>(a.w_post, lane + i * tpr, first[i], tpr, a.H);
            wn[i] = weight_unit<ODD>(a.w_pre, lane + i * tpr, first[i], tpr, a.H);
        }
    RowRing ring = ring_of(ring_mem, group, a.groups, a.depth, 2 * (int)pitch, 2);   // places of [h][y]; with a barrier of the CTA
    // Row t, whose output row is s, into a place: h by the group's first thread, y by one of another warp where there is one.
    const int asked = lane == 0 ? 0 : 1;
    const bool asks = lane == 0 || lane == (tpr > kWarp ? kWarp : 1);
    const unsigned char* from = static_cast<const unsigned char*>(asked ? a.y : a.h);
    auto ask = [&](int t, int s, int place) {
        uint64_t* bar = ring.bars + place;
        unsigned char* to = ring.base + (uint32_t)(place * ring.stage) + asked * pitch;
        const bool wanted = !asked || s >= 0;
        const size_t off = (size_t)(uint32_t)(asked ? s : t) * row_bytes;
        Piece p{off, wanted ? row_bytes : 0u, 0u};
        if constexpr (ODD) {
            if (wanted) p = piece_of(off, row_bytes, (size_t)(asked ? a.rows : a.T) * row_bytes);
            tail_of(to, from, p);
        }
        mbar_expect_tx(bar, p.bytes);
        if (p.bytes) bulk_g2s(to, from + p.from, p.bytes, bar);
    };
    if (asks)
        for (int d = 0; d < a.depth && t_first + (long long)d * t_step < a.T; ++d) ask(t_first + d * t_step, table[d].s, d);
    const int ahead = a.depth * t_step, last_ask = a.T - ahead;
    RowInfo soon{};
    int n = 0;   // the row's number within the group
    for (int t = t_first; t < a.T; t += t_step, ++n) {
        const size_t row = (size_t)t * row_bytes;
        const RowInfo f = table[n & (kTable - 1)];
        if (lane < 32) {
            if ((n & 31) == 0 && n > 0) soon = info_of(a, t + (32 + lane) * (long long)t_step);
            if ((n & 31) == 16 && n > 32) table[(n + 16 + lane) & (kTable - 1)] = soon;
        }
        const unsigned char* place = ring.wait();
        Unit8 h[2], v[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (!FULL && !ODD && !have[i]) { clear(h[i]); clear(v[i]); continue; }
            h[i] = widen<X>(load_raw<X, false, ODD>(place + (ODD ? (uint32_t)row & 15 : 0), off[i], first[i], tpr, a.H));
            v[i] = widen<X>(load_raw<X, false, ODD>(place + pitch + (ODD ? (uint32_t)f.s * row_bytes & 15 : 0), off[i], first[i], tpr, a.H));
            if (f.s < 0) clear(v[i]);   // nothing came
        }
        float2 acc = both(0.0f);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc = __ffma2_rn(v[i].p[j], v[i].p[j], acc);
        float sum = total.one(acc.x + acc.y);
        __syncwarp();
        if (asks && t < last_ask) ask(t + ahead, table[(n + a.depth) & (kTable - 1)].s, ring.place);   // the group has taken the row
        ring.next();
        const float r = rsqrtf(fmaf(sum, inv_h, a.eps));
        if (CKPT && a.r_post && lane == 0) a.r_post[t] = r;
        const float2 g2 = both(f.gate), r2 = both(f.s < 0 ? 0.0f : r), a2 = both(a.res_scale);   // nothing stays 0 where eps is 0 and r infinite
        acc = both(0.0f);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (ODD || have[i]) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[i].p[j] = __fmul2_rn(v[i].p[j], r2);
                    h[i].p[j] = __ffma2_rn(__fmul2_rn(g2, wp[i].p[j]), v[i].p[j], __fmul2_rn(a2, h[i].p[j]));
                    acc = __ffma2_rn(h[i].p[j], h[i].p[j], acc);
                }
                if (a.h_out) store_unit<X, ODD>(static_cast<unsigned char*>(a.h_out) + row, off[i], first[i], tpr, a.H, h[i]);
                if (CKPT && a.u8) store_unit_codes<ODD>(a.u8 + (size_t)t * a.H, (lane + i * tpr) * 8, first[i], tpr, a.H, v[i]);
            }
        if (!want_pre) continue;
        sum = total.one(acc.x + acc.y);
        const float q = rsqrtf(fmaf(sum, inv_h, a.eps));
        if (CKPT && a.r_pre && lane == 0) a.r_pre[t] = q;
        const float2 q2 = both(q);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (ODD || have[i]) {
#pragma unroll
                for (int j = 0; j < 4; ++j) h[i].p[j] = __fmul2_rn(h[i].p[j], q2);
                if (CKPT && a.x8) store_unit_codes<ODD>(a.x8 + (size_t)t * a.H, (lane + i * tpr) * 8, first[i], tpr, a.H, h[i]);
#pragma unroll
                for (int j = 0; j < 4; ++j) h[i].p[j] = __fmul2_rn(h[i].p[j], wn[i].p[j]);
                if (a.n_out) store_unit<X, ODD>(static_cast<unsigned char*>(a.n_out) + row, off[i], first[i], tpr, a.H, h[i]);
            }
    }
    ring.leave();
}

// Gradient.  Written with the raw rows x', u' (x = xs x', u = us u'; codes: xs = us = 1):
//   D = dh' + q dn w_pre - cx x',  cx = q xs^2 sum(dn w_pre x') / H;    dw_post += (R us) D u',  dw_pre += xs dn x'
//   e = D w_post,  k = us sum(e u'),  dv = R r e - cu u',  cu = R r us k / H
// A row's second sum (k) is taken together with the next row's first ones, so that a row costs one meeting of its group.
// Everything but dv is done before it, so that only e and u' are held over it.
// Bound by the instructions of a row and, at one group a CTA, by the length of the chain through its meeting (39 % of the
// issue slots at 65536 x 5120).  Hence two units a thread (554 instructions a warp and row against 2 x 404 with one), the
// weights' columns in registers (WREG; out of shared memory 887 us against 767), and each array of a row asked for by a
// thread of another warp (by four lanes of one warp 789 us against 737).  Not taken: an mbarrier that warps pass later
// than they arrive at it, with the work that needs no sum in between (860 us); widened rows kept over the meeting (1249
// us: what spills comes back through an L1 that the rings leave little of).
// Reached at 65536 x 5120 in bf16: 714-762 us (5.2-5.6 TB/s, 80-85 % of the copy bandwidth), from checkpoints 651-662.
// FULL: every thread has two units.  ALL: both upstream gradients, the branch, dh and dy are there.  ODD: see above (also
// rows of codes that are no whole 16-byte pieces).
constexpr int kGradThreads = 384;   // 168 registers a thread; the weights of rows beyond 16 x 384 lie in shared memory, 512 threads
template <typename X, bool CK, bool WREG, bool FULL, bool ALL, bool ODD>
__global__ void __launch_bounds__(WREG ? kGradThreads : 512) block_norm_grad_ring_kernel(const NormGradArgs a) {
    __shared__ float red_all[kMaxGroups * kRedFloats];
    extern __shared__ __align__(128) unsigned char ring_mem[];
    pdl_wait();
    pdl_trigger();
    constexpr int NV = 2, UB = 8 * sizeof(X), AB = CK ? 8 : UB;   // units of a thread; bytes of one of the rows and of the activations
    const int tpr = a.tpr, group = threadIdx.x / tpr, lane = threadIdx.x - group * tpr;
    GroupSum total(red_all + group * kRedFloats, group, tpr);
    const float inv_h = 1.0f / (float)a.H;
    const int units = (a.H + 7) / 8;
    const bool branch = ALL || (CK ? a.u8 != nullptr : a.y != nullptr);
    const bool has_dn = ALL || a.dn, has_up = ALL || a.dh_out, has_dh = ALL || a.dh, has_dy = ALL || a.dy;
    const int t_first = (int)(blockIdx.x * a.groups + group), t_step = (int)(gridDim.x * a.groups);
    const uint32_t row_bytes = (uint32_t)(a.H * sizeof(X)), act_bytes = CK ? (uint32_t)a.H : row_bytes;
    // of an array in a place
    const uint32_t row_pitch = ODD ? (row_bytes + 30) / 16 * 16 : row_bytes, act_pitch = ODD ? (act_bytes + 30) / 16 * 16 : act_bytes;
    unsigned char* after = ring_mem + (size_t)a.groups * a.depth * (2 * (row_pitch + act_pitch) + 16);
    RowInfo* table = reinterpret_cast<RowInfo*>(after) + group * kTable;
    float* weights = reinterpret_cast<float*>(after + a.groups * kTable * sizeof(RowInfo));   // [2][H]: w_post, w_pre (not WREG)
    for (int i = lane; i < kTable; i += tpr) table[i] = info_of<CK>(a, branch, t_first + (long long)i * t_step);
    for (int c = threadIdx.x; c < a.H && !WREG; c += blockDim.x) {
        weights[c] = a.w_post ? a.w_post[c] : 1.0f;
        weights[a.H + c] = a.w_pre ? a.w_pre[c] : 1.0f;
    }
    // places of [dh_out][dn][h_out or x8][y or u8]; with a barrier of the CTA
    RowRing ring = ring_of(ring_mem, group, a.groups, a.depth, 2 * (int)(row_pitch + act_pitch), 4);
    // Row t, whose output row is s, into a place: by four threads of different warps where there are four, one an array.
    const int wide4 = tpr / kWarp, asked = (lane % kWarp) * wide4 + lane / kWarp;
    const bool asks = lane % kWarp * wide4 < 4 && asked < 4;
    const unsigned char* from = nullptr;
    uint32_t len = 0, at_place = 0;
    if (asks) {
        if (asked == 0) from = static_cast<const unsigned char*>(a.dh_out);
        else if (asked == 1) from = static_cast<const unsigned char*>(a.dn);
        else if (asked == 2) from = !has_dn ? nullptr : CK ? reinterpret_cast<const unsigned char*>(a.x8) : static_cast<const unsigned char*>(a.h_out);
        else from = CK ? reinterpret_cast<const unsigned char*>(a.u8) : static_cast<const unsigned char*>(a.y);
        len = asked < 2 ? row_bytes : act_bytes;
        at_place = asked < 2 ? asked * row_pitch : 2 * row_pitch + (asked - 2) * act_pitch;
    }
    const bool slots = asked == 3 && !CK;   // codes lie in token order, the block's output in slot order
    auto ask = [&](int t, int s, int place) {
        uint64_t* bar = ring.bars + place;
        unsigned char* to = ring.base + (uint32_t)(place * ring.stage) + at_place;
        const bool wanted = from && (asked < 3 || s >= 0);
        const size_t off = (size_t)(uint32_t)(slots ? s : t) * len;
        Piece p{off, wanted ? len : 0u, 0u};
        if constexpr (ODD) {
            if (wanted) p = piece_of(off, len, (size_t)(slots ? a.rows : a.T) * len);
            tail_of(to, from, p);
        }
        mbar_expect_tx(bar, p.bytes);
        if (p.bytes) bulk_g2s(to, from + p.from, p.bytes, bar);
    };
    if (asks)
        for (int d = 0; d < a.depth && t_first + (long long)d * t_step < a.T; ++d) ask(t_first + d * t_step, table[d].s, d);
    const int ahead = a.depth * t_step, last_ask = a.T - ahead;
    // this thread's places in a row, in its activations, in the weights
    bool have[NV];
    uint32_t off[NV], act[NV];
    int first[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int un = lane + i * tpr;
        have[i] = FULL || un < units;
        off[i] = un * UB;
        act[i] = un * AB;
        first[i] = lane + 8 * i * tpr;   // ODD: this thread's elements are first + j * tpr
    }
    Unit8 w_own[WREG ? 2 * NV : 1];
    if constexpr (WREG)
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (FULL || ODD || have[i]) {
                w_own[i] = weight_unit<ODD>(a.w_post, lane + i * tpr, first[i], tpr, a.H);
                w_own[NV + i] = weight_unit<ODD>(a.w_pre, lane + i * tpr, first[i], tpr, a.H);
            }
    auto weight = [&](bool post, int i) {
        const float* w = weights + (post ? 0 : a.H);
        if constexpr (WREG) return w_own[post ? i : NV + i];
        else if constexpr (ODD) return widen<float>(load_raw<float, false, true>(reinterpret_cast<const unsigned char*>(w), 0, first[i], tpr, a.H));
        else return load_pairs<float>(reinterpret_cast<const unsigned char*>(w + (lane + i * tpr) * 8));
    };
    using Raw = typename RawUnit<X, CK>::type;
    // row t's gradients (k = 0, 1), its activations from h_out / x8 and those from y / u8
    auto raw_row = [&](const unsigned char* place, int t, int k, int i) {
        return load_raw<X, false, ODD>(place + k * row_pitch + (ODD ? (uint32_t)t * row_bytes & 15 : 0), off[i], first[i], tpr, a.H);
    };
    auto raw_x = [&](const unsigned char* place, int t, int i) {
        return load_raw<X, CK, ODD>(place + 2 * row_pitch + (ODD ? (uint32_t)t * act_bytes & 15 : 0), act[i], first[i], tpr, a.H);
    };
    auto raw_u = [&](const unsigned char* place, int t, int s, int i) {
        return load_raw<X, CK, ODD>(place + 2 * row_pitch + act_pitch + (ODD ? (uint32_t)(CK ? t : s) * act_bytes & 15 : 0), act[i], first[i], tpr, a.H);
    };
    Unit8 acc_post[NV], acc_pre[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) { clear(acc_post[i]); clear(acc_pre[i]); }
    Unit8 e[NV];                                       // D w_post
    Raw u[NV], x[NV];                                  // u', x' and dn as they lie in memory: half the registers
    typename RawUnit<X, false>::type dn[NV];
    // A row's first sums: x'^2, u'^2, dn w_pre x'.
    auto begin = [&](const unsigned char* place, int t, int s, float& xx, float& uu, float& dot) {
        float2 sx = both(0.0f), su = both(0.0f), sg = both(0.0f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!FULL && !ODD && !have[i]) continue;
            if (has_dn) {
                x[i] = raw_x(place, t, i);
                dn[i] = raw_row(place, t, 1, i);
                const Unit8 xv = widen<X>(x[i]), g = widen<X>(dn[i]), w = weight(false, i);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (!CK) sx = __ffma2_rn(xv.p[j], xv.p[j], sx);
                    sg = __ffma2_rn(__fmul2_rn(g.p[j], xv.p[j]), w.p[j], sg);
                }
            }
            if (!CK && s >= 0) {
                const Unit8 v = widen<X>(raw_u(place, t, s, i));
#pragma unroll
                for (int j = 0; j < 4; ++j) su = __ffma2_rn(v.p[j], v.p[j], su);
            }
        }
        xx = sx.x + sx.y; uu = su.x + su.y; dot = sg.x + sg.y;
    };
    RowInfo soon{}, f{};
    unsigned char* dh_row = static_cast<unsigned char*>(a.dh) + (size_t)t_first * row_bytes;
    const size_t dh_step = (size_t)t_step * row_bytes;
    const unsigned char* place = nullptr;
    int at = 0;                        // the row's place
    float xx = 0.0f, uu = 0.0f, dot = 0.0f;
    if (t_first < a.T) {
        f = table[0];
        place = ring.wait();
        ring.next();
        begin(place, t_first, f.s, xx, uu, dot);
        total.three(xx, uu, dot);
    }
    int n = 0;   // the row's number within the group
    for (int t = t_first; t < a.T; t += t_step, ++n) {
        if (lane < 32) {
            if ((n & 31) == 0 && n > 0) soon = info_of<CK>(a, branch, t + (32 + lane) * (long long)t_step);
            if ((n & 31) == 16 && n > 32) table[(n + 16 + lane) & (kTable - 1)] = soon;
        }
        float q = f.q, r = f.r, xs = 1.0f, us = 1.0f;
        if constexpr (!CK) {
            xs = q = rsqrtf(fmaf(xx, inv_h, a.eps));
            us = r = rsqrtf(fmaf(uu, inv_h, a.eps));
        }
        const float2 q2 = both(q), cx = both(-q * xs * (dot * xs * inv_h)), gu = both(f.gate * us), xs2 = both(xs), a2 = both(a.res_scale);
        float2 sk = both(0.0f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!FULL && !ODD && !have[i]) continue;
            Unit8 D;
            clear(D);
            if (has_up) D = widen<X>(raw_row(place, t, 0, i));
            if (has_dn) {
                if constexpr (sizeof(X) == 4) {   // too many registers to keep
                    x[i] = raw_x(place, t, i);
                    dn[i] = raw_row(place, t, 1, i);
                }
                const Unit8 xv = widen<X>(x[i]), g = widen<X>(dn[i]), w = weight(false, i);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    D.p[j] = __ffma2_rn(cx, xv.p[j], __ffma2_rn(q2, __fmul2_rn(g.p[j], w.p[j]), D.p[j]));
                    acc_pre[i].p[j] = __ffma2_rn(xs2, __fmul2_rn(g.p[j], xv.p[j]), acc_pre[i].p[j]);
                }
            }
            if (f.s >= 0) {
                u[i] = raw_u(place, t, f.s, i);
                const Unit8 v = widen<X>(u[i]), w = weight(true, i);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 du = __fmul2_rn(D.p[j], v.p[j]);
                    acc_post[i].p[j] = __ffma2_rn(gu, du, acc_post[i].p[j]);
                    sk = __ffma2_rn(du, w.p[j], sk);
                    e[i].p[j] = __fmul2_rn(D.p[j], w.p[j]);
                }
            }
            if (has_dh) {
#pragma unroll
                for (int j = 0; j < 4; ++j) D.p[j] = __fmul2_rn(a2, D.p[j]);
                store_unit<X, ODD>(dh_row, off[i], first[i], tpr, a.H, D);
            }
        }
        dh_row += dh_step;
        // the next row's first sums beside this one's last
        const RowInfo here = f;
        const int was = at;
        if (t + (long long)t_step < a.T) {
            f = table[(n + 1) & (kTable - 1)];
            at = ring.place;
            place = ring.wait();
            ring.next();
            begin(place, t + t_step, f.s, xx, uu, dot);
        }
        float k = sk.x + sk.y;
        total.four(k, xx, uu, dot);
        __syncwarp();
        if (asks && t < last_ask) ask(t + ahead, table[(n + a.depth) & (kTable - 1)].s, was);   // the group is done with the row
        k = here.s < 0 ? 0.0f : k * us;
        if (lane == 0 && a.dgate) a.dgate[t] = k;
        if (has_dy && here.s >= 0) {
            const float rg = r * here.gate;
            const float2 rg2 = both(rg), cu = both(-rg * us * (k * inv_h));
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (!FULL && !ODD && !have[i]) continue;
                const Unit8 v = widen<X>(u[i]);
#pragma unroll
                for (int j = 0; j < 4; ++j) e[i].p[j] = __ffma2_rn(cu, v.p[j], __fmul2_rn(rg2, e[i].p[j]));
                store_unit<X, ODD>(static_cast<unsigned char*>(a.dy) + (size_t)here.s * row_bytes, off[i], first[i], tpr, a.H, e[i]);
            }
        }
    }
    ring.leave();
    if (a.part_post || a.part_pre) {   // the groups' columns meet where the rings were (8 H bytes a group fit there), added in group order
        float* cols = reinterpret_cast<float*>(ring_mem);   // [groups][2][H]
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float* to = cols + (size_t)group * 2 * a.H;
            if constexpr (ODD) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int c = first[i] + j * tpr;
                    if (c >= a.H) continue;
                    to[c] = j & 1 ? acc_post[i].p[j / 2].y : acc_post[i].p[j / 2].x;
                    to[a.H + c] = j & 1 ? acc_pre[i].p[j / 2].y : acc_pre[i].p[j / 2].x;
                }
            } else if (FULL || have[i]) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    reinterpret_cast<float2*>(to)[(lane + i * tpr) * 4 + j] = acc_post[i].p[j];
                    reinterpret_cast<float2*>(to + a.H)[(lane + i * tpr) * 4 + j] = acc_pre[i].p[j];
                }
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * a.H; c += blockDim.x) {
            float v = cols[c];
            for (int g = 1; g < a.groups; ++g) v += cols[(size_t)g * 2 * a.H + c];
            if (c < a.H) {
                if (a.part_post) a.part_post[(size_t)blockIdx.x * a.H + c] = v;
            } else if (a.part_pre) {
                a.part_pre[(size_t)blockIdx.x * a.H + c - a.H] = v;
            }
        }
    }
    if (a.dy && a.inv) {   // rows of the slot buffer that no token owns have a zero gradient
        Unit8 z;
        clear(z);
        const int l = threadIdx.x & 31;
        for (long long row0 = (long long)t_first * 32; row0 < a.rows; row0 += (long long)t_step * 32) {   // every warp sees the same 32 rows
            unsigned empty = __ballot_sync(0xffffffffu, row0 + l < a.rows && a.inv[row0 + l] < 0);
            for (; empty; empty &= empty - 1) {
                unsigned char* to = static_cast<unsigned char*>(a.dy) + (size_t)(row0 + __ffs(empty) - 1) * row_bytes;
                if constexpr (ODD) for (int c = lane; c < a.H; c += tpr) reinterpret_cast<X*>(to)[c] = 0;
                else for (int un = lane; un < units; un += tpr) store_pairs<X>(to + un * UB, z);
            }
        }
    }
}

// Column sums: the CTAs' rows of the workspace added in index order (fp32, 16 interleaved chains joined in order).
constexpr int kColThreads = 512, kColChains = 16;
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
#pragma unroll 10
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
RowPlan plan_rows(int units, int nv, int threads, int T) {
    int tpr = nv > 0 ? (units + nv - 1) / nv : threads;
    tpr = (tpr + kWarp - 1) / kWarp * kWarp;
    if (tpr > 1024) tpr = 1024;
    int groups = nv > 0 ? threads / tpr : 1;
    if (groups < 1) groups = 1;
    if (groups > kMaxGroups) groups = kMaxGroups;
    const int share = (T + sm_count() - 1) / sm_count();   // few rows are spread over the SMs
    if (groups > share) groups = share;
    return {tpr, groups};
}

constexpr int kGradCtasPerSm = 1;       // one row of column sums each
constexpr int kRingSmem = 210 << 10;    // shared memory of a CTA for rings and weights, beside the static strips
constexpr int kRingMaxDepth = 4;

bool aligned(const void* p, int n) { return (uintptr_t)p % n == 0; }

// Rings of `groups` groups with `stage` bytes a row beside `extra` bytes: their depth, 0 if two rows do not fit; and the
// shared memory of rings, barriers and tables.
int ring_depth(int groups, int stage, int extra) {
    int d = (kRingSmem - extra - groups * kTable * (int)sizeof(RowInfo)) / (groups * (stage + 16));
    if (d > kRingMaxDepth) d = kRingMaxDepth;
    return d < 2 ? 0 : d;
}
size_t ring_bytes(int groups, int depth, int stage) { return (size_t)groups * (depth * (stage + 16) + kTable * sizeof(RowInfo)); }
int round16(int n) { return (n + 15) / 16 * 16; }
template <typename K>
bool allow_smem(K kernel, size_t bytes) {
    if (bytes <= 32 << 10) return true;   // with the static strips within the 48 KB that need no leave
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess) return true;
    cudaGetLastError();
    return false;
}

template <typename X>
int forward(NormArgs& a, cudaStream_t st) {
    // bulk copies and vectors need arrays that begin at their boundaries; rows may begin anywhere
    const bool based = aligned(a.h, 16) && aligned(a.y, 16) && aligned(a.h_out, 16) && aligned(a.n_out, 16) && aligned(a.w_post, 16) &&
                       aligned(a.w_pre, 16) && aligned(a.u8, 8) && aligned(a.x8, 8);
    const bool wide = based && a.H % 8 == 0;
    const int units = wide ? a.H / 8 : a.H;
    auto launch = [&](auto kernel, const RowPlan& p, int ctas, size_t smem) {
        a.tpr = p.tpr; a.groups = p.groups;
        const int threads = p.tpr * p.groups;
        long long grid = (a.T + p.groups - 1) / p.groups;
        const long long most = (long long)sm_count() * ctas;
        if (grid > most) grid = most;
        if (!allow_smem(kernel, smem)) return (int)LOCMOE_ERR_CUDA;
        return launch_pdl(kernel, dim3((unsigned)grid), dim3(threads), smem, st, a);
    };
    // The ring wherever a row has at most two units a thread (65536 x 5120 in bf16: 418 us against 699 by the kernel that
    // loads its rows itself; gradient of 3001 x 777, rows that begin anywhere: 22 against 33); longer rows, and arrays that
    // bulk copies cannot take, go through that kernel.
    const bool ck = a.u8 || a.x8;
    if (based && a.H <= 16 * kRingThreads) {
        const int eights = (a.H + 7) / 8, row = a.H * (int)sizeof(X);
        const bool fewer = !wide && !ck && sizeof(X) == 4 && eights <= 2 * kOddThreads;
        const RowPlan p = plan_rows(eights, 2, fewer ? kOddThreads : kRingThreads, a.T);
        const int stage = 2 * (wide ? row : round16(row + 15));
        a.depth = ring_depth(p.groups, stage, 0);
        const size_t smem = ring_bytes(p.groups, a.depth, stage);
        if (a.depth) {
            const bool full = eights == 2 * p.tpr;
            if (!wide && ck) return launch(block_norm_ring_kernel<X, false, true, true>, p, 1, smem);
            if constexpr (sizeof(X) == 4)
                if (fewer) return launch(block_norm_ring_kernel<X, false, false, true, kOddThreads>, p, 1, smem);
            if (!wide) return launch(block_norm_ring_kernel<X, false, false, true>, p, 1, smem);
            if (ck) return full ? launch(block_norm_ring_kernel<X, true, true, false>, p, 1, smem) : launch(block_norm_ring_kernel<X, false, true, false>, p, 1, smem);
            return full ? launch(block_norm_ring_kernel<X, true, false, false>, p, 1, smem) : launch(block_norm_ring_kernel<X, false, false, false>, p, 1, smem);
        }
    }
    const int nv = wide ? 0 : (units <= 1024 * 8 ? 8 : 0);
    const RowPlan p = plan_rows(units, nv, 256, a.T);
    const int ctas = 2048 / (p.tpr * p.groups) > 0 ? 2048 / (p.tpr * p.groups) : 1;
    if (wide) return launch(block_norm_kernel<X, 8, 0>, p, ctas, 0);
    return nv ? launch(block_norm_kernel<X, 1, 8>, p, ctas, 0) : launch(block_norm_kernel<X, 1, 0>, p, ctas, 0);
}

template <typename X, bool CK>
int backward(NormGradArgs& a, float* dw_post, float* dw_pre, cudaStream_t st) {
    const bool based = aligned(a.dh_out, 16) && aligned(a.dn, 16) && aligned(a.h_out, 16) && aligned(a.y, 16) && aligned(a.x8, 16) &&
                       aligned(a.u8, 16) && aligned(a.w_post, 16) && aligned(a.w_pre, 16) && aligned(a.dh, 16) && aligned(a.dy, 16);
    const bool wide = based && a.H % 8 == 0;
    const int units = wide ? a.H / 8 : a.H;
    long long grid = 0;
    auto launch = [&](auto kernel, const RowPlan& p, int ctas, size_t smem) {
        a.tpr = p.tpr; a.groups = p.groups;
        const int threads = p.tpr * p.groups;
        grid = (a.T + p.groups - 1) / p.groups;
        const long long most = (long long)sm_count() * ctas;
        if (grid > most) grid = most;
        if (!allow_smem(kernel, smem)) return (int)LOCMOE_ERR_CUDA;
        return launch_pdl(kernel, dim3((unsigned)grid), dim3(threads), smem, st, a);
    };
    int rc = LOCMOE_OK;
    bool done = false;
    // as in the forward pass: the ring where a row has at most two units a thread
    if (based && a.H <= 8 * 1024) {
        const int eights = (a.H + 7) / 8, row = a.H * (int)sizeof(X), act = CK ? a.H : row;
        const bool wreg = eights <= 2 * kGradThreads;   // (one unit a thread with 512 threads: 612 us against 640 at 65536 x 4096, but 531 / 375 at 2560)
        const RowPlan p = plan_rows(eights, 2, wreg ? kGradThreads : 512, a.T);
        const bool whole = wide && act % 16 == 0;   // all rows are whole 16-byte pieces
        const int stage = whole ? 2 * (row + act) : 2 * (round16(row + 15) + round16(act + 15)), extra = wreg ? 0 : 8 * a.H;
        a.depth = ring_depth(p.groups, stage, extra);
        if (a.depth) {
            const size_t smem = ring_bytes(p.groups, a.depth, stage) + extra;
            const bool all = a.dh_out && a.dn && (CK ? (const void*)a.u8 : a.y) && a.dh && a.dy;
            if (!whole) rc = wreg ? launch(block_norm_grad_ring_kernel<X, CK, true, false, false, true>, p, 1, smem)
                                  : launch(block_norm_grad_ring_kernel<X, CK, false, false, false, true>, p, 1, smem);
            else if (!wreg) rc = launch(block_norm_grad_ring_kernel<X, CK, false, false, false, false>, p, 1, smem);
            else if (!all) rc = launch(block_norm_grad_ring_kernel<X, CK, true, false, false, false>, p, 1, smem);
            else if (eights == 2 * p.tpr) rc = launch(block_norm_grad_ring_kernel<X, CK, true, true, true, false>, p, 1, smem);
            else rc = launch(block_norm_grad_ring_kernel<X, CK, true, false, true, false>, p, 1, smem);
            done = true;
        }
    }
    if (!done) {
        // The row in registers where it fits 512 threads (32768 rows of 8192 in fp32 1465 us, read again after each sum 4037; of
        // 8191 3807 / 6825).
        const int nv = wide ? (units <= 512 * 2 ? 2 : 0) : units <= 512 * 8 ? 8 : units <= 512 * 16 ? 16 : 0;
        const RowPlan p = plan_rows(units, nv, 512, a.T);
        const size_t smem = nv && p.groups > 1 ? (size_t)a.H * 8 : 0;
        if (wide) rc = nv ? launch(block_norm_grad_kernel<X, 8, 2, CK>, p, kGradCtasPerSm, smem)
                          : launch(block_norm_grad_kernel<X, 8, 0, CK>, p, kGradCtasPerSm, smem);
        else rc = nv == 8 ? launch(block_norm_grad_kernel<X, 1, 8, CK>, p, kGradCtasPerSm, smem)
                : nv ? launch(block_norm_grad_kernel<X, 1, 16, CK>, p, kGradCtasPerSm, smem)
                     : launch(block_norm_grad_kernel<X, 1, 0, CK>, p, kGradCtasPerSm, smem);
    }
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
               rows, s.T, s.H, 0, 0, 0};
    return s.x_dtype == LOCMOE_F32 ? forward<float>(a, st) : forward<uint16_t>(a, st);
}

int launch_block_norm_grad(const locmoe_shape_t& s, long long rows, const locmoe_block_norm_grad_t& b, void* ws, cudaStream_t st) {
    float* part = static_cast<float*>(ws);
    NormGradArgs a{b.dh_out, b.dn, b.h_out, b.y, b.x8, b.u8, b.r_pre, b.r_post, b.slot, b.slot ? b.inv : nullptr, b.gate_w, b.w_post,
                   b.w_pre, b.res_scale, b.eps, b.dh, b.dy, b.dgate, b.dw_post ? part : nullptr,
                   b.dw_pre ? part + (size_t)sm_count() * kGradCtasPerSm * s.H : nullptr, rows, s.T, s.H, 0, 0, 0};
    const bool ck = b.x8 || b.u8;
    if (s.x_dtype == LOCMOE_F32)
        return ck ? backward<float, true>(a, b.dw_post, b.dw_pre, st) : backward<float, false>(a, b.dw_post, b.dw_pre, st);
    return ck ? backward<uint16_t, true>(a, b.dw_post, b.dw_pre, st) : backward<uint16_t, false>(a, b.dw_post, b.dw_pre, st);
}

int read_norm_flags(int* out, cudaStream_t st) {
    if (cudaMemcpyFromSymbolAsync(out, g_norm_flags, sizeof(int), 0, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaStreamSynchronize(st) != cudaSuccess) {
        cudaGetLastError();
        return LOCMOE_ERR_CUDA;
    }
    return LOCMOE_OK;
}

}  // namespace locmoe
