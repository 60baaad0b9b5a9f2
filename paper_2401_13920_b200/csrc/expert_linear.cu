// The experts' products on rows sorted by expert: group e is the rows [offsets[e], offsets[e + 1]), of any length.
//   forward   y[r]  = act(x[r] W_e^T + b_e) + residual[r]            W_e [N][K]
//   towards x dx[r] = (dy[r] W_e) * act'(z[r])                       W_e [K][N] here: the reduction runs over its rows
//   weights   dW_e  = dy_e^T x_e,  db_e = sum of dy_e's rows         the reduction runs over the group's rows
// One GEMM kernel on the tensor cores (tcgen05, bf16 operands, fp32 accumulators in TMEM) serves all three: 128 x 256 output
// tiles, operands by TMA into a ring of four stages of 64 along the reduction, two accumulators so that a tile's epilogue runs
// beside the next tile's products; or tiles of 256 x 256, an accumulator for each half, where loads are the limit.  An operand whose rows run along the reduction is K-major, else MN-major: the same TMA
// boxes of 64 elements x rows, the matrix descriptor says which way they lie, so nothing is transposed in memory.
// Warp 0 loads, warp 1 issues the products, warps 2..9 drain the accumulators (a row a lane, half of the columns a warp).
//
// A group may begin and end inside a tile.  Forward and towards x that only means rows which are not stored; over the group's
// rows (weights) the last block of the reduction holds rows of the next group, and those are overwritten with zeros in shared
// memory, in both operands, since a zero in one does not undo an infinity in the other.
//
// Work is dealt by tiles (tile i to CTA i modulo the grid), neighbours in time sharing operands in L2, and what is left after the
// last full wave in equal runs of 64-blocks of the reduction, so that every SM gets the same share whatever the groups are.
// A tile that a run begins or ends in leaves fp32 sums in the workspace, which a second kernel adds in order.
//
// A few rows, and the bias's gradient alone, have kernels without tiles.
#include <cuda.h>

#include "common.cuh"
#include "tensor_map.cuh"
#include "umma.cuh"

namespace locmoe {

namespace {

constexpr int BM = 128, BN = 256, BK = 64, UMMA_K = 16;
constexpr uint32_t A_BYTES = BM * BK * 2, B_BYTES = BN * BK * 2;
constexpr uint32_t CHUNK_BYTES = 64 * BK * 2;       // 64 columns of an MN-major tile
constexpr uint32_t TMEM_COLS = 512;
constexpr int kMaxE = 1024;

enum Kind { kForward = 0, kTowardsX = 1, kWeights = 2 };

// Warps after the two that load and issue: the epilogue's (sixteen of them on 16 columns a step were 10 % slower throughout), and
// those of the column sums.
constexpr int kEpiWarps = 8, kEpiThreads = 32 * kEpiWarps;
constexpr int kSumWarps = 4;                        // only where the weights' gradient comes with the bias's
constexpr int kThreads = 64 + kEpiThreads, kWeightsThreads = kThreads + 32 * kSumWarps;

// Shared memory: the ring (four whole stages; more of them where the rows are few and A short), or three stages and two boxes a
// warp (weights' gradients of short groups); then the barriers, the offsets, a tile's bias.
constexpr uint32_t kBoxBytes = 32 * 128;            // 32 rows of 128 bytes on their way out
constexpr int kMaxStages = 6, kBoxStages = 3;
constexpr size_t kRing = kBoxStages * (size_t)(A_BYTES + B_BYTES) + 2 * kEpiWarps * kBoxBytes;
static_assert(kRing >= 4 * (size_t)(A_BYTES + B_BYTES) && kRing >= 6 * (size_t)(16 * BK * 2 + B_BYTES), "the rings fit");
constexpr size_t kOffsetBytes = (kMaxE + 4) * sizeof(int), kBiasBytes = BN * 4 * sizeof(float);
constexpr size_t kSmem = 1024 /*alignment slack*/ + kRing + 256 /*barriers*/ + kOffsetBytes + kBiasBytes;
static_assert(kSmem <= 227 * 1024, "all of it fits");

__device__ int g_linear_flags = 0;   // bit 0: a bounded wait gave up

// A tile whose first blocks are run c's last ones, left to the kernel that joins: written by CTA c, rows = 0 if there is none.
struct __align__(16) Split {
    int e, row, rows, nt;       // expert, the tile's first row in the output, its rows, its column
    int last, pad[3];           // last run that worked on it
};

struct LinearArgs {
    const int32_t* offsets;     // [E + 1]
    void* out;                  // bf16 [R][N], or the weights' gradient [E][M][N], bf16 or fp32
    void* z_out;                // bf16 [R][N] or nullptr
    const float* bias;          // [E][N] or nullptr
    const void* residual;       // bf16 [R][N] or nullptr
    const void* z_in;           // bf16 [R][N]: multiply by act'(z_in); nullptr: no factor
    float* part;                // [grid][2][part_rows][BN]
    float* db;                  // weights only: [E][M] or nullptr
    float* db_part;             // [grid][2][unit]
    Split* split;               // [grid]
    int act, out_f32;
    int E, R, M, N, K;          // M: rows of a weight (weights only)
    int unit;                   // rows of a tile: BM, or 2 BM with an accumulator for each half
    int n_tiles, a_rows;        // rows of one A box
    int stages;                 // of the ring
    int boxes;                  // weights: rows leave as boxes
    int a_chunks, b_chunks;     // 1: one load brings an MN-major tile, else one for each 64 columns
    int part_rows;
    int grid;
};

__device__ __forceinline__ bool wait_or_abort(uint64_t* bar, uint32_t parity, volatile int* abort_word) {
    for (uint32_t i = 0; i < (1u << 22); ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 63u) == 63u && *abort_word) return false;
    }
    *abort_word = 1;
    atomicOr(&g_linear_flags, 1);
    return false;
}

// The same for a warp that stays together: all lanes get one answer.
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, volatile int* abort_word) {
    return __all_sync(0xffffffffu, wait_or_abort(bar, parity, abort_word));
}

// Group e's rows, whatever the offsets hold: inside [0, R) and not negative in number.
struct Group { int lo, n; };
__device__ __forceinline__ Group group_of(const int* offsets, int e, int R) {
    const int lo = min(max(offsets[e], 0), R);
    return {lo, max(min(offsets[e + 1], R) - lo, 0)};
}

// The list of work: the groups' tiles in order, a tile being `kb` blocks of the reduction.
template <int KIND, int HALVES>
struct Tiles {
    static constexpr int UNIT = HALVES * BM;
    const LinearArgs& a;
    const int* offsets;
    __device__ __forceinline__ int kblocks(const Group& g) const { return KIND == kWeights ? (g.n + BK - 1) / BK : (a.K + BK - 1) / BK; }
    __device__ __forceinline__ int m_tiles(const Group& g) const { return ((KIND == kWeights ? a.M : g.n) + UNIT - 1) / UNIT; }
    __device__ __forceinline__ int tiles(const Group& g) const { return g.n > 0 ? m_tiles(g) * a.n_tiles : 0; }
};

constexpr float kWeightsBlock = 0.4f, kJoinUs = 3.0f, kRowUs = 0.05f;     // us, see deal()

// How the work is dealt, the same on every CTA.  Tiles below `whole` go to the CTAs one by one; what they leave, less than a tile
// for every CTA, is cut into `runs` equal runs of blocks, or dealt like the others (whole = all tiles) where that is no slower.
struct Deal {
    int tiles, whole, runs;
    long long each;             // run c begins at each * c + min(c, more) of the rest's blocks
    int more;
    __device__ __forceinline__ long long begin(int c) const { return each * c + min(c, more); }
};

__device__ __forceinline__ long long sum_warp(long long v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// By one warp (all lanes get it).  Splitting the rest saves what its longest tile takes beyond an equal share, at 0.27 us a block
// where the tensor cores are the limit, 0.4 where a few SMs stream the rows of long groups (weights), and up to 0.73 where
// each weight tile is used by one tile of rows and comes out of HBM at 148 x 32 KB a step.  It costs the join's launch, 3 us,
// and the sums' way through memory, 0.05 us for each row of a tile (1981 rows of 304 x 1024 with every tile split 28 against
// 19 us whole; 8 rows of one expert, 10240 x 2560, 10 tiles in all, 20 us split; weights' gradient of 10749 rows in 4 groups, 400 x 160,
// 16 tiles, 52 us whole, 32 split).
template <int KIND, int HALVES>
__device__ __forceinline__ Deal deal(const LinearArgs& a, const int* offsets, int lane) {
    const Tiles<KIND, HALVES> t{a, offsets};
    long long n = 0, rows = 0, rowtiles = 0, groups = 0;
    for (int e = lane; e < a.E; e += 32) {
        const Group g = group_of(offsets, e, a.R);
        n += t.tiles(g);
        rows += g.n;
        if (g.n > 0) { rowtiles += t.m_tiles(g); ++groups; }
    }
    Deal d{(int)sum_warp(n), 0, 0, 0, 0};
    d.whole = d.tiles;
    const int rest = d.tiles % a.grid;
    if (rest == 0 || !a.split) return d;
    // blocks of the last `rest` tiles
    long long units = 0, longest = (a.K + BK - 1) / BK;
    if (KIND == kWeights) {
        longest = 0;
        int before = 0;                                         // tiles of the groups passed
        for (int e0 = 0; e0 < a.E; e0 += 32) {
            const Group g = e0 + lane < a.E ? group_of(offsets, e0 + lane, a.R) : Group{0, 0};
            const unsigned busy = __ballot_sync(0xffffffffu, g.n > 0);
            const int per = t.m_tiles(g) * a.n_tiles, first = before + per * __popc(busy & ((1u << lane) - 1u));
            const int in = g.n > 0 ? max(0, min(per, first + per - (d.tiles - rest))) : 0;
            units += (long long)in * t.kblocks(g);
            if (in > 0) longest = max(longest, (long long)t.kblocks(g));
            before += per * __popc(busy);
        }
        units = sum_warp(units);
#pragma unroll
        for (int o = 16; o; o >>= 1) longest = max(longest, __shfl_xor_sync(0xffffffffu, longest, o));
    } else {
        units = (long long)rest * ((a.K + BK - 1) / BK);
    }
    rows = sum_warp(rows); rowtiles = sum_warp(rowtiles); groups = sum_warp(groups);
    const float block = (float)HALVES * (KIND == kWeights ? kWeightsBlock : fmaxf(0.27f, 0.73f * (float)groups / (float)rowtiles));
    const float tile_rows = KIND == kWeights ? (float)(HALVES * BM) : (float)rows / (float)rowtiles;
    if (((float)longest - (float)units / (float)a.grid) * block < kJoinUs + kRowUs * tile_rows) return d;
    const long long r = units / 4;                              // a run has at least four blocks
    d.whole = d.tiles - rest;
    d.runs = r < 1 ? 1 : r < a.grid ? (int)r : a.grid;
    d.each = units / d.runs;
    d.more = (int)(units - d.each * d.runs);
    return d;
}
// The host's side of that rule: whether any offsets could lead to a split.
template <int KIND>
bool may_split(const LinearArgs& a) {
    const float kb = (float)(((KIND == kWeights ? a.R : a.K) + BK - 1) / BK);
    return KIND == kWeights ? kb * (float)(a.unit / BM) * kWeightsBlock >= kJoinUs + kRowUs * (float)a.unit : kb * (float)(a.unit / BM) * 0.73f >= kJoinUs;
}

struct Item {
    int e, lo, n;               // group, its first row, its rows
    int mt, nt;                 // tile
    int kb0, kb1, kb;           // blocks of this item, blocks of the tile
    long long begin;            // in a run: the tile's first block among the rest's
};

// Halves of a tile that hold rows.
template <int KIND, int HALVES>
__device__ __forceinline__ int halves_of(const LinearArgs& a, const Item& it) {
    return HALVES == 2 && (KIND == kWeights ? a.M : it.n) - it.mt * HALVES * BM > BM ? 2 : 1;
}

// Walks through one CTA's share: its tiles, then its run.
template <int KIND, int HALVES>
struct Cursor {
    const LinearArgs& a;
    const int* offsets;
    const Deal& d;
    int tile, e, base;          // next tile; group; the group's first tile
    long long at, end, ubase;   // next block and end of the run; blocks of the rest before group e
    Group g;
    int kb, per;                // blocks a tile, tiles of group e
    __device__ __forceinline__ Cursor(const LinearArgs& a_, const int* off, const Deal& d_, int c) : a(a_), offsets(off), d(d_), tile(c), e(-1), base(0), ubase(0) {
        g = Group{0, 0};
        kb = per = 0;
        at = c < d.runs ? d.begin(c) : 0;
        end = c < d.runs ? d.begin(c + 1) : 0;
    }
    __device__ __forceinline__ int rest() const { return max(0, min(per, base + per - d.whole)); }     // tiles of group e in runs
    __device__ __forceinline__ bool step() {
        ubase += (long long)rest() * kb;
        base += per;
        if (++e >= a.E) return false;
        const Tiles<KIND, HALVES> t{a, offsets};
        g = group_of(offsets, e, a.R);
        kb = t.kblocks(g);
        per = t.tiles(g);
        return true;
    }
    __device__ __forceinline__ bool next(Item& it) {
        int in;                 // tile inside the group
        if (tile < d.whole) {
            while (e < 0 || tile >= base + per)
                if (!step()) return false;
            in = tile - base;
            it.kb0 = 0;
            it.kb1 = kb;
            tile += a.grid;
        } else if (at < end) {
            while (e < 0 || at >= ubase + (long long)rest() * kb)
                if (!step()) return false;
            const long long rel = at - ubase;
            const int j = (rel >> 32) == 0 ? (int)((uint32_t)rel / (uint32_t)kb) : (int)(rel / kb);
            in = per - rest() + j;
            it.begin = ubase + (long long)j * kb;
            it.kb0 = (int)(at - it.begin);
            const long long left = end - at;
            it.kb1 = left < kb - it.kb0 ? it.kb0 + (int)left : kb;
            at += it.kb1 - it.kb0;
        } else {
            return false;
        }
        it.kb = kb;
        it.e = e; it.lo = g.lo; it.n = g.n;
        if (KIND == kWeights && a.boxes) {      // whole rows of the gradient are written at a time
            it.mt = in / a.n_tiles;
            it.nt = in - it.mt * a.n_tiles;
        } else {                        // tiles that share a weight tile are neighbours
            const int mts = Tiles<KIND, HALVES>{a, offsets}.m_tiles(g);
            it.nt = in / mts;
            it.mt = in - it.nt * mts;
        }
        return true;
    }
};

// Descriptor of an MN-major bf16 tile with 128-byte swizzle, as TMA boxes of 64 elements x 64 rows leave it: a row of 128
// bytes is 64 elements at one step of the reduction, 8 steps are 1024 bytes (stride byte offset), the next 64 elements
// follow a box later (leading byte offset).  16 steps further is 2048 bytes.
__device__ __forceinline__ uint64_t umma_desc_mn(uint32_t smem_addr) {
    return (uint64_t)((smem_addr & 0x3ffffu) >> 4) | ((uint64_t)(CHUNK_BYTES >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) |
           (2ull << 61);
}
// bf16 x bf16 -> fp32, 128 x up to 256 columns; bits 15 and 16: A, B are MN-major.
__device__ __forceinline__ uint32_t idesc(bool a_mn, bool b_mn, int cols) {
    const uint32_t n = cols < BN ? (uint32_t)(cols + 15) / 16 * 16 : BN;     // no products beyond the row's end
    return (1u << 4) | (1u << 7) | (1u << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) | ((n >> 3) << 17) | ((uint32_t)(BM >> 4) << 24);
}
__device__ __forceinline__ void umma_f16(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t id, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(id), "r"(accumulate) : "memory");
}

// ---- epilogue arithmetic on pairs ----
__device__ __forceinline__ float2 unpack2(uint32_t w) { return make_float2(bf16_lo(w), bf16_hi(w)); }

// 8 or 16 columns of a row, by the lane that has them.  Rows are far apart, so that a lane's 32 bytes are a sector of their own:
// stored whole they cost the L2 no merge (first product of 65536 x 2560 x 10240 with GeLU and z 3.85 ms with 16 bytes a
// store, 3.09 with 32).  `wide`: rows begin on 32 bytes.
template <int W>
__device__ __forceinline__ void st_row(void* base, size_t o, const float2 (&v)[W / 2], bool wide) {
    uint16_t* p = static_cast<uint16_t*>(base) + o;
    uint32_t r[W / 2];
#pragma unroll
    for (int i = 0; i < W / 2; ++i) r[i] = cvt_bf16x2(v[i]);
    if (W == 16 && wide) {
        st_global_v8(p, r[0], r[1], r[2], r[3], r[W / 2 - 4], r[W / 2 - 3], r[W / 2 - 2], r[W / 2 - 1]);
    } else {
#pragma unroll
        for (int i = 0; i < W / 8; ++i) reinterpret_cast<uint4*>(p)[i] = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
    }
}
template <int W>
__device__ __forceinline__ void ld_row(const void* base, size_t o, uint32_t* r, bool wide) {
    const uint16_t* p = static_cast<const uint16_t*>(base) + o;
    if (W == 16 && wide) {
        asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "l"(p) : "memory");
    } else {
#pragma unroll
        for (int i = 0; i < W / 8; ++i)
            asm volatile("ld.global.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r[4 * i]), "=r"(r[4 * i + 1]), "=r"(r[4 * i + 2]), "=r"(r[4 * i + 3]) : "l"(p + 8 * i) : "memory");
    }
}
// What comes after z: the activation and the residual, or the slope of the activation before the product.
template <int KIND, int W>
__device__ __forceinline__ void arithmetic(const LinearArgs& a, float2 (&v)[W / 2], const uint32_t* extra) {
    if (KIND == kForward) {
        if (a.act == LOCMOE_ACT_GELU) {
#pragma unroll
            for (int i = 0; i < W / 2; ++i) v[i] = gelu2(v[i]);
        } else if (a.act == LOCMOE_ACT_SILU) {
#pragma unroll
            for (int i = 0; i < W / 2; ++i) v[i] = silu2(v[i]);
        } else if (a.act == LOCMOE_ACT_RELU) {
#pragma unroll
            for (int i = 0; i < W / 2; ++i) v[i] = make_float2(v[i].x < 0.0f ? 0.0f : v[i].x, v[i].y < 0.0f ? 0.0f : v[i].y);
        }
        if (a.residual) {
#pragma unroll
            for (int i = 0; i < W / 2; ++i) v[i] = __fadd2_rn(v[i], unpack2(extra[i]));
        }
    } else if (KIND == kTowardsX) {
        if (a.act == LOCMOE_ACT_GELU) {
#pragma unroll
            for (int i = 0; i < W / 2; ++i) v[i] = __fmul2_rn(v[i], gelu_slope2(unpack2(extra[i])));
        } else if (a.act == LOCMOE_ACT_SILU) {
#pragma unroll
            for (int i = 0; i < W / 2; ++i) v[i] = __fmul2_rn(v[i], silu_slope2(unpack2(extra[i])));
        } else if (a.act == LOCMOE_ACT_RELU) {
#pragma unroll
            for (int i = 0; i < W / 2; ++i) {
                const float2 z = unpack2(extra[i]);
                v[i] = make_float2(z.x > 0.0f ? v[i].x : 0.0f, z.y > 0.0f ? v[i].y : 0.0f);
            }
        }
    }
}
template <int W>
__device__ __forceinline__ void add_bias(float2 (&v)[W / 2], const float4* b) {
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
        v[2 * i] = __fadd2_rn(v[2 * i], make_float2(b[i].x, b[i].y));
        v[2 * i + 1] = __fadd2_rn(v[2 * i + 1], make_float2(b[i].z, b[i].w));
    }
}
// W sums of one row on their whole way; `o` is the first's index in the output, `b` the bias, `extra` what is read along.
template <int KIND, int W>
__device__ __forceinline__ void finish(const LinearArgs& a, size_t o, float2 (&v)[W / 2], const float4* b, const uint32_t* extra, bool wide) {
    if (KIND == kForward && a.bias) add_bias<W>(v, b);
    if (KIND == kForward && a.z_out) st_row<W>(a.z_out, o, v, wide);
    arithmetic<KIND, W>(a, v, extra);
    if (KIND == kWeights && a.out_f32) {
        float4* p = reinterpret_cast<float4*>(static_cast<float*>(a.out) + o);
#pragma unroll
        for (int i = 0; i < W / 4; ++i) p[i] = make_float4(v[2 * i].x, v[2 * i].y, v[2 * i + 1].x, v[2 * i + 1].y);
    } else {
        st_row<W>(a.out, o, v, wide);
    }
}
// 32 columns of a weight's gradient by the lane that has the row, `cols` of them before the row's end.
__device__ __forceinline__ void store_weights32(const LinearArgs& a, size_t o, int cols, const uint32_t (&r)[32], bool wide) {
#pragma unroll
    for (int i = 0; i < 32; i += 8) {
        if (i >= cols) break;
        if (a.out_f32) {
            float* p = static_cast<float*>(a.out) + o + i;
            if (wide) {
                st_global_v8(p, r[i], r[i + 1], r[i + 2], r[i + 3], r[i + 4], r[i + 5], r[i + 6], r[i + 7]);
            } else {
                reinterpret_cast<uint4*>(p)[0] = make_uint4(r[i], r[i + 1], r[i + 2], r[i + 3]);
                reinterpret_cast<uint4*>(p)[1] = make_uint4(r[i + 4], r[i + 5], r[i + 6], r[i + 7]);
            }
        } else if (wide && i % 16 == 0 && i + 16 <= cols) {
            float2 v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = make_float2(__uint_as_float(r[(i & 16) + 2 * k]), __uint_as_float(r[(i & 16) + 2 * k + 1]));
            st_row<16>(a.out, o + i, v, true);
        } else if (!wide || i % 16 == 0) {
            float2 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = make_float2(__uint_as_float(r[i + 2 * k]), __uint_as_float(r[i + 2 * k + 1]));
            st_row<8>(a.out, o + i, v, false);
        }
    }
}
// A 16-byte piece of a lane's row in a box of 32 rows x 128 bytes on its way out, where the map's swizzle wants it (eight lanes fill
// the banks once).
__device__ __forceinline__ void put_piece(unsigned char* box, int lane, int i, const uint4& r) {
    *reinterpret_cast<uint4*>(box + lane * 128 + ((i ^ (lane & 7)) << 4)) = r;
}
// The array read along with the sums, if there is one.
template <int KIND>
__device__ __forceinline__ const void* extra_array(const LinearArgs& a) { return KIND == kForward ? a.residual : KIND == kTowardsX ? a.z_in : nullptr; }

// HALVES: of a tile, 128 rows each with an accumulator.
template <int KIND, int HALVES>
__global__ void __launch_bounds__(KIND == kWeights ? kWeightsThreads : kThreads, 1)
expert_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmOther,
                   const LinearArgs a) {
    constexpr int UNIT = HALVES * BM;
    constexpr bool A_MN = KIND == kWeights, B_MN = KIND != kForward;
    constexpr uint64_t kStepA = (A_MN ? 2048 : UMMA_K * 2) >> 4, kStepB = (B_MN ? 2048 : UMMA_K * 2) >> 4;   // 16 steps of the reduction
    extern __shared__ unsigned char smraw[];
    unsigned char* base = reinterpret_cast<unsigned char*>(((uintptr_t)smraw + 1023) & ~(uintptr_t)1023);
    uint64_t* bars = reinterpret_cast<uint64_t*>(base + kRing);
    uint64_t* full = bars;                   // [stages] operands landed
    uint64_t* empty = bars + kMaxStages;     // [stages] products (and column sums) that read the stage are done
    uint64_t* acc_full = bars + 2 * kMaxStages;  // [2] accumulator complete
    uint64_t* acc_empty = acc_full + 2;      // [2] accumulator drained
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
    volatile int* abort_word = reinterpret_cast<volatile int*>(tmem_slot + 1);
    int* offsets = reinterpret_cast<int*>(base + kRing + 256);   // [E + 1]

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int NSTAGE = a.stages;
    const uint32_t a_bytes = (uint32_t)a.a_rows * BK * 2, STAGE_BYTES = a_bytes + B_BYTES;   // products read on beyond a short A: into B, for rows of no account
    const bool with_db = KIND == kWeights && a.db;
    if (threadIdx.x == 0) {
        for (int s = 0; s < NSTAGE; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], with_db ? 1 + kSumWarps : 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], with_db ? kEpiWarps + kSumWarps : kEpiWarps); }
        *abort_word = 0;
        mbar_init_fence();
        prefetch_map(&tmA);
        prefetch_map(&tmB);
        prefetch_map(&tmOther);
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();
    pdl_trigger();
    for (int i = threadIdx.x; i <= a.E; i += blockDim.x) offsets[i] = __ldg(a.offsets + i);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    const Deal runs = deal<KIND, HALVES>(a, offsets, lane);
    Cursor<KIND, HALVES> cur(a, offsets, runs, blockIdx.x);
    Item it;

    if (warp == 0) {
        if (lane == 0) {  // ---- loads ----
            int stage = 0; uint32_t phase = 0;
            bool ok = true;
            while (ok && cur.next(it)) {
                const int m0 = it.mt * UNIT, n0 = it.nt * BN;
                // a group's last rows come in boxes of 32: what lies behind them is another group's, and would be read for nothing
                // (1000 rows of 1560 x 4104 over 24 experts 76 against 65 us)
                const int few = A_MN || a.a_rows < BM || it.n - m0 > UNIT - 32 ? 0 : (it.n - m0 + 31) / 32;
                const uint32_t bytes = few ? (uint32_t)few * 32 * BK * 2 + B_BYTES : STAGE_BYTES;
                for (int kb = it.kb0; kb < it.kb1; ++kb) {
                    if (!wait_or_abort(&empty[stage], phase ^ 1u, abort_word)) { ok = false; break; }
                    unsigned char* sa = base + (size_t)stage * STAGE_BYTES;
                    unsigned char* sb = sa + a_bytes;
                    mbar_expect_tx(&full[stage], bytes);
                    if (A_MN && a.a_chunks) {
                        tma_load_4d(sa, &tmA, 0, it.lo + kb * BK, m0 / 64, 0, &full[stage]);
                    } else if (A_MN) {
#pragma unroll
                        for (int c = 0; c < UNIT / 64; ++c) tma_load_2d(sa + c * CHUNK_BYTES, &tmA, m0 + 64 * c, it.lo + kb * BK, &full[stage]);
                    } else if (few) {
                        for (int i = 0; i < few; ++i) tma_load_2d(sa + i * (32 * BK * 2), &tmOther, kb * BK, it.lo + m0 + 32 * i, &full[stage]);
                    } else {
                        tma_load_2d(sa, &tmA, kb * BK, it.lo + m0, &full[stage]);
                    }
                    if (KIND == kForward) {
                        tma_load_3d(sb, &tmB, kb * BK, n0, it.e, &full[stage]);
                    } else if (a.b_chunks) {
                        tma_load_4d(sb, &tmB, 0, KIND == kWeights ? it.lo + kb * BK : kb * BK, n0 / 64, KIND == kWeights ? 0 : it.e, &full[stage]);
                    } else {
#pragma unroll
                        for (int c = 0; c < BN / 64; ++c) {
                            if (KIND == kWeights) tma_load_2d(sb + c * CHUNK_BYTES, &tmB, n0 + 64 * c, it.lo + kb * BK, &full[stage]);
                            else tma_load_3d(sb + c * CHUNK_BYTES, &tmB, n0 + 64 * c, kb * BK, it.e, &full[stage]);
                        }
                    }
                    if (++stage == NSTAGE) { stage = 0; phase ^= 1u; }
                }
            }
            // tail: all asynchronous commits to this CTA's stage barriers have arrived before the CTA leaves
            for (int i = 0; i < NSTAGE; ++i) {
                if (!wait_or_abort(&empty[stage], phase ^ 1u, abort_word)) break;
                if (++stage == NSTAGE) { stage = 0; phase ^= 1u; }
            }
        }
    } else if (warp == 1) {  // ---- products: lane 0 issues them alone but for a group's last block, which the warp prepares ----
        int stage = 0; uint32_t phase = 0;
        int acc = 0; uint32_t acc_phase = 0;
        bool ok = true;
        while (ok && cur.next(it)) {
            const int halves = halves_of<KIND, HALVES>(a, it);
            if (!wait_warp(&acc_empty[acc], acc_phase ^ 1u, abort_word)) break;
            if (halves == 2 && !wait_warp(&acc_empty[acc ^ 1], acc == 0 ? acc_phase ^ 1u : acc_phase, abort_word)) break;
            tc_fence_after();
            const uint32_t id = idesc(A_MN, B_MN, a.N - it.nt * BN);
            const int left = KIND == kWeights ? it.n - (it.kb1 - 1) * BK : BK;      // rows of the group in the last block
            const int plain = it.kb1 - it.kb0 - (left < BK ? 1 : 0);                // blocks that are products and nothing else
            if (lane == 0) {
                int s = stage; uint32_t ph = phase;
                for (int i = 0; i < plain; ++i) {
                    if (!wait_or_abort(&full[s], ph, abort_word)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t sa = smem_u32(base) + (uint32_t)s * STAGE_BYTES;
                    const uint64_t da = A_MN ? umma_desc_mn(sa) : umma_desc_sw128(sa), db = B_MN ? umma_desc_mn(sa + a_bytes) : umma_desc_sw128(sa + a_bytes);
                    for (int h = 0; h < halves; ++h) {
#pragma unroll
                        for (int k = 0; k < BK / UMMA_K; ++k)
                            umma_f16(tmem_base + (uint32_t)((acc ^ h) * BN), da + h * (A_BYTES >> 4) + k * kStepA, db + k * kStepB, id, (i > 0 || k > 0) ? 1u : 0u);
                    }
                    umma_commit(&empty[s]);
                    if (with_db && it.nt != 0) mbar_arrive_n(&empty[s], kSumWarps);    // nobody else reads this stage
                    if (++s == NSTAGE) { s = 0; ph ^= 1u; }
                }
            }
            ok = __shfl_sync(0xffffffffu, ok, 0);
            if (!ok) break;
            phase ^= (uint32_t)((stage + plain) / NSTAGE) & 1u;
            stage = (stage + plain) % NSTAGE;
            if constexpr (KIND == kWeights) if (left < BK) {
                if (!wait_warp(&full[stage], phase, abort_word)) { ok = false; break; }
                unsigned char* pa = base + (size_t)stage * STAGE_BYTES;
                const int steps = (left + UMMA_K - 1) / UMMA_K;
                // rows [left, 16 * steps) belong to the next group: zeros.  A row is 128 bytes in each box, whatever the swizzle,
                // which moves bytes inside a row only.
                for (int r = left + (lane >> 3); r < steps * UMMA_K; r += 4) {
                    for (int c = 0; c < (int)(STAGE_BYTES / CHUNK_BYTES); ++c)
                        *reinterpret_cast<uint4*>(pa + c * CHUNK_BYTES + r * 128 + (lane & 7) * 16) = make_uint4(0, 0, 0, 0);
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    tc_fence_after();
                    const uint64_t da = umma_desc_mn(smem_u32(pa)), db = umma_desc_mn(smem_u32(pa) + a_bytes);
                    for (int h = 0; h < halves; ++h)
                        for (int k = 0; k < steps; ++k)
                            umma_f16(tmem_base + (uint32_t)((acc ^ h) * BN), da + h * (A_BYTES >> 4) + k * kStepA, db + k * kStepB, id, (plain > 0 || k > 0) ? 1u : 0u);
                    umma_commit(&empty[stage]);
                    if (with_db && it.nt != 0) mbar_arrive_n(&empty[stage], kSumWarps);
                }
                __syncwarp();
                if (++stage == NSTAGE) { stage = 0; phase ^= 1u; }
            }
            for (int h = 0; h < halves; ++h) {
                if (lane == 0) umma_commit(&acc_full[acc]);
                if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
            }
            __syncwarp();
        }
    } else if (KIND == kWeights && warp >= 2 + kEpiWarps) {
        // ---- column sums of dy, from the A tiles of the first column of output tiles: a warp 32 columns, a lane 8 of them in
        // every eighth row.  Four lanes' units of 16 bytes in rows r and r + 4 fill the banks once, swizzled as they are.
        // Each tile's accumulator is waited for and released like the epilogue does, so that these warps never fall a phase behind.
        if (with_db) {
            const int w = warp - 2 - kEpiWarps, o = w * 4 + (lane & 3), r0 = ((lane >> 2) & 1) * 4 + (lane >> 3);
            const uint32_t at = (uint32_t)(o >> 3) * CHUNK_BYTES + (uint32_t)(((o & 7) ^ r0) << 4) + (uint32_t)r0 * 128;
            int stage = 0; uint32_t phase = 0;
            int acc = 0; uint32_t acc_phase = 0;
            bool ok = true;
            while (ok && cur.next(it)) {
                const int n = it.kb1 - it.kb0;
                const int halves = halves_of<KIND, HALVES>(a, it);
                if (it.nt == 0) {
                    float2 v[HALVES][4] = {};
                    for (int kb = it.kb0; kb < it.kb1; ++kb) {
                        if (!wait_warp(&full[stage], phase, abort_word)) { ok = false; break; }
                        const unsigned char* p = base + (size_t)stage * STAGE_BYTES + at;
                        const int left = it.n - kb * BK;
#pragma unroll
                        for (int h = 0; h < HALVES; ++h) {
                            if (h == halves) break;
#pragma unroll
                            for (int i = 0; i < BK / 8; ++i) {
                                if (r0 + 8 * i >= left) break;
                                const uint4 q = *reinterpret_cast<const uint4*>(p + h * A_BYTES + i * 1024);
                                v[h][0] = __fadd2_rn(v[h][0], unpack2(q.x)); v[h][1] = __fadd2_rn(v[h][1], unpack2(q.y));
                                v[h][2] = __fadd2_rn(v[h][2], unpack2(q.z)); v[h][3] = __fadd2_rn(v[h][3], unpack2(q.w));
                            }
                        }
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&empty[stage]);
                        if (++stage == NSTAGE) { stage = 0; phase ^= 1u; }
                    }
                    if (!ok) break;
#pragma unroll
                    for (int h = 0; h < HALVES; ++h) {
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                v[h][i].x += __shfl_xor_sync(0xffffffffu, v[h][i].x, d);
                                v[h][i].y += __shfl_xor_sync(0xffffffffu, v[h][i].y, d);
                            }
                        }
                        const int in = h * BM + o * 8, col = it.mt * UNIT + in;
                        float* out = n == it.kb ? (col < a.M ? a.db + (size_t)it.e * a.M + col : nullptr)
                                                : a.db_part + ((size_t)blockIdx.x * 2 + (it.kb0 == 0 ? 1 : 0)) * UNIT + in;
                        if (lane < 4 && h < halves && out) {
                            reinterpret_cast<float4*>(out)[0] = make_float4(v[h][0].x, v[h][0].y, v[h][1].x, v[h][1].y);
                            reinterpret_cast<float4*>(out)[1] = make_float4(v[h][2].x, v[h][2].y, v[h][3].x, v[h][3].y);
                        }
                    }
                } else {
                    phase ^= (uint32_t)((stage + n) / NSTAGE) & 1u;
                    stage = (stage + n) % NSTAGE;
                }
                for (int h = 0; ok && h < halves; ++h) {
                    ok = wait_warp(&acc_full[acc], acc_phase, abort_word);
                    if (ok && lane == 0) mbar_arrive(&acc_empty[acc]);
                    if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
                }
            }
        }
    } else {  // ---- epilogue: TMEM lane quadrant = warp % 4, the columns dealt to the warps of a quadrant ----
        constexpr int kCols = BN * 4 / kEpiWarps, kBlock = 32;       // columns of one warp, of a step
        const int q = warp & 3, part0 = ((warp - 2) >> 2) * kCols;
        const int et = threadIdx.x - 64;
        // what no tile covers: rows before the first group and behind the last, weights of experts without rows
        if (KIND != kWeights) {
            const int first = min(max(offsets[0], 0), a.R), kept = max(min(offsets[a.E], a.R), first);
            const long long per = a.N / 8, before = first * per, n = before + ((long long)a.R - kept) * per;
            for (long long i = (long long)blockIdx.x * kEpiThreads + et; i < n; i += (long long)gridDim.x * kEpiThreads) {
                const size_t o = (size_t)(i < before ? i : i - before + kept * per) * 8;
                *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.out) + o) = make_uint4(0, 0, 0, 0);
                if (a.z_out) *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.z_out) + o) = make_uint4(0, 0, 0, 0);
            }
        } else {
            const long long n = (long long)a.M * (a.N / 8);
            for (int e = 0; e < a.E; ++e) {
                if (group_of(offsets, e, a.R).n > 0) continue;
                if (a.db && e % (int)gridDim.x == (int)blockIdx.x)
                    for (int i = et; i < a.M; i += kEpiThreads) a.db[(size_t)e * a.M + i] = 0.0f;
                for (long long i = (long long)blockIdx.x * kEpiThreads + et; i < n; i += (long long)gridDim.x * kEpiThreads) {
                    float2 z[4] = {{0, 0}, {0, 0}, {0, 0}, {0, 0}};
                    finish<KIND, 8>(a, (size_t)(e * n + i) * 8, z, nullptr, nullptr, false);
                }
            }
        }
        if (et == 0 && a.split) a.split[blockIdx.x].rows = 0;
        __syncwarp();
        const void* with = extra_array<KIND>(a);
        const bool wide = a.N % 16 == 0 && (((uintptr_t)a.out | (uintptr_t)a.z_out | (uintptr_t)with) % 32) == 0;
        float* bias = reinterpret_cast<float*>(base + kRing + 256 + kOffsetBytes) + (warp - 2) * kCols;      // of this warp's columns
        unsigned char* boxes = base + (size_t)kBoxStages * (A_BYTES + B_BYTES) + (size_t)(warp - 2) * 2 * kBoxBytes;
        int turn = 0;
        int acc = 0; uint32_t acc_phase = 0;
        bool ok = true;
        while (ok && cur.next(it)) {
            if (it.kb0 == 0 && it.kb1 < it.kb && et == 0) {
                int last = blockIdx.x + 1;
                while (last + 1 < runs.runs && runs.begin(last + 1) < it.begin + it.kb) ++last;
                Split split{it.e, it.mt * UNIT + (KIND == kWeights ? 0 : it.lo), min(UNIT, (KIND == kWeights ? a.M : it.n) - it.mt * UNIT), it.nt, last};
                a.split[blockIdx.x] = split;
            }
            __syncwarp();
            const int halves = halves_of<KIND, HALVES>(a, it);
#pragma unroll 1
            for (int h = 0; h < halves; ++h) {
                const int m0 = it.mt * UNIT + h * BM + q * 32, n0 = it.nt * BN + part0;      // the warp's first row and column
                const int all = KIND == kWeights ? a.M : it.n;
                const bool row_ok = m0 + lane < all, whole = it.kb1 - it.kb0 == it.kb;
                const size_t o0 = ((size_t)(KIND == kWeights ? 0 : it.lo) + m0 + lane) * a.N + n0;      // rows' outputs only
                float* part = whole ? nullptr : a.part + (((size_t)blockIdx.x * 2 + (it.kb0 == 0 ? 1 : 0)) * a.part_rows + h * BM + q * 32 + lane) * BN + part0;
                const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * BN + part0);
                if constexpr (KIND == kWeights) {
                    if (!wait_warp(&acc_full[acc], acc_phase, abort_word)) { ok = false; break; }
                    tc_fence_after();
                    const int step = a.out_f32 ? 32 : 64;       // columns of a box
#pragma unroll 1
                    for (int c = 0; c < kCols; c += step) {
                        if (m0 >= all || n0 + c >= a.N) break;                  // all lanes alike
                        unsigned char* box = boxes + turn * kBoxBytes;
                        if (whole && a.boxes) {
                            if (lane == 0) bulk_wait_read<1>();                 // the box before the last one has left
                            __syncwarp();
                        }
#pragma unroll 1
                        for (int d = 0; d < step; d += 32) {
                            uint32_t r[32];
                            tmem_ld32(taddr + c + d, r);
                            if (!whole) {
                                if (row_ok) {
#pragma unroll
                                    for (int i = 0; i < 32; i += 8) st_global_v8(part + c + d + i, r[i], r[i + 1], r[i + 2], r[i + 3], r[i + 4], r[i + 5], r[i + 6], r[i + 7]);
                                }
                                __syncwarp();
                            } else if (!a.boxes) {
                                if (row_ok) store_weights32(a, ((size_t)it.e * a.M + m0 + lane) * a.N + n0 + c + d, a.N - n0 - c - d, r, wide);
                                __syncwarp();
                            } else if (a.out_f32) {
#pragma unroll
                                for (int i = 0; i < 8; ++i) put_piece(box, lane, i, make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]));
                            } else {
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    uint32_t p[4];
#pragma unroll
                                    for (int k = 0; k < 4; ++k) p[k] = cvt_bf16x2(make_float2(__uint_as_float(r[8 * i + 2 * k]), __uint_as_float(r[8 * i + 2 * k + 1])));
                                    put_piece(box, lane, d / 8 + i, make_uint4(p[0], p[1], p[2], p[3]));
                                }
                            }
                        }
                        if (whole && a.boxes) {
                            fence_async_smem();
                            __syncwarp();
                            if (lane == 0) {                    // what lies beyond the weights' rows and columns is left out
                                tma_store_3d(&tmOther, box, n0 + c, m0, it.e);
                                bulk_commit();
                            }
                            turn ^= 1;
                        }
                    }
                } else {
                    // the bias and the array read along come ahead: the former through shared memory, the latter a block ahead, the
                    // first block's before the sums are there (1000 rows of 1560 x 4104 with both: loads one after the other were
                    // 9 us a tile)
                    if (KIND == kForward && a.bias && whole) {
                        if (4 * lane < kCols && n0 + 4 * lane < a.N)
                            *reinterpret_cast<float4*>(bias + 4 * lane) = __ldg(reinterpret_cast<const float4*>(a.bias + (size_t)it.e * a.N + n0) + lane);
                        __syncwarp();
                    }
                    uint32_t next[kBlock / 2];
                    auto fetch = [&](int c) {
                        if (!row_ok || !whole || !with) return;
#pragma unroll
                        for (int i = 0; i < kBlock; i += 16) {
                            if (n0 + c + i + 16 <= a.N) ld_row<16>(with, o0 + c + i, next + i / 2, wide);
                            else if (n0 + c + i < a.N) ld_row<8>(with, o0 + c + i, next + i / 2, false);
                        }
                    };
                    fetch(0);
                    if (!wait_warp(&acc_full[acc], acc_phase, abort_word)) { ok = false; break; }
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < kCols; c += kBlock) {
                        uint32_t extra[kBlock / 2];
#pragma unroll
                        for (int i = 0; i < kBlock / 2; ++i) extra[i] = next[i];
                        if (c + kBlock < kCols) fetch(c + kBlock);
                        __syncwarp();  // tcgen05.ld is warp-collective: reconverge after the masked stores
                        uint32_t r[kBlock];
                        tmem_ld(taddr + c, r);
                        if (!row_ok || n0 + c >= a.N) continue;
                        if (!whole) {
#pragma unroll
                            for (int i = 0; i < kBlock; i += 8) st_global_v8(part + c + i, r[i], r[i + 1], r[i + 2], r[i + 3], r[i + 4], r[i + 5], r[i + 6], r[i + 7]);
                            continue;
                        }
#pragma unroll
                        for (int i = 0; i < kBlock; i += 16) {
                            float4 b[4];
                            if (KIND == kForward && a.bias) {
#pragma unroll
                                for (int k = 0; k < 4; ++k) b[k] = reinterpret_cast<const float4*>(bias + c + i)[k];
                            }
                            if (n0 + c + i + 16 <= a.N) {
                                float2 v[8];
#pragma unroll
                                for (int k = 0; k < 8; ++k) v[k] = make_float2(__uint_as_float(r[i + 2 * k]), __uint_as_float(r[i + 2 * k + 1]));
                                finish<KIND, 16>(a, o0 + c + i, v, b, extra + i / 2, wide);
                            } else if (n0 + c + i < a.N) {      // the row's last eight
                                float2 v[4];
#pragma unroll
                                for (int k = 0; k < 4; ++k) v[k] = make_float2(__uint_as_float(r[i + 2 * k]), __uint_as_float(r[i + 2 * k + 1]));
                                finish<KIND, 8>(a, o0 + c + i, v, b, extra + i / 2, false);
                            }
                        }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&acc_empty[acc]);
                if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
            }
        }
        if (KIND == kWeights && lane == 0) bulk_wait_all<0>();      // the last boxes are where they belong
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

// Adds up the sums of the tiles that more than one run worked on, in the order of the runs, and finishes them.  CTA (x, y): run
// x's split tile, every gridDim.y-th piece.  What tile that is the GEMM has written down; finding it anew cost every warp
// here a few thousand cycles (200 rows of 1600 x 4096, 23 experts: 15 against 4 us).
constexpr int kJoinThreads = 256, kJoinParts = 8;
static_assert(kJoinThreads >= 2 * BM, "a thread for each row of a tile");
template <int KIND>
__global__ void __launch_bounds__(kJoinThreads) expert_join_kernel(const LinearArgs a) {
    pdl_wait();
    pdl_trigger();
    const int c0 = blockIdx.x;
    const int4 s0 = __ldcg(reinterpret_cast<const int4*>(a.split + c0));
    const int last = __ldcg(&a.split[c0].last);
    const int e = s0.x, rows = s0.z, n0 = s0.w * BN;
    if (rows == 0) return;
    const size_t row0 = KIND == kWeights ? (size_t)e * a.M + s0.y : (size_t)s0.y;
    const int cols = min(BN, a.N - n0) / 8;
    if (KIND == kWeights && a.db && n0 == 0 && blockIdx.y == 0 && (int)threadIdx.x < rows) {
        const int i = threadIdx.x;
        float sum = __ldcg(a.db_part + ((size_t)c0 * 2 + 1) * a.unit + i);
        for (int c = c0 + 1; c <= last; ++c) sum += __ldcg(a.db_part + (size_t)c * 2 * a.unit + i);
        a.db[row0 + i] = sum;
    }
    const size_t step = (size_t)2 * a.part_rows * BN;               // from a run's sums to the next one's
    for (int i = blockIdx.y * kJoinThreads + threadIdx.x; i < rows * cols; i += gridDim.y * kJoinThreads) {
        const int r = i / cols, col = (i - r * cols) * 8;
        const size_t o = (row0 + r) * a.N + n0 + col;
        uint32_t extra[4];
        if (extra_array<KIND>(a)) ld_row<8>(extra_array<KIND>(a), o, extra, false);
        float4 b[2];
        if (KIND == kForward && a.bias) {
            const float4* q = reinterpret_cast<const float4*>(a.bias + (size_t)e * a.N + n0 + col);
            b[0] = __ldg(q); b[1] = __ldg(q + 1);
        }
        // the first run's part is its second slot's, the others' their first
        const float* p = a.part + (((size_t)c0 * 2 + 1) * a.part_rows + r) * BN + col;
        const float4 f0 = __ldcg(reinterpret_cast<const float4*>(p)), f1 = __ldcg(reinterpret_cast<const float4*>(p) + 1);
        float2 v[4] = {{f0.x, f0.y}, {f0.z, f0.w}, {f1.x, f1.y}, {f1.z, f1.w}};
        p = a.part + (((size_t)c0 * 2 + 2) * a.part_rows + r) * BN + col;
        for (int c = c0 + 1; c <= last; c += 4, p += 4 * step) {    // four runs' sums in flight
            float4 q[4][2];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (c + k > last) break;
                q[k][0] = __ldcg(reinterpret_cast<const float4*>(p + k * step));
                q[k][1] = __ldcg(reinterpret_cast<const float4*>(p + k * step) + 1);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (c + k > last) break;
                v[0].x += q[k][0].x; v[0].y += q[k][0].y; v[1].x += q[k][0].z; v[1].y += q[k][0].w;
                v[2].x += q[k][1].x; v[2].y += q[k][1].y; v[3].x += q[k][1].z; v[3].y += q[k][1].w;
            }
        }
        finish<KIND, 8>(a, o, v, b, extra, false);
    }
}

// Forward for a few rows, single tokens' most of all: nothing but the weights to read, and no tile to fill.  A task is four columns of
// an expert with rows; its CTA's threads share the reduction, 16 bytes of each of the four weight rows at a time, twice in
// flight, and two rows of x share them.  The sums of the lanes, then of the warps, in a fixed order.  Weights in a ring in
// shared memory, asynchronously and on into the next task's, were slower (two rows, 2560 x 10240: 26 against 23 us).
constexpr int kFewRows = 8, kFewThreads = 256, kFewWarps = 24;      // kFewWarps: of an SM
constexpr int kFewCols = 4, kFewShare = 2;                          // columns and rows of a task
constexpr int kScan = 8;                                            // offsets a lane in flight (a row of 1024 experts, 256 x 256: 3.8 us, 6.3 with one)
// Four rows (of one expert 20 us either way at 2560 x 10240, of four 41 against 35, two of two 26 against 20, one 19 against 12;
// 16 experts of 3936 x 288 12 against 5), eight where the weights are so small that the tiles' fixed times count (64 of
// 1024 x 1024, eight rows of as many 12 against 6 us, of one expert 9 against 10; 2560 x 10240 20 against 49).
constexpr int kFewWeight = 1 << 21;
template <int ROWS>
__device__ __forceinline__ void few_sums(int K, const uint16_t* __restrict__ x, const uint16_t* __restrict__ w, float* sums) {
    constexpr int DEPTH = ROWS == 1 ? 2 : 1;                        // registers for kFewWarps
    float2 v[ROWS][kFewCols] = {};
    const int step = blockDim.x * 8;
#pragma unroll 1
    for (int k = threadIdx.x * 8; k < K; k += DEPTH * step) {
        uint4 q[DEPTH][kFewCols];
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
#pragma unroll
            for (int c = 0; c < kFewCols; ++c)
                if (i == 0 || k + step < K) q[i][c] = ld_stream(reinterpret_cast<const uint4*>(w + (size_t)c * K + k + i * step));
        }
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
            if (i == 1 && k + step >= K) break;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const uint4 p = __ldg(reinterpret_cast<const uint4*>(x + (size_t)r * K + k + i * step));
                const float2 x0 = unpack2(p.x), x1 = unpack2(p.y), x2 = unpack2(p.z), x3 = unpack2(p.w);
#pragma unroll
                for (int c = 0; c < kFewCols; ++c) {
                    v[r][c] = __ffma2_rn(unpack2(q[i][c].x), x0, v[r][c]);
                    v[r][c] = __ffma2_rn(unpack2(q[i][c].y), x1, v[r][c]);
                    v[r][c] = __ffma2_rn(unpack2(q[i][c].z), x2, v[r][c]);
                    v[r][c] = __ffma2_rn(unpack2(q[i][c].w), x3, v[r][c]);
                }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
#pragma unroll
        for (int c = 0; c < kFewCols; ++c) {
            float f = v[r][c].x + v[r][c].y;
#pragma unroll
            for (int d = 16; d; d >>= 1) f += __shfl_xor_sync(0xffffffffu, f, d);
            if ((threadIdx.x & 31) == 0) sums[((threadIdx.x >> 5) * kFewShare + r) * kFewCols + c] = f;
        }
    }
}
__global__ void __launch_bounds__(kFewThreads, kFewWarps * 32 / kFewThreads) expert_few_kernel(const LinearArgs a, const uint16_t* __restrict__ x,
                                                                                              const uint16_t* __restrict__ w) {
    __shared__ __align__(16) float sums[2][kFewThreads / 32 * kFewShare * kFewCols];
    __shared__ int busy[kFewRows][3], n_busy;       // experts with rows: expert, first row, rows
    pdl_wait();
    pdl_trigger();
    if (threadIdx.x < 32) {
        int n = 0;
        for (int e0 = 0; e0 < a.E; e0 += 32 * kScan) {
            int off[kScan][2];
#pragma unroll
            for (int i = 0; i < kScan; ++i) {
                const int e = e0 + 32 * i + (int)threadIdx.x;
                off[i][0] = e < a.E ? __ldg(a.offsets + e) : 0;
                off[i][1] = e < a.E ? __ldg(a.offsets + e + 1) : 0;
            }
#pragma unroll
            for (int i = 0; i < kScan; ++i) {
                const Group g = group_of(off[i], 0, a.R);
                const unsigned has = __ballot_sync(0xffffffffu, g.n > 0);
                const int at = n + __popc(has & ((1u << threadIdx.x) - 1u));
                if (g.n > 0 && at < kFewRows) { busy[at][0] = e0 + 32 * i + (int)threadIdx.x; busy[at][1] = g.lo; busy[at][2] = g.n; }
                n += __popc(has);
            }
        }
        if (threadIdx.x == 0) n_busy = min(n, kFewRows);       // more only where the offsets descend
    }
    const int first = min(max(__ldg(a.offsets), 0), a.R), kept = max(min(__ldg(a.offsets + a.E), a.R), first);
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < a.R * (a.N / 8); i += gridDim.x * blockDim.x) {
        const int r = i / (a.N / 8);
        if (r >= first && r < kept) continue;
        reinterpret_cast<uint4*>(a.out)[i] = make_uint4(0, 0, 0, 0);
        if (a.z_out) reinterpret_cast<uint4*>(a.z_out)[i] = make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
    const int per = a.N / kFewCols;
    int turn = 0;
    for (int t = blockIdx.x; t < n_busy * per; t += gridDim.x) {
        const int g = t / per, n0 = (t - g * per) * kFewCols, e = busy[g][0];
        for (int r0 = 0; r0 < busy[g][2]; r0 += kFewShare, turn ^= 1) {
            const int rows = min(kFewShare, busy[g][2] - r0), row = busy[g][1] + r0;
            const uint16_t* xr = x + (size_t)row * a.K;
            const uint16_t* wr = w + ((size_t)e * a.N + n0) * a.K;
            if (rows == 1) few_sums<1>(a.K, xr, wr, sums[turn]);
            else few_sums<2>(a.K, xr, wr, sums[turn]);
            __syncthreads();        // the other half of sums is written next
            if ((int)threadIdx.x < rows) {
                const size_t o = (size_t)(row + threadIdx.x) * a.N + n0;
                float2 v[2] = {};
                for (int i = 0; i < (int)blockDim.x / 32; ++i) {
                    const float4 f = *reinterpret_cast<const float4*>(&sums[turn][(i * kFewShare + threadIdx.x) * kFewCols]);
                    v[0] = __fadd2_rn(v[0], make_float2(f.x, f.y));
                    v[1] = __fadd2_rn(v[1], make_float2(f.z, f.w));
                }
                if (a.bias) {
                    const float4 b = __ldg(reinterpret_cast<const float4*>(a.bias + (size_t)e * a.N + n0));
                    add_bias<4>(v, &b);
                }
                if (a.z_out) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.z_out) + o) = make_uint2(cvt_bf16x2(v[0]), cvt_bf16x2(v[1]));
                uint32_t extra[2];
                if (a.residual) {
                    const uint2 h = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(a.residual) + o);
                    extra[0] = h.x; extra[1] = h.y;
                }
                arithmetic<kForward, 4>(a, v, extra);
                *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + o) = make_uint2(cvt_bf16x2(v[0]), cvt_bf16x2(v[1]));
            }
        }
    }
}

// db without dw: db[e] = sum of the group's rows of dy, in a fixed order: a CTA takes 64 columns of one expert, eight lanes a row of
// them, all its warps the group's rows (15818 rows in 4 experts, 192 columns: 98 us with eight warps and 4 bytes a lane, 16 so).
constexpr int kBiasThreads = 1024, kBiasFew = 256, kBiasLong = 192;     // most, those for groups of fewer rows than that
__global__ void __launch_bounds__(kBiasThreads) expert_bias_grad_kernel(const int32_t* __restrict__ offsets, const uint16_t* __restrict__ dy, int R, int N,
                                                                        float* __restrict__ db) {
    __shared__ float sm[kBiasThreads / 32][64];
    pdl_wait();
    pdl_trigger();
    const int e = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Group g = group_of(offsets, e, R);
    const int col = blockIdx.x * 64 + 8 * (lane & 7);       // N is a multiple of 8
    constexpr int kFlight = 4;                              // rows of a lane in flight
    const int step = blockDim.x / 8;
    float2 s[4] = {};
    if (col < N) {
        const uint16_t* p = dy + (size_t)g.lo * N + col;
        for (int r = threadIdx.x >> 3; r < g.n; r += step * kFlight) {
            uint4 q[kFlight];
#pragma unroll
            for (int i = 0; i < kFlight; ++i)
                q[i] = r + step * i < g.n ? __ldg(reinterpret_cast<const uint4*>(p + (size_t)(r + step * i) * N)) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < kFlight; ++i) {
                s[0] = __fadd2_rn(s[0], unpack2(q[i].x)); s[1] = __fadd2_rn(s[1], unpack2(q[i].y));
                s[2] = __fadd2_rn(s[2], unpack2(q[i].z)); s[3] = __fadd2_rn(s[3], unpack2(q[i].w));
            }
        }
    }
#pragma unroll
    for (int d = 8; d < 32; d <<= 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[i].x += __shfl_xor_sync(0xffffffffu, s[i].x, d);
            s[i].y += __shfl_xor_sync(0xffffffffu, s[i].y, d);
        }
    }
    if (lane < 8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<float2*>(&sm[warp][8 * lane + 2 * i]) = s[i];
    }
    __syncthreads();
    const int c = blockIdx.x * 64 + (int)threadIdx.x;
    if (threadIdx.x < 64 && c < N) {
        float sum = 0.0f;
#pragma unroll 8
        for (int w = 0; w < (int)blockDim.x / 32; ++w) sum += sm[w][threadIdx.x];
        db[(size_t)e * N + c] = sum;
    }
}

// Weights' gradients: up to this many rows an expert on average a tile is stores more than products, and its rows leave as boxes of
// 128 bytes a row by TMA; a lane's stores of its own row are 32 bytes each, half sectors where rows do not begin on 32 (72
// rows of 12 experts, weights of 5440 x 8984: 686 against 324 us).  The boxes take the fourth stage of the ring, which long
// reductions need (65536 rows of 10240 x 2560: 64 % of the tensor cores' cycles with three stages, 80 % with four).  Between 128 and
// 512 rows an expert neither is near the copy rate (2560 x 10240 of 32 experts: 64 rows 313 us, 4096 391, 8192 579; 256 to 288 there).
constexpr int kBoxRows = 512;

// Rows of a tile.  256 rows share each weight tile's load: 32 instead of 48 KB for 128 x 256 x 64 products come through the SM's
// port to the L2, which has 64 bytes a cycle: 0.40 us for 48 KB where the products take 0.27, and 0.65 us where rows do not
// begin on sectors of 32 bytes.  But both accumulators belong to one tile then, and its epilogue stands alone.  That pays
// where rows are off the sectors, groups and reductions are long and the tiles last for some waves (18083 rows in 16 experts,
// 3544 x 3520: 535 against 456 us forward, 493 against 436 towards x, 575 against 448 for the weights, whose tiles are
// split more dearly: 12332 rows in 8 experts, 2528 x 1784, 3.8 waves, 123 against 166); with whole sectors only for weights'
// gradients of very many tiles (65536 rows in 32 experts, 2560 x 10240: 3225 against 2957 us; 20893 rows in 8, 2944 x 4672,
// 12 waves: 495 against 549), and not for products with few rows or an epilogue that costs more (65536 rows forward with
// GeLU and z: 3137 against 3696).  Long reductions on whole sectors without such an epilogue were not measured with 256.
constexpr int kTallRows = 1024, kTallK = 1536;
int rows_of_tile(Kind kind, long long R, int E, int M, int N, int K) {
    const long long tiles = (kind == kWeights ? (long long)E * ((M + 2 * BM - 1) / (2 * BM)) : R / (2 * BM)) * ((N + BN - 1) / BN);
    const bool off = kind == kWeights ? (M | N) % 16 != 0 : K % 16 != 0 || (kind == kTowardsX && N % 16 != 0);
    const bool tall = R >= (long long)kTallRows * E && (kind == kWeights ? tiles >= (off ? 8ll : 32ll) * sm_count()
                                                                         : off && K >= kTallK && tiles >= 3ll * sm_count());
    return tall ? 2 * BM : BM;
}

template <int KIND>
int launch_gemm(const LinearArgs& a0, const void* A, const void* B, void* ws, cudaStream_t st) {
    LinearArgs a = a0;
    CUtensorMap tmA, tmB, tmOther;
    a.n_tiles = (a.N + BN - 1) / BN;
    a.grid = sm_count();
    a.part = static_cast<float*>(ws);
    a.unit = rows_of_tile((Kind)KIND, a.R, a.E, a.M, a.N, a.K);
    a.part_rows = KIND == kWeights ? a.unit : min(a.R, a.unit);
    a.db_part = a.part + (size_t)a.grid * 2 * a.part_rows * BN;
    a.a_rows = a.unit;
    a.b_chunks = KIND != kForward && a.N % 64 == 0;
    if (KIND == kWeights) {         // dy [R][M], x [R][N]
        const uint64_t da[2] = {(uint64_t)a.M, (uint64_t)a.R}, db[2] = {(uint64_t)a.N, (uint64_t)a.R};
        a.a_chunks = a.M % 64 == 0;
        if (!(a.a_chunks ? make_map_chunks(&tmA, A, a.M, a.R, 1, BK, a.unit / 64) : make_map(&tmA, A, 2, da, BK))) return LOCMOE_ERR_CUDA;
        if (!(a.b_chunks ? make_map_chunks(&tmB, B, a.N, a.R, 1, BK, BN / 64) : make_map(&tmB, B, 2, db, BK))) return LOCMOE_ERR_CUDA;
    } else {
        while (a.a_rows > 16 && a.a_rows / 2 >= a.R) a.a_rows /= 2;     // few rows: smaller boxes, the tile's other rows hold what they held
        const uint64_t da[2] = {(uint64_t)a.K, (uint64_t)a.R};
        const uint64_t db[3] = {(uint64_t)(KIND == kForward ? a.K : a.N), (uint64_t)(KIND == kForward ? a.N : a.K), (uint64_t)a.E};
        if (!make_map(&tmA, A, 2, da, a.a_rows)) return LOCMOE_ERR_CUDA;
        if (!(a.b_chunks ? make_map_chunks(&tmB, B, a.N, a.K, a.E, BK, BN / 64) : make_map(&tmB, B, 3, db, KIND == kForward ? BN : BK))) return LOCMOE_ERR_CUDA;
    }
    // the weights' gradient on its way out, or A in boxes of 32 rows
    const uint64_t dims[2] = {(uint64_t)a.K, (uint64_t)a.R};
    if (!(KIND == kWeights ? make_store_map(&tmOther, a.out, a.out_f32, a.N, a.M, a.E) : make_map(&tmOther, A, 2, dims, 32))) return LOCMOE_ERR_CUDA;
    a.boxes = KIND == kWeights && a.unit == BM && (long long)a.R < (long long)kBoxRows * a.E;
    a.stages = a.boxes ? kBoxStages : (int)(kRing / ((size_t)a.a_rows * BK * 2 + B_BYTES));
    if (a.stages > kMaxStages) a.stages = kMaxStages;
    auto* kernel = a.unit > BM ? expert_gemm_kernel<KIND, 2> : expert_gemm_kernel<KIND, 1>;
    static bool attr_done_dev[2][64] = {};     // the attribute is per device
    int dev = 0;
    cudaGetDevice(&dev);
    bool& attr_done = attr_done_dev[a.unit > BM][dev & 63];
    if (!attr_done) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem) != cudaSuccess) {
            cudaGetLastError();
            return LOCMOE_ERR_CUDA;
        }
        attr_done = true;
    }
    const bool join = may_split<KIND>(a);
    a.split = join ? reinterpret_cast<Split*>(a.db_part + (KIND == kWeights ? (size_t)a.grid * 2 * a.unit : 0)) : nullptr;
    int rc = launch_pdl(kernel, dim3(a.grid), dim3(KIND == kWeights && a.db ? kWeightsThreads : kThreads), kSmem, st, tmA, tmB, tmOther, a);
    if (rc) return rc;
    if (join) {
        const int parts = (a.part_rows * (BN / 8) + kJoinThreads - 1) / kJoinThreads;
        rc = launch_pdl(expert_join_kernel<KIND>, dim3(a.grid, parts < kJoinParts ? parts : kJoinParts), dim3(kJoinThreads), 0, st, a);
    }
    return rc ? rc : check_launch();
}

}  // namespace

// Two tiles' sums a CTA, and what its split tile is.
size_t expert_linear_ws_bytes(const locmoe_shape_t& s, int N, int grad) {
    const int unit = grad ? max(rows_of_tile(kTowardsX, s.T, s.E, 0, s.H, N), rows_of_tile(kWeights, s.T, s.E, N, s.H, 0)) : rows_of_tile(kForward, s.T, s.E, 0, N, s.H);
    const size_t rows = grad || s.T > unit ? unit : s.T, sums = rows * BN + (grad ? unit : 0);
    return ((size_t)sm_count() * (2 * sums * sizeof(float) + sizeof(Split)) + 255) & ~(size_t)255;
}

int launch_expert_linear(const locmoe_shape_t& s, int N, const locmoe_expert_linear_t& l, void* ws, cudaStream_t st) {
    LinearArgs a{};
    a.offsets = l.offsets; a.out = l.y; a.z_out = l.z; a.bias = l.bias; a.residual = l.residual; a.act = l.act;
    a.E = s.E; a.R = s.T; a.N = N; a.K = s.H;
    if (s.T <= (s.H <= kFewWeight / N ? kFewRows : kFewRows / 2)) {
        // warps a task: the fewest turns of all, each as long as a warp's part of the reduction
        const long long tasks = (long long)s.T * (N / kFewCols), warps = (long long)kFewWarps * sm_count();
        int best = 1;
        double cost = 1e30;
        for (int n = 1; n * 32 <= kFewThreads && (n == 1 || n * 32 <= s.H / 8); n *= 2) {
            const double c = (double)((tasks * n + warps - 1) / warps) * ((s.H / 8 + 32 * n - 1) / (32 * n) + 1);
            if (c <= cost) { cost = c; best = n; }
        }
        const long long resident = warps / best;
        const int rc = launch_pdl(expert_few_kernel, dim3((unsigned)(tasks < resident ? tasks : resident)), dim3(32 * best), 0, st, a,
                                  static_cast<const uint16_t*>(l.x), static_cast<const uint16_t*>(l.w));
        return rc ? rc : check_launch();
    }
    return launch_gemm<kForward>(a, l.x, l.w, ws, st);
}

int launch_expert_linear_grad(const locmoe_shape_t& s, int N, const locmoe_expert_linear_grad_t& l, void* ws, cudaStream_t st) {
    int rc = LOCMOE_OK;
    if (l.dx) {
        LinearArgs a{};
        a.offsets = l.offsets; a.out = l.dx;
        if (l.z && l.act != LOCMOE_ACT_NONE) { a.z_in = l.z; a.act = l.act; }
        a.E = s.E; a.R = s.T; a.N = s.H; a.K = N;
        rc = launch_gemm<kTowardsX>(a, l.dy, l.w, ws, st);
        if (rc) return rc;
    }
    if (l.dw) {
        LinearArgs a{};
        a.offsets = l.offsets; a.out = l.dw; a.out_f32 = l.dw_dtype == LOCMOE_F32; a.db = l.db;
        a.E = s.E; a.R = s.T; a.M = N; a.N = s.H;
        rc = launch_gemm<kWeights>(a, l.dy, l.x, ws, st);
        if (rc) return rc;
    }
    if (l.db && !l.dw) {
        const int threads = (long long)s.T < (long long)kBiasLong * s.E ? kBiasFew : kBiasThreads;
        rc = launch_pdl(expert_bias_grad_kernel, dim3((N + 63) / 64, s.E), dim3(threads), 0, st, l.offsets, static_cast<const uint16_t*>(l.dy), (int)s.T, N, l.db);
        if (rc) return rc;
    }
    return check_launch();
}

int read_linear_flags(int* out, cudaStream_t st) {
    if (cudaMemcpyFromSymbolAsync(out, g_linear_flags, sizeof(int), 0, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaStreamSynchronize(st) != cudaSuccess) {
        cudaGetLastError();
        return LOCMOE_ERR_CUDA;
    }
    return LOCMOE_OK;
}

}  // namespace locmoe
