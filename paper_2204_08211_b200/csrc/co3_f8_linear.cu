// Products of 8-bit blocks on the tensor cores: y = x W^T + b and its counterpart towards the inputs, x W.
//
// The weights are the first operand, 128 of their rows (or, transposed, of their columns) per tile, and the rows of x the second,
// 16 to 256 of them: tensor memory then holds an output feature per lane and a row of x per column, so that a warp's 32 lanes
// write neighbouring entries of y, and few rows of x cost little.  The tensor core applies both operands' scales while it multiplies
// (kind::mxf8f6f4, an exponent byte for each 32 columns of the sum: the same four times); sums are fp32 in tensor memory, and in
// registers every so many columns.
//
// A block of threads: one warp issues bulk copies, one the products, eight warps take the sums out.  A stage of the ring is a
// block of 128 columns of the sum; exponent bytes come with every fourth.  Few tiles: the blocks of a cluster divide the
// sum's length, and add their parts through shared memory in order.
#include <algorithm>
#include <atomic>

#include "co3_f8.cuh"
#include "co3_launch.cuh"
#include "co3_orth.cuh"

namespace co3 {

namespace {

constexpr uint32_t kMaxSplit = 8;
constexpr uint32_t kTmemScales = 256;        // first column of the exponent bytes; eight turns of 16 columns
constexpr uint32_t kScaleTurns = 8, kScaleCols = 16;
// The tensor core cuts what it adds towards zero, about 2^-25 of the sum each time: a sum is taken out and added up in registers,
// to nearest, after so many blocks.  Results of 16 bits round by 2^-12 and more.  For fp32 results, us and error relative to the
// result's norm after 8, 4 and 2 blocks (fp32 products in PyTorch): 6400 x 512 x 512 14.3, 14.2, 15.0 and 3.3, 3.3, 2.5e-8 (2.6);
// 2048 x 2048 x 2048 23.7, 25.2, 28.3 and 6.5, 5.0, 4.8e-8 (5.9); 16384 x 4096 x 4096 291, 324, 401 and 7.2, 6.2, 6.5e-8 (8.5).  Beside
// the 2^-4 by which operands of 8 bits are off none of it counts: 8.
constexpr uint32_t kBlocksF32 = 8, kBlocks16 = 32;

struct LinearArgs {
    const uint8_t *a, *a_scales, *b, *b_scales;
    uint64_t a_block, a_tile;                // bytes between blocks of the sum, between tiles
    uint64_t a_group, b_group;               // bytes between groups of four blocks' exponent bytes
    uint64_t b_block;
    uint32_t kb;                             // blocks of the sum
    uint32_t features, rows;
    uint32_t m_tiles, n_tiles;
    uint32_t split;
    uint32_t pair_rows;                      // rows of x in a pair's tile, 128 or 256
    uint32_t blocks;                         // blocks that tensor memory adds up
    void* y;
    uint64_t y_stride;
    int y_type;
    const float* bias;
    co3_result* res;
};

constexpr uint32_t kScaleBytes = 2 * kF8Scales;  // of a stage: first operand's, then the second's
template <int kN>
struct Shape {
    static constexpr uint32_t kStages = kN == 128 ? 6 : 8;
    static constexpr uint32_t kStageBytes = kF8Tile + kN * 128;
    static constexpr uint32_t kRing = kStages * kStageBytes;
    static constexpr uint32_t kSmem = 1024 + kRing + kStages * kScaleBytes + 256;
    static_assert(kN * 128 * 4 <= kRing, "a tile's sums fit the ring");
};

template <int kN>
struct LinearSmem {
    uint64_t full[Shape<kN>::kStages], empty[Shape<kN>::kStages], sum_full[2], sum_empty[2], done;
    uint32_t tmem, failed;
};

// D fp32, A and B e4m3, scales of eight bits of exponent; `block` says which byte of the scales' columns counts.
__host__ __device__ constexpr uint32_t f8_instr(bool a_transposed, uint32_t cols, uint32_t block) {
    return (block << 4) | ((uint32_t)a_transposed << 15) | ((cols / 8u) << 17) | (1u << 23) | (1u << 27) | (block << 29);
}
__device__ __forceinline__ void f8_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t instr, uint32_t sa, uint32_t sb, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(instr), "r"(sa),
        "r"(sb), "r"((uint32_t)accumulate)
        : "memory");
}
// 512 bytes of shared memory, 32 rows of 16, to four columns of tensor memory, the same for each 32 lanes.
__device__ __forceinline__ void f8_scales_in(uint32_t to, uint32_t from) {
    const uint64_t desc = (uint64_t)((from >> 4) & 0x3fffu) | (8ull << 32) | (1ull << 46);
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(to), "l"(desc) : "memory");
}
// Operands as co3_orth.cuh has them, here of one-byte elements: 32 columns of the sum are 32 bytes of a row or, transposed, 32 rows
// of 128 bytes.
__device__ __forceinline__ uint64_t f8_desc(uint32_t addr) { return (uint64_t)((addr >> 4) & 0x3fffu) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61); }
__host__ __device__ constexpr uint32_t f8_step(bool transposed) { return transposed ? 4096u >> 4 : 32u >> 4; }

// The four products of a stage.
template <bool kTransposed, uint32_t kBlock4>
__device__ __forceinline__ void multiply_block(uint32_t d, uint32_t a, uint32_t b, uint32_t cols, uint32_t sa, uint32_t sb, bool accumulate) {
    const uint64_t da = f8_desc(a), db = f8_desc(b);
    const uint32_t instr = f8_instr(kTransposed, 0, kBlock4) | ((cols / 8u) << 17);
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) f8_mma(d, da + e * f8_step(kTransposed), db + e * f8_step(false), instr, sa, sb, accumulate || e > 0);
}

__device__ __forceinline__ void tc_load8(uint32_t addr, float (&v)[8]) {
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(addr)
                 : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
// Adds a half tile's columns to acc, or (first) puts them there.
template <int kHalf>
__device__ __forceinline__ void take_sums(uint32_t from, bool first, float (&acc)[kHalf]) {
    constexpr int kLoad = kHalf < 32 ? kHalf : 32;
    if (first) {
        if constexpr (kHalf == 8) tc_load8(from, acc);
        else tc_load(from, acc);
    } else {
#pragma unroll
        for (int h = 0; h < kHalf; h += kLoad) {
            float w[kLoad];
            if constexpr (kHalf == 8) tc_load8(from + h, w);
            else tc_load(from + h, w);
#pragma unroll
            for (int i = 0; i < kLoad; ++i) acc[h + i] = __fadd_rn(acc[h + i], w[i]);
        }
    }
}

// The sums of four neighbouring entries over the cluster's blocks, in order, from the same place in each one's shared memory.
__device__ __forceinline__ float4 add_parts(uint32_t addr, uint32_t split) {
    float4 v[kMaxSplit];
#pragma unroll
    for (uint32_t p = 0; p < kMaxSplit; ++p) {
        if (p >= split) break;
        uint32_t at;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(p));
        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[p].x), "=f"(v[p].y), "=f"(v[p].z), "=f"(v[p].w) : "r"(at) : "memory");
    }
    float4 s = v[0];
#pragma unroll
    for (uint32_t p = 1; p < kMaxSplit; ++p) {
        if (p >= split) break;
        s = make_float4(__fadd_rn(s.x, v[p].x), __fadd_rn(s.y, v[p].y), __fadd_rn(s.z, v[p].z), __fadd_rn(s.w, v[p].w));
    }
    return s;
}
// This block's part of a tile whose parts lie in shared memory, 128 features for each row of x: `rows` of them from row n0 on, by 256
// threads.
template <typename T>
__device__ __forceinline__ void join_parts(const LinearArgs& a, uint32_t sums, uint32_t part, uint32_t feature0, uint32_t n0, uint32_t rows, uint32_t tid) {
    const uint32_t all = rows * 32u, i1 = all * (part + 1) / a.split, f = feature0 + (tid & 31u) * 4u;
    for (uint32_t i = all * part / a.split / 32u * 32u + tid; i < i1; i += 256u) {
        if (i < all * part / a.split) continue;
        const uint32_t r = i >> 5;
        const float4 v = add_parts(sums + i * 16u, a.split);
        const float w[4] = {v.x, v.y, v.z, v.w};
        T* p = static_cast<T*>(a.y) + (uint64_t)(n0 + r) * a.y_stride + f;
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
            if (f + k < a.features) p[k] = from_float<T>(a.bias ? __fadd_rn(w[k], a.bias[f + k]) : w[k]);
    }
}
__device__ __forceinline__ void join_parts_any(const LinearArgs& a, uint32_t sums, uint32_t part, uint32_t feature0, uint32_t n0, uint32_t rows, uint32_t tid) {
    if (a.y_type == CO3_F32) join_parts<float>(a, sums, part, feature0, n0, rows, tid);
    else if (a.y_type == CO3_F16) join_parts<__half>(a, sums, part, feature0, n0, rows, tid);
    else join_parts<__nv_bfloat16>(a, sums, part, feature0, n0, rows, tid);
}

// A lane's sums of kCount rows of x, from row `first` on.
template <typename T, int kCount>
__device__ __forceinline__ void write_sums(const LinearArgs& a, uint32_t feature, uint32_t first, float bias, const float* v) {
    T* p = static_cast<T*>(a.y) + (uint64_t)first * a.y_stride + feature;
#pragma unroll
    for (int i = 0; i < kCount; ++i)
        if (first + i < a.rows) p[i * a.y_stride] = from_float<T>(__fadd_rn(v[i], bias));
}
template <int kCount>
__device__ __forceinline__ void write_any(const LinearArgs& a, uint32_t feature, uint32_t first, float bias, const float* v) {
    if (feature >= a.features) return;
    if (a.y_type == CO3_F32) write_sums<float, kCount>(a, feature, first, bias, v);
    else if (a.y_type == CO3_F16) write_sums<__half, kCount>(a, feature, first, bias, v);
    else write_sums<__nv_bfloat16, kCount>(a, feature, first, bias, v);
}

template <int kN, bool kTransposed, bool kSplit>
__global__ void __launch_bounds__(kF8Threads, 1) f8_linear_kernel(const __grid_constant__ LinearArgs a) {
    extern __shared__ unsigned char smem_raw[];
    using S = Shape<kN>;
    constexpr uint32_t kStages = S::kStages;
    unsigned char* ring = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    unsigned char* scales = ring + S::kRing;
    LinearSmem<kN>& sm = *reinterpret_cast<LinearSmem<kN>*>(scales + kStages * kScaleBytes);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < kStages; ++i) { mbar_init(&sm.full[i], 1); mbar_init(&sm.empty[i], 1); }
        for (uint32_t i = 0; i < 2; ++i) { mbar_init(&sm.sum_full[i], 1); mbar_init(&sm.sum_empty[i], 8); }
        mbar_init(&sm.done, 1);
        sm.failed = 0;
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&sm.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm.tmem;
    volatile uint32_t* failed = &sm.failed;
    wait_for_previous_kernel();

    const uint32_t tiles = a.m_tiles * a.n_tiles;
    const uint32_t part = kSplit ? blockIdx.x % a.split : 0u, step = kSplit ? gridDim.x / a.split : gridDim.x;
    const uint32_t first = kSplit ? blockIdx.x / a.split : blockIdx.x;  // one tile a cluster when split
    const uint32_t k0 = kSplit ? (uint32_t)((uint64_t)a.kb * part / a.split) : 0u, k1 = kSplit ? (uint32_t)((uint64_t)a.kb * (part + 1) / a.split) : a.kb;

    if (warp < 4) few_registers();
    const bool issues = warp < 2 && elected();
    if (warp == 0) {
        uint32_t st = 0, turn = 0;
        for (uint32_t t = first; t < tiles && !*failed; t += step) {
            const uint32_t mt = t % a.m_tiles, nt = t / a.m_tiles, n0 = nt * kN;
            const uint32_t n = min((uint32_t)kN, (a.rows - n0 + 15u) & ~15u);
            for (uint32_t q = k0; q < k1; ++q) {
                if (turn > 0 && !f8_wait(&sm.empty[st], (turn - 1) & 1u)) { *failed = 1; break; }
                if (issues) {
                    unsigned char* to = ring + st * S::kStageBytes;
                    const bool with_scales = q == k0 || (q & 3u) == 0;
                    mbar_arrive_expect_tx(&sm.full[st], kF8Tile + n * 128u + (with_scales ? 2 * kF8Scales : 0u));
                    bulk_copy_g2s(to, a.a + q * a.a_block + mt * a.a_tile, kF8Tile, &sm.full[st]);
                    bulk_copy_g2s(to + kF8Tile, a.b + q * a.b_block + (uint64_t)n0 * 128u, n * 128u, &sm.full[st]);
                    if (with_scales) {
                        unsigned char* s = scales + st * kScaleBytes;
                        bulk_copy_g2s(s, a.a_scales + (q >> 2) * a.a_group + (uint64_t)mt * kF8Scales, kF8Scales, &sm.full[st]);
                        bulk_copy_g2s(s + kF8Scales, a.b_scales + (q >> 2) * a.b_group + (uint64_t)(n0 >> 7) * kF8Scales, kF8Scales, &sm.full[st]);
                    }
                }
                if (++st == kStages) { st = 0; ++turn; }
            }
        }
        // copies in flight end before the block does, whoever else has given up
        for (uint32_t i = 0; i < kStages; ++i) {
            const uint32_t begun = turn + (i < st ? 1u : 0u);
            if (begun > 0) f8_wait(&sm.full[i], (begun - 1) & 1u);
        }
    } else if (warp == 1) {
        uint32_t st = 0, turn = 0, sum = 0, sum_turn = 0, group = 0;
        bool ok = true;
        for (uint32_t t = first; t < tiles && ok && !*failed; t += step) {
            const uint32_t n0 = t / a.m_tiles * kN, n = min((uint32_t)kN, (a.rows - n0 + 15u) & ~15u);
            uint32_t left = 0;  // blocks that the present sum still takes
            for (uint32_t q = k0; q < k1; ++q) {
                const bool fresh = left == 0;
                if (fresh) {
                    left = min(a.blocks, k1 - q);
                    if (sum_turn > 0 && !f8_wait(&sm.sum_empty[sum], (sum_turn - 1) & 1u)) { ok = false; break; }
                }
                --left;
                if (!f8_wait(&sm.full[st], turn & 1u)) { ok = false; break; }
                tc_fence_after();
                const bool with_scales = q == k0 || (q & 3u) == 0;
                // the columns of eight groups ago are free: fewer than kStages <= 8 blocks are under way
                if (with_scales) group = (group + 1) % kScaleTurns;
                if (issues) {
                    const uint32_t d = tmem + sum * kN, sa = tmem + kTmemScales + group * kScaleCols;
                    if (with_scales) {
                        const uint32_t from = smem_addr(scales + st * kScaleBytes);
                        f8_scales_in(sa, from);
                        f8_scales_in(sa + 4, from + kF8Scales);
                    }
                    const uint32_t sb = sa + 4 + ((n0 & 127u) >> 5), at = smem_addr(ring + st * S::kStageBytes), bt = at + kF8Tile;
                    switch (q & 3u) {
                        case 0: multiply_block<kTransposed, 0>(d, at, bt, n, sa, sb, !fresh); break;
                        case 1: multiply_block<kTransposed, 1>(d, at, bt, n, sa, sb, !fresh); break;
                        case 2: multiply_block<kTransposed, 2>(d, at, bt, n, sa, sb, !fresh); break;
                        default: multiply_block<kTransposed, 3>(d, at, bt, n, sa, sb, !fresh); break;
                    }
                    tc_commit(&sm.empty[st]);
                    if (left == 0) tc_commit(&sm.sum_full[sum]);
                }
                if (left == 0 && ++sum == 2) { sum = 0; ++sum_turn; }
                if (++st == kStages) { st = 0; ++turn; }
            }
        }
        if (!ok) *failed = 1;
        if (issues) tc_commit(&sm.done);
        f8_wait(&sm.done, 0);
    } else if (warp >= 4) {
        many_registers();
        // lanes of a tile by quarters, columns by halves
        constexpr int kHalf = kN / 2;
        const uint32_t quad = warp & 3u, half = (warp - 4u) >> 2, row = quad * 32u + lane;
        uint32_t sum = 0, sum_turn = 0;
        for (uint32_t t = first; t < tiles; t += step) {
            const uint32_t mt = t % a.m_tiles, n0 = t / a.m_tiles * kN, feature = mt * 128u + row;
            bool ok = true;
            float acc[kHalf];
            for (uint32_t q = k0; q < k1; q += a.blocks) {
                ok = lane != 0 || f8_wait(&sm.sum_full[sum], sum_turn & 1u);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                const uint32_t from = tmem + ((quad * 32u) << 16) + sum * kN + half * kHalf;
                take_sums(from, q == k0, acc);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.sum_empty[sum]);
                if (++sum == 2u) { sum = 0; ++sum_turn; }
            }
            if (!ok) { *failed = 1; break; }
            if constexpr (kSplit) {  // into the ring, of which no copy and no product is left
                float* to = reinterpret_cast<float*>(ring) + (uint64_t)half * kHalf * 128u + row;
#pragma unroll
                for (int i = 0; i < kHalf; ++i) to[i * 128] = acc[i];
            } else {
                const float bias = a.bias && feature < a.features ? a.bias[feature] : 0.0f;
                write_any<kHalf>(a, feature, n0 + half * kHalf, bias, acc);
            }
        }
        if constexpr (kSplit) {
            // everybody's part is there; each block takes some of the columns
            __syncwarp();
            cluster_sync();
            const uint32_t n0 = first / a.m_tiles * kN;
            if (!*failed) join_parts_any(a, smem_addr(ring), part, first % a.m_tiles * 128u, n0, min((uint32_t)kN, a.rows - n0), threadIdx.x - 128u);
        }
    }
    __syncwarp();
    if constexpr (kSplit) {
        if (warp < 4) cluster_sync();
        cluster_sync();  // nobody leaves while its part is read
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    if (threadIdx.x == 0 && *failed && a.res) atomicExch(&a.res->status, CO3_ERR_CUDA);
}

// ------------------------------------------------------------------------------------------------
// Tiles of 256 features by 256 (or 128) rows of x, by pairs of blocks.
// ------------------------------------------------------------------------------------------------
constexpr uint32_t kPairCols = 256, kPairStages = 6;
constexpr uint32_t kPairStageBytes = 2 * kF8Tile, kPairScaleBytes = 3 * kF8Scales;  // the second operand's scales for all 256 rows
constexpr uint32_t kPairSmem = 1024 + kPairStages * (kPairStageBytes + kPairScaleBytes) + 256;

struct PairSmem {
    uint64_t full[kPairStages], empty[kPairStages], sum_full, sum_empty, done;
    uint32_t tmem, failed;
};
static_assert(sizeof(PairSmem) <= 256, "barriers");

__device__ __forceinline__ void pair_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t instr, uint32_t sa, uint32_t sb, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(instr), "r"(sa),
        "r"(sb), "r"((uint32_t)accumulate)
        : "memory");
}
// In each of the two blocks, from its own shared memory.
__device__ __forceinline__ void pair_scales_in(uint32_t to, uint32_t from) {
    const uint64_t desc = (uint64_t)((from >> 4) & 0x3fffu) | (8ull << 32) | (1ull << 46);
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(to), "l"(desc) : "memory");
}
template <bool kTransposed, uint32_t kBlock4>
__device__ __forceinline__ void multiply_block_pair(uint32_t d, uint32_t a, uint32_t b, uint32_t cols, uint32_t sa, uint32_t sb, bool accumulate) {
    const uint64_t da = f8_desc(a), db = f8_desc(b);
    const uint32_t instr = (f8_instr(kTransposed, 0, kBlock4) + (1u << 27)) | ((cols / 8u) << 17);  // 256 rows of A
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) pair_mma(d, da + e * f8_step(kTransposed), db + e * f8_step(false), instr, sa, sb, accumulate || e > 0);
}

template <bool kTransposed>
__global__ void __launch_bounds__(kF8Threads, 1) f8_pair_kernel(const __grid_constant__ LinearArgs a) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* ring = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    unsigned char* scales = ring + kPairStages * kPairStageBytes;
    PairSmem& sm = *reinterpret_cast<PairSmem*>(scales + kPairStages * kPairScaleBytes);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, rank = cluster_rank();
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < kPairStages; ++i) { mbar_init(&sm.full[i], rank == 0 ? 2 : 1); mbar_init(&sm.empty[i], 1); }
        mbar_init(&sm.sum_full, 1);
        mbar_init(&sm.sum_empty, 16);
        mbar_init(&sm.done, 1);
        sm.failed = 0;
    }
    if (warp == 1) tmem_alloc_pair(&sm.tmem);
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = sm.tmem;
    volatile uint32_t* failed = &sm.failed;
    wait_for_previous_kernel();
    const uint32_t m_pairs = (a.m_tiles + 1) / 2, tiles = m_pairs * a.n_tiles, first = blockIdx.x >> 1, step = gridDim.x >> 1;

    if (warp < 4) {
        few_registers();
        const bool issues = elected();
        if (warp == 0) {
            uint32_t st = 0, turn = 0;
            for (uint32_t t = first; t < tiles && !*failed; t += step) {
                const uint32_t mt = min(2 * (t % m_pairs) + rank, a.m_tiles - 1);  // (an odd last tile: the second block's sums go nowhere)
                const uint32_t n0 = t / m_pairs * a.pair_rows, n = min(a.pair_rows, (a.rows - n0 + 15u) & ~15u);
                const uint32_t b_scales = n > 128 ? 2 * kF8Scales : kF8Scales, half = n / 2;
                const uint8_t *from_a = a.a + mt * a.a_tile, *from_b = a.b + (n0 + rank * half) * 128ull;
                for (uint32_t q = 0; q < a.kb; ++q) {
                    if (turn > 0 && !f8_wait(&sm.empty[st], (turn - 1) & 1u)) { *failed = 1; break; }
                    if (issues) {
                        unsigned char* to = ring + st * kPairStageBytes;
                        // exponent bytes of a tile's first group, and then of each next one a few blocks ahead
                        const uint32_t group = q == 0 ? 0u : (q >> 2) + 1;
                        const bool with_scales = q == 0 || ((q & 3u) == 1u && group * 4u < a.kb);
                        mbar_arrive_expect_tx(&sm.full[st], kF8Tile + half * 128u + (with_scales ? kF8Scales + b_scales : 0u));
                        bulk_copy_g2s(to, from_a + q * a.a_block, kF8Tile, &sm.full[st]);
                        bulk_copy_g2s(to + kF8Tile, from_b + q * a.b_block, half * 128u, &sm.full[st]);
                        if (with_scales) {
                            unsigned char* s = scales + st * kPairScaleBytes;
                            bulk_copy_g2s(s, a.a_scales + group * a.a_group + (uint64_t)mt * kF8Scales, kF8Scales, &sm.full[st]);
                            bulk_copy_g2s(s + kF8Scales, a.b_scales + group * a.b_group + (uint64_t)(n0 >> 7) * kF8Scales, b_scales, &sm.full[st]);
                        }
                    }
                    if (++st == kPairStages) { st = 0; ++turn; }
                }
            }
            // copies in flight end before the block does, whoever else has given up
            for (uint32_t i = 0; i < kPairStages; ++i) {
                const uint32_t begun = turn + (i < st ? 1u : 0u);
                if (begun > 0) f8_wait(&sm.full[i], (begun - 1) & 1u);
            }
        } else if (warp == 1 && rank == 1) {
            // tells the first block what has arrived here: its barrier waits for both
            uint32_t st = 0, turn = 0;
            bool ok = true;
            for (uint32_t t = first; t < tiles && ok; t += step)
                for (uint32_t q = 0; q < a.kb; ++q) {
                    if (!f8_wait(&sm.full[st], turn & 1u)) { ok = false; break; }
                    if (issues) mbar_arrive_at(&sm.full[st], 0);
                    if (++st == kPairStages) { st = 0; ++turn; }
                }
            if (!ok) *failed = 1;
        } else if (warp == 1) {
            uint32_t st = 0, turn = 0, sums = 0, group = 0;  // sums: begun
            bool ok = true;
            for (uint32_t t = first; t < tiles && ok; t += step) {
                const uint32_t n = min(a.pair_rows, (a.rows - t / m_pairs * a.pair_rows + 15u) & ~15u);
                uint32_t left = 0;  // blocks that the present sum still takes
                for (uint32_t q = 0; q < a.kb; ++q) {
                    const bool fresh = left == 0;
                    if (fresh) {
                        left = min(a.blocks, a.kb - q);
                        if (sums > 0 && !f8_wait(&sm.sum_empty, (sums - 1) & 1u)) { ok = false; break; }
                        ++sums;
                    }
                    --left;
                    if (!f8_wait(&sm.full[st], turn & 1u)) { ok = false; break; }
                    tc_fence_after();
                    if ((q & 3u) == 0) group = (group + 1) % kScaleTurns;
                    if (issues) {
                        const uint32_t sa = tmem + kTmemScales + group * kScaleCols, sb = sa + 4;
                        const uint32_t from = smem_addr(scales + st * kPairScaleBytes), at = smem_addr(ring + st * kPairStageBytes), bt = at + kF8Tile;
                        // to columns of eight groups ago, which are free: fewer than kPairStages blocks are under way
                        auto bring_scales = [&](uint32_t to) {
                            pair_scales_in(to, from);
                            pair_scales_in(to + 4, from + kF8Scales);
                            if (n > 128) pair_scales_in(to + 8, from + 2 * kF8Scales);
                        };
                        if (q == 0) bring_scales(sa);
                        switch (q & 3u) {
                            case 0: multiply_block_pair<kTransposed, 0>(tmem, at, bt, n, sa, sb, !fresh); break;
                            case 1: multiply_block_pair<kTransposed, 1>(tmem, at, bt, n, sa, sb, !fresh); break;
                            case 2: multiply_block_pair<kTransposed, 2>(tmem, at, bt, n, sa, sb, !fresh); break;
                            default: multiply_block_pair<kTransposed, 3>(tmem, at, bt, n, sa, sb, !fresh); break;
                        }
                        // the next group's, while this one is multiplied: right before their use they cost 25 us of 16384 x 4096 x 4096's
                        // 245, here 14
                        if ((q & 3u) == 1u && ((q >> 2) + 1) * 4u < a.kb) bring_scales(tmem + kTmemScales + (group + 1) % kScaleTurns * kScaleCols);
                        tc_commit_pair(&sm.empty[st]);
                        if (left == 0) tc_commit_pair(&sm.sum_full);
                    }
                    if (++st == kPairStages) { st = 0; ++turn; }
                }
            }
            if (!ok) *failed = 1;
            if (issues) tc_commit_first(&sm.done);
            f8_wait(&sm.done, 0);
        }
    } else {
        many_registers();
        constexpr int kHalf = kPairCols / 2;
        const uint32_t quad = warp & 3u, half = (warp - 4u) >> 2, row = quad * 32u + lane;
        const uint32_t cols = a.pair_rows / 2;  // of a warp
        uint32_t sums = 0;
        bool ok = true;
        for (uint32_t t = first; t < tiles && ok; t += step) {
            const uint32_t n0 = t / m_pairs * a.pair_rows, feature = (2 * (t % m_pairs) + rank) * 128u + row;
            float acc[kHalf];
            for (uint32_t q = 0; q < a.kb; q += a.blocks, ++sums) {
                ok = lane != 0 || f8_wait(&sm.sum_full, sums & 1u);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                const uint32_t from = tmem + ((quad * 32u) << 16) + half * cols;
                if (cols == kHalf) take_sums(from, q == 0, acc);
                else take_sums(from, q == 0, *reinterpret_cast<float(*)[kHalf / 2]>(acc));
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_at(&sm.sum_empty, 0);
            }
            if (!ok) break;
            const float bias = a.bias && feature < a.features ? a.bias[feature] : 0.0f;
            if (cols == kHalf) write_any<kHalf>(a, feature, n0 + half * cols, bias, acc);
            else write_any<kHalf / 2>(a, feature, n0 + half * cols, bias, acc);
        }
        if (!ok) *failed = 1;
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // the other block's arrivals and products need this one's shared memory
    tc_fence_after();
    if (warp == 1) tmem_free_pair(tmem);
    if (threadIdx.x == 0 && *failed && a.res) atomicExch(&a.res->status, CO3_ERR_CUDA);
}

// ------------------------------------------------------------------------------------------------
// Up to 16 rows of x (tokens of a decoding loop): a cluster's blocks divide the sum, each brings its own columns of x into shared
// memory as 8-bit blocks while the first tiles of the weights are on their way, so that there is one launch, and the packed rows go
// to memory from the first tile's blocks alone.
// ------------------------------------------------------------------------------------------------
constexpr uint32_t kFewRows = 16, kFewStages = 8, kFewBlocks = 32;  // blocks of columns of x that a block of threads holds
constexpr uint32_t kFewRing = kFewStages * kF8Tile, kFewX = kFewBlocks * kFewRows * 128;
constexpr uint32_t kFewSmem = 1024 + kFewRing + kFewX + (kFewStages + kFewBlocks / 4 + 1) * kF8Scales + 256;

struct FewArgs {
    LinearArgs l;
    const void* x;           // nullable: the blocks are in l.b
    int x_type;
    uint64_t x_stride;
    uint32_t cols, wide;     // wide: rows are aligned for four values at a time
    uint8_t *x8, *x8_scales;
};
// Two warps issue products, for every other group of four blocks, each into sums of its own that are added up at the end: one alone takes
// 0.35 us for the 16 KB of a stage (1 x 8192 x 8192 22.4 us, with two 17.6; the weights' bytes 10).
constexpr uint32_t kFewSums = 4;
static_assert(kFewStages == 8 && (kFewBlocks / 4 + 2) / 2 * 4 <= kFewSums * kBlocksF32 && kFewBlocks <= kBlocks16, "a warp's sums");
struct FewSmem {
    uint64_t full[kFewStages], empty[kFewStages], sum_full[2], ready, done[2];
    uint32_t tmem, failed;
};
static_assert(sizeof(FewSmem) <= 256, "barriers");

// Four neighbouring values, zeros beyond the row's end.
template <typename T>
__device__ __forceinline__ void load4(const T* p, uint32_t left, bool wide, float (&v)[4]) {
    if (wide && left >= 4) {
        if constexpr (sizeof(T) == 4) {
            const float4 f = *reinterpret_cast<const float4*>(p);
            v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
        } else {
            const uint2 raw = *reinterpret_cast<const uint2*>(p);
            const T* e = reinterpret_cast<const T*>(&raw);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = to_float(e[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (uint32_t)i < left ? to_float(p[i]) : 0.0f;
    }
}
__device__ __forceinline__ void load4_any(const FewArgs& a, uint32_t row, uint64_t col, float (&v)[4]) {
    const uint32_t left = col < a.cols ? (uint32_t)(a.cols - col) : 0u;
    const uint64_t at = row * a.x_stride + col;
    if (a.x_type == CO3_F32) load4(static_cast<const float*>(a.x) + at, left, a.wide, v);
    else if (a.x_type == CO3_F16) load4(static_cast<const __half*>(a.x) + at, left, a.wide, v);
    else load4(static_cast<const __nv_bfloat16*>(a.x) + at, left, a.wide, v);
}

template <bool kTransposed>
__global__ void __launch_bounds__(kF8Threads, 1) f8_few_kernel(const __grid_constant__ FewArgs few) {
    extern __shared__ unsigned char smem_raw[];
    const LinearArgs& a = few.l;
    unsigned char* ring = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    unsigned char* xs = ring + kFewRing;                              // its blocks, 16 rows of 128 bytes each
    unsigned char* scales = xs + kFewX;                               // the weights' for each stage, then x's for each group
    unsigned char* x_scales = scales + kFewStages * kF8Scales;
    FewSmem& sm = *reinterpret_cast<FewSmem*>(x_scales + (kFewBlocks / 4 + 1) * kF8Scales);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < kFewStages; ++i) { mbar_init(&sm.full[i], 1); mbar_init(&sm.empty[i], 1); }
        for (uint32_t i = 0; i < 2; ++i) { mbar_init(&sm.sum_full[i], 1); mbar_init(&sm.done[i], 1); }
        mbar_init(&sm.ready, 8);
        sm.failed = 0;
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&sm.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm.tmem;
    volatile uint32_t* failed = &sm.failed;
    wait_for_previous_kernel();

    const uint32_t part = blockIdx.x % a.split, mt = blockIdx.x / a.split;
    const uint32_t k0 = (uint32_t)((uint64_t)a.kb * part / a.split), k1 = (uint32_t)((uint64_t)a.kb * (part + 1) / a.split);
    const bool issues = warp < 3 && elected();
    if (warp == 0) {
        uint32_t st = 0, turn = 0;
        for (uint32_t q = k0; q < k1; ++q) {
            if (turn > 0 && !f8_wait(&sm.empty[st], (turn - 1) & 1u)) { *failed = 1; break; }
            if (issues) {
                const bool with_scales = q == k0 || (q & 3u) == 0;
                mbar_arrive_expect_tx(&sm.full[st], kF8Tile + (with_scales ? kF8Scales : 0u));
                bulk_copy_g2s(ring + st * kF8Tile, a.a + q * a.a_block + mt * a.a_tile, kF8Tile, &sm.full[st]);
                if (with_scales) bulk_copy_g2s(scales + st * kF8Scales, a.a_scales + (q >> 2) * a.a_group + (uint64_t)mt * kF8Scales, kF8Scales, &sm.full[st]);
            }
            if (++st == kFewStages) { st = 0; ++turn; }
        }
        // copies in flight end before the block does, whoever else has given up
        for (uint32_t i = 0; i < kFewStages; ++i) {
            const uint32_t begun = turn + (i < st ? 1u : 0u);
            if (begun > 0) f8_wait(&sm.full[i], (begun - 1) & 1u);
        }
    } else if (warp < 3) {
        const uint32_t which = warp - 1u;
        uint32_t mine = 0, group = 0;  // blocks and groups of this warp
        bool ok = f8_wait(&sm.ready, 0);
        for (uint32_t q = k0; q < k1 && ok; ++q) {
            if ((((q >> 2) - (k0 >> 2)) & 1u) != which) continue;
            const uint32_t st = (q - k0) % kFewStages, turn = (q - k0) / kFewStages;
            if (!f8_wait(&sm.full[st], turn & 1u)) { ok = false; break; }
            tc_fence_after();
            const bool with_scales = q == k0 || (q & 3u) == 0;
            // the columns of four groups of this warp ago are free: only two groups are under way
            if (with_scales) group = (group + 1) % (kScaleTurns / 2);
            if (issues) {
                const uint32_t d = tmem + (which * kFewSums + mine / a.blocks) * kFewRows, sa = tmem + kTmemScales + (which * (kScaleTurns / 2) + group) * kScaleCols, sb = sa + 4;
                const bool fresh = mine % a.blocks == 0;
                if (with_scales) {
                    f8_scales_in(sa, smem_addr(scales + st * kF8Scales));
                    f8_scales_in(sb, smem_addr(x_scales + ((q >> 2) - (k0 >> 2)) * kF8Scales));
                }
                const uint32_t at = smem_addr(ring + st * kF8Tile), bt = smem_addr(xs + (q - k0) * (kFewRows * 128u));
                switch (q & 3u) {
                    case 0: multiply_block<kTransposed, 0>(d, at, bt, kFewRows, sa, sb, !fresh); break;
                    case 1: multiply_block<kTransposed, 1>(d, at, bt, kFewRows, sa, sb, !fresh); break;
                    case 2: multiply_block<kTransposed, 2>(d, at, bt, kFewRows, sa, sb, !fresh); break;
                    default: multiply_block<kTransposed, 3>(d, at, bt, kFewRows, sa, sb, !fresh); break;
                }
                tc_commit(&sm.empty[st]);
            }
            ++mine;
        }
        if (!ok) *failed = 1;
        if (issues) {
            tc_commit(&sm.sum_full[which]);
            tc_commit(&sm.done[which]);
        }
        f8_wait(&sm.done[which], 0);
    } else if (warp >= 4) {
        // rows of a block by warps, four columns a lane; rows that are not there stay as they are: they reach no sum that counts
        const uint32_t units = (k1 - k0) * a.rows;
        constexpr uint32_t kAtOnce = 4;
        for (uint32_t u0 = warp - 4u; u0 < units; u0 += 8 * kAtOnce) {
            float v[kAtOnce][4];
            uint32_t copied[kAtOnce], byte[kAtOnce];
#pragma unroll
            for (uint32_t i = 0; i < kAtOnce; ++i) {
                const uint32_t u = u0 + 8 * i, q = k0 + u / a.rows, r = u % a.rows;
                if (u >= units) continue;
                if (few.x) {
                    load4_any(few, r, q * 128ull + lane * 4u, v[i]);
                } else {
                    copied[i] = *reinterpret_cast<const uint32_t*>(a.b + q * a.b_block + r * 128u + lane * 4u);
                    byte[i] = a.b_scales[(q >> 2) * a.b_group + f8_scale_at(r, q)];
                }
            }
#pragma unroll
            for (uint32_t i = 0; i < kAtOnce; ++i) {
                const uint32_t u = u0 + 8 * i, q = k0 + u / a.rows, r = u % a.rows;
                if (u >= units) continue;
                const uint32_t piece = f8_piece(r, lane >> 2) + (lane & 3u) * 4u;
                unsigned char* to = xs + (q - k0) * (kFewRows * 128u) + r * 128u;
                if (few.x) {
                    uint32_t m = max(max(f8_magnitude(v[i][0]), f8_magnitude(v[i][1])), max(f8_magnitude(v[i][2]), f8_magnitude(v[i][3])));
                    m = __reduce_max_sync(0xffffffffu, m);
                    int e = f8_exponent(m);
                    if (m > kF8Rare) {
                        m = 0;
#pragma unroll
                        for (int k = 0; k < 4; ++k) m = max(m, f8_finite_magnitude(v[i][k]));
                        e = f8_exponent(__reduce_max_sync(0xffffffffu, m));
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[i][k] = f8_rare(v[i][k], e);
                    }
                    const float inverse = power_of_two(-e);
                    const uint32_t w = f8_from4(__fmul_rn(v[i][0], inverse), __fmul_rn(v[i][1], inverse), __fmul_rn(v[i][2], inverse), __fmul_rn(v[i][3], inverse));
                    byte[i] = (uint32_t)(e + 127);
                    *reinterpret_cast<uint32_t*>(to + piece) = w;
                    if (mt == 0) {
                        *reinterpret_cast<uint32_t*>(few.x8 + q * a.b_block + r * 128u + piece) = w;
                        if (lane == 0) few.x8_scales[(q >> 2) * a.b_group + f8_scale_at(r, q)] = (uint8_t)byte[i];
                    }
                } else {
                    *reinterpret_cast<uint32_t*>(to + lane * 4u) = copied[i];  // (swizzled already)
                }
                if (lane == 0) x_scales[((q >> 2) - (k0 >> 2)) * kF8Scales + f8_scale_at(r, q)] = (uint8_t)byte[i];
            }
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.ready);

        const uint32_t quad = warp & 3u, half = (warp - 4u) >> 2, row = quad * 32u + lane;
        constexpr int kHalf = kFewRows / 2;
        uint32_t blocks[2] = {0, 0};  // of the two warps
        for (uint32_t q = k0; q < k1; ++q) ++blocks[((q >> 2) - (k0 >> 2)) & 1u];
        float acc[kHalf];
        bool ok = lane != 0 || (f8_wait(&sm.sum_full[0], 0) && f8_wait(&sm.sum_full[1], 0));
        ok = __all_sync(0xffffffffu, ok);
        if (ok) {
            tc_fence_after();
            for (uint32_t w = 0; w < 2; ++w)
                for (uint32_t i = 0; i * a.blocks < blocks[w]; ++i)
                    take_sums(tmem + ((quad * 32u) << 16) + (w * kFewSums + i) * kFewRows + half * kHalf, w == 0 && i == 0, acc);
            tc_fence_before();
        }
        if (!ok) {
            *failed = 1;
        } else {  // into the ring, of which no copy and no product is left
            float* to = reinterpret_cast<float*>(ring) + half * kHalf * 128u + row;
#pragma unroll
            for (int i = 0; i < kHalf; ++i) to[i * 128] = acc[i];
        }
    }
    __syncwarp();
    __syncthreads();
    cluster_sync();
    // everybody's part is there; each block adds some of the entries in order
    if (!*failed && warp >= 4) join_parts_any(a, smem_addr(ring), part, mt * 128u, 0, a.rows, threadIdx.x - 128u);
    tc_fence_before();
    cluster_sync();  // nobody leaves while its part is read
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    if (threadIdx.x == 0 && *failed && a.res) atomicExch(&a.res->status, CO3_ERR_CUDA);
}

// Clusters of 1, 2, 4 and 8 blocks that run at once, a block on each of 148 multiprocessors (clusters stay within a group of 16 to 20 of them).
// What is chosen for a call follows from these numbers and its sizes, never from what a device or a part of one reports: the same call
// gives the same bits everywhere.
constexpr uint32_t kAtOnce[4] = {148, 74, 33, 15};

int multiprocessors(uint32_t* out) {
    static std::atomic<int> known[64];
    int dev = 0;
    CO3_CUDA(cudaGetDevice(&dev));
    int n = dev < 64 ? known[dev].load(std::memory_order_relaxed) : 0;
    if (n == 0) {
        CO3_CUDA(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev));
        if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
    }
    *out = (uint32_t)n;
    return CO3_OK;
}

// Blocks of a cluster (1: none) work on kernel<smem>.
template <auto* kKernel, uint32_t kSmem, typename Args>
int launch_clusters(const Args& a, uint32_t blocks, uint32_t cluster, cudaStream_t st) {
    static std::atomic<bool> ready[64];
    int dev = 0;
    CO3_CUDA(cudaGetDevice(&dev));
    if (dev >= 64 || !ready[dev].load(std::memory_order_relaxed)) {
        CO3_CUDA(cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem));
        if (dev < 64) ready[dev].store(true, std::memory_order_relaxed);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(kF8Threads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    CO3_CUDA(cudaLaunchKernelEx(&cfg, kKernel, a));
    return CO3_OK;
}
template <int kN, bool kTransposed>
int launch_linear(const LinearArgs& a, uint32_t sms, cudaStream_t st) {
    const uint32_t tiles = a.m_tiles * a.n_tiles;
    if (a.split > 1) return launch_clusters<f8_linear_kernel<kN, kTransposed, true>, Shape<kN>::kSmem>(a, tiles * a.split, a.split, st);
    return launch_clusters<f8_linear_kernel<kN, kTransposed, false>, Shape<kN>::kSmem>(a, std::min(tiles, sms), 1, st);
}
int launch_pairs(LinearArgs a, uint32_t rows_of_tile, bool transposed, uint32_t sms, cudaStream_t st) {
    a.pair_rows = rows_of_tile;
    a.n_tiles = (a.rows + rows_of_tile - 1) / rows_of_tile;
    const uint64_t tiles = (uint64_t)((a.m_tiles + 1) / 2) * a.n_tiles;
    const uint32_t blocks = 2 * (uint32_t)std::min<uint64_t>(tiles, std::max(1u, sms / 2));
    return transposed ? launch_clusters<f8_pair_kernel<true>, kPairSmem>(a, blocks, 2, st) : launch_clusters<f8_pair_kernel<false>, kPairSmem>(a, blocks, 2, st);
}
// Blocks that divide a tile's sum: as many as leave no cluster waiting (16 x 8192 x 4608: 51 us in two rounds of clusters, 21 in one), two
// blocks of columns each at least.
uint32_t split_of(uint64_t tiles, uint32_t kb) {
    uint32_t split = 1;
    for (uint32_t i = 1; i < 4 && tiles <= kAtOnce[i] && kb >= (2u << i); ++i) split = 1u << i;
    return split;
}
template <int kN>
int launch_tile(LinearArgs a, bool transposed, uint32_t sms, cudaStream_t st) {
    a.n_tiles = (a.rows + kN - 1) / kN;
    a.split = split_of((uint64_t)a.m_tiles * a.n_tiles, a.kb);
    return transposed ? launch_linear<kN, true>(a, sms, st) : launch_linear<kN, false>(a, sms, st);
}

}  // namespace
}  // namespace co3

using namespace co3;

extern "C" {

int co3_f8_linear(const void* x, int x_type, uint64_t x_row_stride, void* x8, size_t x8_bytes, const void* w8, size_t w8_bytes, uint32_t outs, uint32_t ins,
                  int transposed, const float* bias, void* y, int y_type, uint64_t y_row_stride, uint64_t rows, co3_result* res, void* stream) {
    F8Layout lx, lw;
    const uint32_t from = transposed ? outs : ins, to = transposed ? ins : outs;
    if ((x && (x_type < CO3_F32 || x_type > CO3_BF16)) || y_type < CO3_F32 || y_type > CO3_BF16 || !f8_layout(outs, ins, CO3_F8_SQUARE, &lw) ||
        !f8_layout(rows, from, CO3_F8_ROWS, &lx))
        return CO3_ERR_INVALID_ARG;
    if (rows == 0 || to == 0) return CO3_OK;
    if (from == 0) return CO3_ERR_INVALID_ARG;
    if ((x && !f8_valid_rows(x_type, x, x_row_stride, from)) || !f8_valid(x8) || !f8_valid(w8) || !f8_valid_rows(y_type, y, y_row_stride, to) ||
        !aligned(bias, 4) || !aligned(res, 8) || (uint64_t)((to + 127u) / 128u) * ((rows + 15u) / 16u) >= (1ull << 30))
        return CO3_ERR_INVALID_ARG;
    if (x8_bytes < lx.bytes || w8_bytes < lw.bytes) return CO3_ERR_CAPACITY;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint32_t sms = 0;
    int e = multiprocessors(&sms);
    if (e != CO3_OK) return e;
    const uint8_t *w = static_cast<const uint8_t*>(w8), *b = static_cast<const uint8_t*>(x8);
    LinearArgs a = {};
    a.a = w;
    a.a_block = transposed ? kF8Tile : lw.rows * 128u;
    a.a_tile = transposed ? lw.rows * 128u : kF8Tile;
    a.a_scales = w + (transposed ? lw.scales_t : lw.scales);
    a.a_group = transposed ? (uint64_t)lw.kb * kF8Scales : lw.rows / 128u * kF8Scales;
    a.b = b;
    a.b_block = lx.rows * 128u;
    a.b_scales = b + lx.scales;
    a.b_group = lx.rows / 128u * kF8Scales;
    a.kb = lx.kb;
    a.features = to;
    a.rows = (uint32_t)rows;
    a.m_tiles = (to + 127u) / 128u;
    a.y = y;
    a.y_stride = y_row_stride;
    a.y_type = y_type;
    a.blocks = y_type == CO3_F32 ? kBlocksF32 : kBlocks16;
    a.bias = bias;
    a.res = res;
    if (rows <= kFewRows) {
        // while a warp packs two rounds of rows at most; beyond, packing apart and the kernel below are faster (16 x 8192 x 2048: 30 and 20 us)
        a.split = split_of(a.m_tiles, a.kb);
        const uint64_t own = (a.kb + a.split - 1) / a.split;
        if (own <= kFewBlocks && own * rows <= 64) {
            FewArgs f = {a, x, x_type, x_row_stride, from, 0, static_cast<uint8_t*>(x8), static_cast<uint8_t*>(x8) + lx.scales};
            f.wide = x && aligned(x, 4 * type_size(x_type)) && x_row_stride % 4 == 0;
            return transposed ? launch_clusters<f8_few_kernel<true>, kFewSmem>(f, a.m_tiles * a.split, a.split, st)
                              : launch_clusters<f8_few_kernel<false>, kFewSmem>(f, a.m_tiles * a.split, a.split, st);
        }
    }
    if (x) {
        e = co3_f8_pack(x, x_type, rows, from, x_row_stride, CO3_F8_ROWS, x8, x8_bytes, stream);
        if (e != CO3_OK) return e;
    }
    // The estimated time of each kind of tile, in ns: rounds of tiles, a stage of each kind, what a tile costs besides, and the join of a
    // divided sum.  us measured, pairs with 256 and 128 rows / one block with 128 and 64: 512 x 4096 x 4096 21.6 and 19.3 / 25 and 37, 2048 x
    // 2048 x 2048 19.2 and 21.5 / 28 and 39, 1501 x 1023 x 1001 15.5 and 12.5 / 13.2 and 15.5, 3000 x 128 x 1000 12.2 and 12.5 / 11.6 and 10.4.
    auto single = [&](uint32_t n, uint32_t stage, uint32_t besides) {
        const uint64_t tiles = (uint64_t)a.m_tiles * ((rows + n - 1) / n);
        const uint32_t split = split_of(tiles, a.kb);
        return (split > 1 ? 1 : (tiles + kAtOnce[0] - 1) / kAtOnce[0]) * ((uint64_t)(a.kb + split - 1) / split * stage + besides + (split > 1 ? 1500 : 0));
    };
    auto by_pairs = [&](uint32_t n, uint32_t stage, uint32_t besides) {
        const uint64_t pairs = (uint64_t)((a.m_tiles + 1) / 2) * ((rows + n - 1) / n);
        return (pairs + kAtOnce[1] - 1) / kAtOnce[1] * ((uint64_t)a.kb * stage + besides);
    };
    const uint64_t ns[4] = {by_pairs(256, 370, 5500), by_pairs(128, 300, 3500), single(128, 470, 2500), single(64, 430, 1500)};
    const int best = (int)(std::min_element(ns, ns + 4) - ns);
    if (best < 2) return launch_pairs(a, best == 0 ? 256 : 128, transposed != 0, sms, st);
    return best == 2 ? launch_tile<128>(a, transposed != 0, sms, st) : launch_tile<64>(a, transposed != 0, sms, st);
}

}  // extern "C"
