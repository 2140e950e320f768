// Gradients of a linear layer's weights and biases from the inputs that were kept in 8 bits, for each client into its own vector:
//     dW_u = sum over the client's rows r of dy[r]^T x[r],    db_u = sum of dy[r].
//
// The sum runs along the rows, along which the 8-bit blocks' scales differ, so the tensor cores cannot apply them: values are
// brought to bf16, which is exact (four significant bits times a power of two).  dy is cut into parts of eight significant
// bits, one for bf16, two for fp16, three for fp32, so that nothing of it is lost: the products are exact and the sums fp32.
//
// A first kernel writes both operands, as the tensor cores read them, to the workspace (doing this inside the product costs every
// tile the conversion of all its rows: 16384 x 4096 x 4096 bf16 2.02 ms), and sums dy; bf16 gradients with rows on 16-byte boundaries
// stay where they are, and the products' copies swizzle them (459 us with them rearranged, 442 so).  The products are
// tiles of 256 inputs (tensor memory's lanes, so that a warp writes neighbouring entries of dW) by 256 or 128 outputs, by pairs of
// blocks; a stage is 64 rows, a row of the batch per row of shared memory.  After every 256 rows the sums are taken out and
// added up in registers (the tensor core cuts what it adds towards zero).  Few tiles: the rows are divided, and a last kernel adds
// the parts in order.
#include <cuda.h>
#include <cudaTypedefs.h>
#include <stddef.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "co3_f8.cuh"
#include "co3_launch.cuh"
#include "co3_orth.cuh"

namespace co3 {
namespace {

constexpr uint32_t kChunk = 64;              // rows of a stage
constexpr uint32_t kSumChunks = 4;           // chunks that tensor memory adds up
constexpr uint32_t kOuts = 256;              // outputs of a tile at most; two groups of 128
constexpr uint32_t kAtom = kChunk * 128;     // bytes of 64 columns of a chunk
constexpr uint32_t kPlane16 = 2 * kAtom;     // bytes of 128 columns of a chunk
constexpr uint32_t kRing = 196608;           // bytes of the ring of stages
constexpr uint32_t kMaxStagesW = 6;
constexpr uint32_t kSmemW = 1024 + kRing + 256;
constexpr uint32_t kPairsAssumed = 74, kSmsAssumed = 148;  // how rows are divided does not depend on the device

// Parts of eight significant bits of a value of this type.
__host__ __device__ constexpr uint32_t parts_of(int type) { return type == CO3_F32 ? 3u : type == CO3_F16 ? 2u : 1u; }

// Where the operands lie in the workspace: for each client and 128 columns, chunk after chunk, 64 rows of two atoms of 64
// columns, swizzled; of dy the parts one after the other within a chunk.
struct WeightArgs {
    const void* dy;
    uint64_t dy_stride;
    const uint8_t *x, *x_scales;
    uint64_t x_rows;                         // rows of the packed inputs, padded
    uint64_t rows;                           // of a client
    uint32_t outs, ins, clients;
    uint32_t k_tiles, groups, chunks;        // blocks of 128 inputs, of 128 outputs, chunks of a client
    uint32_t tile_outs, n_tiles;             // outputs of a tile (128 or 256), tiles of outputs
    uint32_t parts, db_parts;                // row parts of the products, and of the sums of dy
    unsigned char *ws_x, *ws_dy;
    float *dw_parts, *db_parts_at;           // parts x clients x outs x ins; db_parts x clients x outs
    float *dw, *db;
    uint64_t client_stride;
    int accumulate;
    int direct;                              // dy is read where it is
    co3_result* res;
};

// ------------------------------------------------------------------------------------------------
// Operands
// ------------------------------------------------------------------------------------------------
// The parts of a value, each exact in bf16, as the upper halves of fp32 patterns.
template <int kParts>
__device__ __forceinline__ void cut(float v, uint32_t (&part)[kParts]) {
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
        const uint32_t top = __float_as_uint(v) & 0xffff0000u;
        part[k] = top;
        // an infinity is its own first part
        if (k + 1 < kParts) v = f8_magnitude(v) == 0x7f800000u ? 0.0f : __fsub_rn(v, __uint_as_float(top));
    }
}

// A chunk of a block of x: two pieces of 16 columns a thread.
__device__ __forceinline__ void bring_x(const WeightArgs& a, uint32_t u, uint32_t kt, uint32_t c) {
    const uint64_t row0 = u * a.rows + (uint64_t)c * kChunk;
    const uint32_t rows = (uint32_t)min((uint64_t)kChunk, a.rows - (uint64_t)c * kChunk);
    unsigned char* chunk = a.ws_x + (((uint64_t)u * a.k_tiles + kt) * a.chunks + c) * kPlane16;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t i = (threadIdx.x >> 3) + 32u * j;
        uint4 x = make_uint4(0, 0, 0, 0);
        float s = 1.0f;
        const uint64_t row = row0 + i;
        if (i < rows) {
            x = __ldcs(reinterpret_cast<const uint4*>(a.x + f8_row(a.x_rows, kt, row) + ((threadIdx.x & 7u) << 4)));
            s = __uint_as_float((uint32_t)a.x_scales[((kt >> 2) * (a.x_rows >> 7) + (row >> 7)) * kF8Scales + f8_scale_at((uint32_t)row & 127u, kt)] << 23);
        }
        const uint32_t piece = (threadIdx.x & 7u) ^ ((uint32_t)row & 7u);  // columns 16 piece ..
        const uint32_t q[4] = {x.x, x.y, x.z, x.w};
        uint32_t w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float2 v = f8_to2(q[k >> 1] >> (16 * (k & 1)));
            const __nv_bfloat162 b = __floats2bfloat162_rn(__fmul_rn(v.x, s), __fmul_rn(v.y, s));
            w[k] = *reinterpret_cast<const uint32_t*>(&b);
        }
        unsigned char* to = chunk + (piece >> 2) * kAtom + i * 128u;
        *reinterpret_cast<uint4*>(to + f8_piece(i, (piece & 3u) * 2u)) = make_uint4(w[0], w[1], w[2], w[3]);
        *reinterpret_cast<uint4*>(to + f8_piece(i, (piece & 3u) * 2u + 1u)) = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

// Eight columns of a row from column `col` on, zeros beyond the last.
template <typename T, bool kWide>
__device__ __forceinline__ void load8(const T* row, uint32_t col, uint32_t cols, float (&v)[8]) {
    if constexpr (kWide) {
        constexpr int kVec = 16 / sizeof(T);
#pragma unroll
        for (int l = 0; l < 8 / kVec; ++l) {
            uint4 raw = make_uint4(0, 0, 0, 0);
            if (col + l * kVec < cols) raw = __ldcs(reinterpret_cast<const uint4*>(row + col + l * kVec));
            const T* e = reinterpret_cast<const T*>(&raw);
#pragma unroll
            for (int k = 0; k < kVec; ++k) v[l * kVec + k] = to_float(e[k]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = col + k < cols ? to_float(row[col + k]) : 0.0f;
    }
}

// Chunks of 128 columns of dy: 16 neighbouring threads have a row, eight columns each, a thread four rows of a chunk.
template <typename T, bool kWide>
__device__ __forceinline__ void bring_dy(const WeightArgs& a, uint32_t u, uint32_t g, uint32_t part) {
    constexpr int kParts = (int)parts_of(sizeof(T) == 4 ? CO3_F32 : std::is_same<T, __half>::value ? CO3_F16 : CO3_BF16);
    __shared__ float sums[8][128];
    const uint32_t c0 = (uint32_t)((uint64_t)a.chunks * part / a.db_parts), c1 = (uint32_t)((uint64_t)a.chunks * (part + 1) / a.db_parts);
    const uint32_t p = threadIdx.x & 15u, r0 = threadIdx.x >> 4, col = g * 128u + p * 8u;
    float db[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) db[k] = 0.0f;
    for (uint32_t c = c0; c < c1; ++c) {
        const uint32_t rows = (uint32_t)min((uint64_t)kChunk, a.rows - (uint64_t)c * kChunk);
        const T* from = static_cast<const T*>(a.dy) + (u * a.rows + (uint64_t)c * kChunk) * a.dy_stride;
        float v[4][8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t i = r0 + 16u * j;
            if (i < rows) {
                load8<T, kWide>(from + i * a.dy_stride, col, a.outs, v[j]);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[j][k] = 0.0f;
            }
        }
        if (a.dw && !a.direct) {
            unsigned char* chunk = a.ws_dy + (((uint64_t)u * a.groups + g) * a.chunks + c) * (kParts * kPlane16) + (p >> 3) * kAtom;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t i = r0 + 16u * j;
                uint32_t w[kParts][4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint32_t lo[kParts], hi[kParts];
                    cut(v[j][2 * k], lo);
                    cut(v[j][2 * k + 1], hi);
#pragma unroll
                    for (int m = 0; m < kParts; ++m) w[m][k] = __byte_perm(lo[m], hi[m], 0x7632);
                }
#pragma unroll
                for (int m = 0; m < kParts; ++m)
                    *reinterpret_cast<uint4*>(chunk + m * kPlane16 + i * 128u + f8_piece(i, p & 7u)) = make_uint4(w[m][0], w[m][1], w[m][2], w[m][3]);
            }
        }
        if (a.db) {
#pragma unroll
            for (int k = 0; k < 8; ++k) db[k] = __fadd_rn(db[k], __fadd_rn(__fadd_rn(v[0][k], v[1][k]), __fadd_rn(v[2][k], v[3][k])));
        }
    }
    if (!a.db) return;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
#pragma unroll
    for (int k = 0; k < 8; ++k) db[k] = __fadd_rn(db[k], __shfl_xor_sync(0xffffffffu, db[k], 16));
    if (lane < 16)
#pragma unroll
        for (int k = 0; k < 8; ++k) sums[warp][p * 8u + k] = db[k];
    __syncthreads();
    const uint32_t o = g * 128u + threadIdx.x;
    if (threadIdx.x >= 128 || o >= a.outs) return;
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s = __fadd_rn(s, sums[w][threadIdx.x]);
    if (a.db_parts > 1) {
        a.db_parts_at[((uint64_t)part * a.clients + u) * a.outs + o] = s;
    } else {
        float* to = a.db + u * a.client_stride + o;
        *to = a.accumulate ? __fadd_rn(*to, s) : s;
    }
}

// Blocks for dy first (one for each client, 128 columns and part of the chunks), then for x (one for each client, block of columns
// and chunk).
template <typename T, bool kWide>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 5 : 3) f8_operands_kernel(const __grid_constant__ WeightArgs a) {
    wait_for_previous_kernel();
    const uint32_t of_dy = a.direct && !a.db ? 0u : a.clients * a.groups * a.db_parts;
    uint32_t b = blockIdx.x;
    if (b < of_dy) {
        const uint32_t part = b / (a.clients * a.groups);
        b -= part * a.clients * a.groups;
        bring_dy<T, kWide>(a, b / a.groups, b % a.groups, part);
    } else {
        b -= of_dy;
        const uint32_t kt = b % a.k_tiles, uc = b / a.k_tiles;
        bring_x(a, uc / a.chunks, kt, uc % a.chunks);
    }
}

// ------------------------------------------------------------------------------------------------
// Products
// ------------------------------------------------------------------------------------------------
struct WeightSmem {
    uint64_t full[kMaxStagesW], empty[kMaxStagesW], sum_full[2], sum_empty[2], done;
    uint32_t tmem, failed;
};
static_assert(sizeof(WeightSmem) <= 256, "barriers");

// D fp32, A and B bf16, both with the sum along their rows; 256 rows of A by the pair
__host__ __device__ constexpr uint32_t weight_instr(uint32_t cols) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((cols / 8u) << 17) | (16u << 24);
}
__device__ __forceinline__ void pair_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t instr, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(instr), "r"((uint32_t)accumulate)
        : "memory");
}

// A pair's tiles one after the other, and the chunks of rows that each sums.  Tiles are counted by blocks of inputs, outputs, parts of the
// rows, clients; going on by so many tiles is adding these four digits with their carries (dividing anew for each tile took about 1000
// cycles, a fifth of a small tile).
struct Walk {
    uint32_t t, tiles, step;
    uint32_t kp, n, part, u;          // the tile
    uint32_t d_kp, d_n, d_part, d_u;  // the step
    __device__ __forceinline__ explicit Walk(const WeightArgs& a) {
        const uint32_t pairs = (a.k_tiles + 1) / 2;
        tiles = pairs * a.n_tiles * a.parts * a.clients;
        t = blockIdx.x >> 1;
        step = gridDim.x >> 1;
        auto digits = [&](uint32_t v, uint32_t& k, uint32_t& nn, uint32_t& pp, uint32_t& uu) {
            k = v % pairs;
            v /= pairs;
            nn = v % a.n_tiles;
            v /= a.n_tiles;
            pp = v % a.parts;
            uu = v / a.parts;
        };
        digits(t, kp, n, part, u);
        digits(step, d_kp, d_n, d_part, d_u);
    }
    __device__ __forceinline__ bool more() const { return t < tiles; }
    __device__ __forceinline__ void next(const WeightArgs& a) {
        t += step;
        const uint32_t pairs = (a.k_tiles + 1) / 2;
        kp += d_kp;
        n += d_n;
        part += d_part;
        u += d_u;
        if (kp >= pairs) { kp -= pairs; ++n; }
        if (n >= a.n_tiles) { n -= a.n_tiles; ++part; }
        if (part >= a.parts) { part -= a.parts; ++u; }
    }
    __device__ __forceinline__ uint32_t n0(const WeightArgs& a) const { return n * a.tile_outs; }
    __device__ __forceinline__ uint32_t c0(const WeightArgs& a) const { return a.parts == 1 ? 0u : (uint32_t)((uint64_t)a.chunks * part / a.parts); }
    __device__ __forceinline__ uint32_t c1(const WeightArgs& a) const { return a.parts == 1 ? a.chunks : (uint32_t)((uint64_t)a.chunks * (part + 1) / a.parts); }
};
// Outputs of a tile that are multiplied: 128, half of them in each block, or 256.
__device__ __forceinline__ uint32_t tile_cols(const WeightArgs& a, uint32_t n0) { return a.outs - n0 > 128u ? a.tile_outs : 128u; }

// 64 columns of 64 rows of a client's dy, swizzled; zeros beyond the last column and row.
__device__ __forceinline__ void copy_box(unsigned char* to, const CUtensorMap& map, uint32_t col, uint32_t row, uint32_t client, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_addr(to)), "l"(&map),
                 "r"(col), "r"(row), "r"(client), "r"(smem_addr(bar))
                 : "memory");
}

template <int kParts, bool kDirect>
__global__ void __launch_bounds__(kF8Threads, 1) f8_weight_kernel(const __grid_constant__ WeightArgs a, const __grid_constant__ CUtensorMap dy_map) {
    extern __shared__ unsigned char smem_raw[];
    constexpr uint32_t kStageBytes = kPlane16 * (1 + kParts), kStages = kRing / kStageBytes;
    static_assert(kStages <= kMaxStagesW, "stages");
    unsigned char* ring = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    WeightSmem& sm = *reinterpret_cast<WeightSmem*>(ring + kRing);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, rank = cluster_rank();
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < kStages; ++i) { mbar_init(&sm.full[i], rank == 0 ? 2 : 1); mbar_init(&sm.empty[i], 1); }
        for (uint32_t i = 0; i < 2; ++i) { mbar_init(&sm.sum_full[i], 1); mbar_init(&sm.sum_empty[i], 16); }
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

    if (warp < 4) {
        few_registers();
        const bool issues = elected();
        if (warp == 0) {
            uint32_t st = 0, turn = 0;
            for (Walk p(a); p.more() && !*failed; p.next(a)) {
                const uint32_t n0 = p.n0(a), c1 = p.c1(a);
                const uint32_t kt = min(2 * p.kp + rank, a.k_tiles - 1);  // (an odd last tile: the second block's sums go nowhere)
                const bool both = tile_cols(a, n0) == 256u;
                const uint32_t g = (n0 >> 7) + (both ? rank : 0u);
                const unsigned char* x = a.ws_x + ((uint64_t)p.u * a.k_tiles + kt) * a.chunks * kPlane16;
                const unsigned char* dy = a.ws_dy + ((uint64_t)p.u * a.groups + g) * a.chunks * (kParts * kPlane16);
                for (uint32_t c = p.c0(a); c < c1; ++c) {
                    if (turn > 0 && !f8_wait(&sm.empty[st], (turn - 1) & 1u)) { *failed = 1; break; }
                    if (issues) {
                        unsigned char* to = ring + st * kStageBytes;
                        mbar_arrive_expect_tx(&sm.full[st], kPlane16 + kParts * (both ? kPlane16 : kAtom));
                        bulk_copy_g2s(to, x + (uint64_t)c * kPlane16, kPlane16, &sm.full[st]);
                        if constexpr (kDirect) {
                            const uint32_t col = n0 + (both ? 128u : 64u) * rank;
                            copy_box(to + kPlane16, dy_map, col, c * kChunk, p.u, &sm.full[st]);
                            if (both) copy_box(to + kPlane16 + kAtom, dy_map, col + 64u, c * kChunk, p.u, &sm.full[st]);
                        } else {
                            const unsigned char* from = dy + (uint64_t)c * (kParts * kPlane16);
                            if (both) {
                                bulk_copy_g2s(to + kPlane16, from, kParts * kPlane16, &sm.full[st]);
                            } else {
                                for (uint32_t m = 0; m < kParts; ++m) bulk_copy_g2s(to + kPlane16 * (1 + m), from + m * kPlane16 + rank * kAtom, kAtom, &sm.full[st]);
                            }
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
        } else if (warp == 1 && rank == 1) {
            // tells the first block what has arrived here: its barrier waits for both
            uint32_t st = 0, turn = 0;
            bool ok = true;
            for (Walk p(a); p.more() && ok; p.next(a)) {
                const uint32_t c1 = p.c1(a);
                for (uint32_t c = p.c0(a); c < c1; ++c) {
                    if (!f8_wait(&sm.full[st], turn & 1u)) { ok = false; break; }
                    if (issues) mbar_arrive_at(&sm.full[st], 0);
                    if (++st == kStages) { st = 0; ++turn; }
                }
            }
            if (!ok) *failed = 1;
        } else if (warp == 1) {
            uint32_t st = 0, turn = 0, sum = 0, sum_turn = 0;
            bool ok = true;
            for (Walk p(a); p.more() && ok; p.next(a)) {
                const uint32_t instr = weight_instr(0) | ((tile_cols(a, p.n0(a)) / 8u) << 17), c0 = p.c0(a), c1 = p.c1(a);
                for (uint32_t c = c0; c < c1; ++c) {
                    const uint32_t in_sum = (c - c0) % kSumChunks;
                    if (in_sum == 0 && sum_turn > 0 && !f8_wait(&sm.sum_empty[sum], (sum_turn - 1) & 1u)) { ok = false; break; }
                    if (!f8_wait(&sm.full[st], turn & 1u)) { ok = false; break; }
                    tc_fence_after();
                    const bool last = in_sum == kSumChunks - 1 || c + 1 == c1;
                    if (issues) {
                        const uint32_t d = tmem + sum * kOuts, at = smem_addr(ring + st * kStageBytes);
                        const uint64_t dx = smem_desc(at, true, kAtom);
#pragma unroll
                        for (int m = kParts - 1; m >= 0; --m) {
                            const uint64_t dd = smem_desc(at + kPlane16 * (1 + m), true, kAtom);
#pragma unroll
                            for (uint32_t e = 0; e < kChunk / 16u; ++e)
                                pair_mma(d, dx + e * desc_step(true), dd + e * desc_step(true), instr, in_sum > 0 || m < kParts - 1 || e > 0);
                        }
                        tc_commit_pair(&sm.empty[st]);
                        if (last) tc_commit_pair(&sm.sum_full[sum]);
                    }
                    if (last && ++sum == 2) { sum = 0; ++sum_turn; }
                    if (++st == kStages) { st = 0; ++turn; }
                }
            }
            if (!ok) *failed = 1;
            if (issues) tc_commit_first(&sm.done);
            f8_wait(&sm.done, 0);
        }
    } else {
        many_registers();
        const uint32_t quad = warp & 3u, half = (warp - 4u) >> 2, row = quad * 32u + lane;
        uint32_t sum = 0, sum_turn = 0;
        bool ok = true;
        const uint32_t cols = a.tile_outs / 2;  // of a warp
        for (Walk p(a); p.more() && ok; p.next(a)) {
            const uint32_t o0 = p.n0(a) + half * cols, c0 = p.c0(a), c1 = p.c1(a);
            float acc[kOuts / 2];
            for (uint32_t c = c0; c < c1; c += kSumChunks) {
                ok = lane != 0 || f8_wait(&sm.sum_full[sum], sum_turn & 1u);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                const uint32_t from = tmem + ((quad * 32u) << 16) + sum * kOuts + half * cols;
                if (o0 < a.outs && c == c0) {
                    if (cols == kOuts / 2) tc_load(from, acc);
                    else tc_load(from, *reinterpret_cast<float(*)[kOuts / 4]>(acc));
                } else if (o0 < a.outs) {
#pragma unroll
                    for (int h = 0; h < (int)kOuts / 2; h += 64) {
                        if ((uint32_t)h >= cols) break;
                        float w[64];
                        tc_load(from + h, w);
#pragma unroll
                        for (int i = 0; i < 64; ++i) acc[h + i] = __fadd_rn(acc[h + i], w[i]);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_at(&sm.sum_empty[sum], 0);
                if (++sum == 2) { sum = 0; ++sum_turn; }
            }
            if (!ok) break;
            const uint32_t k = (2 * p.kp + rank) * 128u + row;
            if (k < a.ins && o0 < a.outs) {
                const uint32_t count = min(cols, a.outs - o0);
                const bool add = a.parts == 1 && a.accumulate;
                float* to = (a.parts > 1 ? a.dw_parts + ((uint64_t)p.part * a.clients + p.u) * a.outs * a.ins : a.dw + p.u * a.client_stride) + (uint64_t)o0 * a.ins + k;
#pragma unroll
                for (int i0 = 0; i0 < (int)kOuts / 2; i0 += 16) {
                    if ((uint32_t)i0 >= count) break;
                    if (add)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if ((uint32_t)(i0 + i) < count) acc[i0 + i] = __fadd_rn(to[(uint64_t)i * a.ins], acc[i0 + i]);
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if ((uint32_t)(i0 + i) < count) to[(uint64_t)i * a.ins] = acc[i0 + i];
                    to += 16ull * a.ins;
                }
            }
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
// to[u][i] (+)= sum over the parts of from[part][u][i], in order; with no parts: zeros.  Two such sums in one launch: db, of few
// columns and up to hundreds of parts, first (eight threads a column), then dw.
// ------------------------------------------------------------------------------------------------
struct Join {
    const float* from;
    float* to;
    uint64_t count;
    uint32_t parts;
};
struct JoinArgs {
    Join db, dw;
    uint64_t client_stride;
    uint32_t clients, db_blocks;
    int accumulate;
};
constexpr uint32_t kJoinEach = 4;  // entries of a thread
__global__ void __launch_bounds__(256) f8_join_kernel(const __grid_constant__ JoinArgs a) {
    __shared__ float sums[8][32];
    wait_for_previous_kernel();
    if (blockIdx.x < a.db_blocks) {
        const uint64_t i = blockIdx.x * 32ull + (threadIdx.x & 31u), all = a.db.count * a.clients;
        const float* from = a.db.from + blockIdx.y * a.db.count + i;
        float s = 0.0f;
        if (i < a.db.count)
#pragma unroll 4
            for (uint32_t p = threadIdx.x >> 5; p < a.db.parts; p += 8) s = __fadd_rn(s, __ldcs(from + p * all));
        sums[threadIdx.x >> 5][threadIdx.x & 31u] = s;
        __syncthreads();
        if (threadIdx.x >= 32 || i >= a.db.count) return;
        for (uint32_t w = 1; w < 8; ++w) s = __fadd_rn(s, sums[w][threadIdx.x]);
        float* to = a.db.to + blockIdx.y * a.client_stride + i;
        *to = a.accumulate ? __fadd_rn(*to, s) : s;
        return;
    }
    const uint64_t all = a.dw.count * a.clients, i0 = (blockIdx.x - a.db_blocks) * (256ull * kJoinEach) + threadIdx.x;
    float* to = a.dw.to + blockIdx.y * a.client_stride;
    const float* from = a.dw.from + blockIdx.y * a.dw.count;
    float s[kJoinEach];
#pragma unroll
    for (uint32_t e = 0; e < kJoinEach; ++e) s[e] = 0.0f;
#pragma unroll 4
    for (uint32_t p = 0; p < a.dw.parts; ++p)
#pragma unroll
        for (uint32_t e = 0; e < kJoinEach; ++e)
            if (i0 + e * 256u < a.dw.count) s[e] = __fadd_rn(s[e], __ldcs(from + p * all + i0 + e * 256u));
#pragma unroll
    for (uint32_t e = 0; e < kJoinEach; ++e)
        if (i0 + e * 256u < a.dw.count) to[i0 + e * 256u] = a.accumulate ? __fadd_rn(to[i0 + e * 256u], s[e]) : s[e];
}
int launch_join(const Join& dw, const Join& db, uint32_t clients, uint64_t client_stride, int accumulate, cudaStream_t st) {
    JoinArgs a = {db, dw, client_stride, clients, 0, accumulate};
    if (!a.db.to) a.db.count = 0;
    if (!a.dw.to) a.dw.count = 0;
    a.db_blocks = (uint32_t)((a.db.count + 31u) / 32u);
    const uint32_t blocks = a.db_blocks + (uint32_t)((a.dw.count + 256u * kJoinEach - 1) / (256u * kJoinEach));
    if (blocks == 0) return CO3_OK;
    // (a grid's second dimension ends at 65535)
    for (uint32_t u0 = 0; u0 < clients; u0 += 65535u) {
        const uint32_t n = std::min(clients - u0, 65535u);
        CO3_CUDA(launch_behind(f8_join_kernel, dim3(blocks, n), dim3(256), 0, st, a));
        for (Join* j : {&a.db, &a.dw}) {
            if (j->to) j->to += n * client_stride;
            if (j->from) j->from += n * j->count;
        }
    }
    return CO3_OK;
}

// ------------------------------------------------------------------------------------------------
// Small gradients in one launch, without the tensor cores: 32 outputs by 128 inputs a block, 4 x 4 entries a thread, 32 rows
// at a time in shared memory as fp32, the next ones on their way.
// ------------------------------------------------------------------------------------------------
constexpr uint32_t kFewOuts = 32, kFewRowsW = 32;
struct alignas(16) SmallSmem {  // rows are written and read 16 bytes at a time
    float x[kFewRowsW][132];
    float dy[kFewRowsW][kFewOuts];
};
static_assert(alignof(SmallSmem) % 16 == 0 && sizeof(SmallSmem::x[0]) % 16 == 0 && offsetof(SmallSmem, dy) % 16 == 0 && sizeof(SmallSmem::dy[0]) % 16 == 0, "16-byte accesses");
template <typename T>
__global__ void __launch_bounds__(256) f8_weight_small_kernel(const __grid_constant__ WeightArgs a) {
    __shared__ SmallSmem sm;
    auto &xs = sm.x;
    auto &ds = sm.dy;
    wait_for_previous_kernel();
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const uint32_t o_tiles = (a.outs + kFewOuts - 1) / kFewOuts, i_tiles = a.dw ? a.k_tiles : 1u;
    const uint32_t kt = blockIdx.x % i_tiles, ot = blockIdx.x / i_tiles % o_tiles, u = blockIdx.x / i_tiles / o_tiles;
    const uint64_t row0 = u * a.rows;
    const uint32_t xr = threadIdx.x >> 3, xp = threadIdx.x & 7u;   // this thread's row and piece of x, its column of dy
    const uint32_t o = ot * kFewOuts + lane;
    uint4 x;
    float s, d[4];
    auto fetch = [&](uint64_t r0) {
        x = make_uint4(0, 0, 0, 0);
        s = 1.0f;
        const uint64_t row = row0 + r0 + xr;
        if (a.dw && r0 + xr < a.rows) {
            x = *reinterpret_cast<const uint4*>(a.x + f8_row(a.x_rows, kt, row) + f8_piece((uint32_t)row & 7u, xp));
            s = __uint_as_float((uint32_t)a.x_scales[((kt >> 2) * (a.x_rows >> 7) + (row >> 7)) * kF8Scales + f8_scale_at((uint32_t)row & 127u, kt)] << 23);
        }
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            const uint64_t r = r0 + warp + 8 * j;
            d[j] = r < a.rows && o < a.outs ? to_float(static_cast<const T*>(a.dy)[(row0 + r) * a.dy_stride + o]) : 0.0f;
        }
    };
    float acc[4][4], db = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[j][k] = 0.0f;
    fetch(0);
    for (uint64_t r0 = 0; r0 < a.rows; r0 += kFewRowsW) {
        const uint32_t q[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 lo = f8_to2(q[k]), hi = f8_to2(q[k] >> 16);
            *reinterpret_cast<float4*>(&xs[xr][xp * 16u + 4u * k]) = make_float4(__fmul_rn(lo.x, s), __fmul_rn(lo.y, s), __fmul_rn(hi.x, s), __fmul_rn(hi.y, s));
        }
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) ds[warp + 8 * j][lane] = d[j];
        __syncthreads();
        if (r0 + kFewRowsW < a.rows) fetch(r0 + kFewRowsW);
        const uint32_t n = (uint32_t)min((uint64_t)kFewRowsW, a.rows - r0);
        for (uint32_t r = 0; r < n; ++r) {
            const float4 g = *reinterpret_cast<const float4*>(&ds[r][warp * 4u]);
            const float gs[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float v = xs[r][lane + 32u * k];
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j][k] = __fmaf_rn(gs[j], v, acc[j][k]);
            }
        }
        if (kt == 0 && warp == 0)
            for (uint32_t r = 0; r < n; ++r) db = __fadd_rn(db, ds[r][lane]);
        __syncthreads();
    }
    if (a.dw)
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            const uint32_t out = ot * kFewOuts + warp * 4u + j;
            float* to = a.dw + u * a.client_stride + (uint64_t)out * a.ins + kt * 128u + lane;
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k)
                if (out < a.outs && kt * 128u + lane + 32u * k < a.ins) to[32u * k] = a.accumulate ? __fadd_rn(to[32u * k], acc[j][k]) : acc[j][k];
        }
    if (a.db && kt == 0 && warp == 0 && o < a.outs) {
        float* to = a.db + u * a.client_stride + o;
        *to = a.accumulate ? __fadd_rn(*to, db) : db;
    }
}
// Whether that is the faster way: one launch against two or three, as long as the rows are few turns, the products below 2^26 (about
// 8 us without the tensor cores) and the entries below 2^22 (us, a call with its arguments: 1 x 64 x 1024 x 1024 15.5 and 18.5, 30 x 200 x
// 100 x 100 15.9 and 20.9; 1 x 1 x 8192 x 8192 66 and 55).
bool small_gradient(uint64_t rows, uint32_t outs, uint32_t ins, uint32_t clients) {
    const uint64_t entries = (uint64_t)outs * ins * clients;
    return rows <= 256 && entries <= (1ull << 22) && rows * entries <= (1ull << 26);
}
template <typename T>
int launch_small(const WeightArgs& a, cudaStream_t st) {
    const uint32_t blocks = (a.dw ? a.k_tiles : 1u) * ((a.outs + kFewOuts - 1) / kFewOuts) * a.clients;
    CO3_CUDA(launch_behind(f8_weight_small_kernel<T>, dim3(blocks), dim3(256), 0, st, a));
    return CO3_OK;
}

// ------------------------------------------------------------------------------------------------
// Sizes: they follow from the call's alone, so that the same call gives the same bits everywhere.
// ------------------------------------------------------------------------------------------------
struct WeightPlan {
    uint32_t k_tiles, groups, tile_outs, n_tiles, chunks, parts, db_parts;
    uint64_t x, dy, dw, db, bytes;  // offsets in the workspace
};
bool weight_plan(uint64_t rows, uint32_t outs, uint32_t ins, uint32_t clients, uint32_t pieces, WeightPlan* w) {
    if (clients == 0 || rows >= (1ull << 31) || outs >= (1u << 31) || ins >= (1u << 31) || rows * clients >= (1ull << 31) ||
        (uint64_t)outs * ins >= (1ull << 40) / clients)
        return false;
    w->k_tiles = (ins + 127u) / 128u;
    w->groups = (outs + 127u) / 128u;
    w->chunks = (uint32_t)((rows + kChunk - 1) / kChunk);
    const uint64_t all = (uint64_t)clients * w->chunks;
    if (all * std::max(w->k_tiles, w->groups) >= (1ull << 40) / kPlane16 / 4) return false;
    // Outputs of a tile, and how many parts the rows are divided into: the least estimated time, in ns.  Rounds of tiles; a chunk's
    // products and handing over; what a tile costs besides, its sums written at 30 bytes a cycle above all; for the join a launch of 2500
    // and 5 bytes a ns.  (us: 2 x 1501 x 1023 x 1001 fp16 divided 36.4, whole 31.8, of 128 outputs 25.7.)
    const uint64_t pairs_k = (w->k_tiles + 1) / 2, size = (uint64_t)clients * outs * ins * 4, most = std::min<uint64_t>(kPairsAssumed, w->chunks / 2);
    uint64_t best = ~0ull;
    for (uint32_t outs_of_tile : {256u, 128u})
        for (uint32_t p = 1; p <= std::max<uint64_t>(1, most); ++p) {
            const uint64_t n_tiles = (outs + outs_of_tile - 1) / outs_of_tile, rounds = (pairs_k * n_tiles * clients * p + kPairsAssumed - 1) / kPairsAssumed;
            const uint64_t chunk = outs_of_tile == 256 ? 280 * pieces + 70 : 140 * pieces + 110;
            const uint64_t ns = rounds * ((w->chunks + p - 1) / p * chunk + 600 + outs_of_tile * 10) + (p > 1 ? 2500 + (2ull * p + 1) * size / 5000 : 0);
            if (ns < best) {
                best = ns;
                w->tile_outs = outs_of_tile;
                w->n_tiles = (uint32_t)n_tiles;
                w->parts = p;
            }
        }
    const uint64_t tiles = pairs_k * w->n_tiles * clients;
    // the sums of dy: as many blocks as the device takes at once, about
    const uint64_t columns = std::max<uint64_t>(1, (uint64_t)w->groups * clients);
    w->db_parts = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>((4 * kSmsAssumed + columns - 1) / columns, w->chunks));
    if (tiles * w->parts >= (1ull << 30) || all * w->k_tiles + columns * w->db_parts >= (1ull << 31)) return false;
    w->x = 0;
    w->dy = all * w->k_tiles * kPlane16;
    w->dw = w->dy + all * w->groups * kPlane16 * pieces;
    w->db = w->dw + (w->parts > 1 ? (uint64_t)w->parts * clients * outs * ins * 4 : 0);
    w->bytes = w->db + (w->db_parts > 1 ? (uint64_t)w->db_parts * clients * outs * 4 : 0);
    w->bytes = std::max<uint64_t>(256, (w->bytes + 255u) & ~(uint64_t)255u);
    return true;
}

// The driver's call that describes a tensor to the copies, or null.
PFN_cuTensorMapEncodeTiled_v12000 tensor_map_call() {
    static std::atomic<void*> known{nullptr};
    void* f = known.load(std::memory_order_relaxed);
    if (!f) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            return nullptr;
        }
        known.store(f, std::memory_order_relaxed);
    }
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
}
// dy of bf16 as clients x rows x outputs; false: it has to be rearranged.
bool describe(const WeightArgs& a, CUtensorMap* map) {
    const cuuint64_t sizes[3] = {a.outs, a.rows, a.clients}, strides[2] = {a.dy_stride * 2, a.rows * a.dy_stride * 2};
    const cuuint32_t box[3] = {64, kChunk, 1}, each[3] = {1, 1, 1};
    if (strides[1] >= (1ull << 40)) return false;
    const auto call = tensor_map_call();
    return call && call(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(a.dy), sizes, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int kParts, bool kDirect = false>
int launch_weight(const WeightArgs& a, const CUtensorMap& map, cudaStream_t st) {
    auto* kernel = f8_weight_kernel<kParts, kDirect>;
    static std::atomic<int> sms[64];
    int dev = 0;
    CO3_CUDA(cudaGetDevice(&dev));
    int n = dev < 64 ? sms[dev].load(std::memory_order_relaxed) : 0;
    if (n == 0) {
        CO3_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemW));
        CO3_CUDA(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev));
        if (dev < 64) sms[dev].store(n, std::memory_order_relaxed);
    }
    const uint32_t tiles = (a.k_tiles + 1) / 2 * a.n_tiles * a.parts * a.clients;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * std::min(tiles, (uint32_t)n / 2));
    cfg.blockDim = dim3(kF8Threads);
    cfg.dynamicSmemBytes = kSmemW;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    CO3_CUDA(cudaLaunchKernelEx(&cfg, kernel, a, map));
    return CO3_OK;
}
template <typename T, bool kWide>
int launch_operands(const WeightArgs& a, cudaStream_t st) {
    const uint32_t blocks = (a.direct && !a.db ? 0u : a.clients * a.groups * a.db_parts) + (a.dw ? a.clients * a.k_tiles * a.chunks : 0u);
    CO3_CUDA(launch_behind(f8_operands_kernel<T, kWide>, dim3(blocks), dim3(256), 0, st, a));
    return CO3_OK;
}

}  // namespace
}  // namespace co3

using namespace co3;

extern "C" {

int co3_f8_weight_gradient_workspace_bytes(uint64_t rows, uint32_t outs, uint32_t ins, uint32_t n_clients, size_t* out) {
    uint64_t most = 0;  // of the three types
    for (int type : {CO3_F32, CO3_F16, CO3_BF16}) {
        WeightPlan w;
        if (!out || !weight_plan(rows, outs, ins, n_clients, parts_of(type), &w)) return CO3_ERR_INVALID_ARG;
        most = std::max(most, w.bytes);
    }
    *out = (size_t)most;
    return CO3_OK;
}

int co3_f8_weight_gradient(const void* dy, int type, uint64_t dy_row_stride, const void* x8, size_t x8_bytes, uint64_t rows, uint32_t outs, uint32_t ins,
                           float* dw, float* db, uint32_t n_clients, uint64_t client_stride_elems, int accumulate, void* workspace, size_t workspace_bytes,
                           co3_result* res, void* stream) {
    F8Layout l;
    WeightPlan w;
    if (type < CO3_F32 || type > CO3_BF16 || !weight_plan(rows, outs, ins, n_clients, parts_of(type), &w) ||
        !f8_layout(rows * n_clients, ins, CO3_F8_ROWS, &l))
        return CO3_ERR_INVALID_ARG;
    if (ins == 0) dw = nullptr;
    if (outs == 0 || (!dw && !db)) return CO3_OK;
    if (!aligned(dw, 4) || !aligned(db, 4) || !aligned(res, 8) || client_stride_elems >= (1ull << 40) ||
        (n_clients > 1 && ((dw && client_stride_elems < (uint64_t)outs * ins) || (db && client_stride_elems < outs))))
        return CO3_ERR_INVALID_ARG;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows == 0)  // no terms: zeros
        return accumulate ? CO3_OK
                          : launch_join({nullptr, dw, (uint64_t)outs * ins, 0}, {nullptr, db, outs, 0}, n_clients, client_stride_elems, 0, st);
    if (!dy || !aligned(dy, type_size(type)) || dy_row_stride < outs || dy_row_stride >= (1ull << 40) || (dw && (!x8 || !aligned(x8, 256))) || !workspace ||
        !aligned(workspace, 256))
        return CO3_ERR_INVALID_ARG;
    if ((dw && x8_bytes < l.bytes) || workspace_bytes < w.bytes) return CO3_ERR_CAPACITY;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    WeightArgs a = {};
    a.dy = dy;
    a.dy_stride = dy_row_stride;
    a.x = static_cast<const uint8_t*>(x8);
    a.x_scales = a.x + l.scales;
    a.x_rows = l.rows;
    a.rows = rows;
    a.outs = outs;
    a.ins = ins;
    a.clients = n_clients;
    a.k_tiles = w.k_tiles;
    a.groups = w.groups;
    a.chunks = w.chunks;
    a.tile_outs = w.tile_outs;
    a.n_tiles = w.n_tiles;
    a.parts = w.parts;
    a.db_parts = w.db_parts;
    a.ws_x = ws + w.x;
    a.ws_dy = ws + w.dy;
    a.dw_parts = reinterpret_cast<float*>(ws + w.dw);
    a.db_parts_at = reinterpret_cast<float*>(ws + w.db);
    a.dw = dw;
    a.db = db;
    a.client_stride = client_stride_elems;
    a.accumulate = accumulate;
    a.res = res;
    if (small_gradient(rows, outs, ins, n_clients))
        return type == CO3_F32 ? launch_small<float>(a, st) : type == CO3_F16 ? launch_small<__half>(a, st) : launch_small<__nv_bfloat16>(a, st);
    const size_t s = type_size(type);
    const bool wide = aligned(dy, 16) && dy_row_stride * s % 16 == 0 && outs * s % 16 == 0;
    CUtensorMap map = {};
    a.direct = type == CO3_BF16 && wide && dw && describe(a, &map);
    int e = type == CO3_F32   ? (wide ? launch_operands<float, true>(a, st) : launch_operands<float, false>(a, st))
            : type == CO3_F16 ? (wide ? launch_operands<__half, true>(a, st) : launch_operands<__half, false>(a, st))
                              : (wide ? launch_operands<__nv_bfloat16, true>(a, st) : launch_operands<__nv_bfloat16, false>(a, st));
    if (e == CO3_OK && dw)
        e = type == CO3_F32   ? launch_weight<3>(a, map, st)
            : type == CO3_F16 ? launch_weight<2>(a, map, st)
            : a.direct        ? launch_weight<1, true>(a, map, st)
                              : launch_weight<1>(a, map, st);
    if (e != CO3_OK) return e;
    return launch_join({a.dw_parts, w.parts > 1 ? dw : nullptr, (uint64_t)outs * ins, w.parts}, {a.db_parts_at, w.db_parts > 1 ? db : nullptr, outs, w.db_parts},
                       n_clients, client_stride_elems, accumulate, st);
}

}  // extern "C"
