// Orthogonalised updates: Newton-Schulz steps X <- a X + (b A + c A A) X, A = X X^T, for many matrices at once, on the
// fifth-generation tensor cores.
//
//   orth_begin_kernel   (momentum update +) sum of squares of every matrix
//   orth_load_kernel    X_0 = G / (norm + eps) as operand blocks
//   orth_steps_kernel   all products of all steps in one cooperative launch: per step A = X X^T; B = b A + c A A;
//                       X <- a X + B X; the last product writes the result (or steps the parameters) instead of X
#include <cuda_runtime.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

#include "co3.h"
#include "co3_device.cuh"
#include "co3_launch.cuh"
#include "co3_orth.cuh"
#include "co3_orth_small.h"
#include "co3_types.cuh"

namespace co3 {

constexpr uint32_t kOrthMats = 96;                  // matrices of one batch of launches
constexpr uint32_t kBeginElems = 8192;              // elements per block of orth_begin_kernel
constexpr int kBeginThreads = 256;
constexpr int kLoadThreads = 256;
enum OrthPhase { kGram = 0, kPoly = 1, kApply = 2 };

struct OrthMat {
    uint64_t in_off, in_stride, out_off, out_stride;
    uint32_t rows, cols;
    float scale;
    uint32_t plain;
    uint32_t block0;     // first operand block of the matrix in the workspace
    uint32_t chunk0;     // first block of orth_begin_kernel that works on it
    uint32_t full0;      // tiles of X of the matrices before it
    uint32_t slot0;      // first partial-sum slot
    uint32_t arrive0;    // first arrival counter of split tiles
    uint32_t task0[3];   // tasks of the matrices before it, per phase
    uint32_t splits[3];  // tasks per tile (the summed dimension in that many parts), per phase
    uint32_t pad;
};

struct OrthBatch {
    OrthMat mat[kOrthMats];
    uint32_t n_mats, n_chunks, n_full, n_arrive;
    uint32_t n_tasks[3];
    uint32_t index0;  // index of mat[0] in the caller's list
    uint32_t first;   // 1: the call's first batch, which clears the result
    uint32_t tile;    // OrthTile
};

struct OrthCtrl {
    uint32_t abort;
    uint32_t done[kOrthMats];  // tiles finished since the start of the call, per matrix
};

struct OrthWs {
    OrthBatch* batch;
    OrthCtrl* ctrl;
    uint32_t* arrive;  // [n_arrive]
    double* partial;   // [n_chunks] sums of squares
    float* slots;      // [n_slots][128 * 128] partial sums of split tiles
    unsigned char* blocks;
};

// Tiles of a product: 128 x 64 or 128 x 128.
enum OrthTile { kNarrow = 0, kSquare = 1 };
template <int kTile>
struct Tiling {
    static constexpr uint32_t kCols = kTile == kNarrow ? 64 : 128;
    static constexpr uint32_t kSums = 512 / kCols;                                   // tiles that tensor memory holds
    static constexpr uint32_t kColPlane = kTile == kNarrow ? kHalfPlane : kPlane;    // of the columns' operand
    static constexpr uint32_t kStageBytes = kBlock + 2 * kColPlane, kStages = kTile == kNarrow ? 4 : 3;
    static constexpr uint32_t kOwnBytes = kTile == kNarrow ? kBlock : 2 * kBlock;    // of the tile's own blocks
};

struct OrthShape {
    uint32_t m, n;         // small side, long side
    uint32_t mb, nb;       // both in blocks of 128, which are the rows of tiles
    uint32_t mc, nc;       // both in tile columns
    uint32_t sym, per_row; // tiles of a symmetric product; tile columns per block
    bool tall;             // rows > cols: X is the transposed matrix
};

__host__ __device__ inline OrthShape orth_shape(uint32_t rows, uint32_t cols, uint32_t tile) {
    OrthShape s;
    const uint32_t tc = tile == kNarrow ? 64u : 128u;
    s.tall = rows > cols;
    s.m = s.tall ? cols : rows;
    s.n = s.tall ? rows : cols;
    s.mb = (s.m + 127u) / 128u;
    s.nb = (s.n + 127u) / 128u;
    s.mc = (s.m + tc - 1u) / tc;
    s.nc = (s.n + tc - 1u) / tc;
    s.per_row = 128u / tc;
    // up to and including the diagonal: (i + 1) per_row tiles in row i, as far as the matrix reaches
    s.sym = s.mb ? s.per_row * s.mb * (s.mb - 1u) / 2u + s.mc : 0u;
    return s;
}
// Tiles of the apply product, and of its last one, whose rows are the long side unless the matrix is tall.
__host__ __device__ inline uint32_t orth_apply_tiles(const OrthShape& s, bool last) { return last && !s.tall ? s.nb * s.mc : s.mb * s.nc; }

// Operand blocks of one matrix: X twice [mb][2 nb], A and B [mb][2 mb] (their lower triangles of tiles are used).
__host__ __device__ inline uint64_t orth_blocks(const OrthShape& s) {
    return 4ull * s.mb * s.nb + 4ull * s.mb * s.mb;
}
struct OrthOperands {
    unsigned char *x[2], *a, *b;
};
__device__ inline OrthOperands orth_operands(const OrthWs& ws, const OrthMat& t, const OrthShape& s) {
    OrthOperands o;
    const uint64_t xs = 2ull * s.mb * s.nb * kBlock;
    o.x[0] = ws.blocks + (uint64_t)t.block0 * kBlock;
    o.x[1] = o.x[0] + xs;
    o.a = o.x[1] + xs;
    o.b = o.a + 2ull * s.mb * s.mb * kBlock;
    return o;
}

// Index of the matrix that owns item `x`: largest k with first(k) <= x.  Matrices without items are skipped because
// the next one starts at the same item.
template <typename F>
__device__ __forceinline__ uint32_t orth_find(uint32_t n_mats, uint32_t x, F first) {
    uint32_t lo = 0, hi = n_mats;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) >> 1;
        if (first(mid) <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// ------------------------------------------------------------------------------------------------
// begin: one block per kBeginElems elements of a matrix.  Sums of squares in fp64, in a fixed order.  Momentum: buf is
// updated here, and plain layers take their whole step.
// ------------------------------------------------------------------------------------------------
struct BeginArgs {
    const void* in;
    float* momentum;  // null: orthogonalize only
    float* params;
    float mu, lr, shrink;
    int nesterov;
    co3_result* res;
    OrthWs ws;
};

template <typename T>
__global__ void __launch_bounds__(kBeginThreads) orth_begin_kernel(const __grid_constant__ OrthBatch batch, BeginArgs a) {
    wait_for_previous_kernel();
    if (blockIdx.x == 0) {
        const uint32_t* src = reinterpret_cast<const uint32_t*>(&batch);
        uint32_t* dst = reinterpret_cast<uint32_t*>(a.ws.batch);
        for (uint32_t i = threadIdx.x; i < sizeof(OrthBatch) / 4; i += kBeginThreads) dst[i] = src[i];
        if (threadIdx.x == 0) {
            if (batch.first) {
                co3_result r = {};
                r.first_bad_chunk = 0xffffffffu;
                *a.res = r;
            }
        }
    }
    {
        uint32_t* ctrl = reinterpret_cast<uint32_t*>(a.ws.ctrl);
        const uint32_t at = blockIdx.x * kBeginThreads + threadIdx.x, step = gridDim.x * kBeginThreads;
        for (uint32_t i = at; i < sizeof(OrthCtrl) / 4; i += step) ctrl[i] = 0u;
        for (uint32_t i = at; i < batch.n_arrive; i += step) a.ws.arrive[i] = 0u;
    }
    if (blockIdx.x >= batch.n_chunks) return;
    const uint32_t k = orth_find(batch.n_mats, blockIdx.x, [&](uint32_t i) { return batch.mat[i].chunk0; });
    const OrthMat& t = batch.mat[k];
    const uint64_t e0 = (uint64_t)(blockIdx.x - t.chunk0) * kBeginElems;
    const uint64_t total = (uint64_t)t.rows * t.cols;
    const uint32_t cnt = (uint32_t)min((uint64_t)kBeginElems, total - e0);
    const T* in = static_cast<const T*>(a.in);
    double sum = 0.0;
    const bool flat = t.in_stride == t.cols;
    for (uint32_t i = threadIdx.x; i < cnt; i += kBeginThreads) {
        const uint64_t e = e0 + i;
        uint64_t at;
        if (flat) {
            at = t.in_off + e;
        } else {
            const uint64_t r = e / t.cols;
            at = t.in_off + r * t.in_stride + (e - r * t.cols);
        }
        float u = to_float(in[at]);
        if (a.momentum) {
            const float g = u;
            const float buf = __fmaf_rn(a.mu, a.momentum[at], g);
            a.momentum[at] = buf;
            u = a.nesterov ? __fmaf_rn(a.mu, buf, g) : buf;
            if (t.plain) a.params[at] = __fmaf_rn(-a.lr * t.scale, u, a.shrink * a.params[at]);
        }
        sum += (double)u * (double)u;
    }
    __shared__ double s_sum[kBeginThreads / 32];
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int w = 0; w < kBeginThreads / 32; ++w) s += s_sum[w];
        a.ws.partial[blockIdx.x] = s;
    }
}

// A layer that holds a NaN or an infinity goes into the result.  By kernels behind orth_begin_kernel only: block 0 of that
// clears the result, in no order with its other blocks.
__device__ __forceinline__ void report_nonfinite(co3_result* res, uint32_t index) {
    set_status(res, CO3_ERR_NONFINITE);
    atomicMin(&res->first_bad_chunk, index);
    atomicAdd(reinterpret_cast<unsigned long long*>(&res->n_nonfinite), 1ull);
}

// ------------------------------------------------------------------------------------------------
// load: one block per 64 x 64 piece of X (padding included): S * G / (norm + eps).  If there are plain layers, one block
// more looks at their sums of squares, a warp to a layer.
// ------------------------------------------------------------------------------------------------
struct LoadArgs {
    const void* in;
    const float* momentum;  // null: orthogonalize only
    float mu, eps;
    int nesterov;
    co3_result* res;
    OrthWs ws;
};

template <typename T>
__global__ void __launch_bounds__(kLoadThreads) orth_load_kernel(LoadArgs a) {
    wait_for_previous_kernel();
    __shared__ float s_v[64][65];
    __shared__ double s_sum[kLoadThreads / 32];
    __shared__ double s_f;
    const OrthBatch& batch = *a.ws.batch;
    const uint32_t tile = blockIdx.x >> 2;  // tile of 128 x 128, quarter blockIdx.x & 3
    if (tile == batch.n_full) {
        for (uint32_t k = threadIdx.x >> 5; k < batch.n_mats; k += kLoadThreads / 32) {
            const OrthMat& t = batch.mat[k];
            if (!t.plain) continue;
            const uint32_t n_part = (uint32_t)(((uint64_t)t.rows * t.cols + kBeginElems - 1) / kBeginElems);
            bool good = true;
            for (uint32_t i = threadIdx.x & 31u; i < n_part; i += 32) good = good && isfinite(a.ws.partial[t.chunk0 + i]);
            if (!__all_sync(0xffffffffu, good) && (threadIdx.x & 31u) == 0) report_nonfinite(a.res, batch.index0 + k);
        }
        return;
    }
    const uint32_t k = orth_find(batch.n_mats, tile, [&](uint32_t i) { return batch.mat[i].full0; });
    const OrthMat t = batch.mat[k];
    const OrthShape s = orth_shape(t.rows, t.cols, batch.tile);
    // the norm: this matrix' partial sums in order
    const uint32_t n_part = (uint32_t)(((uint64_t)t.rows * t.cols + kBeginElems - 1) / kBeginElems);
    double sum = 0.0;
    for (uint32_t i = threadIdx.x; i < n_part; i += kLoadThreads) sum += a.ws.partial[t.chunk0 + i];
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double total = 0.0;
        for (int w = 0; w < kLoadThreads / 32; ++w) total += s_sum[w];
        const double d = sqrt(total) + (double)a.eps;
        s_f = d > 0.0 ? (double)orth_s(s.m, s.n) / d : 0.0;  // an all-zero matrix without eps stays zero
        if (!isfinite(total) && tile == t.full0 && (blockIdx.x & 3u) == 0) report_nonfinite(a.res, batch.index0 + k);
        if (!isfinite(total)) s_f = (double)NAN;
    }
    __syncthreads();
    const double f = s_f;
    const uint32_t local = tile - t.full0;
    const uint32_t x_row0 = (local / s.nb) * 128u + (blockIdx.x & 1u) * 64u;         // row of X (small side)
    const uint32_t x_col0 = (local % s.nb) * 128u + ((blockIdx.x >> 1) & 1u) * 64u;  // column of X (long side)
    const uint32_t r0 = s.tall ? x_col0 : x_row0, c0 = s.tall ? x_row0 : x_col0;     // place in the caller's matrix
    const T* in = static_cast<const T*>(a.in);
    // s_v holds X's piece by (row of X, column of X)
    for (uint32_t i = threadIdx.x; i < 64 * 64; i += kLoadThreads) {
        const uint32_t r = i >> 6, c = i & 63u;
        float v = 0.0f;
        if (r0 + r < t.rows && c0 + c < t.cols) {
            const uint64_t at = t.in_off + (uint64_t)(r0 + r) * t.in_stride + (c0 + c);
            float u = to_float(in[at]);
            if (a.momentum) {
                const float buf = a.momentum[at];
                u = a.nesterov ? __fmaf_rn(a.mu, buf, u) : buf;
            }
            v = (float)((double)u * f);
        }
        if (s.tall) s_v[c][r] = v; else s_v[r][c] = v;
    }
    __syncthreads();
    const OrthOperands op = orth_operands(a.ws, t, s);
    unsigned char* xb = op.x[0] + ((uint64_t)(x_row0 >> 7) * (2 * s.nb) + (x_col0 >> 6)) * kBlock;
    for (uint32_t i = threadIdx.x; i < 64 * 8; i += kLoadThreads) {
        const uint32_t row = i >> 3, piece = i & 7u;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = s_v[row][piece * 8 + e];
        uint4 hi, lo;
        split8(v, hi, lo);
        unsigned char* p = xb + swizzled((x_row0 & 64u) + row, piece);
        *reinterpret_cast<uint4*>(p) = hi;
        *reinterpret_cast<uint4*>(p + kPlane) = lo;
    }
}

// ------------------------------------------------------------------------------------------------
// steps: persistent blocks (all resident: a cooperative launch).  The products of all steps form one list of tasks,
// phase by phase; a task is a tile, or a part of its sum where there are fewer tiles than SMs.  Block b takes
// tasks b, b + number of blocks, ... in order, and before a task's operands are fetched it waits until the matrix' tiles
// of the phases before it are finished (a counter per matrix): the tasks waited for stand earlier in the list, so that
// waiting always ends, and one matrix' tail is filled with other matrices' work.
//
// Warps 0 and 10 copy operand blocks into a ring (one thread each, for the rows' and the columns' operand: a copy costs its
// thread about 100 cycles), warps 1 and 11 issue the products, every other stage each: looking at a barrier takes a thread 100 to
// 200 cycles during which it issues nothing (12 products 770 cycles; with the looks by one thread 1000).  Warps 2..9 take the sums: each of them 32 rows x half of the tile's
// columns in registers, and from there on each works on its own.  Behind a task's operands the ring carries its linear
// term (b A or a X, the tile's own blocks); the warps put the finished values in its place, from where they go to memory.
//
// Which tiles: a stage (64 columns of the sum, 12 products) of a 128 x 128 tile takes about 0.6 us, of a 128 x 64 tile
// 0.45: the smaller ones win while there are fewer tiles than SMs (1000 x 513: 0.19 against 0.22 ms, 2048 x 2048: 0.88
// against 0.55).  Tiles of 256 x 256 by pairs of blocks, which read half as much per product, were no faster where the
// power limit holds the clock down (4096 x 4096: 4.36 against 4.15 ms) and much slower for small matrices.
// ------------------------------------------------------------------------------------------------
constexpr int kEpiThreads = 256;
constexpr int kStepThreads = 64 + kEpiThreads + 64;
constexpr int kMaxStages = 4;
// The tensor core cuts what it adds to 26 bits below the largest term, always towards zero: sums of one sign (the
// diagonal of A) drift.  The sum of each stage is therefore taken out and added up in registers, where fp32 rounds to
// nearest.  1000 x 513, five steps, error against 64 bits: 1.3e-5 if the tensor core adds up all stages, 6.1e-6 if
// four, 2.1e-6 if one (2.9e-6 with all sums in fp32 arithmetic).
constexpr size_t kRingBytes = 192 << 10;
static_assert(Tiling<kNarrow>::kStages * Tiling<kNarrow>::kStageBytes == kRingBytes && Tiling<kSquare>::kStages * Tiling<kSquare>::kStageBytes == kRingBytes, "one size of ring");

struct Task {
    uint32_t step, phase, mat;
    uint32_t rb, cg;      // block row, and first group of 64 columns, of the tile
    uint32_t k0, k1;      // operand blocks of the summed dimension
    uint32_t part, parts;
    uint32_t tile;        // index within the matrix and phase
    uint32_t before;      // warps' parts of this matrix' tiles that have to be finished
    bool swap;            // kApply: the tile's rows are the long side
    bool diagonal;        // both operands are the same blocks
    bool skip;            // no such tile
};

struct MatView {
    OrthMat t;
    OrthShape s;
    OrthOperands op;
};

struct StepSmem {
    // A barrier tells its last phase from the one before and no more: who waits on it has to see every phase.  So each
    // stage of the ring has one per reader: warp 1, warp 11, warps 2..9.
    uint64_t full[3][kMaxStages];
    uint64_t empty[kMaxStages];      // a stage of operands has been multiplied, or one of the tile's own blocks stored
    uint32_t stored[kMaxStages];     // warps that are done with a stage of the tile's own blocks
    uint64_t sum_full[8], sum_empty[8];
    uint64_t done[2];
    uint32_t tmem, failed;
    uint32_t task0[3][kOrthMats];
    Task task[8];  // what warps 2..9 work on: in shared memory, the sums need the registers
    MatView view[8];
};
constexpr size_t kSmemOff = kRingBytes;
constexpr size_t kStepSmem = 1024 + kSmemOff + sizeof(StepSmem);
static_assert(kStepSmem <= 227 * 1024 && kSmemOff % 8 == 0, "shared memory of a block");

struct StepArgs {
    OrthWs ws;
    co3_ns ns;
    int out_kind;
    void* out;
    float lr, shrink;
    uint64_t limit_ns;  // longest wait
    co3_result* res;
};

template <int kTile>
__device__ __forceinline__ Task find_task(const StepArgs& a, const StepSmem& sm, const uint32_t* n_tasks, uint32_t n_mats, uint32_t g, MatView& v) {
    using L = Tiling<kTile>;
    Task k;
    const uint32_t per_step = n_tasks[0] + n_tasks[1] + n_tasks[2];
    k.step = g / per_step;
    uint32_t x = g - k.step * per_step;
    k.phase = 0;
    while (x >= n_tasks[k.phase]) x -= n_tasks[k.phase++];
    const uint32_t* first = sm.task0[k.phase];
    k.mat = orth_find(n_mats, x, [&](uint32_t i) { return first[i]; });
    v.t = a.ws.batch->mat[k.mat];
    v.s = orth_shape(v.t.rows, v.t.cols, kTile);
    v.op = orth_operands(a.ws, v.t, v.s);
    x -= first[k.mat];
    k.parts = v.t.splits[k.phase];
    k.tile = x / k.parts;
    k.part = x - k.tile * k.parts;
    k.before = 8 * (k.step * (2 * v.s.sym + orth_apply_tiles(v.s, false)) + k.phase * v.s.sym);
    k.swap = k.diagonal = k.skip = false;
    uint32_t i, j, blocks;
    if (k.phase == kApply) {
        // in the last product of a matrix that is not tall the tile's rows are the long side, so that a warp's rows
        // are neighbours in the caller's memory
        const bool last = k.step + 1 == a.ns.steps;
        k.swap = last && !v.s.tall;
        k.skip = k.tile >= orth_apply_tiles(v.s, last);
        const uint32_t cols = k.swap ? v.s.mc : v.s.nc;
        i = k.tile / cols;
        j = k.tile - i * cols;
        blocks = (v.s.m + 63u) / 64u;
    } else {  // tiles on and below the diagonal
        const uint32_t t = k.tile / (128u / L::kCols);
        i = (uint32_t)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
        while (v.s.per_row * i * (i + 1) / 2 > k.tile) --i;
        while (v.s.per_row * (i + 1) * (i + 2) / 2 <= k.tile) ++i;
        j = k.tile - v.s.per_row * i * (i + 1) / 2;
        k.diagonal = kTile == kSquare && i == j;
        blocks = ((k.phase == kGram ? v.s.n : v.s.m) + 63u) / 64u;
    }
    k.rb = i;
    k.cg = j * (L::kCols / 64u);
    k.k0 = (uint32_t)((uint64_t)blocks * k.part / k.parts);
    k.k1 = (uint32_t)((uint64_t)blocks * (k.part + 1) / k.parts);
    return k;
}

// Whether the apply product of a step adds a X in fp32.  In the last step a I is part of B instead: the result's tiles may
// lie the other way round there, where X has no blocks to add.  In the steps before, the rounding of B + a I to pairs
// would grow with the small singular values (130 x 70: error 2.5e-6 instead of 1.5e-6).
__device__ __forceinline__ bool adds_x(const StepArgs& a, uint32_t step) { return step + 1 < a.ns.steps; }

// The tile's own blocks of the linear term, in a row; null if there is none.
__device__ __forceinline__ const unsigned char* linear_term(const StepArgs& a, const Task& k, const MatView& v) {
    if (k.phase == kPoly) return v.op.a + ((uint64_t)k.rb * (2 * v.s.mb) + k.cg) * kBlock;
    if (k.phase == kApply && adds_x(a, k.step)) return v.op.x[k.step & 1u] + ((uint64_t)k.rb * (2 * v.s.nb) + k.cg) * kBlock;
    return nullptr;
}

// bulk_copy_g2s and mbar_arrive_expect_tx with shared-memory addresses as they are
__device__ __forceinline__ void copy_in(uint32_t dst, const unsigned char* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void arrive_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

// How one of a task's operands is fetched: columns 64 q .. 64 q + 63 of the sum, for 128 rows of block row r, or for 64
// rows (r counts groups of 64).
struct Operand {
    const unsigned char* base;
    uint64_t row;      // bytes between block rows
    uint32_t r;
    uint32_t from;     // stages from this one on are fetched transposed
    __device__ __forceinline__ void fetch128(uint32_t dst, uint32_t q, uint32_t bar) const {
        if (q < from) {
            copy_in(dst, base + r * row + (uint64_t)q * kBlock, kBlock, bar);
        } else {  // rows 64 q .. of block row q / 2, columns of blocks 2 r and 2 r + 1
            const unsigned char* p = base + (q >> 1) * row + (uint64_t)(2 * r) * kBlock + (q & 1u) * kHalfPlane;
            copy_in(dst, p, kHalfPlane, bar);
            copy_in(dst + kHalfPlane, p + kBlock, kHalfPlane, bar);
            copy_in(dst + kPlane, p + kPlane, kHalfPlane, bar);
            copy_in(dst + kPlane + kHalfPlane, p + kBlock + kPlane, kHalfPlane, bar);
        }
    }
    __device__ __forceinline__ void fetch64(uint32_t dst, uint32_t q, uint32_t bar) const {
        const unsigned char* p = q < from ? base + (r >> 1) * row + (uint64_t)q * kBlock + (r & 1u) * kHalfPlane
                                          : base + (q >> 1) * row + (uint64_t)r * kBlock + (q & 1u) * kHalfPlane;
        copy_in(dst, p, kHalfPlane, bar);
        copy_in(dst + kHalfPlane, p + kPlane, kHalfPlane, bar);
    }
};
// The operand of the tile's rows (which == 0) or columns (1).
template <int kTile>
__device__ __forceinline__ Operand operand(const Task& k, const MatView& v, int which) {
    const uint32_t r = which == 0 ? k.rb : kTile == kNarrow ? k.cg : k.cg / 2;
    const uint32_t block_row = which == 1 && kTile == kNarrow ? r / 2 : r;
    const uint64_t row_x = (uint64_t)(2 * v.s.nb) * kBlock, row_m = (uint64_t)(2 * v.s.mb) * kBlock;
    if (k.phase == kGram) return {v.op.x[k.step & 1u], row_x, r, 0xffffffffu};
    if (k.phase == kApply && (which == 1) != k.swap) return {v.op.x[k.step & 1u], row_x, r, 0u};
    // a symmetric matrix: stored up to and including the block on the diagonal
    return {k.phase == kPoly ? v.op.a : v.op.b, row_m, r, (block_row + 1) * 2};
}

__device__ __forceinline__ uint32_t load_acquire(const uint32_t* p) {
    uint32_t v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, uint64_t limit_ns) {
    if (mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = global_timer_ns();
    for (;;) {
        for (int i = 0; i < 64; ++i)
            if (mbar_try_wait(bar, parity)) return true;
        if (global_timer_ns() - t0 > limit_ns) return false;
    }
}

// Waits until at least `need` parts of a matrix' tiles are finished.
__device__ __forceinline__ bool wait_tiles(const OrthCtrl* ctrl, uint32_t mat, uint32_t need, uint64_t limit_ns) {
    if (load_acquire(&ctrl->done[mat]) >= need) return true;
    const uint64_t t0 = global_timer_ns();
    for (uint32_t i = 1;; ++i) {
        if (load_acquire(&ctrl->done[mat]) >= need) return true;
        if ((i & 255u) == 0 && (load_acquire(&ctrl->abort) != 0u || global_timer_ns() - t0 > limit_ns)) return false;
    }
}

__device__ __forceinline__ void bulk_copy_s2g(void* dst_gmem, const void* src_smem, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst_gmem), "r"(smem_addr(src_smem)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_stores_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void bulk_stores_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// The products of one stage: 64 columns of the sum, operands at a and b in shared memory.
template <int kTile, bool kTa, bool kTb>
__device__ __forceinline__ void multiply_stage(uint32_t d, uint32_t a, uint32_t b) {
    using L = Tiling<kTile>;
    constexpr uint32_t instr = instr_desc(kTa, kTb, 128, L::kCols), da = desc_step(kTa), db = desc_step(kTb);
    const uint64_t ah = smem_desc(a, kTa), bh = smem_desc(b, kTb);
    const uint64_t al = ah + (kPlane >> 4), bl = bh + (L::kColPlane >> 4);
    // the corrections first, 2^11 times too large; the first product of the hi planes scales them down
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) tc_mma(d, ah + e * da, bl + e * db, instr, e > 0);
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) tc_mma(d, al + e * da, bh + e * db, instr, true);
    tc_mma<kLoBits>(d, ah, bh, instr, true);
#pragma unroll
    for (uint32_t e = 1; e < 4; ++e) tc_mma(d, ah + e * da, bh + e * db, instr, true);
}

template <int kTile>
__global__ void __launch_bounds__(kStepThreads, 1) orth_steps_kernel(const __grid_constant__ StepArgs a) {
    extern __shared__ unsigned char smem_raw[];
    using L = Tiling<kTile>;
    constexpr uint32_t kCols = L::kCols, kSums = L::kSums, kStages = L::kStages, kStageBytes = L::kStageBytes;
    unsigned char* ring = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    StepSmem& sm = *reinterpret_cast<StepSmem*>(ring + kSmemOff);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const uint32_t n_mats = a.ws.batch->n_mats;
    const uint32_t n_tasks[3] = {a.ws.batch->n_tasks[0], a.ws.batch->n_tasks[1], a.ws.batch->n_tasks[2]};
    const uint32_t total = a.ns.steps * (n_tasks[0] + n_tasks[1] + n_tasks[2]);
    for (uint32_t i = threadIdx.x; i < n_mats; i += kStepThreads)
        for (int p = 0; p < 3; ++p) sm.task0[p][i] = a.ws.batch->mat[i].task0[p];
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < kStages; ++i) {
            for (int w = 0; w < 3; ++w) mbar_init(&sm.full[w][i], 2);
            mbar_init(&sm.empty[i], 1);
            sm.stored[i] = 0;
        }
        for (uint32_t i = 0; i < kSums; ++i) { mbar_init(&sm.sum_full[i], 1); mbar_init(&sm.sum_empty[i], 8); }
        mbar_init(&sm.done[0], 1);
        mbar_init(&sm.done[1], 1);
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
    MatView v;

    if ((warp == 0 || warp == 10) && lane == 0) {
        const int which = warp == 0 ? 0 : 1;
        uint32_t st = 0, turn = 0;  // the ring's next stage, and how often the ring has been gone through
        uint32_t unit = 0;          // stages of operands begun: warps 1 and 11 multiply every other one
        uint32_t filled = 0;        // phases of sm.full begun, modulo 2: bit 4 reader + stage
        const uint32_t ring_addr = smem_addr(ring), full0 = smem_addr(&sm.full[0][0]);
        for (uint32_t g = blockIdx.x; g < total && !*failed; g += gridDim.x) {
            const Task k = find_task<kTile>(a, sm, n_tasks, n_mats, g, v);
            if (k.skip) continue;
            const Operand o = operand<kTile>(k, v, which);
            if (!wait_tiles(a.ws.ctrl, k.mat, k.before, a.limit_ns)) { *failed = 1; break; }
            fence_async_all();  // orders what the counter says after the copies that follow
            auto begin = [&]() {
                if (turn > 0 && !wait_for(&sm.empty[st], (turn - 1) & 1u, a.limit_ns)) { *failed = 1; return false; }
                return true;
            };
            auto next = [&](uint32_t reader) {
                filled ^= 1u << (4 * reader + st);
                if (++st == kStages) { st = 0; ++turn; }
            };
            const bool half_width = which == 1 && kTile == kNarrow;
            const uint32_t bytes = half_width ? kPlane : kBlock;  // of a stage
            for (uint32_t q = k.k0; q < k.k1; ++q) {
                if (!begin()) break;
                const uint32_t reader = unit & 1u, bar = full0 + (reader * kMaxStages + st) * 8u;
                const uint32_t dst = ring_addr + st * kStageBytes + (which ? kBlock : 0u);
                if (which == 1 && k.diagonal) {
                    mbar_arrive(&sm.full[reader][st]);
                } else {
                    arrive_expect(bar, bytes);
                    if (half_width) o.fetch64(dst, q, bar); else o.fetch128(dst, q, bar);
                }
                next(reader);
                ++unit;
            }
            const unsigned char* lin = which == 0 ? linear_term(a, k, v) : nullptr;
            if (!*failed && begin()) {
                const uint32_t bar = full0 + (2 * kMaxStages + st) * 8u;
                if (lin) {
                    arrive_expect(bar, L::kOwnBytes);
                    copy_in(ring_addr + st * kStageBytes, lin, L::kOwnBytes, bar);
                } else {
                    mbar_arrive(&sm.full[2][st]);  // nothing to fetch: the stage is there for the results
                }
                next(2);
            }
        }
        // copies in flight end before the block does, whoever else has given up
        for (uint32_t b = 0; b < 12; ++b)
            if (b % 4 < kStages) mbar_wait(&sm.full[b / 4][b % 4], ((filled >> b) & 1u) ^ 1u);
    } else if ((warp == 1 || warp == 11) && lane == 0) {
        const uint32_t mine = warp == 1 ? 0u : 1u;
        uint32_t unit = 0, seen = 0;             // stages begun; phases of this warp's sm.full, modulo 2, by stage
        uint32_t st = 0, buf = 0, buf_turn = 0;  // next stage of the ring; next sum in tensor memory, and how often round
        const uint32_t ring_addr = smem_addr(ring);
        for (uint32_t g = blockIdx.x; g < total && !*failed; g += gridDim.x) {
            const Task k = find_task<kTile>(a, sm, n_tasks, n_mats, g, v);
            if (k.skip) continue;
            const uint32_t from_a = operand<kTile>(k, v, 0).from, from_b = operand<kTile>(k, v, 1).from;
            bool ok = true;
            for (uint32_t q = k.k0; q < k.k1; ++q) {
                if ((unit & 1u) == mine) {
                    if (!wait_for(&sm.full[mine][st], (seen >> st) & 1u, a.limit_ns)) { ok = false; break; }
                    seen ^= 1u << st;
                    if (buf_turn > 0 && !wait_for(&sm.sum_empty[buf], (buf_turn - 1) & 1u, a.limit_ns)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t d = tmem + buf * kCols, at = ring_addr + st * kStageBytes, bt = k.diagonal ? at : at + kBlock;
                    if (q >= from_a) {
                        if (q >= from_b) multiply_stage<kTile, true, true>(d, at, bt);
                        else multiply_stage<kTile, true, false>(d, at, bt);
                    } else {
                        if (q >= from_b) multiply_stage<kTile, false, true>(d, at, bt);
                        else multiply_stage<kTile, false, false>(d, at, bt);
                    }
                    tc_commit(&sm.sum_full[buf]);
                    tc_commit(&sm.empty[st]);
                }
                ++unit;
                if (++st == kStages) st = 0;
                if (++buf == kSums) { buf = 0; ++buf_turn; }
            }
            if (!ok) { *failed = 1; break; }
            if (++st == kStages) st = 0;  // the tile's own blocks pass from the copies to warps 2..9
        }
        tc_commit(&sm.done[mine]);
        mbar_wait(&sm.done[mine], 0);
    } else if (warp >= 2 && warp < 10) {
        constexpr int kAcc = kCols / 2;  // columns of this warp
        const uint32_t quad = warp & 3u, half = (warp - 2u) >> 2, row = quad * 32u + lane;
        const uint32_t lane_base = tmem + ((quad * 32u) << 16) + half * kAcc;
        uint32_t it = 0, chunk = 0, seen = 0;  // seen: phases of sm.full[2], modulo 2, by stage
        for (uint32_t g = blockIdx.x; g < total; g += gridDim.x) {
            if (lane == 0) sm.task[warp - 2] = find_task<kTile>(a, sm, n_tasks, n_mats, g, sm.view[warp - 2]);
            __syncwarp();
            const Task& k = sm.task[warp - 2];
            const MatView& v = sm.view[warp - 2];
            if (k.skip) { __syncwarp(); continue; }
            const uint32_t chunks = k.k1 - k.k0;
            float acc[kAcc];
#pragma unroll
            for (int i = 0; i < kAcc; ++i) acc[i] = 0.0f;
            bool ok = true;
            for (uint32_t q = 0; q < chunks; ++q, ++chunk) {
                const uint32_t buf = chunk % kSums;
                // one lane looks: 256 threads at the barriers would slow down the one that issues the products
                ok = lane != 0 || wait_for(&sm.sum_full[buf], (chunk / kSums) & 1u, a.limit_ns);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                tc_fence_after();
#pragma unroll
                for (int h = 0; h < kAcc / 32; ++h) {
                    float w[32];
                    tc_load32(lane_base + buf * kCols + h * 32u, w);
#pragma unroll
                    for (int i = 0; i < 32; ++i) acc[h * 32 + i] = __fadd_rn(acc[h * 32 + i], w[i]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.sum_empty[buf]);
            }
            it += chunks;
            const uint32_t out_st = it % kStages;  // the stage with the tile's own blocks
            ++it;
            ok = ok && (lane != 0 || wait_for(&sm.full[2][out_st], (seen >> out_st) & 1u, a.limit_ns));
            seen ^= 1u << out_st;
            if (!__all_sync(0xffffffffu, ok)) { *failed = 1; break; }

            bool mine = true;  // this warp finishes its part of the tile
            if (k.parts > 1) {
                // the sums of this part of the summed dimension into its slot; whoever arrives last adds all of them
                // in order
                const uint64_t slot0 = v.t.slot0 + (uint64_t)k.tile * k.parts;
                float* to = a.ws.slots + (slot0 + k.part) * (128 * kCols);
#pragma unroll
                for (int i = 0; i < kAcc; ++i) __stcg(to + (half * kAcc + i) * 128 + row, acc[i]);
                __threadfence();
                __syncwarp();
                uint32_t old = 0;
                if (lane == 0) {
                    old = atomicAdd(a.ws.arrive + v.t.arrive0 + (k.phase * v.s.sym + k.tile) * 8 + warp - 2, 1u);
                    __threadfence();
                }
                old = __shfl_sync(0xffffffffu, old, 0);
                mine = old == k.step * k.parts + k.parts - 1;
                if (mine) {
#pragma unroll
                    for (int i = 0; i < kAcc; ++i) acc[i] = 0.0f;
                    for (uint32_t p = 0; p < k.parts; ++p) {
                        const float* from = a.ws.slots + (slot0 + p) * (128 * kCols);
#pragma unroll
                        for (int i = 0; i < kAcc; ++i) acc[i] = __fadd_rn(acc[i], __ldcg(from + (half * kAcc + i) * 128 + row));
                    }
                }
            }

            const bool last = k.phase == kApply && k.step + 1 == a.ns.steps, has_lin = k.phase == kPoly || (k.phase == kApply && adds_x(a, k.step));
            const uint32_t n_rows = k.swap ? v.s.n : v.s.m, n_cols = k.phase == kApply && !k.swap ? v.s.n : v.s.m;
            const uint32_t row0 = k.rb * 128u, col0 = k.cg * 64u;
            // Rows and columns up to a multiple of 64 are written: beyond, no product reads them.
            // This warp's block of the tile, of which it has all columns or half of them, from piece p0 on.
            const uint32_t cg = kTile == kNarrow ? 0u : half, p0 = kTile == kNarrow ? half * 4u : 0u, c0 = col0 + cg * 64u + p0 * 8u;
            if (mine && row0 + (quad & 2u) * 32u < n_rows && col0 + cg * 64u < n_cols) {
                const float inv_s = 1.0f / orth_s(v.s.m, v.s.n);
                float fl = 0.0f, fa = inv_s;  // value = fl * linear + fa * sum
                if (k.phase == kPoly) { fl = a.ns.coef[k.step][1]; fa = __fmul_rn(a.ns.coef[k.step][2], inv_s); }
                if (k.phase == kApply) fl = a.ns.coef[k.step][0];
                if (last) {
                    const float f = __fmul_rn(v.t.scale, inv_s);
                    fl = __fmul_rn(fl, f);
                    fa = __fmul_rn(fa, f);
                }
                // B takes a I in where the apply product does not add a X
                const bool add_diag = k.phase == kPoly && !adds_x(a, k.step);
                const float diag = __fmul_rn(a.ns.coef[k.step][0], orth_s(v.s.m, v.s.n));
                unsigned char* dst = nullptr;  // this block's part of the tile, its blocks in a row
                if (k.phase != kApply) dst = (k.phase == kGram ? v.op.a : v.op.b) + ((uint64_t)k.rb * (2 * v.s.mb) + k.cg) * kBlock;
                else if (!last) dst = v.op.x[(k.step & 1u) ^ 1u] + ((uint64_t)k.rb * (2 * v.s.nb) + k.cg) * kBlock;
                unsigned char* own = ring + (size_t)out_st * kStageBytes + cg * kBlock;
#pragma unroll
                for (int p = 0; p < kAcc / 8; ++p) {
                    float* w = acc + p * 8;
                    const uint32_t at = swizzled(row, p0 + p);
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] = __fmul_rn(fa, w[e]);
                    if (has_lin) {
                        float l[8];
                        join8(*reinterpret_cast<const uint4*>(own + at), *reinterpret_cast<const uint4*>(own + at + kPlane), l);
#pragma unroll
                        for (int e = 0; e < 8; ++e) w[e] = __fmaf_rn(fl, l[e], w[e]);
                    }
                    if (add_diag) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (c0 + p * 8 + e == row0 + row) w[e] = __fadd_rn(w[e], diag);
                    }
                    if (!last) {
                        uint4 hi, lo;
                        split8(w, hi, lo);
                        *reinterpret_cast<uint4*>(own + at) = hi;
                        *reinterpret_cast<uint4*>(own + at + kPlane) = lo;
                    }
                }
                if (!last && kTile == kNarrow) {
                    // half a block's columns: 64 bytes of each row, four lanes to a row
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t r = quad * 32u + (i & 3) * 8u + (lane >> 2), off = (i >> 2) * kPlane + swizzled(r, p0 + (lane & 3u));
                        *reinterpret_cast<uint4*>(dst + off) = *reinterpret_cast<const uint4*>(own + off);
                    }
                } else if (!last) {
                    fence_async_smem();
                    __syncwarp();
                    if (lane < 2) {  // 32 rows of either plane lie in a row
                        const uint32_t off = lane * kPlane + quad * 32u * 128u;
                        bulk_copy_s2g(dst + (uint64_t)cg * kBlock + off, own + off, 32u * 128u);
                        bulk_stores_commit();
                    }
                } else {
                    // the tile's rows run along the caller's rows, its columns across them
                    const uint32_t c = row0 + row;
                    const uint64_t first = v.t.out_off + (uint64_t)c0 * v.t.out_stride + c;
                    const uint32_t n = c < v.t.cols && c0 < v.t.rows ? min((uint32_t)kAcc, v.t.rows - c0) : 0u;
                    put_result<kAcc>(a.out, a.out_kind, first, v.t.out_stride, n, 1.0f, acc, a.lr, a.shrink);
                }
            }
            // the ring's stage is free as soon as the copies have read it, the tile finished when they have written it
            if (last || kTile == kNarrow) fence_async_all();  // ordinary accesses before the copies of others
            if (lane < 2) bulk_stores_read();
            __syncwarp();
            if (lane == 0) {
                __threadfence_block();
                if (atomicAdd(&sm.stored[out_st], 1u) == 7) {
                    sm.stored[out_st] = 0;
                    __threadfence_block();
                    mbar_arrive(&sm.empty[out_st]);
                }
            }
            if (mine && !last) {
                if (lane < 2) {
                    bulk_stores_done();
                    fence_async_all();
                }
                __syncwarp();  // and the release takes all lanes' writes along
                if (lane == 0) asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(&a.ws.ctrl->done[k.mat]) : "memory");
            }
            __syncwarp();
        }
    }
    __syncwarp();
    __syncthreads();
    if (warp == 1) {
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
    if (threadIdx.x == 0 && *failed) {
        a.ws.ctrl->abort = 1u;
        __threadfence();
        set_status(a.res, CO3_ERR_CUDA);
    }
}

}  // namespace co3

// ================================================================================================
// Host side
// ================================================================================================
using namespace co3;

namespace {

uint64_t up256(uint64_t x) { return (x + 255u) & ~(uint64_t)255u; }

bool valid_mat(const co3_mat& t) {
    if (t.rows == 0 || t.cols == 0) return true;
    if (t.rows >= (1u << 31) || t.cols >= (1u << 31) || (uint64_t)t.rows * t.cols >= (1ull << 40)) return false;
    if (t.row_stride < t.cols || (t.flags & ~CO3_MAT_PLAIN) != 0u) return false;
    return t.offset < (1ull << 60) && t.row_stride < (1ull << 40);
}

struct WsPlan {
    uint64_t batch, ctrl, arrive, partial, slots, blocks, total;
};
struct BatchNeeds {
    uint64_t slots, blocks;  // workspace
    uint64_t work;           // stages of one step
    uint64_t ns;             // their time, about
};
WsPlan ws_plan(const OrthBatch* b, const BatchNeeds& needs) {
    WsPlan w;
    w.batch = 0;
    w.ctrl = up256(sizeof(OrthBatch));
    w.arrive = w.ctrl + up256(sizeof(OrthCtrl));
    w.partial = w.arrive + up256(b ? 4ull * b->n_arrive : 0);
    w.slots = w.partial + up256(b ? 8ull * b->n_chunks : 0);
    w.blocks = w.slots + needs.slots * (128ull * 4) * 128;
    w.total = w.blocks + needs.blocks * kBlock;
    return w;
}

// A tile whose sum is long is split so that the tasks of a phase are about as long as the phase's work spread over
// all SMs, but no part is shorter than kMinPart stages.
constexpr uint64_t kPlanSms = 148, kMinPart = 8, kMaxParts = 16;
// Time of a stage and of what a phase takes besides, in nanoseconds, by kind of tile.
constexpr uint64_t kStageNs[2] = {450, 600}, kTilePhaseNs[2] = {6500, 7500};

// Takes matrices from `at` on into one batch with the given tiles; returns how many, 0 if one is unusable.
uint32_t plan_batch(const co3_mat* in, const co3_mat* out, uint32_t n_mats, uint32_t at, bool muon, uint32_t tile, OrthBatch* b,
                    BatchNeeds* needs) {
    uint32_t n = 0;
    uint64_t work[3] = {0, 0, 0};
    for (; at + n < n_mats && n < kOrthMats; ++n) {
        const co3_mat &ti = in[at + n], &to = out[at + n];
        if (!valid_mat(ti) || !valid_mat(to) || ti.rows != to.rows || ti.cols != to.cols) return 0;
        const bool plain = (to.flags & CO3_MAT_PLAIN) != 0u;
        if (plain && !muon) return 0;
        if (plain || ti.rows == 0 || ti.cols == 0) continue;
        const OrthShape s = orth_shape(ti.rows, ti.cols, tile);
        const uint64_t km = (s.m + 63u) / 64u, kn = (s.n + 63u) / 64u;
        if (s.mb >= (1u << 12) || (uint64_t)s.mb * s.nb >= (1u << 23)) return 0;
        work[kGram] += s.sym * kn;
        work[kPoly] += s.sym * km;
        work[kApply] += orth_apply_tiles(s, false) * km;
    }
    uint64_t chunks = 0, full = 0, arrive = 0, slots = 0, blocks = 0, tasks[3] = {0, 0, 0};
    for (uint32_t k = 0; k < n; ++k) {
        const co3_mat &ti = in[at + k], &to = out[at + k];
        const bool plain = (to.flags & CO3_MAT_PLAIN) != 0u;
        OrthMat& m = b->mat[k];
        m = {};
        m.in_off = ti.offset; m.in_stride = ti.row_stride;
        m.out_off = to.offset; m.out_stride = to.row_stride;
        m.rows = ti.rows; m.cols = ti.cols;
        m.scale = to.scale;
        m.plain = plain ? 1u : 0u;
        m.block0 = (uint32_t)blocks; m.chunk0 = (uint32_t)chunks; m.full0 = (uint32_t)full;
        m.slot0 = (uint32_t)slots; m.arrive0 = (uint32_t)arrive;
        for (int p = 0; p < 3; ++p) { m.task0[p] = (uint32_t)tasks[p]; m.splits[p] = 1u; }
        if (ti.rows == 0 || ti.cols == 0) continue;
        chunks += ((uint64_t)ti.rows * ti.cols + kBeginElems - 1) / kBeginElems;
        if (!plain) {
            const OrthShape s = orth_shape(ti.rows, ti.cols, tile);
            const uint64_t sym = s.sym, all = std::max(orth_apply_tiles(s, false), orth_apply_tiles(s, true));
            uint64_t most = 0;
            for (int p = 0; p < 3; ++p) {
                const uint64_t depth = ((p == kGram ? s.n : s.m) + 63u) / 64u, tiles = p == kApply ? all : sym;
                const uint64_t part = std::max(kMinPart, (work[p] + kPlanSms - 1) / kPlanSms);
                const uint64_t parts = std::min(kMaxParts, std::max<uint64_t>(1, depth / part));
                m.splits[p] = (uint32_t)parts;
                tasks[p] += tiles * parts;
                if (parts > 1) most = std::max(most, tiles * parts);
            }
            slots += most;
            arrive += (2 * sym + all) * 8;
            full += (uint64_t)s.mb * s.nb;
            blocks += orth_blocks(s);
        }
        if (chunks >= (1u << 30) || tasks[0] + tasks[1] + tasks[2] >= (1u << 26) || blocks >= (1ull << 32)) return 0;
    }
    b->n_mats = n;
    b->n_chunks = (uint32_t)chunks;
    b->n_full = (uint32_t)full;
    b->n_arrive = (uint32_t)arrive;
    uint64_t ns = 0;
    for (int p = 0; p < 3; ++p) {
        b->n_tasks[p] = (uint32_t)tasks[p];
        if (tasks[p]) ns += (tasks[p] + kPlanSms - 1) / kPlanSms * work[p] * kStageNs[tile] / tasks[p] + kTilePhaseNs[tile];
    }
    b->index0 = at;
    b->first = at == 0 ? 1u : 0u;
    b->tile = tile;
    *needs = {slots, blocks, work[0] + work[1] + work[2], ns};
    return n;
}

// Times in nanoseconds that decide whether small matrices go to clusters of their own: a step of
// a cluster of one block and of several, and what either call takes besides.
constexpr uint64_t kSmallStepNs[2] = {4000, 7000}, kCallNs = 10000;

// Fills `small` with a batch's matrices and returns true if they are all small and clusters take less time for them.
bool small_batch(const co3_mat* in, const co3_mat* out, uint32_t n_mats, uint32_t at, const OrthBatch& b, const BatchNeeds& needs,
                 uint32_t steps, SmallBatch* small) {
    uint64_t ns = 0, blocks[kSmallCluster + 1] = {};
    small->n_mats = 0;
    for (uint32_t k = 0; k < b.n_mats; ++k) {
        const co3_mat &ti = in[at + k], &to = out[at + k];
        if ((to.flags & CO3_MAT_PLAIN) != 0u || ti.rows == 0 || ti.cols == 0) continue;
        const uint32_t c = small_ctas(ti.rows, ti.cols);
        if (c == 0 || small->n_mats == kSmallMats) return false;
        blocks[c] += c;
        small->mat[small->n_mats++] = {ti.offset, ti.row_stride, to.offset, to.row_stride, ti.rows, ti.cols, to.scale, at + k};
    }
    // clusters that fit the SMs at a time: whole ones within a group of about 16
    for (uint32_t c = 1; c <= kSmallCluster; c *= 2)
        if (blocks[c]) ns += (blocks[c] + (c > 4 ? 127 : 147)) / (c > 4 ? 128 : 148) * steps * kSmallStepNs[c > 1] + kCallNs;
    return small->n_mats > 0 && ns <= steps * needs.ns + 2 * kCallNs;
}

// With the kind of tile that takes the least time.
uint32_t make_batch(const co3_mat* in, const co3_mat* out, uint32_t n_mats, uint32_t at, bool muon, OrthBatch* b, BatchNeeds* needs) {
    uint32_t best = kNarrow;
    uint64_t ns = ~0ull;
    for (uint32_t tile = kNarrow; tile <= kSquare; ++tile) {
        if (plan_batch(in, out, n_mats, at, muon, tile, b, needs) == 0) return 0;
        if (needs->ns < ns) { ns = needs->ns; best = tile; }
    }
    return plan_batch(in, out, n_mats, at, muon, best, b, needs);
}

// Whether every singular value in [0, 1] keeps within the limits.  What a step makes of an interval is an interval, whose
// ends it takes at the ends or where its derivative vanishes; it is widened by kSlack a step for what the products round
// (a few 2^-22), so that an iteration which holds the limits in exact arithmetic alone is refused too.
bool valid_ns(const co3_ns& ns) {
    constexpr double kSlack = 1.0 / 65536, kRoom = 1.0 + 1.0 / 1024;  // fp16 pairs hold four times the limits
    if (ns.steps < 1 || ns.steps > CO3_NS_MAX_STEPS || !(ns.eps >= 0.0f) || !isfinite(ns.eps)) return false;
    double lo = 0.0, hi = 1.0;
    for (uint32_t k = 0; k < ns.steps; ++k) {
        const double a = ns.coef[k][0], b = ns.coef[k][1], c = ns.coef[k][2];
        if (!isfinite(a) || !isfinite(b) || !isfinite(c)) return false;
        lo -= kSlack;
        hi += kSlack;
        // factors b q + c q^2 and a + b q + c q^2 over the squares q
        const double q0 = lo < 0.0 && hi > 0.0 ? 0.0 : std::min(lo * lo, hi * hi), q1 = std::max(lo * lo, hi * hi);
        const double q_top = c != 0.0 ? -b / (2.0 * c) : -1.0;
        for (double q : {q0, q1, q_top > q0 && q_top < q1 ? q_top : q0}) {
            const double g = q * (b + q * c);
            if (!(fabs(g) <= 4.0 * kRoom) || !(fabs(a + g) <= 4.0 * kRoom)) return false;
        }
        auto step = [&](double x) { return x * (a + x * x * (b + x * x * c)); };
        double least = std::min(step(lo), step(hi)), most = std::max(step(lo), step(hi));
        auto turn = [&](double q) {  // a + 3 b q + 5 c q^2 = 0
            if (!(q > 0.0)) return;
            for (double x : {sqrt(q), -sqrt(q)})
                if (x > lo && x < hi) {
                    least = std::min(least, step(x));
                    most = std::max(most, step(x));
                }
        };
        if (c != 0.0) {
            const double d = 9.0 * b * b - 20.0 * a * c;
            if (d >= 0.0) {
                turn((-3.0 * b + sqrt(d)) / (10.0 * c));
                turn((-3.0 * b - sqrt(d)) / (10.0 * c));
            }
        } else if (b != 0.0) {
            turn(-a / (3.0 * b));
        }
        if (!(most <= 2.0 * kRoom) || !(least >= -2.0 * kRoom)) return false;
        lo = least;
        hi = most;
    }
    return true;
}

// Leaves orth_begin_kernel and orth_load_kernel with the plain layers.
void only_plain(OrthBatch* b) {
    uint32_t chunks = 0;
    for (uint32_t k = 0; k < b->n_mats; ++k) {
        OrthMat& m = b->mat[k];
        m.chunk0 = chunks;
        if (m.plain) chunks += (uint32_t)(((uint64_t)m.rows * m.cols + kBeginElems - 1) / kBeginElems);
    }
    b->n_chunks = chunks;
    b->n_full = 0;
}

// All blocks have to be resident at once: one per SM.
template <int kTile>
int launch_steps(const StepArgs& a, uint32_t widest, cudaStream_t st) {
    static std::atomic<int> sms[64];
    int dev = 0;
    CO3_CUDA(cudaGetDevice(&dev));
    int n = dev < 64 ? sms[dev].load(std::memory_order_relaxed) : 0;
    if (n == 0) {
        CO3_CUDA(cudaFuncSetAttribute(orth_steps_kernel<kTile>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kStepSmem));
        CO3_CUDA(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev));
        if (dev < 64) sms[dev].store(n, std::memory_order_relaxed);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(std::min(widest, (uint32_t)n));
    cfg.blockDim = dim3(kStepThreads);
    cfg.dynamicSmemBytes = kStepSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeCooperative;
    attr[0].val.cooperative = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    CO3_CUDA(cudaLaunchKernelEx(&cfg, orth_steps_kernel<kTile>, a));
    return CO3_OK;
}

// The momentum update with the sums of squares, and what it takes of orth_load_kernel's blocks.
template <typename T>
int enqueue_load(const OrthBatch& batch, const BeginArgs& ba, const LoadArgs& la, cudaStream_t st) {
    CO3_CUDA(launch_behind(orth_begin_kernel<T>, dim3(std::max(1u, batch.n_chunks)), dim3(kBeginThreads), 0, st, batch, ba));
    uint32_t blocks = 4u * batch.n_full;
    for (uint32_t k = 0; k < batch.n_mats; ++k)
        if (batch.mat[k].plain) { ++blocks; break; }
    if (blocks) CO3_CUDA(launch_behind(orth_load_kernel<T>, dim3(blocks), dim3(kLoadThreads), 0, st, la));
    return CO3_OK;
}

struct OrthCall {
    const void* in;
    int in_type;
    const co3_mat* in_mats;
    void* out;
    int out_type;
    const co3_mat* out_mats;
    uint32_t n_mats;
    float* momentum;  // null: co3_orthogonalize
    float mu, lr, shrink;
    int nesterov;
};

int orth_run(const OrthCall& c, const co3_ns* ns_in, co3_result* res, void* workspace, size_t workspace_bytes, void* stream) {
    co3_ns ns;
    if (ns_in) ns = *ns_in; else co3_ns_default(&ns);
    if ((ns_in && !valid_ns(ns)) || !res || !aligned(res, 8) || !workspace || !aligned(workspace, 256)) return CO3_ERR_INVALID_ARG;
    size_t need = 0;
    if (c.n_mats && (!c.in || !c.out || !c.in_mats)) return CO3_ERR_INVALID_ARG;
    if (!aligned(c.in, type_size(c.in_type)) || !aligned(c.out, type_size(c.out_type))) return CO3_ERR_INVALID_ARG;
    const bool muon = c.momentum != nullptr;
    OrthBatch batch;
    BatchNeeds needs = {};
    // every matrix is checked before anything is enqueued
    for (uint32_t at = 0; at < c.n_mats;) {
        const uint32_t k = make_batch(c.in_mats, c.out_mats, c.n_mats, at, muon, &batch, &needs);
        if (!k) return CO3_ERR_INVALID_ARG;
        const uint64_t total = ws_plan(&batch, needs).total;
        if (total > need) need = total;
        at += k;
    }
    const uint64_t least = ws_plan(nullptr, BatchNeeds{}).total;
    if (workspace_bytes < (need > least ? need : least)) return CO3_ERR_CAPACITY;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint32_t at = 0;
    do {
        const uint32_t k = make_batch(c.in_mats, c.out_mats, c.n_mats, at, muon, &batch, &needs);
        SmallBatch small;
        const bool is_small = small_batch(c.in_mats, c.out_mats, c.n_mats, at, batch, needs, ns.steps, &small);
        const WsPlan w = ws_plan(&batch, needs);
        if (is_small) only_plain(&batch);
        unsigned char* base = static_cast<unsigned char*>(workspace);
        OrthWs ws = {reinterpret_cast<OrthBatch*>(base + w.batch), reinterpret_cast<OrthCtrl*>(base + w.ctrl),
                     reinterpret_cast<uint32_t*>(base + w.arrive), reinterpret_cast<double*>(base + w.partial),
                     reinterpret_cast<float*>(base + w.slots), base + w.blocks};
        BeginArgs ba = {c.in, c.momentum, static_cast<float*>(c.out), c.mu, c.lr, c.shrink, c.nesterov, res, ws};
        LoadArgs la = {c.in, c.momentum, c.mu, ns.eps, c.nesterov, res, ws};
        int e = CO3_OK;
        if (!is_small || c.n_mats > 1)  // a lone small matrix starts the result itself
            e = c.in_type == CO3_F32 ? enqueue_load<float>(batch, ba, la, st)
                : c.in_type == CO3_F16 ? enqueue_load<__half>(batch, ba, la, st) : enqueue_load<__nv_bfloat16>(batch, ba, la, st);
        if (e != CO3_OK) return e;
        if (is_small) {
            const SmallCall sc = {c.in, c.momentum, c.out, muon ? (int)kOutParams : c.out_type, c.mu, c.lr, c.shrink, c.nesterov, c.n_mats == 1 ? 1 : 0, ns, res};
            e = orth_small_run(small, sc, c.in_type, st);
            if (e != CO3_OK) return e;
        }
        if (batch.n_full) {
            StepArgs sa = {};
            sa.ws = ws;
            sa.ns = ns;
            sa.out_kind = muon ? kOutParams : c.out_type;
            sa.out = c.out;
            sa.lr = c.lr;
            sa.shrink = c.shrink;
            sa.limit_ns = 500000000ull + ns.steps * needs.work * 64ull;
            sa.res = res;
            const uint32_t widest = std::max(batch.n_tasks[0], std::max(batch.n_tasks[1], batch.n_tasks[2]));
            e = batch.tile == kNarrow ? launch_steps<kNarrow>(sa, widest, st) : launch_steps<kSquare>(sa, widest, st);
            if (e != CO3_OK) return e;
        }
        at += k;
    } while (at < c.n_mats);
    return CO3_OK;
}

}  // namespace

extern "C" {

int co3_ns_default(co3_ns* out) {
    if (!out) return CO3_ERR_INVALID_ARG;
    *out = co3_ns{};
    out->steps = 5;
    out->eps = 1e-7f;
    for (uint32_t k = 0; k < 5; ++k) {
        out->coef[k][0] = 3.4445f;
        out->coef[k][1] = -4.7750f;
        out->coef[k][2] = 2.0315f;
    }
    return CO3_OK;
}

int co3_orthogonalize_workspace_bytes(const co3_mat* mats, uint32_t n_mats, size_t* out) {
    if (!out || (n_mats && !mats)) return CO3_ERR_INVALID_ARG;
    uint64_t need = ws_plan(nullptr, BatchNeeds{}).total;
    OrthBatch batch;
    for (uint32_t at = 0; at < n_mats;) {
        BatchNeeds needs = {};
        const uint32_t k = make_batch(mats, mats, n_mats, at, true, &batch, &needs);
        if (!k) return CO3_ERR_INVALID_ARG;
        const uint64_t total = ws_plan(&batch, needs).total;
        if (total > need) need = total;
        at += k;
    }
    *out = (size_t)need;
    return CO3_OK;
}

int co3_orthogonalize(const void* in, int in_type, const co3_mat* in_mats, void* out, int out_type, const co3_mat* out_mats,
                      uint32_t n_mats, const co3_ns* ns, co3_result* res, void* workspace, size_t workspace_bytes, void* stream) {
    if (in_type < CO3_F32 || in_type > CO3_BF16 || out_type < CO3_F32 || out_type > CO3_BF16) return CO3_ERR_INVALID_ARG;
    OrthCall c = {in, in_type, in_mats, out, out_type, out_mats ? out_mats : in_mats, n_mats, nullptr, 0.0f, 0.0f, 0.0f, 0};
    return orth_run(c, ns, res, workspace, workspace_bytes, stream);
}

int co3_muon_update(const float* grad, float* momentum, float* params, const co3_mat* mats, uint32_t n_mats, float mu,
                    int nesterov, float lr, float weight_decay, const co3_ns* ns, co3_result* res, void* workspace,
                    size_t workspace_bytes, void* stream) {
    if (!momentum || !aligned(momentum, 4) || !(mu >= 0.0f && mu <= 1.0f) || !isfinite(lr) || !isfinite(weight_decay))
        return CO3_ERR_INVALID_ARG;
    const float shrink = (float)(1.0 - (double)lr * (double)weight_decay);
    OrthCall c = {grad, CO3_F32, mats, params, CO3_F32, mats, n_mats, momentum, mu, lr, shrink, nesterov};
    return orth_run(c, ns, res, workspace, workspace_bytes, stream);
}

}  // extern "C"
