// Orthogonalised updates: Newton-Schulz steps X <- a X + (b A + c A A) X, A = X X^T, for many matrices at once, on the
// fifth-generation tensor cores.
//
//   orth_begin_kernel   (momentum update +) sum of squares of every matrix
//   orth_load_kernel    X_0 = G / (norm + eps) as operand blocks, as it is and transposed
//   orth_steps_kernel   all products of all steps in one cooperative launch: per step A = X X^T; B = b A + c A A;
//                       X <- a X + B X; the last product writes the result (or steps the parameters) instead of X
//
// Operands live in the workspace as blocks of 128 rows x 64 columns, each a pair of fp16 planes of 16 KB: hi = the
// value rounded, lo = 2^11 times the remainder rounded, together 22 significant bits.  A plane is stored exactly as
// the tensor core wants it in shared memory (128-byte rows, 16-byte pieces XORed with the row number modulo 8), so
// that a tile is fetched by one plain bulk copy, and padding of the matrix to whole blocks is stored as zeros.  A
// product is hi*hi + 2^-11 (hi*lo + lo*hi): the part left out, lo*lo, is below 2^-22 of the whole.
#include <cuda_runtime.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "co3.h"
#include "co3_device.cuh"
#include "co3_launch.cuh"
#include "co3_types.cuh"

namespace co3 {

constexpr uint32_t kOrthMats = 96;                  // matrices of one batch of launches
constexpr uint32_t kPlane = 128 * 64 * 2;           // bytes of a plane of a block
constexpr uint32_t kBlock = 2 * kPlane;             // hi, then lo
constexpr uint32_t kBeginElems = 8192;              // elements per block of orth_begin_kernel
constexpr int kBeginThreads = 256;
constexpr int kLoadThreads = 256;
constexpr float kLoScale = 2048.0f;
constexpr int kMaxLogS = 13;                        // values are held times S = 2^min(13, log2 sqrt(m n)): entries about 1

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
    uint32_t pad;
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

struct OrthShape {
    uint32_t m, n, mb, nb;  // small side, long side, and both in blocks of 128
    bool tall;              // rows > cols: X is the transposed matrix
};

__host__ __device__ inline OrthShape orth_shape(uint32_t rows, uint32_t cols) {
    OrthShape s;
    s.tall = rows > cols;
    s.m = s.tall ? cols : rows;
    s.n = s.tall ? rows : cols;
    s.mb = (s.m + 127u) / 128u;
    s.nb = (s.n + 127u) / 128u;
    return s;
}

// Operand blocks of one matrix: X [mb][2 nb], X^T twice [nb][2 mb], A and B [mb][2 mb].
__host__ __device__ inline uint64_t orth_blocks(const OrthShape& s) {
    return 6ull * s.mb * s.nb + 4ull * s.mb * s.mb;
}
struct OrthOperands {
    unsigned char *x, *xt[2], *a, *b;
};
__device__ inline OrthOperands orth_operands(const OrthWs& ws, const OrthMat& t, const OrthShape& s) {
    OrthOperands o;
    const uint64_t xs = 2ull * s.mb * s.nb * kBlock;
    o.x = ws.blocks + (uint64_t)t.block0 * kBlock;
    o.xt[0] = o.x + xs;
    o.xt[1] = o.xt[0] + xs;
    o.a = o.xt[1] + xs;
    o.b = o.a + 2ull * s.mb * s.mb * kBlock;
    return o;
}

__host__ __device__ inline float orth_s(const OrthShape& s) {
    const uint64_t p = (uint64_t)s.m * s.n;
    int k = 0;
    while (k < kMaxLogS && (1ull << (2 * (k + 1))) <= p) ++k;
    return (float)(1u << k);
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
        if (!isfinite(s) && a.momentum && t.plain) set_status(a.res, CO3_ERR_NONFINITE);
    }
}

// ------------------------------------------------------------------------------------------------
// load: one block per 64 x 64 piece of X (padding included): both operand layouts of S * G / (norm + eps).
// ------------------------------------------------------------------------------------------------
struct LoadArgs {
    const void* in;
    const float* momentum;  // null: orthogonalize only
    float mu, eps;
    int nesterov;
    co3_result* res;
    OrthWs ws;
};

__device__ __forceinline__ uint32_t swizzled(uint32_t row, uint32_t piece) { return row * 128u + ((piece ^ (row & 7u)) << 4); }

__device__ __forceinline__ uint32_t pack_halves(__half a, __half b) {
    return (uint32_t)__half_as_ushort(a) | ((uint32_t)__half_as_ushort(b) << 16);
}

// hi and lo of eight values, as 16-byte pieces.
__device__ __forceinline__ void split8(const float (&v)[8], uint4& hi, uint4& lo) {
    __half h[8], l[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        h[i] = __float2half_rn(v[i]);
        l[i] = __float2half_rn(__fmul_rn(__fsub_rn(v[i], __half2float(h[i])), kLoScale));
    }
    hi = make_uint4(pack_halves(h[0], h[1]), pack_halves(h[2], h[3]), pack_halves(h[4], h[5]), pack_halves(h[6], h[7]));
    lo = make_uint4(pack_halves(l[0], l[1]), pack_halves(l[2], l[3]), pack_halves(l[4], l[5]), pack_halves(l[6], l[7]));
}

__device__ __forceinline__ void join8(const uint4& hi, const uint4& lo, float (&v)[8]) {
    const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w}, l[4] = {lo.x, lo.y, lo.z, lo.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = __half2float(__ushort_as_half((unsigned short)(h[i / 2] >> (16 * (i & 1)))));
        const float b = __half2float(__ushort_as_half((unsigned short)(l[i / 2] >> (16 * (i & 1)))));
        v[i] = __fmaf_rn(b, 1.0f / kLoScale, a);
    }
}

template <typename T>
__global__ void __launch_bounds__(kLoadThreads) orth_load_kernel(LoadArgs a) {
    wait_for_previous_kernel();
    __shared__ float s_v[64][65];
    __shared__ double s_sum[kLoadThreads / 32];
    __shared__ double s_f;
    const OrthBatch& batch = *a.ws.batch;
    const uint32_t tile = blockIdx.x >> 2;  // tile of 128 x 128, quarter blockIdx.x & 3
    const uint32_t k = orth_find(batch.n_mats, tile, [&](uint32_t i) { return batch.mat[i].full0; });
    const OrthMat t = batch.mat[k];
    const OrthShape s = orth_shape(t.rows, t.cols);
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
        s_f = d > 0.0 ? (double)orth_s(s) / d : 0.0;  // an all-zero matrix without eps stays zero
        if (!isfinite(total) && tile == t.full0 && (blockIdx.x & 3u) == 0) {
            set_status(a.res, CO3_ERR_NONFINITE);
            atomicMin(&a.res->first_bad_chunk, batch.index0 + k);
            atomicAdd(reinterpret_cast<unsigned long long*>(&a.res->n_nonfinite), 1ull);
            s_f = (double)NAN;
        }
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
    unsigned char* xb = op.x + ((uint64_t)(x_row0 >> 7) * (2 * s.nb) + (x_col0 >> 6)) * kBlock;
    unsigned char* tb = op.xt[0] + ((uint64_t)(x_col0 >> 7) * (2 * s.mb) + (x_row0 >> 6)) * kBlock;
    const uint32_t xr = x_row0 & 64u, tr = x_col0 & 64u;
    for (uint32_t i = threadIdx.x; i < 2 * 64 * 8; i += kLoadThreads) {
        const bool tr_part = i >= 64 * 8;
        const uint32_t row = (i >> 3) & 63u, piece = i & 7u;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tr_part ? s_v[piece * 8 + e][row] : s_v[row][piece * 8 + e];
        uint4 hi, lo;
        split8(v, hi, lo);
        unsigned char* p = (tr_part ? tb : xb) + swizzled(row + (tr_part ? tr : xr), piece);
        *reinterpret_cast<uint4*>(p) = hi;
        *reinterpret_cast<uint4*>(p + kPlane) = lo;
    }
}

// ------------------------------------------------------------------------------------------------
// tcgen05: operands in shared memory (K-major, 128-byte swizzle), fp32 accumulators in tensor memory.
// ------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr) {
    // start address, leading offset 16 (unused with this swizzle), 1024 bytes between groups of eight rows, the
    // fixed version bit of this architecture, 128-byte swizzle
    return (uint64_t)((addr >> 4) & 0x3fffu) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// D fp32, A and B fp16, both K-major, M = 128, N = 128
constexpr uint32_t kInstrDesc = (1u << 4) | ((128u / 8u) << 17) | ((128u / 16u) << 24);

__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(kInstrDesc),
        "r"((uint32_t)accumulate)
        : "memory");
}
__device__ __forceinline__ void tc_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}
// 32 columns of this warp's 32 lanes
__device__ __forceinline__ void tc_load32(uint32_t addr, float (&v)[32]) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// ------------------------------------------------------------------------------------------------
// steps: persistent blocks (all resident: a cooperative launch).  The products of all steps form one list of tasks,
// phase by phase; a task is a 128 x 128 tile, or a part of its sum where there are fewer tiles than SMs.  Block b takes
// tasks b, b + gridDim.x, ... in order, and before a task's operands are fetched it waits until the matrix' tiles of
// the phases before it are finished (a counter per matrix): the tasks waited for stand earlier in the list, so that
// waiting always ends, and one matrix' tail is filled with other matrices' work.
//
// Warp 0 copies operand blocks into a ring, warp 1 issues the products, warps 2..9 take the accumulators: each of them
// 32 rows x 64 columns of the tile in registers.
// ------------------------------------------------------------------------------------------------
constexpr int kEpiThreads = 256;
constexpr int kStepThreads = 64 + kEpiThreads;
constexpr int kStages = 3;
// The tensor core cuts what it adds to 26 bits below the largest term, always towards zero: sums of one sign (the
// diagonal of A) drift.  Sums of this many stages (64 columns each) are therefore added up in registers, where fp32
// rounds to nearest.  1000 x 513, five steps, error against 64 bits: 1.3e-5 if never, 6.1e-6 every 4 stages, 2.1e-6
// every stage (2.9e-6 with all sums in fp32 arithmetic).
constexpr uint32_t kDrain = 1;
constexpr uint32_t kStageBytes = 2 * kBlock;
constexpr uint32_t kPitch = 129;  // floats between columns of the staged half tile

struct StepSmem {
    uint64_t full[kStages], empty[kStages];
    uint64_t main_full[2], main_empty[2], corr_full[2], corr_empty[2];
    uint64_t done;
    uint32_t tmem, failed, last;
    uint32_t task0[3][kOrthMats];
};
constexpr size_t kStageOff = (size_t)kStages * kStageBytes;
constexpr size_t kSmemOff = kStageOff + 64 * kPitch * 4;
constexpr size_t kStepSmem = 1024 + kSmemOff + sizeof(StepSmem);
static_assert(kStepSmem <= 227 * 1024 && kSmemOff % 8 == 0, "shared memory of a block");

enum OrthOut { kOutF32 = 0, kOutF16 = 1, kOutBf16 = 2, kOutParams = 3 };

struct StepArgs {
    OrthWs ws;
    co3_ns ns;
    uint32_t pairs;  // bit k: step k multiplies pairs (three products), otherwise the hi planes alone
    int out_kind;
    void* out;
    float lr, shrink;
    uint64_t limit_ns;  // longest wait
    co3_result* res;
};

struct Task {
    uint32_t step, phase, mat;
    uint32_t i, j;           // block row and column of the tile (kApply: i of the small side, j of the long side)
    uint32_t part, parts;
    uint32_t k0, k1;         // operand blocks of the summed dimension
    uint32_t tile;           // index within the matrix and phase
    uint32_t before;         // tiles of this matrix that have to be finished
    bool swap;               // kApply: the tile's rows are the long side
};

struct MatView {
    OrthMat t;
    OrthShape s;
    OrthOperands op;
};

__device__ __forceinline__ Task find_task(const StepArgs& a, const StepSmem& sm, const uint32_t* n_tasks, uint32_t n_mats, uint32_t g, MatView& v) {
    Task k;
    const uint32_t per_step = n_tasks[0] + n_tasks[1] + n_tasks[2];
    k.step = g / per_step;
    uint32_t x = g - k.step * per_step;
    k.phase = 0;
    while (x >= n_tasks[k.phase]) x -= n_tasks[k.phase++];
    const uint32_t* first = sm.task0[k.phase];
    k.mat = orth_find(n_mats, x, [&](uint32_t i) { return first[i]; });
    v.t = a.ws.batch->mat[k.mat];
    v.s = orth_shape(v.t.rows, v.t.cols);
    v.op = orth_operands(a.ws, v.t, v.s);
    x -= first[k.mat];
    k.parts = v.t.splits[k.phase];
    k.tile = x / k.parts;
    k.part = x - k.tile * k.parts;
    const uint32_t sym = v.s.mb * (v.s.mb + 1) / 2;
    k.before = k.step * (2 * sym + v.s.mb * v.s.nb) + k.phase * sym;
    k.swap = false;
    uint32_t blocks;
    if (k.phase == kApply) {
        k.i = k.tile / v.s.nb;
        k.j = k.tile - k.i * v.s.nb;
        // in the last product of a matrix that is not tall the tile's rows are the long side, so that a warp's rows
        // are neighbours in the caller's memory
        k.swap = k.step + 1 == a.ns.steps && !v.s.tall;
        blocks = (v.s.m + 63u) / 64u;
    } else {  // the triangle i >= j
        uint32_t i = (uint32_t)((sqrtf(8.0f * (float)k.tile + 1.0f) - 1.0f) * 0.5f);
        while (i * (i + 1) / 2 > k.tile) --i;
        while ((i + 1) * (i + 2) / 2 <= k.tile) ++i;
        k.i = i;
        k.j = k.tile - i * (i + 1) / 2;
        blocks = ((k.phase == kGram ? v.s.n : v.s.m) + 63u) / 64u;
    }
    k.k0 = (uint32_t)((uint64_t)blocks * k.part / k.parts);
    k.k1 = (uint32_t)((uint64_t)blocks * (k.part + 1) / k.parts);
    return k;
}

__device__ __forceinline__ uint32_t load_acquire(const uint32_t* p) {
    uint32_t v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void fence_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }

__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, uint64_t limit_ns) {
    if (mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = global_timer_ns();
    for (;;) {
        for (int i = 0; i < 64; ++i)
            if (mbar_try_wait(bar, parity)) return true;
        if (global_timer_ns() - t0 > limit_ns) return false;
    }
}

// Waits until at least `need` tiles of a matrix are finished.
__device__ __forceinline__ bool wait_tiles(const OrthCtrl* ctrl, uint32_t mat, uint32_t need, uint64_t limit_ns) {
    if (load_acquire(&ctrl->done[mat]) >= need) return true;
    const uint64_t t0 = global_timer_ns();
    for (uint32_t i = 1;; ++i) {
        if (load_acquire(&ctrl->done[mat]) >= need) return true;
        if ((i & 255u) == 0 && (load_acquire(&ctrl->abort) != 0u || global_timer_ns() - t0 > limit_ns)) return false;
    }
}

__device__ __forceinline__ void epi_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
// The same, and whether any of the threads says so.
__device__ __forceinline__ bool epi_any(bool x) {
    uint32_t any;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 q, %1, 0;\n\t"
        "bar.red.or.pred p, 1, 256, q;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(any)
        : "r"((uint32_t)x)
        : "memory");
    return any != 0u;
}

__global__ void __launch_bounds__(kStepThreads, 1) orth_steps_kernel(const __grid_constant__ StepArgs a) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* ring = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    float* stage = reinterpret_cast<float*>(ring + kStageOff);
    StepSmem& sm = *reinterpret_cast<StepSmem*>(ring + kSmemOff);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const uint32_t n_mats = a.ws.batch->n_mats;
    const uint32_t n_tasks[3] = {a.ws.batch->n_tasks[0], a.ws.batch->n_tasks[1], a.ws.batch->n_tasks[2]};
    const uint32_t total = a.ns.steps * (n_tasks[0] + n_tasks[1] + n_tasks[2]);
    for (uint32_t i = threadIdx.x; i < n_mats; i += kStepThreads)
        for (int p = 0; p < 3; ++p) sm.task0[p][i] = a.ws.batch->mat[i].task0[p];
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) { mbar_init(&sm.full[i], 1); mbar_init(&sm.empty[i], 1); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm.main_full[i], 1);
            mbar_init(&sm.main_empty[i], kEpiThreads);
            mbar_init(&sm.corr_full[i], 1);
            mbar_init(&sm.corr_empty[i], kEpiThreads);
        }
        mbar_init(&sm.done, 1);
        sm.failed = 0;
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&sm.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm.tmem;  // columns: main 0..127, 128..255; corrections 256..383, 384..511
    volatile uint32_t* failed = &sm.failed;
    MatView v;

    if (warp == 0 && lane == 0) {
        uint32_t it = 0;
        for (uint32_t g = blockIdx.x; g < total && !*failed; g += gridDim.x) {
            const Task k = find_task(a, sm, n_tasks, n_mats, g, v);
            const unsigned char *pa, *pb;
            if (k.phase == kGram) {
                pa = v.op.x + (uint64_t)k.i * (2 * v.s.nb) * kBlock;
                pb = v.op.x + (uint64_t)k.j * (2 * v.s.nb) * kBlock;
            } else if (k.phase == kPoly) {
                pa = v.op.a + (uint64_t)k.i * (2 * v.s.mb) * kBlock;
                pb = v.op.a + (uint64_t)k.j * (2 * v.s.mb) * kBlock;
            } else {
                const unsigned char* b = v.op.b + (uint64_t)k.i * (2 * v.s.mb) * kBlock;
                const unsigned char* x = v.op.xt[k.step & 1u] + (uint64_t)k.j * (2 * v.s.mb) * kBlock;
                pa = k.swap ? x : b;
                pb = k.swap ? b : x;
            }
            const uint32_t bytes = (a.pairs >> k.step) & 1u ? kBlock : kPlane;
            if (!wait_tiles(a.ws.ctrl, k.mat, k.before, a.limit_ns)) { *failed = 1; break; }
            fence_async_all();  // the blocks were written by ordinary stores of other SMs
            for (uint32_t q = k.k0; q < k.k1; ++q, ++it) {
                const uint32_t st = it % kStages;
                if (it >= (uint32_t)kStages && !wait_for(&sm.empty[st], (it / kStages - 1) & 1u, a.limit_ns)) { *failed = 1; break; }
                unsigned char* dst = ring + (size_t)st * kStageBytes;
                mbar_arrive_expect_tx(&sm.full[st], 2 * bytes);
                bulk_copy_g2s(dst, pa + (uint64_t)q * kBlock, bytes, &sm.full[st]);
                bulk_copy_g2s(dst + kBlock, pb + (uint64_t)q * kBlock, bytes, &sm.full[st]);
            }
        }
        // copies in flight end before the block does, whoever else has given up
        for (uint32_t q = it > (uint32_t)kStages ? it - kStages : 0; q < it; ++q) mbar_wait(&sm.full[q % kStages], (q / kStages) & 1u);
    } else if (warp == 1 && lane == 0) {
        uint32_t it = 0, chunk = 0, tile = 0;
        for (uint32_t g = blockIdx.x; g < total && !*failed; g += gridDim.x) {
            const Task k = find_task(a, sm, n_tasks, n_mats, g, v);
            const bool pairs = (a.pairs >> k.step) & 1u;
            const uint32_t drain = pairs ? kDrain : k.k1 - k.k0;
            const uint32_t tb = tile & 1u, corr = tmem + 256u + tb * 128u;
            if (pairs && tile >= 2 && !wait_for(&sm.corr_empty[tb], (tile / 2 - 1) & 1u, a.limit_ns)) { *failed = 1; break; }
            bool ok = true;
            for (uint32_t q = k.k0; q < k.k1; ++q, ++it) {
                const uint32_t st = it % kStages, n = q - k.k0, in_chunk = n % drain;
                const uint32_t cb = chunk & 1u, main = tmem + cb * 128u;
                if (in_chunk == 0 && chunk >= 2 && !wait_for(&sm.main_empty[cb], (chunk / 2 - 1) & 1u, a.limit_ns)) { ok = false; break; }
                if (!wait_for(&sm.full[st], (it / kStages) & 1u, a.limit_ns)) { ok = false; break; }
                tc_fence_after();
                const uint32_t at = smem_addr(ring + (size_t)st * kStageBytes);
                const uint64_t ah = smem_desc(at), al = smem_desc(at + kPlane);
                const uint64_t bh = smem_desc(at + kBlock), bl = smem_desc(at + kBlock + kPlane);
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) tc_mma(main, ah + 2 * e, bh + 2 * e, in_chunk + e > 0);
                if (in_chunk == drain - 1 || q + 1 == k.k1) { tc_commit(&sm.main_full[cb]); ++chunk; }
                if (pairs) {
#pragma unroll
                    for (uint32_t e = 0; e < 4; ++e) tc_mma(corr, ah + 2 * e, bl + 2 * e, n + e > 0);
#pragma unroll
                    for (uint32_t e = 0; e < 4; ++e) tc_mma(corr, al + 2 * e, bh + 2 * e, true);
                }
                tc_commit(&sm.empty[st]);
            }
            if (!ok) { *failed = 1; break; }
            if (pairs) { tc_commit(&sm.corr_full[tb]); ++tile; }
        }
        tc_commit(&sm.done);
        mbar_wait(&sm.done, 0);
    } else if (warp >= 2) {
        const uint32_t et = threadIdx.x - 64u, quad = warp & 3u, half = (warp - 2u) >> 2;
        const uint32_t row = quad * 32u + lane;
        const uint32_t lane_base = tmem + ((quad * 32u) << 16) + half * 64u;
        uint32_t chunk = 0, tile = 0;
        for (uint32_t g = blockIdx.x; g < total; g += gridDim.x) {
            const Task k = find_task(a, sm, n_tasks, n_mats, g, v);
            const bool pairs = (a.pairs >> k.step) & 1u;
            const uint32_t drain = pairs ? kDrain : k.k1 - k.k0;
            float acc[64];
#pragma unroll
            for (int i = 0; i < 64; ++i) acc[i] = 0.0f;
            bool ok = true;
            for (uint32_t q = k.k0; q < k.k1; q += drain, ++chunk) {
                const uint32_t cb = chunk & 1u;
                ok = wait_for(&sm.main_full[cb], (chunk / 2) & 1u, a.limit_ns);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                tc_fence_after();
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float w[32];
                    tc_load32(lane_base + cb * 128u + h * 32u, w);
#pragma unroll
                    for (int i = 0; i < 32; ++i) acc[h * 32 + i] = __fadd_rn(acc[h * 32 + i], w[i]);
                }
                tc_fence_before();
                mbar_arrive(&sm.main_empty[cb]);
            }
            if (ok && pairs) {
                const uint32_t tb = tile & 1u;
                ok = __all_sync(0xffffffffu, wait_for(&sm.corr_full[tb], (tile / 2) & 1u, a.limit_ns));
                if (ok) {
                    tc_fence_after();
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float w[32];
                        tc_load32(lane_base + 256u + tb * 128u + h * 32u, w);
#pragma unroll
                        for (int i = 0; i < 32; ++i) acc[h * 32 + i] = __fmaf_rn(w[i], 1.0f / kLoScale, acc[h * 32 + i]);
                    }
                    tc_fence_before();
                    mbar_arrive(&sm.corr_empty[tb]);
                    ++tile;
                }
            }
            if (epi_any(!ok)) { *failed = 1; break; }

            if (k.parts > 1) {
                // this part's sums into its slot; the part that arrives last adds all of them in order
                float* mine = a.ws.slots + ((uint64_t)v.t.slot0 + k.tile * k.parts + k.part) * (128 * 128);
#pragma unroll
                for (int i = 0; i < 64; ++i) __stcg(mine + (half * 64 + i) * 128 + row, acc[i]);
                __threadfence();
                epi_sync();
                if (et == 0) {
                    const uint32_t sym = v.s.mb * (v.s.mb + 1) / 2;
                    const uint32_t old = atomicAdd(a.ws.arrive + v.t.arrive0 + k.phase * sym + k.tile, 1u);
                    __threadfence();
                    sm.last = old == k.step * k.parts + k.parts - 1 ? 1u : 0u;
                }
                epi_sync();
                if (!sm.last) continue;
#pragma unroll
                for (int i = 0; i < 64; ++i) acc[i] = 0.0f;
                for (uint32_t p = 0; p < k.parts; ++p) {
                    const float* from = a.ws.slots + ((uint64_t)v.t.slot0 + k.tile * k.parts + p) * (128 * 128);
#pragma unroll
                    for (int i = 0; i < 64; ++i) acc[i] = __fadd_rn(acc[i], __ldcg(from + (half * 64 + i) * 128 + row));
                }
            }

            const float s_val = orth_s(v.s), inv_s = 1.0f / s_val;
            const bool last = k.phase == kApply && k.step + 1 == a.ns.steps;
            const float ca = a.ns.coef[k.step][0], cb = a.ns.coef[k.step][1], cc = a.ns.coef[k.step][2];
            const uint32_t row_blk = k.swap ? k.j : k.i, col_blk = k.swap ? k.i : k.j;
            const uint32_t n_rows = k.phase == kApply ? (k.swap ? v.s.n : v.s.m) : v.s.m;
            const uint32_t n_cols = k.phase == kApply ? (k.swap ? v.s.m : v.s.n) : v.s.m;
            // rows and columns up to a multiple of 64 are written: beyond, no product reads them
            const uint32_t rows_used = n_rows - row_blk * 128u > 64u ? 128u : 64u;
            const uint32_t halves = n_cols - col_blk * 128u > 64u ? 2u : 1u;
            // the tile's own blocks: linear term, destination, destination of the transposed tile
            const uint64_t at_m = ((uint64_t)k.i * (2 * v.s.mb) + 2 * k.j) * kBlock;  // in an m x m operand
            const uint64_t at_mt = ((uint64_t)k.j * (2 * v.s.mb) + 2 * k.i) * kBlock;
            const uint64_t at_x = ((uint64_t)k.i * (2 * v.s.nb) + 2 * k.j) * kBlock;
            const unsigned char* lin = nullptr;
            unsigned char *dst = nullptr, *dst_t = nullptr;
            float fl, fa;  // value = fl * linear + fa * sum
            if (k.phase == kGram) {
                dst = v.op.a + at_m;
                dst_t = k.i != k.j ? v.op.a + at_mt : nullptr;
                fl = 0.0f; fa = inv_s;
            } else if (k.phase == kPoly) {
                lin = v.op.a + at_m;
                dst = v.op.b + at_m;
                dst_t = k.i != k.j ? v.op.b + at_mt : nullptr;
                fl = cb; fa = __fmul_rn(cc, inv_s);
            } else {
                lin = k.swap ? v.op.xt[k.step & 1u] + at_mt : v.op.x + at_x;
                dst = last ? nullptr : v.op.x + at_x;
                dst_t = last ? nullptr : v.op.xt[(k.step & 1u) ^ 1u] + at_mt;
                fl = ca; fa = inv_s;
                if (last) {
                    const float f = __fmul_rn(v.t.scale, inv_s);
                    fl = __fmul_rn(fl, f);
                    fa = __fmul_rn(fa, f);
                }
            }
            for (uint32_t h = 0; h < halves; ++h) {
                if (half == h) {
#pragma unroll
                    for (int i = 0; i < 64; ++i) stage[i * kPitch + row] = acc[i];
                }
                epi_sync();
                for (uint32_t i = et; i < rows_used * 8u; i += kEpiThreads) {
                    const uint32_t r = i >> 3, piece = i & 7u;
                    const uint64_t at = (uint64_t)h * kBlock + swizzled(r, piece);
                    float w[8], l[8];
                    if (lin) join8(__ldcg(reinterpret_cast<const uint4*>(lin + at)), __ldcg(reinterpret_cast<const uint4*>(lin + at + kPlane)), l);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        w[e] = __fmul_rn(fa, stage[(piece * 8 + e) * kPitch + r]);
                        if (lin) w[e] = __fmaf_rn(fl, l[e], w[e]);
                    }
                    if (last) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) stage[(piece * 8 + e) * kPitch + r] = w[e];
                    } else {
                        uint4 hi, lo;
                        split8(w, hi, lo);
                        *reinterpret_cast<uint4*>(dst + at) = hi;
                        *reinterpret_cast<uint4*>(dst + at + kPlane) = lo;
                        if (dst_t) {
                            const uint32_t hs[4] = {hi.x, hi.y, hi.z, hi.w}, ls[4] = {lo.x, lo.y, lo.z, lo.w};
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                stage[(piece * 8 + e) * kPitch + r] = __uint_as_float(__byte_perm(hs[e / 2], ls[e / 2], e & 1 ? 0x7632 : 0x5410));
                        }
                    }
                }
                epi_sync();
                if (last) {
                    const uint32_t c = row_blk * 128u + (et & 127u);
                    if (c < v.t.cols) {
                        for (uint32_t i = et >> 7; i < 64u; i += 2) {
                            const uint32_t r = col_blk * 128u + h * 64u + i;
                            if (r >= v.t.rows) break;
                            const float o = stage[i * kPitch + (et & 127u)];
                            const uint64_t at = v.t.out_off + (uint64_t)r * v.t.out_stride + c;
                            if (a.out_kind == kOutF32) static_cast<float*>(a.out)[at] = o;
                            else if (a.out_kind == kOutF16) static_cast<__half*>(a.out)[at] = __float2half_rn(o);
                            else if (a.out_kind == kOutBf16) static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(o);
                            else {
                                float* p = static_cast<float*>(a.out) + at;
                                *p = __fmaf_rn(-a.lr, o, __fmul_rn(a.shrink, *p));
                            }
                        }
                    }
                } else if (dst_t) {
                    for (uint32_t i = et; i < 64u * 16u; i += kEpiThreads) {
                        const uint32_t c = i >> 4, piece = i & 15u;
                        if (piece * 8u >= rows_used) continue;
                        uint32_t hs[4], ls[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t p = __float_as_uint(stage[c * kPitch + piece * 8 + 2 * e]);
                            const uint32_t q = __float_as_uint(stage[c * kPitch + piece * 8 + 2 * e + 1]);
                            hs[e] = __byte_perm(p, q, 0x5410);
                            ls[e] = __byte_perm(p, q, 0x7632);
                        }
                        unsigned char* to = dst_t + (uint64_t)(piece >> 3) * kBlock + swizzled(h * 64u + c, piece & 7u);
                        *reinterpret_cast<uint4*>(to) = make_uint4(hs[0], hs[1], hs[2], hs[3]);
                        *reinterpret_cast<uint4*>(to + kPlane) = make_uint4(ls[0], ls[1], ls[2], ls[3]);
                    }
                }
                if (h + 1 < halves) epi_sync();
            }
            if (!last) {
                fence_async_all();  // the next products fetch these blocks with bulk copies
                __threadfence();
                epi_sync();
                if (et == 0) asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(&a.ws.ctrl->done[k.mat]) : "memory");
            } else {
                epi_sync();  // the staged half is free again
            }
        }
    }
    __syncthreads();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
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
};
WsPlan ws_plan(const OrthBatch* b, const BatchNeeds& needs) {
    WsPlan w;
    w.batch = 0;
    w.ctrl = up256(sizeof(OrthBatch));
    w.arrive = w.ctrl + up256(sizeof(OrthCtrl));
    w.partial = w.arrive + up256(b ? 4ull * b->n_arrive : 0);
    w.slots = w.partial + up256(b ? 8ull * b->n_chunks : 0);
    w.blocks = w.slots + needs.slots * (128 * 128 * 4);
    w.total = w.blocks + needs.blocks * kBlock;
    return w;
}

// A tile whose sum is long is split so that the tasks of a phase are about as long as the phase's work spread over
// all SMs, but no part is shorter than kMinPart stages.
constexpr uint64_t kPlanSms = 148, kMinPart = 8, kMaxParts = 16;

// Takes matrices from `at` on into one batch; returns how many, 0 if one is unusable.
uint32_t make_batch(const co3_mat* in, const co3_mat* out, uint32_t n_mats, uint32_t at, bool muon, OrthBatch* b,
                    BatchNeeds* needs) {
    uint32_t n = 0;
    uint64_t work[3] = {0, 0, 0};
    for (; at + n < n_mats && n < kOrthMats; ++n) {
        const co3_mat &ti = in[at + n], &to = out[at + n];
        if (!valid_mat(ti) || !valid_mat(to) || ti.rows != to.rows || ti.cols != to.cols) return 0;
        const bool plain = (to.flags & CO3_MAT_PLAIN) != 0u;
        if (plain && !muon) return 0;
        if (plain || ti.rows == 0 || ti.cols == 0) continue;
        const OrthShape s = orth_shape(ti.rows, ti.cols);
        const uint64_t sym = (uint64_t)s.mb * (s.mb + 1) / 2, km = (s.m + 63u) / 64u, kn = (s.n + 63u) / 64u;
        if (sym >= (1u << 24) || (uint64_t)s.mb * s.nb >= (1u << 24)) return 0;
        work[kGram] += sym * kn;
        work[kPoly] += sym * km;
        work[kApply] += (uint64_t)s.mb * s.nb * km;
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
            const OrthShape s = orth_shape(ti.rows, ti.cols);
            const uint64_t sym = (uint64_t)s.mb * (s.mb + 1) / 2;
            uint64_t most = 0;
            for (int p = 0; p < 3; ++p) {
                const uint64_t depth = ((p == kGram ? s.n : s.m) + 63u) / 64u, tiles = p == kApply ? (uint64_t)s.mb * s.nb : sym;
                const uint64_t part = std::max(kMinPart, (work[p] + kPlanSms - 1) / kPlanSms);
                const uint64_t parts = std::min(kMaxParts, std::max<uint64_t>(1, depth / part));
                m.splits[p] = (uint32_t)parts;
                tasks[p] += tiles * parts;
                if (parts > 1) most = std::max(most, tiles * parts);
            }
            slots += most;
            arrive += 2 * sym + (uint64_t)s.mb * s.nb;
            full += (uint64_t)s.mb * s.nb;
            blocks += orth_blocks(s);
        }
        if (chunks >= (1u << 30) || tasks[0] + tasks[1] + tasks[2] >= (1u << 26) || blocks >= (1ull << 32)) return 0;
    }
    b->n_mats = n;
    b->n_chunks = (uint32_t)chunks;
    b->n_full = (uint32_t)full;
    b->n_arrive = (uint32_t)arrive;
    for (int p = 0; p < 3; ++p) b->n_tasks[p] = (uint32_t)tasks[p];
    b->index0 = at;
    b->first = at == 0 ? 1u : 0u;
    *needs = {slots, blocks, work[0] + work[1] + work[2]};
    return n;
}

bool valid_ns(const co3_ns& ns) {
    if (ns.steps < 1 || ns.steps > CO3_NS_MAX_STEPS || !(ns.eps >= 0.0f) || !isfinite(ns.eps)) return false;
    for (uint32_t k = 0; k < ns.steps; ++k)
        for (int j = 0; j < 3; ++j)
            if (!isfinite(ns.coef[k][j])) return false;
    for (int i = 0; i <= 4096; ++i) {
        double x = i / 4096.0;
        for (uint32_t k = 0; k < ns.steps; ++k) {
            const double q = x * x, g = q * (ns.coef[k][1] + q * ns.coef[k][2]);
            if (!(fabs(g) <= 4.0)) return false;
            x *= ns.coef[k][0] + g;
            if (!(fabs(x) <= 2.0)) return false;
        }
    }
    return true;
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
    if (!valid_ns(ns) || !res || !aligned(res, 8) || !workspace || !aligned(workspace, 256)) return CO3_ERR_INVALID_ARG;
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
    int dev = 0, sms = 0;
    CO3_CUDA(cudaGetDevice(&dev));
    CO3_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint32_t at = 0;
    do {
        const uint32_t k = make_batch(c.in_mats, c.out_mats, c.n_mats, at, muon, &batch, &needs);
        const WsPlan w = ws_plan(&batch, needs);
        unsigned char* base = static_cast<unsigned char*>(workspace);
        OrthWs ws = {reinterpret_cast<OrthBatch*>(base + w.batch), reinterpret_cast<OrthCtrl*>(base + w.ctrl),
                     reinterpret_cast<uint32_t*>(base + w.arrive), reinterpret_cast<double*>(base + w.partial),
                     reinterpret_cast<float*>(base + w.slots), base + w.blocks};
        BeginArgs ba = {c.in, c.momentum, static_cast<float*>(c.out), c.mu, c.lr, c.shrink, c.nesterov, res, ws};
        LoadArgs la = {c.in, c.momentum, c.mu, ns.eps, c.nesterov, res, ws};
        const dim3 bg(batch.n_chunks ? batch.n_chunks : 1u), lg(4u * batch.n_full);
        if (c.in_type == CO3_F32) {
            CO3_CUDA(launch_behind(orth_begin_kernel<float>, bg, dim3(kBeginThreads), 0, st, batch, ba));
            if (batch.n_full) CO3_CUDA(launch_behind(orth_load_kernel<float>, lg, dim3(kLoadThreads), 0, st, la));
        } else if (c.in_type == CO3_F16) {
            CO3_CUDA(launch_behind(orth_begin_kernel<__half>, bg, dim3(kBeginThreads), 0, st, batch, ba));
            if (batch.n_full) CO3_CUDA(launch_behind(orth_load_kernel<__half>, lg, dim3(kLoadThreads), 0, st, la));
        } else {
            CO3_CUDA(launch_behind(orth_begin_kernel<__nv_bfloat16>, bg, dim3(kBeginThreads), 0, st, batch, ba));
            if (batch.n_full) CO3_CUDA(launch_behind(orth_load_kernel<__nv_bfloat16>, lg, dim3(kLoadThreads), 0, st, la));
        }
        if (batch.n_full) {
            StepArgs sa = {};
            sa.ws = ws;
            sa.ns = ns;
            sa.pairs = 0xffffffffu;
            sa.out_kind = muon ? kOutParams : c.out_type;
            sa.out = c.out;
            sa.lr = c.lr;
            sa.shrink = c.shrink;
            sa.limit_ns = 500000000ull + ns.steps * needs.work * 64ull;
            sa.res = res;
            const uint32_t widest = std::max(batch.n_tasks[0], std::max(batch.n_tasks[1], batch.n_tasks[2]));
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(std::min(widest, (uint32_t)sms));
            cfg.blockDim = dim3(kStepThreads);
            cfg.dynamicSmemBytes = kStepSmem;
            cfg.stream = st;
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeCooperative;
            attr[0].val.cooperative = 1;
            cfg.attrs = attr;
            cfg.numAttrs = 1;
            CO3_CUDA(cudaFuncSetAttribute(orth_steps_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kStepSmem));
            CO3_CUDA(cudaLaunchKernelEx(&cfg, orth_steps_kernel, sa));
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
