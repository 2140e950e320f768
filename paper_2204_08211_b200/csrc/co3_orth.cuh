// What the kernels of the orthogonalised updates share: how operands are held, and the tensor core's instructions.
//
// Operands are blocks of 128 rows x 64 columns, each a pair of fp16 planes of 16 KB: hi = the
// value rounded, lo = 2^11 times the remainder rounded, together 22 significant bits.  A plane is stored, in the workspace
// too, exactly as the tensor core wants it in shared memory (128-byte rows, 16-byte pieces XORed with the row number
// modulo 8), so that a tile is fetched by plain bulk copies, and padding of the matrix to whole blocks is stored as zeros.
// The same bytes serve as the transposed operand (a row of the block runs along the operand's rows instead of along the
// sum): X is not stored transposed, and of the symmetric A and B only the tiles on and below the diagonal are computed
// and stored.  A product is hi*hi + 2^-11 (hi*lo + lo*hi): the part left out, lo*lo, is below 2^-22 of the whole.
#pragma once

#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "co3.h"
#include "co3_device.cuh"
#include "co3_types.cuh"

namespace co3 {

constexpr uint32_t kPlane = 128 * 64 * 2;           // bytes of a plane of a block
constexpr uint32_t kBlock = 2 * kPlane;             // hi, then lo
constexpr uint32_t kHalfPlane = kPlane / 2;         // 64 rows
constexpr int kLoBits = 11;
constexpr float kLoScale = 2048.0f;
constexpr int kMaxLogS = 13;


enum OrthOut { kOutF32 = 0, kOutF16 = 1, kOutBf16 = 2, kOutParams = 3 };

// Values are held times this power of two, so that the entries of X are about 1: 2^min(13, log2 sqrt(m n)).
__host__ __device__ inline float orth_s(uint32_t m, uint32_t n) {
    const uint64_t p = (uint64_t)m * n;
    int k = 0;
    while (k < kMaxLogS && (1ull << (2 * (k + 1))) <= p) ++k;
    return (float)(1u << k);
}

__device__ __forceinline__ uint32_t swizzled(uint32_t row, uint32_t piece) { return row * 128u + ((piece ^ (row & 7u)) << 4); }

// hi and lo of eight values, as 16-byte pieces.
__device__ __forceinline__ void split8(const float* v, uint4& hi, uint4& lo) {
    uint32_t h[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 a = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        const float2 f = __half22float2(a);
        const __half2 b = __floats2half2_rn(__fmul_rn(__fsub_rn(v[2 * i], f.x), kLoScale), __fmul_rn(__fsub_rn(v[2 * i + 1], f.y), kLoScale));
        h[i] = *reinterpret_cast<const uint32_t*>(&a);
        l[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    hi = make_uint4(h[0], h[1], h[2], h[3]);
    lo = make_uint4(l[0], l[1], l[2], l[3]);
}

__device__ __forceinline__ void join8(const uint4& hi, const uint4& lo, float (&v)[8]) {
    const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w}, l[4] = {lo.x, lo.y, lo.z, lo.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&h[i])), b = __half22float2(*reinterpret_cast<const __half2*>(&l[i]));
        v[2 * i] = __fmaf_rn(b.x, 1.0f / kLoScale, a.x);
        v[2 * i + 1] = __fmaf_rn(b.y, 1.0f / kLoScale, a.y);
    }
}

// ------------------------------------------------------------------------------------------------
// tcgen05: operands in shared memory (K-major, 128-byte swizzle), fp32 accumulators in tensor memory.
// ------------------------------------------------------------------------------------------------
// An operand of 128 rows and 64 columns of the sum in shared memory.  As it lies in memory: rows of 128 bytes along the
// sum, 1024 bytes between groups of eight.  Transposed: two halves of 64 operand rows, some distance apart, each with a row of
// 128 bytes per column of the sum, 1024 bytes between groups of eight columns.  Both swizzled.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, bool transposed, uint32_t between_halves = kHalfPlane) {
    return (uint64_t)((addr >> 4) & 0x3fffu) | ((uint64_t)(transposed ? between_halves >> 4 : 1u) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// 16 columns of the sum further.  Descriptors reach the tensor core through the warp's uniform registers: with a step
// that is not known to the compiler each product costs about 120 cycles to issue, with one that is, 64 or 128 to do.
__host__ __device__ constexpr uint32_t desc_step(bool transposed) { return transposed ? 2048u >> 4 : 32u >> 4; }
// D fp32, A and B fp16
__host__ __device__ constexpr uint32_t instr_desc(bool a_transposed, bool b_transposed, uint32_t rows, uint32_t cols) {
    return (1u << 4) | ((uint32_t)a_transposed << 15) | ((uint32_t)b_transposed << 16) | ((cols / 8u) << 17) | ((rows / 16u) << 24);
}

// kScale: what is there already counts 2^-kScale.
template <int kScale = 0>
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t instr, bool accumulate) {
    if constexpr (kScale == 0)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(instr), "r"((uint32_t)accumulate)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p, %5;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(instr), "r"((uint32_t)accumulate),
            "n"(kScale)
            : "memory");
}
// The products issued so far arrive on this barrier when they are done.
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

__device__ __forceinline__ void fence_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }

// A thread's kN sums times f into column `first` of the caller's matrix, down the rows from there on (cnt of them): as the
// result, or as the step of parameters.  A warp's threads have neighbouring columns.
template <int kN>
__device__ __forceinline__ void put_result(void* out_base, int kind, uint64_t first, uint64_t stride, uint32_t cnt, float f,
                                           const float* acc, float lr, float shrink) {
    if (kind == kOutParams) {
        float* out = static_cast<float*>(out_base) + first;
#pragma unroll
        for (int i0 = 0; i0 < kN; i0 += 16) {
            float old[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) old[i] = (uint32_t)(i0 + i) < cnt ? out[(uint64_t)(i0 + i) * stride] : 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if ((uint32_t)(i0 + i) < cnt) out[(uint64_t)(i0 + i) * stride] = __fmaf_rn(-lr, __fmul_rn(f, acc[i0 + i]), __fmul_rn(shrink, old[i]));
        }
    } else if (kind == kOutF32) {
        float* out = static_cast<float*>(out_base) + first;
#pragma unroll
        for (int i = 0; i < kN; ++i)
            if ((uint32_t)i < cnt) out[(uint64_t)i * stride] = __fmul_rn(f, acc[i]);
    } else {
        uint16_t* out = static_cast<uint16_t*>(out_base) + first;
        const bool f16 = kind == kOutF16;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const float v = __fmul_rn(f, acc[i]);
            if ((uint32_t)i < cnt) out[(uint64_t)i * stride] = f16 ? __half_as_ushort(__float2half_rn(v)) : __bfloat16_as_ushort(__float2bfloat16_rn(v));
        }
    }
}

}  // namespace co3
