// What the kernels on 8-bit blocks share: where values and scales lie, and the conversions.
//
// A block of 128 columns of a row (or of 128 x 128 entries, CO3_F8_SQUARE) has one scale, the smallest power of two s with
// max|x| <= 448 s, and its entries are x / s in e4m3 (sign, four bits of exponent, three of mantissa), rounded to nearest, ties
// to even.  A power of two loses nothing against an fp32 scale but at most one bit of the smallest, sub-normal steps; x / s, the
// value read back and its bf16 form are exact; and the tensor cores apply such scales themselves (an exponent byte, 2^(byte - 127)).
//
// The memory holds what the tensor cores read: for each 128 columns, rows of 128 bytes one behind the other, the 16-byte pieces
// of a row XORed with the row number modulo 8.  Any rows that start at a multiple of 8 are fetched by one plain bulk copy, and the
// same bytes serve as the operand and as the transposed operand.  Exponent bytes lie in tiles of 512 bytes for 128 rows and four
// blocks of columns: byte 16 (r % 32) + 4 (r / 32) + block, as they are copied into tensor memory.  Square blocks have
// them once more for the transposed operand.
#pragma once

#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "co3.h"
#include "co3_device.cuh"
#include "co3_types.cuh"

namespace co3 {

// All of these kernels are launched behind the one before them, which may still be writing what they will read once it has completed: they
// use ordinary loads, not those for what is never written while a kernel runs.
constexpr uint32_t kF8Block = 128;
constexpr uint32_t kF8Tile = 128 * 128;        // bytes of 128 rows of a block of columns
constexpr uint32_t kF8Scales = 512;            // bytes of a tile of exponent bytes
constexpr int kF8MinExp = -126, kF8MaxExp = 120;

struct F8Layout {
    uint64_t rows;         // rows padded to whole tiles
    uint32_t kb;           // blocks of columns
    uint64_t scales;       // byte offset of the exponent bytes
    uint64_t scales_t;     // the same for the transposed operand (square blocks)
    uint64_t bytes;
};

inline bool f8_layout(uint64_t rows, uint64_t cols, int kind, F8Layout* out) {
    if (kind != CO3_F8_ROWS && kind != CO3_F8_SQUARE) return false;
    if (rows >= (1ull << 31) || cols >= (1ull << 31)) return false;
    out->rows = (rows + 127u) & ~(uint64_t)127u;
    out->kb = (uint32_t)((cols + 127u) / 128u);
    if (out->kb && out->rows >= (1ull << 40) / 128u / out->kb) return false;
    const uint64_t tiles = out->rows / 128u;
    out->scales = out->rows * out->kb * 128u;
    out->scales_t = out->scales + (uint64_t)((out->kb + 3u) / 4u) * tiles * kF8Scales;
    out->bytes = out->scales_t + (kind == CO3_F8_SQUARE ? (tiles + 3u) / 4u * out->kb * kF8Scales : 0u);
    if (out->bytes < 256u) out->bytes = 256u;
    return true;
}

// Arguments that name a matrix of `type` elements, or a buffer of 8-bit blocks.
inline bool f8_valid_rows(int type, const void* p, uint64_t stride, uint32_t cols) {
    return type >= CO3_F32 && type <= CO3_BF16 && p && reinterpret_cast<uintptr_t>(p) % type_size(type) == 0 && stride >= cols && stride < (1ull << 40);
}
inline bool f8_valid(const void* p) { return p && reinterpret_cast<uintptr_t>(p) % 256u == 0; }

// Offset of a row's 128 bytes of a block of columns, and of a 16-byte piece in them.
__device__ __forceinline__ uint64_t f8_row(uint64_t rows_padded, uint32_t block, uint64_t row) { return (block * rows_padded + row) * 128u; }
__device__ __forceinline__ uint32_t f8_piece(uint32_t row, uint32_t piece) { return (piece ^ (row & 7u)) << 4; }
// Offset of a row's exponent byte among those of a tile.
__host__ __device__ inline uint32_t f8_scale_at(uint32_t row_in_tile, uint32_t block) {
    return (row_in_tile & 31u) * 16u + (row_in_tile >> 5) * 4u + (block & 3u);
}

// Exponent of the scale of a block whose largest magnitude has these bits (finite; 448 = 1.75 * 2^8).  Never below -126, so that
// the scale and its inverse are normal numbers: entries below 2^-136 become zero.
__device__ __forceinline__ int f8_exponent(uint32_t most) {
    const int e = (int)(most >> 23) - 127 - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0);
    return max(e, kF8MinExp);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Two fp32 operations in one instruction.
struct F2 {
    float x, y;
};
__device__ __forceinline__ unsigned long long f2_bits(F2 v) { return (unsigned long long)__float_as_uint(v.x) | ((unsigned long long)__float_as_uint(v.y) << 32); }
__device__ __forceinline__ F2 f2_from(unsigned long long b) { return {__uint_as_float((uint32_t)b), __uint_as_float((uint32_t)(b >> 32))}; }
__device__ __forceinline__ F2 f2_both(float v) { return {v, v}; }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(f2_bits(a)), "l"(f2_bits(b)), "l"(f2_bits(c)));
    return f2_from(r);
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(f2_bits(a)), "l"(f2_bits(b)));
    return f2_from(r);
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(f2_bits(a)), "l"(f2_bits(b)));
    return f2_from(r);
}

// Four values to e4m3, the first in the lowest byte.  NaN stays NaN.
__device__ __forceinline__ uint32_t f8_from4(float a, float b, float c, float d) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)lo | ((uint32_t)hi << 16);
}
// Two of them back.
__device__ __forceinline__ float2 f8_to2(uint32_t two) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// Bits of the largest magnitude from which a block is not on the short way: infinities and NaN, and magnitudes whose nearest value
// may be 2^128.
constexpr uint32_t kF8Rare = 0x7f600000u;

__device__ __forceinline__ uint32_t f8_magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// What a non-finite value counts in its block's largest magnitude, and what it becomes.
__device__ __forceinline__ uint32_t f8_finite_magnitude(float v) {
    const uint32_t m = f8_magnitude(v);
    return m < 0x7f800000u ? m : 0u;
}
__device__ __forceinline__ float f8_rare(float v, int exponent) {
    if (f8_magnitude(v) >= 0x7f800000u) return __uint_as_float(0x7fffffffu);
    const float most = exponent == kF8MaxExp ? __uint_as_float(0x7f700000u) : __uint_as_float(0x7f600000u);  // 240 or 448 scales
    return fminf(fmaxf(v, -most), most);
}

// Registers are shared out between three groups of four warps that start with 168 each: the first group's warps issue
// copies and products, the eight others hold a tile's sums.
constexpr uint32_t kF8Threads = 384;
constexpr uint32_t kFewRegs = 56, kManyRegs = 224;
static_assert(kFewRegs + 2 * kManyRegs == 3 * 168, "registers of the block");
__device__ __forceinline__ void few_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegs)); }
__device__ __forceinline__ void many_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegs)); }

// kCount columns (a multiple of 32) of this warp's 32 lanes, all loads under way at once.  (Volatile statements keep their order, so
// that no sum is used before the wait.)
template <int kCount>
__device__ __forceinline__ void tc_load(uint32_t addr, float (&v)[kCount]) {
    static_assert(kCount % 32 == 0, "whole loads");
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
#pragma unroll
    for (int h = 0; h < kCount; h += 32)
        asm volatile(
            "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
            "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
            "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
            : "=r"(r[h + 0]), "=r"(r[h + 1]), "=r"(r[h + 2]), "=r"(r[h + 3]), "=r"(r[h + 4]), "=r"(r[h + 5]), "=r"(r[h + 6]), "=r"(r[h + 7]), "=r"(r[h + 8]),
              "=r"(r[h + 9]), "=r"(r[h + 10]), "=r"(r[h + 11]), "=r"(r[h + 12]), "=r"(r[h + 13]), "=r"(r[h + 14]), "=r"(r[h + 15]), "=r"(r[h + 16]), "=r"(r[h + 17]),
              "=r"(r[h + 18]), "=r"(r[h + 19]), "=r"(r[h + 20]), "=r"(r[h + 21]), "=r"(r[h + 22]), "=r"(r[h + 23]), "=r"(r[h + 24]), "=r"(r[h + 25]), "=r"(r[h + 26]),
              "=r"(r[h + 27]), "=r"(r[h + 28]), "=r"(r[h + 29]), "=r"(r[h + 30]), "=r"(r[h + 31])
            : "r"(addr + h)
            : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < kCount; ++i) asm volatile("" : "+r"(r[i]));
}

// ------------------------------------------------------------------------------------------------
// Pairs of blocks (a cluster of two) that multiply together: each holds 128 rows of the first operand and half of the second,
// and gets the sums of its own 128 rows.  The pair's first block issues the products for both, which halves what each of
// them reads and keeps of the second operand.
// ------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// An arrival at the barrier that lies at the same place in block `rank` of the cluster.  What it tells of lies in shared or tensor
// memory and is touched by copies and products alone: what a copy brought lies in its block's shared memory before the copy's barrier
// says so, and the products read it there.  So no wider order than the block's is asked for; a release for the cluster takes some 1500
// cycles (16384 x 4096 x 4096 weight gradient 1225 against 433 us, 550 with three warps that take turns).
__device__ __forceinline__ void mbar_arrive_at(uint64_t* bar, uint32_t rank) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_addr(bar)), "r"(rank));
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(at) : "memory");
}
// One lane of a converged warp.  The warps that issue copies and products run their loops with all lanes and let this one issue:
// addresses and descriptors then stay in the warp's uniform registers.
__device__ __forceinline__ bool elected() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
// mbar_wait with the clock looked at less often, here too for at most half a second or so.  What is already there is found by the
// first try: 50 cycles, against 240 through the loop, of which a stage has two while its products take 512.
__device__ __forceinline__ bool f8_wait(uint64_t* bar, uint32_t parity) {
    if (__builtin_expect(mbar_try_wait(bar, parity), 1)) return true;
    uint64_t t0 = 0;
#pragma unroll 1
    for (uint32_t i = 1;; ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 255u) == 0) {
            const uint64_t t = global_timer_ns();
            if (t0 == 0) t0 = t;
            if (t - t0 > 500000000ull) return false;
        }
    }
}
// The products issued so far arrive at the barrier of both blocks, or of this one, when they are done.
__device__ __forceinline__ void tc_commit_pair(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_addr(bar)), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void tc_commit_first(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void tmem_alloc_pair(uint32_t* to) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(to)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free_pair(uint32_t at) { asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(at) : "memory"); }

}  // namespace co3
