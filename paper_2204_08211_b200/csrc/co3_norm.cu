// Layer norm of many rows, forward and backward, the latter with the gradients of gain and bias per client.
//
//   norm_forward_kernel / norm_backward_kernel   a warp or a block per row, the row read from memory once
//   norm_reduce_kernel                           per-block sums of the gain's and bias' gradients added in order
//   norm_*_long_kernel                           rows beyond kMaxCols columns: two passes over the row
//
// All of it is bound by memory: forward moves 2 n s bytes a row (s the element size), backward 3 n s.  Blocks are
// persistent: a thread owns the same columns in every row it works on, so gain and bias stay in its registers (they
// are fp32: read again for every row they would cost four times what a 16-bit row does) and the sums for their
// gradients never leave registers until the last row.  A warp owns a stretch of columns (of one row, or of the row its
// block works on) and fetches it some rows ahead into a ring of its own in shared memory with asynchronous 16-byte
// copies, which hides the memory's latency without registers and takes rows at any alignment: the copies cover the
// 16-byte pieces the stretch touches, and lanes pick their elements out of shared memory, 16 bytes at a time where all
// rows are aligned, one element at a time (neighbouring lanes, neighbouring elements) where they are not.  With 16-bit
// elements the instructions count as much as the bytes: arithmetic is done on pairs of fp32.
#include <cuda_runtime.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

#include "co3.h"
#include "co3_device.cuh"
#include "co3_launch.cuh"
#include "co3_types.cuh"

namespace co3 {

constexpr uint32_t kMaxCols = 16384;   // 512 threads x 32 elements
// Block of the kernels with one warp per row: with 32 elements a lane registers leave room for 12 warps on an SM, in one
// block.  Backward in fp32 they do not quite suffice for that.  (us, 8 against 12 warps: backward 65536 x 1024 bf16 82.5
// and 72.4, fp32 131 and 144; forward 47.4 and 46.1; 3001 x 1023 f16 backward 19.2 and 14.0, forward 9.5 and 7.3.  With
// 16 warps registers spill: backward 65536 x 1024 bf16 124.)
template <typename T, int kElems, bool kBackward>
constexpr int kWarpRowThreads = kElems < 32 || (kBackward && sizeof(T) == 4) ? 256 : 384;
constexpr size_t kRingBytes = 200 << 10;  // shared memory of an SM for rings
constexpr int kLongThreads = 1024;
constexpr uint64_t kPlanBlocks = 148 * 8;

struct NormArgs {
    const void *x, *dy;
    const float *weight, *bias;
    void* out;  // y or dx
    float *mean, *rstd;
    uint64_t rows;      // forward: all; backward: of one client
    uint64_t all_rows;  // backward: of all clients
    uint32_t ring;      // rows a warp has in shared memory: 8, 4, 3, 2 or 1
    uint32_t cols;
    uint64_t x_stride, dy_stride, out_stride;
    float eps;
    // backward
    float *dweight, *dbias;
    uint64_t client_stride;
    uint32_t parts;  // blocks per client
    int accumulate;
    float* partial;  // [client][part][2][cols], used if parts > 1
};

__device__ __forceinline__ void copy16_async(uint32_t dst, const void* src, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <uint32_t kLeft>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }
// All but the newest ring - 2 groups: the oldest row has arrived.
__device__ __forceinline__ void copies_wait_ring(uint32_t ring) {
    if (ring == 8) copies_wait<6>();
    else if (ring == 4) copies_wait<2>();
    else if (ring == 3) copies_wait<1>();
    else copies_wait<0>();
}

// Two fp32 values, and the arithmetic that takes one instruction for both.
struct F2 {
    float x, y;
};
__device__ __forceinline__ unsigned long long bits(const F2& a) {
    unsigned long long v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a.x), "f"(a.y));
    return v;
}
__device__ __forceinline__ F2 pair(unsigned long long v) {
    F2 a;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a.x), "=f"(a.y) : "l"(v));
    return a;
}
__device__ __forceinline__ F2 both(float v) { return {v, v}; }
__device__ __forceinline__ F2 fma2(const F2& a, const F2& b, const F2& c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)), "l"(bits(c)));
    return pair(r);
}
__device__ __forceinline__ F2 add2(const F2& a, const F2& b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)));
    return pair(r);
}
__device__ __forceinline__ F2 mul2(const F2& a, const F2& b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)));
    return pair(r);
}

template <typename T>
__device__ __forceinline__ F2 unpack(uint32_t v);
template <>
__device__ __forceinline__ F2 unpack<__nv_bfloat16>(uint32_t v) { return {__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)}; }
template <>
__device__ __forceinline__ F2 unpack<__half>(uint32_t v) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v));
    return {f.x, f.y};
}
template <typename T>
__device__ __forceinline__ uint32_t repack(const F2& f);
template <>
__device__ __forceinline__ uint32_t repack<__nv_bfloat16>(const F2& f) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <>
__device__ __forceinline__ uint32_t repack<__half>(const F2& f) {
    const __half2 v = __floats2half2_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// A warp's stretch of the rows of one buffer: kCh times 32 x kVec columns, lane l owning columns (32 c + l) kVec + e.
// kVec > 1: 16 bytes, all rows aligned to them and ending on them.  kVec == 1: anything.
template <typename T, int kVec, int kCh>
struct Stretch {
    static_assert(kVec == 1 || kVec * sizeof(T) == 16, "one element, or one 16-byte access");
    static constexpr uint32_t kElems = 32 * kVec * kCh;
    static constexpr uint32_t kBytes = kElems * sizeof(T) + (kVec > 1 ? 0u : 16u);  // in shared memory
    static constexpr int kPairs = kVec * kCh / 2;

    // Copies the stretch that starts at `p`.  The copies cover whole 16-byte pieces, so they may reach into the
    // stretch's neighbours in the buffer, which begins at `lo` and ends at `hi`: within 16 bytes of these a piece that
    // p cuts is fetched element by element, and the last piece is cut short.
    static __device__ __forceinline__ void fetch(unsigned char* dst, const T* p, uint32_t bytes, const bool (&valid)[kCh], const T* lo, const T* hi) {
        const uint32_t lane = threadIdx.x & 31u, to = smem_addr(dst) + lane * 16u;
        if (kVec > 1) {
#pragma unroll
            for (int c = 0; c < kCh; ++c)
                if (valid[c]) copy16_async(to + c * 512u, p + (c * 32 + lane) * kVec, 16u);
        } else {
            const uint32_t ph = (uint32_t)reinterpret_cast<uintptr_t>(p) & 15u, len = ph + bytes;
            const unsigned char* src = reinterpret_cast<const unsigned char*>(p) - ph;
            const bool starts = p - lo < int(16 / sizeof(T)), ends = (hi - p) * int(sizeof(T)) < (int64_t)bytes + 16;
            if (!starts && !ends) {
#pragma unroll
                for (uint32_t c = 0; c < (kBytes + 511u) / 512u; ++c) {
                    const uint32_t off = c * 512u + lane * 16u;
                    if (off < len) copy16_async(to + c * 512u, src + off, 16u);
                }
            } else {
                for (uint32_t off = lane * 16u; off < len; off += 512u) {
                    if (starts && off == 0 && ph) {
                        for (uint32_t i = ph; i < 16u && i < len; i += sizeof(T)) *reinterpret_cast<T*>(dst + i) = p[(i - ph) / sizeof(T)];
                    } else {
                        copy16_async(smem_addr(dst) + off, src + off, ends ? min(16u, len - off) : 16u);
                    }
                }
            }
        }
    }
    // kVec > 1: zeros where no copy ever writes, so that `take` needs no conditions (kCleared).  Forward in blocks that
    // is worth it (16384 x 2048 bf16 41.6 -> 27.5 us); elsewhere the loads then come too early for the registers
    // (65536 x 1024 bf16: forward 46.3 -> 48.4, backward 72 -> 95).
    static __device__ __forceinline__ void clear(unsigned char* dst, const bool (&valid)[kCh]) {
        if constexpr (kVec > 1) {
#pragma unroll
            for (int c = 0; c < kCh; ++c)
                if (!valid[c]) *reinterpret_cast<uint4*>(dst + c * 512u + (threadIdx.x & 31u) * 16u) = make_uint4(0u, 0u, 0u, 0u);
        }
    }
    // The lane's elements, zeros beyond the row.  ph: the stretch's place within its first piece.
    template <bool kCleared = false>
    static __device__ __forceinline__ void take(const unsigned char* from, uint32_t ph, const bool (&valid)[kCh], F2 (&v)[kPairs]) {
        const uint32_t lane = threadIdx.x & 31u;
        if (kVec > 1) {
#pragma unroll
            for (int c = 0; c < kCh; ++c) {
                uint4 q = make_uint4(0u, 0u, 0u, 0u);
                if (kCleared || valid[c]) q = *reinterpret_cast<const uint4*>(from + c * 512u + lane * 16u);
                const uint32_t w[4] = {q.x, q.y, q.z, q.w};
                if constexpr (sizeof(T) == 4) {
                    v[2 * c] = {__uint_as_float(w[0]), __uint_as_float(w[1])};
                    v[2 * c + 1] = {__uint_as_float(w[2]), __uint_as_float(w[3])};
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[4 * c + i] = unpack<T>(w[i]);
                }
            }
        } else {
            const T* p = reinterpret_cast<const T*>(from + ph) + lane;
#pragma unroll
            for (int i = 0; i < kPairs; ++i)
                v[i] = {valid[2 * i] ? to_float(p[64 * i]) : 0.0f, valid[2 * i + 1] ? to_float(p[64 * i + 32]) : 0.0f};
        }
    }
    static __device__ __forceinline__ void put(T* p, const F2 (&v)[kPairs], const bool (&valid)[kCh]) {
        const uint32_t lane = threadIdx.x & 31u;
        if (kVec > 1) {
#pragma unroll
            for (int c = 0; c < kCh; ++c) {
                if (!valid[c]) continue;
                uint4 q;
                if constexpr (sizeof(T) == 4)
                    q = make_uint4(__float_as_uint(v[2 * c].x), __float_as_uint(v[2 * c].y), __float_as_uint(v[2 * c + 1].x), __float_as_uint(v[2 * c + 1].y));
                else
                    q = make_uint4(repack<T>(v[4 * c]), repack<T>(v[4 * c + 1]), repack<T>(v[4 * c + 2]), repack<T>(v[4 * c + 3]));
                __stcs(reinterpret_cast<uint4*>(p + (c * 32 + lane) * kVec), q);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                if (valid[2 * i]) p[64 * i + lane] = from_float<T>(v[i].x);
                if (valid[2 * i + 1]) p[64 * i + 32 + lane] = from_float<T>(v[i].y);
            }
        }
    }
    // Index of element `half` of pair i, and whether the row has it.
    static __device__ __forceinline__ uint32_t column(int i, int half) {
        const uint32_t lane = threadIdx.x & 31u;
        return kVec > 1 ? ((2 * i) / kVec * 32 + lane) * kVec + (2 * i) % kVec + half : (2 * i + half) * 32 + lane;
    }
    static __device__ __forceinline__ bool has(int i, int half, const bool (&valid)[kCh]) {
        return kVec > 1 ? valid[(2 * i) / kVec] : valid[kVec > 1 ? 0 : 2 * i + half];
    }
    static __device__ __forceinline__ void load_vector(const float* from, uint32_t col0, float otherwise, const bool (&valid)[kCh], F2 (&v)[kPairs]) {
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            v[i].x = from && has(i, 0, valid) ? __ldg(from + col0 + column(i, 0)) : otherwise;
            v[i].y = from && has(i, 1, valid) ? __ldg(from + col0 + column(i, 1)) : otherwise;
        }
    }
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

template <typename T, int kVec, int kCh, bool kWarpRow, int kMaxThreads>
__global__ void __launch_bounds__(kMaxThreads) norm_forward_kernel(const NormArgs a) {
    wait_for_previous_kernel();
    using S = Stretch<T, kVec, kCh>;
    // blocks of up to 512 threads have 128 registers a thread: 16-bit rows are taken from shared memory again after their
    // sums (8192 x 8192 bf16 66 -> 50 us; in the smaller blocks, 16384 x 4096, 48 -> 51; fp32 4096 x 16384 89 -> 95)
    constexpr bool kAgain = kMaxThreads > 384 && sizeof(T) == 2;
    extern __shared__ __align__(16) unsigned char s_ring[];
    constexpr uint32_t kWarps = kMaxThreads / 32;
    __shared__ float4 s_part[2][kWarpRow ? 1 : kWarps];
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, warps = blockDim.x / 32u;
    const uint32_t col0 = kWarpRow ? 0u : warp * S::kElems, n_cols = min(a.cols - col0, S::kElems), bytes = n_cols * (uint32_t)sizeof(T);
    const uint64_t first = kWarpRow ? (uint64_t)blockIdx.x * warps + warp : blockIdx.x, step = kWarpRow ? (uint64_t)gridDim.x * warps : gridDim.x;
    unsigned char* ring = s_ring + (size_t)warp * a.ring * S::kBytes;
    bool valid[kCh];
#pragma unroll
    for (int c = 0; c < kCh; ++c) valid[c] = (c * 32 + lane) * kVec < n_cols;
    for (uint32_t k = 0; !kWarpRow && k < a.ring; ++k) S::clear(ring + k * S::kBytes, valid);
    if (!kWarpRow && threadIdx.x < 32) {
        for (uint32_t k = warps + lane; k < kWarps; k += 32) s_part[0][k] = s_part[1][k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    const T *lo = static_cast<const T*>(a.x), *hi = lo + (a.rows - 1) * a.x_stride + a.cols;
    const T* src = lo + first * a.x_stride + col0;  // the row to be fetched next
    uint64_t ahead = first;
    uint32_t slot = 0;
    const uint64_t src_step = step * a.x_stride;
    auto fetch = [&]() {
        if (ahead < a.rows) S::fetch(ring + slot * S::kBytes, src, bytes, valid, lo, hi);
        copies_commit();
        ahead += step;
        src += src_step;
        slot = slot + 1 == a.ring ? 0u : slot + 1;
    };
    for (uint32_t k = 0; k + 1 < a.ring; ++k) fetch();
    F2 w[S::kPairs], b[S::kPairs];
    S::load_vector(a.weight, col0, 1.0f, valid, w);
    S::load_vector(a.bias, col0, 0.0f, valid, b);
    const float inv_n = __fdiv_rn(1.0f, (float)a.cols);
    // element counts of the sets that are put together, and for each of the five levels of a warp the factors
    // sqrt(n1 n2 / (n1 + n2)) / n1 and / n2
    float fm[5], fo[5], warp_n, warp_inv;
    float n_own = 0.0f;
#pragma unroll
    for (int c = 0; c < kCh; ++c) n_own += valid[c] ? (float)kVec : 0.0f;
    const float inv_own = n_own > 0.0f ? __fdiv_rn(1.0f, n_own) : 0.0f;
    {
        float n1 = n_own;
#pragma unroll
        for (int k = 0; k < 5; ++k) {
            const float n2 = __shfl_xor_sync(0xffffffffu, n1, 1 << k);
            const bool some = n1 > 0.0f && n2 > 0.0f;  // an empty set adds nothing
            fm[k] = some ? __fsqrt_rn(__fdiv_rn(n2, n1 * (n1 + n2))) : 0.0f;
            fo[k] = some ? -__fsqrt_rn(__fdiv_rn(n1, n2 * (n1 + n2))) : 0.0f;
            n1 += n2;
        }
        warp_n = n1;
        warp_inv = n1 > 0.0f ? __fdiv_rn(1.0f, n1) : 0.0f;
    }
    T* y = static_cast<T*>(a.out) + first * a.out_stride + col0;
    const T* x_now = static_cast<const T*>(a.x) + first * a.x_stride + col0;
    const uint64_t out_step = step * a.out_stride;
    uint32_t now = 0, flip = 0;  // now: the ring's slot of this row
    for (uint64_t row = first; row < a.rows; row += step, y += out_step, x_now += src_step, flip ^= 1u) {
        if (a.ring == 1) fetch();
        copies_wait_ring(a.ring);
        __syncwarp();  // the row has arrived for all lanes, and the slot of the row before is free
        if (a.ring > 1) fetch();
        // Sum, and sum of squares about the mean, of ever larger sets put together in pairs: the squares of two sets
        // with n1 and n2 elements grow by n1 n2 / (n1 + n2) (mean1 - mean2)^2 (Chan, Golub, LeVeque 1979).  One
        // reduction, and none of the cancellation of sum(x^2) - sum(x)^2 / n.
        F2 v[S::kPairs], s2 = both(0.0f), q2 = both(0.0f);
        const unsigned char* at = ring + now * S::kBytes;
        const uint32_t ph = (uint32_t)reinterpret_cast<uintptr_t>(x_now) & 15u;
        S::template take<!kWarpRow>(at, ph, valid, v);
        now = now + 1 == a.ring ? 0u : now + 1;
#pragma unroll
        for (int i = 0; i < S::kPairs; ++i) s2 = add2(s2, v[i]);
        float sum = s2.x + s2.y;
        const float own = sum * inv_own;
#pragma unroll
        for (int i = 0; i < S::kPairs; ++i) {
            v[i] = add2(v[i], both(-own));
            if (kVec > 1) {
                if (valid[(2 * i) / kVec]) q2 = fma2(v[i], v[i], q2);
            } else {
                const F2 d = {S::has(i, 0, valid) ? v[i].x : 0.0f, S::has(i, 1, valid) ? v[i].y : 0.0f};
                q2 = fma2(d, d, q2);
            }
        }
        float sq = q2.x + q2.y;
#pragma unroll
        for (int k = 0; k < 5; ++k) {
            const float so = __shfl_xor_sync(0xffffffffu, sum, 1 << k), qo = __shfl_xor_sync(0xffffffffu, sq, 1 << k);
            const float d = __fmaf_rn(so, fo[k], sum * fm[k]);
            sum += so;
            sq = __fmaf_rn(d, d, sq + qo);
        }
        float mean;
        if (kWarpRow) {
            mean = sum * inv_n;
            sq = __shfl_sync(0xffffffffu, sq, 0);  // the same bits in every lane
        } else {
            // two buffers in turn: a row's sums are read before its successor's barrier
            if (lane == 0) s_part[flip][warp] = make_float4(sum, sq, warp_n, warp_inv);
            __syncthreads();
            sum = sq = 0.0f;
            if (kWarps <= 4) {  // absent warps' entries are zero
                float4 p[kWarps];
#pragma unroll
                for (uint32_t k = 0; k < kWarps; ++k) { p[k] = s_part[flip][k]; sum += p[k].x; }
                mean = sum * inv_n;
#pragma unroll
                for (uint32_t k = 0; k < kWarps; ++k) {
                    const float d = __fmaf_rn(p[k].x, p[k].w, -mean);
                    sq += __fmaf_rn(d * p[k].z, d, p[k].y);
                }
            } else {
#pragma unroll 4
                for (uint32_t k = 0; k < warps; ++k) sum += s_part[flip][k].x;
                mean = sum * inv_n;
#pragma unroll 4
                for (uint32_t k = 0; k < warps; ++k) {
                    const float4 p = s_part[flip][k];
                    const float d = __fmaf_rn(p.x, p.w, -mean);
                    sq += __fmaf_rn(d * p.z, d, p.y);
                }
            }
        }
        const float rstd = rsqrtf(__fmaf_rn(sq, inv_n, a.eps));
        const F2 r2 = both(rstd);
        if (kAgain) {
            S::template take<!kWarpRow>(at, ph, valid, v);
#pragma unroll
            for (int i = 0; i < S::kPairs; ++i) v[i] = fma2(mul2(add2(v[i], both(-mean)), r2), w[i], b[i]);
        } else {
            const F2 k2 = both((own - mean) * rstd);
#pragma unroll
            for (int i = 0; i < S::kPairs; ++i) v[i] = fma2(fma2(v[i], r2, k2), w[i], b[i]);
        }
        S::put(y, v, valid);
        if (threadIdx.x == (kWarpRow ? warp * 32u : 0u)) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        if (a.ring == 1) __syncwarp();
    }
    copies_wait<0>();
}

__device__ __forceinline__ void put_sum(float* to, float v, int accumulate) { *to = accumulate ? *to + v : v; }

template <typename T, int kVec, int kCh, bool kWarpRow, int kMaxThreads>
__global__ void __launch_bounds__(kMaxThreads) norm_backward_kernel(const NormArgs a) {
    wait_for_previous_kernel();
    using S = Stretch<T, kVec, kCh>;
    // up to 16 elements a thread: what the sums were formed from stays in registers, otherwise it is taken from shared
    // memory again
    constexpr bool kKeep = kCh * kVec <= 16;
    constexpr uint32_t kSlot = 2 * S::kBytes + 16;  // x, dy, mean and rstd of a row
    extern __shared__ __align__(16) unsigned char s_ring[];
    constexpr uint32_t kWarps = kMaxThreads / 32;
    __shared__ __align__(16) float2 s_part[2][kWarpRow ? 2 : kWarps];
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, warps = blockDim.x / 32u;
    const uint32_t client = blockIdx.x / a.parts, part = blockIdx.x - client * a.parts;
    const uint32_t col0 = kWarpRow ? 0u : warp * S::kElems, n_cols = min(a.cols - col0, S::kElems), bytes = n_cols * (uint32_t)sizeof(T);
    const uint64_t end = (uint64_t)(client + 1) * a.rows, step = kWarpRow ? (uint64_t)a.parts * warps : a.parts;
    const uint64_t first = (uint64_t)client * a.rows + (kWarpRow ? (uint64_t)part * warps + warp : part);
    unsigned char* ring = s_ring + (size_t)warp * a.ring * kSlot;
    bool valid[kCh];
#pragma unroll
    for (int c = 0; c < kCh; ++c) valid[c] = (c * 32 + lane) * kVec < n_cols;
    if (!kWarpRow && threadIdx.x < 32) {
        for (uint32_t k = warps + lane; k < kWarps; k += 32) s_part[0][k] = s_part[1][k] = make_float2(0.0f, 0.0f);
    }
    const T *x_lo = static_cast<const T*>(a.x), *d_lo = static_cast<const T*>(a.dy);
    const T *x_hi = x_lo + (a.all_rows - 1) * a.x_stride + a.cols, *d_hi = d_lo + (a.all_rows - 1) * a.dy_stride + a.cols;
    const T *x_next = x_lo + first * a.x_stride + col0, *d_next = d_lo + first * a.dy_stride + col0;
    const T *x_now = x_next, *d_now = d_next;
    const uint64_t x_step = step * a.x_stride, d_step = step * a.dy_stride, out_step = step * a.out_stride;
    uint64_t ahead = first;
    uint32_t slot = 0;
    auto fetch = [&]() {
        if (ahead < end) {
            unsigned char* dst = ring + slot * kSlot;
            S::fetch(dst, x_next, bytes, valid, x_lo, x_hi);
            S::fetch(dst + S::kBytes, d_next, bytes, valid, d_lo, d_hi);
            if (lane < 2)
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_addr(dst) + 2 * S::kBytes + lane * 4u), "l"((lane ? a.rstd : a.mean) + ahead) : "memory");
        }
        copies_commit();
        ahead += step;
        x_next += x_step;
        d_next += d_step;
        slot = slot + 1 == a.ring ? 0u : slot + 1;
    };
    for (uint32_t k = 0; k + 1 < a.ring; ++k) fetch();
    F2 w[S::kPairs], dw[S::kPairs], db[S::kPairs];
    S::load_vector(a.weight, col0, 1.0f, valid, w);
#pragma unroll
    for (int i = 0; i < S::kPairs; ++i) dw[i] = db[i] = both(0.0f);
    const float inv_n = __fdiv_rn(1.0f, (float)a.cols);
    T* dx = static_cast<T*>(a.out) + first * a.out_stride + col0;
    uint32_t now = 0, flip = 0;  // now: the ring's slot of this row
    for (uint64_t row = first; row < end; row += step, dx += out_step, x_now += x_step, d_now += d_step, flip ^= 1u) {
        if (a.ring == 1) fetch();
        copies_wait_ring(a.ring);
        __syncwarp();  // the row has arrived for all lanes, and the slot of the row before is free
        if (a.ring > 1) fetch();
        const unsigned char* at = ring + now * kSlot;
        now = now + 1 == a.ring ? 0u : now + 1;
        const uint32_t px = (uint32_t)reinterpret_cast<uintptr_t>(x_now) & 15u, pd = (uint32_t)reinterpret_cast<uintptr_t>(d_now) & 15u;
        const float2 stat = *reinterpret_cast<const float2*>(at + 2 * S::kBytes);
        const F2 r2 = both(stat.y), m2 = both(-stat.x);
        F2 h[S::kPairs], g[S::kPairs], c1 = both(0.0f), c2 = both(0.0f);
        S::take(at, px, valid, h);
        S::take(at + S::kBytes, pd, valid, g);
#pragma unroll
        for (int i = 0; i < S::kPairs; ++i) {
            // beyond the row dy is zero: nothing reaches the sums, and the element is not written
            h[i] = mul2(add2(h[i], m2), r2);
            dw[i] = fma2(g[i], h[i], dw[i]);
            db[i] = add2(db[i], g[i]);
            g[i] = mul2(g[i], w[i]);
            c1 = add2(c1, g[i]);
            c2 = fma2(g[i], h[i], c2);
        }
        if (a.out) {
            float s1 = warp_sum(c1.x + c1.y), s2 = warp_sum(c2.x + c2.y);
            if (!kWarpRow) {
                if (lane == 0) s_part[flip][warp] = make_float2(s1, s2);
                __syncthreads();  // two buffers: the next row's sums go into the other one
                s1 = s2 = 0.0f;
                if (kWarps <= 8) {  // absent warps' entries are zero
#pragma unroll
                    for (uint32_t k = 0; k < kWarps; k += 2) {
                        const float4 p = *reinterpret_cast<const float4*>(&s_part[flip][k]);
                        s1 += p.x; s2 += p.y;
                        s1 += p.z; s2 += p.w;
                    }
                } else {
#pragma unroll 4
                    for (uint32_t k = 0; k < warps; ++k) { s1 += s_part[flip][k].x; s2 += s_part[flip][k].y; }
                }
            }
            // rstd (g - s1 / n - xh s2 / n) by two multiplications with additions
            const float n2 = -s2 * inv_n * stat.y, n1 = -s1 * inv_n * stat.y;
            if (kKeep) {
#pragma unroll
                for (int i = 0; i < S::kPairs; ++i) g[i] = fma2(g[i], r2, fma2(h[i], both(n2), both(n1)));
            } else {
                S::take(at, px, valid, h);
                S::take(at + S::kBytes, pd, valid, g);
#pragma unroll
                for (int i = 0; i < S::kPairs; ++i)
                    g[i] = fma2(mul2(g[i], w[i]), r2, fma2(add2(h[i], m2), both(n2 * stat.y), both(n1)));
            }
            S::put(dx, g, valid);
        }
        if (a.ring == 1) __syncwarp();
    }
    copies_wait<0>();
    if (!a.dweight && !a.dbias) return;
    float* to = a.parts > 1 ? a.partial + (uint64_t)blockIdx.x * 2 * a.cols : nullptr;
    if (kWarpRow) {
        // the warps' sums side by side, then added in order; warps without a row have nothing to add
        float* s_sum = reinterpret_cast<float*>(s_ring);
        const uint64_t left = a.rows - min(a.rows, (uint64_t)part * warps);
        const uint32_t used = (uint32_t)min((uint64_t)warps, max(left, (uint64_t)1));
        __syncthreads();
        if (warp < used) {
            float* mine = s_sum + (size_t)warp * 2 * a.cols;
#pragma unroll
            for (int i = 0; i < 2 * S::kPairs; ++i)
                if (S::has(i / 2, i & 1, valid)) {
                    const uint32_t col = S::column(i / 2, i & 1);
                    mine[col] = i & 1 ? dw[i / 2].y : dw[i / 2].x;
                    mine[a.cols + col] = i & 1 ? db[i / 2].y : db[i / 2].x;
                }
        }
        __syncthreads();
        for (uint32_t q = threadIdx.x; q < 2 * a.cols; q += blockDim.x) {
            float v = s_sum[q];
            for (uint32_t k = 1; k < used; ++k) v += s_sum[(size_t)k * 2 * a.cols + q];
            if (to) {
                to[q] = v;
            } else {
                float* dst = q < a.cols ? a.dweight : a.dbias;
                if (dst) put_sum(dst + client * a.client_stride + (q < a.cols ? q : q - a.cols), v, a.accumulate);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2 * S::kPairs; ++i)
            if (S::has(i / 2, i & 1, valid)) {
                const uint32_t col = col0 + S::column(i / 2, i & 1);
                const float x = i & 1 ? dw[i / 2].y : dw[i / 2].x, y = i & 1 ? db[i / 2].y : db[i / 2].x;
                if (to) {
                    to[col] = x;
                    to[a.cols + col] = y;
                } else {
                    if (a.dweight) put_sum(a.dweight + client * a.client_stride + col, x, a.accumulate);
                    if (a.dbias) put_sum(a.dbias + client * a.client_stride + col, y, a.accumulate);
                }
            }
    }
}

// Sums over the parts of a client: a block's threads are kGroups of parts x columns, groups added in order.  As many
// groups as there are parts, 16 at most: with 16 for 2 parts 100 x 8 x 4096 bf16 took 61 us instead of 27.
constexpr uint32_t kReduceThreads = 512;
template <uint32_t kGroups>
__global__ void __launch_bounds__(kReduceThreads) norm_reduce_kernel(const NormArgs a) {
    wait_for_previous_kernel();
    __shared__ float s_v[kReduceThreads];
    constexpr uint32_t width = kReduceThreads / kGroups;
    const uint32_t group = threadIdx.x / width, lane = threadIdx.x % width;
    const uint32_t col_blocks = (a.cols + width - 1) / width;
    const uint32_t cb = blockIdx.x % col_blocks, rest = blockIdx.x / col_blocks, which = rest & 1u, client = rest >> 1;
    const uint32_t col = cb * width + lane;
    float* dst = which ? a.dbias : a.dweight;
    if (!dst) return;
    float sum = 0.0f;
    if (col < a.cols) {
        const float* p = a.partial + ((uint64_t)client * a.parts * 2 + which) * a.cols + col;
#pragma unroll 8
        for (uint32_t k = group; k < a.parts; k += kGroups) sum += p[(uint64_t)k * 2 * a.cols];
    }
    s_v[threadIdx.x] = sum;
    __syncthreads();
    if (group == 0 && col < a.cols) {
        for (uint32_t k = 1; k < kGroups; ++k) sum += s_v[k * width + lane];
        put_sum(dst + (uint64_t)client * a.client_stride + col, sum, a.accumulate);
    }
}

// Count, mean and sum of squared deviations of two sets put together (Chan, Golub, LeVeque 1979).
struct Moments {
    float n, mean, m2;
    __device__ __forceinline__ void add(const Moments& o) {
        const float total = n + o.n;
        const float share = total > 0.0f ? __fdiv_rn(o.n, total) : 0.0f;
        const float d = o.mean - mean;
        mean = __fmaf_rn(d, share, mean);
        m2 = m2 + o.m2 + d * d * (n * share);
        n = total;
    }
    __device__ __forceinline__ void add_warp() {  // valid in lane 0
#pragma unroll
        for (int d = 16; d; d >>= 1)
            add({__shfl_down_sync(0xffffffffu, n, d), __shfl_down_sync(0xffffffffu, mean, d), __shfl_down_sync(0xffffffffu, m2, d)});
    }
};

template <typename T>
__global__ void __launch_bounds__(kLongThreads) norm_forward_long_kernel(const NormArgs a) {
    wait_for_previous_kernel();
    __shared__ Moments s_m[32];
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        T* y = static_cast<T*>(a.out) + row * a.out_stride;
        Moments m = {0.0f, 0.0f, 0.0f};
        for (uint32_t c0 = 0; c0 < a.cols; c0 += 8 * kLongThreads) {
            float v[8], sum = 0.0f;
            int n = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t c = c0 + i * kLongThreads + threadIdx.x;
                v[i] = c < a.cols ? to_float(x[c]) : 0.0f;
                n += c < a.cols;
                sum += v[i];
            }
            if (n == 0) continue;
            Moments o = {(float)n, __fdiv_rn(sum, (float)n), 0.0f};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) { const float d = v[i] - o.mean; o.m2 = __fmaf_rn(d, d, o.m2); }
            m.add(o);
        }
        m.add_warp();
        __syncthreads();
        if ((threadIdx.x & 31) == 0) s_m[threadIdx.x >> 5] = m;
        __syncthreads();
        m = s_m[0];
        for (int k = 1; k < kLongThreads / 32; ++k) m.add(s_m[k]);
        const float rstd = __fdiv_rn(1.0f, __fsqrt_rn(__fdiv_rn(m.m2, (float)a.cols) + a.eps));
        for (uint32_t c = threadIdx.x; c < a.cols; c += kLongThreads)
            y[c] = from_float<T>(__fmaf_rn((to_float(x[c]) - m.mean) * rstd, a.weight ? a.weight[c] : 1.0f, a.bias ? a.bias[c] : 0.0f));
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = m.mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kLongThreads) norm_dx_long_kernel(const NormArgs a, uint64_t rows) {
    wait_for_previous_kernel();
    __shared__ float2 s_c[32];
    for (uint64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
        T* dx = static_cast<T*>(a.out) + row * a.out_stride;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float c1 = 0.0f, c2 = 0.0f;
#pragma unroll 4
        for (uint32_t c = threadIdx.x; c < a.cols; c += kLongThreads) {
            const float g = to_float(dy[c]) * (a.weight ? a.weight[c] : 1.0f);
            c1 += g;
            c2 = __fmaf_rn(g, (to_float(x[c]) - mean) * rstd, c2);
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            c1 += __shfl_xor_sync(0xffffffffu, c1, d);
            c2 += __shfl_xor_sync(0xffffffffu, c2, d);
        }
        __syncthreads();
        if ((threadIdx.x & 31) == 0) s_c[threadIdx.x >> 5] = make_float2(c1, c2);
        __syncthreads();
        c1 = c2 = 0.0f;
        for (int k = 0; k < kLongThreads / 32; ++k) { c1 += s_c[k].x; c2 += s_c[k].y; }
        const float inv_n = __fdiv_rn(1.0f, (float)a.cols);
        c1 *= inv_n;
        c2 *= inv_n;
        for (uint32_t c = threadIdx.x; c < a.cols; c += kLongThreads) {
            const float g = to_float(dy[c]) * (a.weight ? a.weight[c] : 1.0f);
            dx[c] = from_float<T>(rstd * (g - __fmaf_rn((to_float(x[c]) - mean) * rstd, c2, c1)));
        }
    }
}

// Column sums of a part of a client's rows, a thread per column.
template <typename T>
__global__ void __launch_bounds__(256) norm_dw_long_kernel(const NormArgs a) {
    wait_for_previous_kernel();
    const uint32_t col_blocks = (a.cols + 255u) / 256u;
    const uint32_t cb = blockIdx.x % col_blocks, slot = blockIdx.x / col_blocks;  // slot = client * parts + part
    const uint32_t client = slot / a.parts, part = slot - client * a.parts, c = cb * 256u + threadIdx.x;
    if (c >= a.cols) return;
    float dw = 0.0f, db = 0.0f;
#pragma unroll 4
    for (uint64_t r = part; r < a.rows; r += a.parts) {
        const uint64_t row = (uint64_t)client * a.rows + r;
        const float d = to_float(static_cast<const T*>(a.dy)[row * a.dy_stride + c]);
        dw = __fmaf_rn(d, (to_float(static_cast<const T*>(a.x)[row * a.x_stride + c]) - a.mean[row]) * a.rstd[row], dw);
        db += d;
    }
    if (a.parts > 1) {
        float* p = a.partial + (uint64_t)slot * 2 * a.cols;
        p[c] = dw;
        p[a.cols + c] = db;
    } else {
        if (a.dweight) put_sum(a.dweight + client * a.client_stride + c, dw, a.accumulate);
        if (a.dbias) put_sum(a.dbias + client * a.client_stride + c, db, a.accumulate);
    }
}

}  // namespace co3

// ================================================================================================
// Host side
// ================================================================================================
using namespace co3;

namespace {

// Parts of a client's rows that the workspace has room for: enough for a full GPU whatever the number of clients, no
// part without a row.
uint64_t max_parts(uint64_t rows, uint32_t n_clients) {
    const uint64_t p = (kPlanBlocks + n_clients - 1) / n_clients;
    return std::max<uint64_t>(1, std::min(p, rows));
}

// What the launches need to know of the device and of a kernel, asked for once per device and kept: it does not change.
constexpr int kDevices = 64;

int sm_count(int* sms) {
    static std::atomic<int> known[kDevices];
    int dev = 0;
    CO3_CUDA(cudaGetDevice(&dev));
    int n = dev < kDevices ? known[dev].load(std::memory_order_relaxed) : 0;
    if (n == 0) {
        CO3_CUDA(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev));
        if (dev < kDevices) known[dev].store(n, std::memory_order_relaxed);
    }
    *sms = n;
    return CO3_OK;
}

// Lets a kernel have kRingBytes of shared memory, and says how many of its blocks an SM holds.
template <auto* kKernel>
int blocks_per_sm(uint32_t threads, size_t smem, int* per_sm) {
    static std::atomic<int> regs[kDevices];
    int dev = 0;
    CO3_CUDA(cudaGetDevice(&dev));
    int r = dev < kDevices ? regs[dev].load(std::memory_order_relaxed) : 0;
    if (r == 0) {
        cudaFuncAttributes f;
        CO3_CUDA(cudaFuncGetAttributes(&f, kKernel));
        CO3_CUDA(cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRingBytes));
        r = f.numRegs;
        if (dev < kDevices) regs[dev].store(r, std::memory_order_relaxed);
    }
    // an SM: 2048 threads, 32 blocks, 64 K registers handed out to warps 256 at a time, 228 KB of shared memory of
    // which 1 KB a block is the system's (and 1 KB at most these kernels' static arrays)
    const uint32_t warp_regs = ((uint32_t)r * 32u + 255u) / 256u * 256u;
    const uint32_t by_regs = 65536u / warp_regs / (threads / 32u), by_smem = (uint32_t)((228u << 10) / (smem + 2048));
    *per_sm = (int)std::max(1u, std::min(std::min(by_regs, by_smem), std::min(2048u / threads, 32u)));
    return CO3_OK;
}

struct Launch {
    bool backward;
    uint32_t n_clients;
    int sms;
    cudaStream_t st;
};

template <uint32_t kGroups>
int launch_groups(const NormArgs& a, const Launch& l) {
    constexpr uint32_t width = kReduceThreads / kGroups;
    const uint64_t blocks = (uint64_t)((a.cols + width - 1) / width) * 2 * l.n_clients;
    CO3_CUDA(launch_behind(norm_reduce_kernel<kGroups>, dim3((uint32_t)blocks), dim3(kReduceThreads), 0, l.st, a));
    return CO3_OK;
}

int launch_reduce(const NormArgs& a, const Launch& l) {
    if (a.parts < 2 || (!a.dweight && !a.dbias)) return CO3_OK;
    return a.parts < 4 ? launch_groups<2>(a, l) : a.parts < 8 ? launch_groups<4>(a, l) : a.parts < 16 ? launch_groups<8>(a, l) : launch_groups<16>(a, l);
}

template <typename T, int kVec, int kCh, bool kWarpRow, bool kBackward, int kMaxThreads>
int launch_rows(NormArgs a, const Launch& l, uint32_t threads) {
    const uint32_t warps = threads / 32u, rows_at_once = kWarpRow ? warps : 1;
    // the deepest ring with which two blocks fit an SM, or else one block
    const size_t turn = (size_t)warps * (kBackward ? 2 * Stretch<T, kVec, kCh>::kBytes + 16 : Stretch<T, kVec, kCh>::kBytes);
    a.ring = 1;
    for (uint32_t r : {8u, 4u, 3u, 2u})
        if (r * turn <= (r > 4 ? kRingBytes / 8 : r > 2 ? kRingBytes / 2 : kRingBytes)) { a.ring = r; break; }
    size_t smem = a.ring * turn;
    int per_sm = 0;
    if constexpr (!kBackward) {
        auto* kernel = norm_forward_kernel<T, kVec, kCh, kWarpRow, kMaxThreads>;
        const int e = blocks_per_sm<norm_forward_kernel<T, kVec, kCh, kWarpRow, kMaxThreads>>(threads, smem, &per_sm);
        if (e != CO3_OK) return e;
        const uint64_t want = (a.rows + rows_at_once - 1) / rows_at_once;
        const uint32_t grid = (uint32_t)std::min<uint64_t>(want, (uint64_t)l.sms * per_sm);
        CO3_CUDA(launch_behind(kernel, dim3(grid), dim3(threads), smem, l.st, a));
        return CO3_OK;
    } else {
        auto* kernel = norm_backward_kernel<T, kVec, kCh, kWarpRow, kMaxThreads>;
        if (kWarpRow) smem = std::max(smem, (size_t)8 * a.cols * warps);
        const int e = blocks_per_sm<norm_backward_kernel<T, kVec, kCh, kWarpRow, kMaxThreads>>(threads, smem, &per_sm);
        if (e != CO3_OK) return e;
        const uint64_t fill = std::max<uint64_t>(1, (uint64_t)l.sms * per_sm / l.n_clients);
        const uint64_t most = std::max<uint64_t>(1, (a.rows + rows_at_once - 1) / rows_at_once);
        a.parts = (uint32_t)std::min(std::min(fill, most), max_parts(a.rows, l.n_clients));
        // One block a client needs no second launch and no partial sums: taken where the turns it adds cost less, a turn
        // about 40 ns an element of a lane, the launch 4.6 us, partial sums 5000 bytes a ns.  (us, one block against
        // several: 100 clients x 64 x 512 fp32 15.8 and 20.3, 100 x 16 x 4096 bf16 19 and 31, 30 x 64 x 1024 bf16 17 and 14.)
        const uint64_t added = most - (most + a.parts - 1) / a.parts;
        if ((a.dweight || a.dbias) && added * 40 * kVec * kCh < 4600 + l.n_clients * (uint64_t)a.parts * a.cols * 16 / 5000) a.parts = 1;
        CO3_CUDA(launch_behind(kernel, dim3(a.parts * l.n_clients), dim3(threads), smem, l.st, a));
        return launch_reduce(a, l);
    }
}

template <typename T, int kVec, int kElems, int kMaxThreads>
int launch_block(const NormArgs& a, const Launch& l) {
    constexpr int kCh = kElems / kVec;
    const uint32_t chunks = (a.cols + kVec - 1) / kVec, threads = (chunks + 32u * kCh - 1) / (32u * kCh) * 32u;
    if (threads > (uint32_t)kMaxThreads) return -1;
    return l.backward ? launch_rows<T, kVec, kCh, false, true, kMaxThreads>(a, l, threads) : launch_rows<T, kVec, kCh, false, false, kMaxThreads>(a, l, threads);
}
template <typename T, int kVec, int kCh>
int launch_warp(const NormArgs& a, const Launch& l) {
    if ((uint64_t)kCh * kVec * 32 < a.cols) return -1;
    constexpr int kForward = kWarpRowThreads<T, kCh * kVec, false>, kBackward = kWarpRowThreads<T, kCh * kVec, true>;
    return l.backward ? launch_rows<T, kVec, kCh, true, true, kBackward>(a, l, kBackward) : launch_rows<T, kVec, kCh, true, false, kForward>(a, l, kForward);
}

// Elements a thread.  A warp takes the row if up to 32 elements a lane suffice, the fewest that do; wider rows go to
// blocks of up to 512 threads, forward with 32 elements a thread, backward with 16 as far as they reach, since its sums
// take registers too (unaligned rows of up to 4096 columns excepted: 128 threads suffice for them).  us, 32 against 16
// elements: forward bf16 16384 x 4096 48 and 66, 16384 x 2048 27 and 32; backward bf16 16384 x 4096 87 and 82, 16384 x
// 2048 60 and 50, 8192 x 8191 f16 265 and 140; backward 65536 x 1024, a warp with 32 against two with 16: 72 and 90.
template <typename T, int kVec, int... kChs>
int launch_width(const NormArgs& a, const Launch& l) {
    int e = -1;
    (void)(((e = launch_warp<T, kVec, kChs>(a, l)) >= 0) || ...);
    if (e >= 0) return e;
    if (l.backward && kVec > 1) {
        e = launch_block<T, kVec, 16, 256>(a, l);
        if (e < 0) e = launch_block<T, kVec, 16, 512>(a, l);
    } else {
        e = launch_block<T, kVec, 32, 128>(a, l);
        if (e < 0 && l.backward) e = launch_block<T, kVec, 16, 512>(a, l);
    }
    return e >= 0 ? e : launch_block<T, kVec, 32, 512>(a, l);
}

template <typename T>
int launch_type(NormArgs a, const Launch& l) {
    if (a.cols > kMaxCols) {
        const uint64_t rows = l.backward ? a.rows * l.n_clients : a.rows;
        const uint32_t grid = (uint32_t)std::min<uint64_t>(rows, 2ull * l.sms);
        if (!l.backward) {
            CO3_CUDA(launch_behind(norm_forward_long_kernel<T>, dim3(grid), dim3(kLongThreads), 0, l.st, a));
            return CO3_OK;
        }
        if (a.dweight || a.dbias) {  // before dx, which may lie over dy or x
            const uint64_t col_blocks = (a.cols + 255u) / 256u;
            const uint64_t fill = std::max<uint64_t>(1, 8ull * l.sms / (col_blocks * l.n_clients));
            a.parts = (uint32_t)std::min(fill, max_parts(a.rows, l.n_clients));
            CO3_CUDA(launch_behind(norm_dw_long_kernel<T>, dim3((uint32_t)(col_blocks * l.n_clients * a.parts)), dim3(256), 0, l.st, a));
            const int e = launch_reduce(a, l);
            if (e != CO3_OK) return e;
        }
        if (a.out && rows) CO3_CUDA(launch_behind(norm_dx_long_kernel<T>, dim3(grid), dim3(kLongThreads), 0, l.st, a, rows));
        return CO3_OK;
    }
    constexpr int kVec = 16 / sizeof(T);
    const size_t s = sizeof(T);
    // 16 bytes at a time where every row starts and ends on a 16-byte boundary
    const bool wide = a.cols % kVec == 0 && aligned(a.x, 16) && aligned(a.out, 16) && aligned(a.dy, 16) && a.x_stride * s % 16 == 0 &&
                      a.out_stride * s % 16 == 0 && a.dy_stride * s % 16 == 0;
    if constexpr (sizeof(T) == 4) {
        if (wide) return launch_width<T, kVec, 1, 2, 4, 8>(a, l);
    } else {
        if (wide) return launch_width<T, kVec, 1, 2, 4>(a, l);
    }
    return launch_width<T, 1, 2, 4, 8, 16, 32>(a, l);
}

int launch_norm(int type, const NormArgs& a, const Launch& l) {
    if (type == CO3_F32) return launch_type<float>(a, l);
    if (type == CO3_F16) return launch_type<__half>(a, l);
    return launch_type<__nv_bfloat16>(a, l);
}

bool valid_layout(int type, const void* p, uint64_t stride, uint64_t rows, uint32_t cols) {
    return p && aligned(p, type_size(type)) && stride >= cols && stride < (1ull << 40) && rows < (1ull << 40);
}

}  // namespace

extern "C" {

int co3_layer_norm_workspace_bytes(uint64_t rows, uint32_t cols, uint32_t n_clients, size_t* out) {
    if (!out || n_clients == 0 || rows >= (1ull << 40)) return CO3_ERR_INVALID_ARG;
    const uint64_t parts = max_parts(rows, n_clients);
    const uint64_t bytes = parts > 1 ? parts * n_clients * 2 * cols * 4 : 0;
    *out = (size_t)std::max<uint64_t>(256, (bytes + 255u) & ~(uint64_t)255u);
    return CO3_OK;
}

int co3_layer_norm(const void* x, int type, const float* weight, const float* bias, void* y, uint64_t rows, uint32_t cols,
                   uint64_t x_row_stride, uint64_t y_row_stride, float eps, float* mean, float* rstd, void* stream) {
    if (type < CO3_F32 || type > CO3_BF16 || !(eps >= 0.0f) || !isfinite(eps) || cols >= (1u << 31)) return CO3_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return CO3_OK;
    if (!valid_layout(type, x, x_row_stride, rows, cols) || !valid_layout(type, y, y_row_stride, rows, cols) ||
        !aligned(weight, 4) || !aligned(bias, 4) || !aligned(mean, 4) || !aligned(rstd, 4))
        return CO3_ERR_INVALID_ARG;
    NormArgs a = {};
    a.x = x; a.weight = weight; a.bias = bias; a.out = y;
    a.mean = mean; a.rstd = rstd;
    a.rows = rows; a.cols = cols;
    a.x_stride = x_row_stride; a.out_stride = y_row_stride;
    a.eps = eps;
    Launch l = {false, 1, 0, static_cast<cudaStream_t>(stream)};
    const int e = sm_count(&l.sms);
    return e != CO3_OK ? e : launch_norm(type, a, l);
}

int co3_layer_norm_backward(const void* dy, const void* x, int type, const float* weight, const float* mean, const float* rstd,
                            void* dx, float* dweight, float* dbias, uint64_t rows, uint32_t cols, uint64_t dy_row_stride,
                            uint64_t x_row_stride, uint64_t dx_row_stride, uint32_t n_clients, uint64_t client_stride_elems,
                            int accumulate, void* workspace, size_t workspace_bytes, void* stream) {
    if (type < CO3_F32 || type > CO3_BF16 || n_clients == 0 || cols >= (1u << 31)) return CO3_ERR_INVALID_ARG;
    if (cols == 0 || (!dx && !dweight && !dbias)) return CO3_OK;
    if (rows && (!valid_layout(type, dy, dy_row_stride, rows, cols) || !valid_layout(type, x, x_row_stride, rows, cols) || !mean || !rstd))
        return CO3_ERR_INVALID_ARG;
    if (rows && dx && !valid_layout(type, dx, dx_row_stride, rows, cols)) return CO3_ERR_INVALID_ARG;
    if (!aligned(weight, 4) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dweight, 4) || !aligned(dbias, 4) ||
        rows >= ((1ull << 40) + n_clients - 1) / n_clients ||  // 2^40 rows of all clients
        (n_clients > 1 && (dweight || dbias) && client_stride_elems < cols))
        return CO3_ERR_INVALID_ARG;
    size_t need = 0;
    co3_layer_norm_workspace_bytes(rows, cols, n_clients, &need);
    if (!workspace || !aligned(workspace, 256)) return CO3_ERR_INVALID_ARG;
    if (workspace_bytes < need) return CO3_ERR_CAPACITY;
    // grids of the reductions: 2^31 - 1 blocks at most
    if ((uint64_t)((cols + 31u) / 32u) * 2 * n_clients >= (1ull << 31)) return CO3_ERR_INVALID_ARG;
    NormArgs a = {};
    a.x = x; a.dy = dy; a.weight = weight; a.out = dx;
    a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
    a.rows = rows; a.all_rows = rows * n_clients; a.cols = cols;
    a.x_stride = x_row_stride; a.dy_stride = dy_row_stride; a.out_stride = dx ? dx_row_stride : 0;
    a.dweight = dweight; a.dbias = dbias;
    a.client_stride = client_stride_elems;
    a.parts = 1;
    a.accumulate = accumulate;
    a.partial = static_cast<float*>(workspace);
    Launch l = {true, n_clients, 0, static_cast<cudaStream_t>(stream)};
    const int e = sm_count(&l.sms);
    return e != CO3_OK ? e : launch_norm(type, a, l);
}

}  // extern "C"
