// Orthogonalised updates of small matrices: the whole of one matrix (norm, all steps, result) in one cluster of blocks,
// without a trip through memory in between.
//
// The short side has at most 128 entries, the long side is cut into slices of 128, one per block: X stays in shared
// memory as an operand (64 KB a slice), A and then B are held whole by every block.  Per step: the block's share of A from
// its slice, added up over the cluster (every block sends the rows of its share to the blocks that add them up, and these
// send the sums to all, through distributed shared memory); B, by every block for itself; X <- a X + B X, slice by
// slice.  What it costs is latency: three short products and an exchange a step.
#include <cuda_runtime.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "co3.h"
#include "co3_device.cuh"
#include "co3_launch.cuh"
#include "co3_orth.cuh"
#include "co3_orth_small.h"
#include "co3_types.cuh"

namespace co3 {

constexpr int kSmallThreads = 512;  // a thread has 32 columns of a row of every product
constexpr uint32_t kOperand = 2 * kBlock;  // 128 x 128
constexpr uint32_t kRawPitch = 129;        // floats between rows of X before it is scaled
constexpr uint32_t kRawBytes = 128 * kRawPitch * 4;
// From A's operand to the shares that other blocks send.  X before it is scaled lies over A's operand, and as no barrier
// of the cluster stands between its last use in one block and the first shares sent by another, it has to end before them.
constexpr uint32_t kSharesOff = kRawBytes > kOperand ? kRawBytes : kOperand;
static_assert(kSharesOff >= kRawBytes && kSharesOff >= kOperand && kSharesOff % 16 == 0, "nothing that others write overlaps");

struct SmallSmem {
    double sums[kSmallCluster];
    double warp_sum[kSmallThreads / 32];
    uint64_t done, arrived;
    uint32_t tmem;
    double factor;
};
constexpr size_t kSmallBytes = 1024 + kOperand + kSharesOff + kOperand + sizeof(SmallSmem);
static_assert(kSmallBytes <= 227 * 1024, "shared memory of a block");

struct SmallKernelArgs {
    SmallBatch batch;
    SmallCall call;
    uint32_t first, ctas;  // matrices from `first` on, with this many blocks each
};

__device__ __forceinline__ void cluster_sync() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void peer_store16(uint32_t addr, float x, float y, float z, float w) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(x), "f"(y), "f"(z), "f"(w) : "memory");
}
// Bytes of this block's shared memory to the same place of another block, counted by that block's barrier.
__device__ __forceinline__ void peer_copy(uint32_t addr, uint32_t rank, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(peer_addr(addr, rank)),
                 "r"(addr), "r"(bytes), "r"(peer_addr(bar, rank))
                 : "memory");
}
__device__ __forceinline__ void peer_store_f64(uint32_t addr, double v) {
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(addr), "d"(v) : "memory");
}

// Sums of 32 columns each of a product of 128 x 128 x (16 steps), into up to four accumulators of tensor memory.
template <bool kTa, bool kTb>
__device__ __forceinline__ void small_product(uint32_t tmem, uint32_t a, uint32_t b, uint32_t steps, uint64_t* done) {
    constexpr uint32_t instr = instr_desc(kTa, kTb, 128, 128), lo = kPlane >> 4;
    const uint64_t a0 = smem_desc(a, kTa, kBlock), b0 = smem_desc(b, kTb, kBlock);
    auto at = [](uint64_t base, bool t, uint32_t s) { return base + (t ? s * (2048u >> 4) : (s >> 2) * (kBlock >> 4) + (s & 3u) * (32u >> 4)); };
#pragma unroll
    for (uint32_t s = 0; s < 8; s += 2) {
        const uint32_t d = tmem + (s / 2) * 128u;
        // the corrections first, 2^11 times too large; the first product of the hi planes scales them down
        if (s + 1 < steps) {
            tc_mma(d, at(a0, kTa, s), at(b0, kTb, s) + lo, instr, false);
            tc_mma(d, at(a0, kTa, s + 1), at(b0, kTb, s + 1) + lo, instr, true);
            tc_mma(d, at(a0, kTa, s) + lo, at(b0, kTb, s), instr, true);
            tc_mma(d, at(a0, kTa, s + 1) + lo, at(b0, kTb, s + 1), instr, true);
            tc_mma<kLoBits>(d, at(a0, kTa, s), at(b0, kTb, s), instr, true);
            tc_mma(d, at(a0, kTa, s + 1), at(b0, kTb, s + 1), instr, true);
        } else if (s < steps) {
            tc_mma(d, at(a0, kTa, s), at(b0, kTb, s) + lo, instr, false);
            tc_mma(d, at(a0, kTa, s) + lo, at(b0, kTb, s), instr, true);
            tc_mma<kLoBits>(d, at(a0, kTa, s), at(b0, kTb, s), instr, true);
        }
    }
    tc_commit(done);
}

template <typename T>
__global__ void __launch_bounds__(kSmallThreads, 1) orth_small_kernel(const __grid_constant__ SmallKernelArgs a) {
    wait_for_previous_kernel();
    extern __shared__ unsigned char smem_raw[];
    unsigned char* op_x = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    unsigned char *op_a = op_x + kOperand, *shares = op_a + kSharesOff;  // op_a: A, then B in its place
    SmallSmem& sm = *reinterpret_cast<SmallSmem*>(shares + kOperand);
    float* raw = reinterpret_cast<float*>(op_a);  // [128][kRawPitch], before the first step
    const SmallCall& call = a.call;
    const SmallMat& t = a.batch.mat[a.first + blockIdx.x / a.ctas];
    const uint32_t rank = blockIdx.x % a.ctas, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
    const bool tall = t.rows > t.cols;
    const uint32_t m = tall ? t.cols : t.rows, n = tall ? t.rows : t.cols;
    const uint32_t n0 = rank * 128u, nn = n > n0 ? min(n - n0, 128u) : 0u;  // this block's columns of X
    const uint32_t mr = (m + 15u) / 16u * 16u, steps_m = mr / 16u, steps_n = (nn + 15u) / 16u;
    if (call.clear_result && blockIdx.x == 0 && tid == 0) {
        co3_result r = {};
        r.first_bad_chunk = 0xffffffffu;
        *call.res = r;
        __threadfence();
    }
    if (tid == 0) { mbar_init(&sm.done, 1); mbar_init(&sm.arrived, 1); }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&sm.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    __syncwarp();
    if (a.ctas > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");

    // X before scaling (zeros up to mr x 128), its sum of squares; momentum
    double sum = 0.0;
    const T* in = static_cast<const T*>(call.in);
    const uint32_t lines = tall ? 128u : mr;
    for (uint32_t i0 = 0; i0 < lines * 128u; i0 += 16 * kSmallThreads) {
        float u[16];
        uint64_t at[16];
        bool have[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const uint32_t i = i0 + j * kSmallThreads + tid, hi = i >> 7, lo = i & 127u;  // lo runs along the caller's rows
            const uint32_t r = tall ? lo : hi, c = tall ? hi : lo;
            have[j] = r < m && c < nn;
            at[j] = t.in_off + (tall ? (uint64_t)(n0 + c) * t.in_stride + r : (uint64_t)r * t.in_stride + n0 + c);
            u[j] = have[j] ? to_float(in[at[j]]) : 0.0f;
        }
        if (call.momentum) {
            float buf[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) buf[j] = have[j] ? call.momentum[at[j]] : 0.0f;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                buf[j] = __fmaf_rn(call.mu, buf[j], u[j]);
                if (have[j]) call.momentum[at[j]] = buf[j];
                u[j] = call.nesterov ? __fmaf_rn(call.mu, buf[j], u[j]) : buf[j];
            }
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const uint32_t i = i0 + j * kSmallThreads + tid, hi = i >> 7, lo = i & 127u;
            const uint32_t r = tall ? lo : hi, c = tall ? hi : lo;
            if (r < mr && c < 128u) raw[r * kRawPitch + c] = u[j];
            sum = fma((double)u[j], (double)u[j], sum);
        }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (lane == 0) sm.warp_sum[warp] = sum;
    __syncwarp();
    if (a.ctas > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // all blocks have started
    __syncthreads();
    if (tid < a.ctas) {
        double s = 0.0;
        for (int w = 0; w < kSmallThreads / 32; ++w) s += sm.warp_sum[w];
        if (a.ctas > 1) peer_store_f64(peer_addr(smem_addr(&sm.sums[rank]), tid), s);
        else sm.sums[0] = s;
    }
    tc_fence_before();
    if (a.ctas > 1) cluster_sync(); else __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm.tmem;
    const float s_val = orth_s(m, n), inv_s = 1.0f / s_val;
    if (tid == 0) {
        double total = 0.0;
        for (uint32_t p = 0; p < a.ctas; ++p) total += sm.sums[p];
        const double d = sqrt(total) + (double)call.ns.eps;
        sm.factor = d > 0.0 ? (double)s_val / d : 0.0;  // an all-zero matrix without eps stays zero
        if (!isfinite(total)) {
            sm.factor = (double)NAN;
            if (rank == 0) {
                set_status(call.res, CO3_ERR_NONFINITE);
                atomicMin(&call.res->first_bad_chunk, t.index);
                atomicAdd(reinterpret_cast<unsigned long long*>(&call.res->n_nonfinite), 1ull);
            }
        }
    }
    __syncthreads();
    {
        const double f = sm.factor;
        for (uint32_t i = tid; i < 128u * 16u; i += kSmallThreads) {
            const uint32_t r = i & 127u, piece = i >> 7;
            if (r >= mr) continue;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (float)((double)raw[r * kRawPitch + piece * 8 + e] * f);
            uint4 hi, lo;
            split8(v, hi, lo);
            unsigned char* p = op_x + (piece >> 3) * kBlock + swizzled(r, piece & 7u);
            *reinterpret_cast<uint4*>(p) = hi;
            *reinterpret_cast<uint4*>(p + kPlane) = lo;
        }
    }

    // this thread's row and first of 32 columns of a product; what lies beyond mr is not read
    const uint32_t quad = warp & 3u, row = quad * 32u + lane, col0 = (warp >> 2) * 32u;
    const bool in_m = quad * 32u < mr && col0 < mr, in_x = quad * 32u < mr && col0 < nn;
    // rows of A that a block adds up
    const uint32_t sum_rows = (mr + a.ctas - 1) / a.ctas, my_row0 = rank * sum_rows, my_rows = my_row0 < mr ? min(sum_rows, mr - my_row0) : 0u;
    uint32_t parity = 0;
    bool good = true;
    float acc[32];
    const std::false_type as_is;
    const std::true_type transposed;
    // One product, all threads: acc <- this thread's 32 sums.
    auto product = [&](unsigned char* pa, auto ta, unsigned char* pb, auto tb, uint32_t steps) {
        fence_async_all();  // operands were written by ordinary stores
        __syncthreads();
        if (tid == 0 && steps > 0) {
            tc_fence_after();
            small_product<decltype(ta)::value, decltype(tb)::value>(tmem, smem_addr(pa), smem_addr(pb), steps, &sm.done);
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[i] = 0.0f;
        if (steps == 0) return;
        good = mbar_wait(&sm.done, parity) && good;
        parity ^= 1u;
        tc_fence_after();
        for (uint32_t ch = 0; ch < (steps + 1) / 2; ++ch) {
            float w[32];
            tc_load32(tmem + ((quad * 32u) << 16) + ch * 128u + col0, w);
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[i] = __fadd_rn(acc[i], w[i]);
        }
        tc_fence_before();
    };

    for (uint32_t k = 0; k < call.ns.steps; ++k) {
        const float ca = call.ns.coef[k][0], cb = call.ns.coef[k][1], cc = call.ns.coef[k][2];
        const bool last = k + 1 == call.ns.steps;
        // A = X X^T
        product(op_x, as_is, op_x, as_is, steps_n);
        if (a.ctas == 1) {
            if (in_m) {
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    float w[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] = __fmul_rn(inv_s, acc[p * 8 + e]);
                    uint4 hi, lo;
                    split8(w, hi, lo);
                    unsigned char* to = op_a + (col0 >> 6) * kBlock + swizzled(row, ((col0 & 32u) >> 3) + p);
                    *reinterpret_cast<uint4*>(to) = hi;
                    *reinterpret_cast<uint4*>(to + kPlane) = lo;
                }
            }
        } else {
            // [source block][4 columns][rows]: a warp's rows lie side by side
            if (row < mr && col0 < mr) {
                const uint32_t dest = row / sum_rows, at = ((rank * 32u + col0 / 4u) * sum_rows + row - dest * sum_rows) * 16u;
                const uint32_t to = peer_addr(smem_addr(shares) + at, dest);
#pragma unroll
                for (int p = 0; p < 8; ++p) peer_store16(to + p * sum_rows * 16u, acc[4 * p], acc[4 * p + 1], acc[4 * p + 2], acc[4 * p + 3]);
            }
            if (tid == 0) mbar_arrive_expect_tx(&sm.arrived, 2u * (mr > 64u ? 2u : 1u) * (mr - my_rows) * 128u);
            cluster_sync();
            for (uint32_t i = tid; i < my_rows * (mr / 8u); i += kSmallThreads) {
                const uint32_t piece = i / my_rows, r = i - piece * my_rows;
                float w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = 0.0f;
#pragma unroll 4
                for (uint32_t p = 0; p < a.ctas; ++p) {
                    const float4 x = *reinterpret_cast<const float4*>(shares + ((p * 32u + 2 * piece) * sum_rows + r) * 16u);
                    const float4 y = *reinterpret_cast<const float4*>(shares + ((p * 32u + 2 * piece + 1) * sum_rows + r) * 16u);
                    w[0] += x.x; w[1] += x.y; w[2] += x.z; w[3] += x.w;
                    w[4] += y.x; w[5] += y.y; w[6] += y.z; w[7] += y.w;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = __fmul_rn(inv_s, w[e]);
                uint4 hi, lo;
                split8(w, hi, lo);
                unsigned char* to = op_a + (piece >> 3) * kBlock + swizzled(my_row0 + r, piece & 7u);
                *reinterpret_cast<uint4*>(to) = hi;
                *reinterpret_cast<uint4*>(to + kPlane) = lo;
            }
            fence_async_smem();
            __syncthreads();
            {
                const uint32_t peer = tid >> 2, plane = tid & 1u, block = (tid >> 1) & 1u;
                if (peer < a.ctas && peer != rank && my_rows > 0 && (block == 0 || mr > 64u))
                    peer_copy(smem_addr(op_a) + block * kBlock + plane * kPlane + my_row0 * 128u, peer, my_rows * 128u, smem_addr(&sm.arrived));
            }
            good = mbar_wait(&sm.arrived, k & 1u) && good;
        }
        // B = b A + c A A, in the last step + a I
        product(op_a, as_is, op_a, as_is, steps_m);
        if (in_m) {
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const uint32_t at = (col0 >> 6) * kBlock + swizzled(row, ((col0 & 32u) >> 3) + p);
                float l[8], w[8];
                join8(*reinterpret_cast<const uint4*>(op_a + at), *reinterpret_cast<const uint4*>(op_a + at + kPlane), l);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    w[e] = __fmaf_rn(cb, l[e], __fmul_rn(__fmul_rn(cc, inv_s), acc[p * 8 + e]));
                    if (last && col0 + p * 8u + e == row) w[e] = __fmaf_rn(ca, s_val, w[e]);
                }
                uint4 hi, lo;
                split8(w, hi, lo);
                *reinterpret_cast<uint4*>(op_a + at) = hi;
                *reinterpret_cast<uint4*>(op_a + at + kPlane) = lo;
            }
        }
        if (!last) {  // X <- a X + B X
            product(op_a, as_is, op_x, transposed, nn ? steps_m : 0u);
            if (in_x) {
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    unsigned char* at = op_x + (col0 >> 6) * kBlock + swizzled(row, ((col0 & 32u) >> 3) + p);
                    float l[8], w[8];
                    join8(*reinterpret_cast<const uint4*>(at), *reinterpret_cast<const uint4*>(at + kPlane), l);
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] = __fmaf_rn(ca, l[e], __fmul_rn(inv_s, acc[p * 8 + e]));
                    uint4 hi, lo;
                    split8(w, hi, lo);
                    *reinterpret_cast<uint4*>(at) = hi;
                    *reinterpret_cast<uint4*>(at + kPlane) = lo;
                }
            }
        } else if (tall) {  // rows of the product run along the caller's rows
            product(op_a, as_is, op_x, transposed, nn ? steps_m : 0u);
        } else {
            product(op_x, transposed, op_a, as_is, nn ? steps_m : 0u);
        }
    }
    {
        // thread's row: the caller's column c; its columns: the caller's rows r0 ..
        const uint32_t c = tall ? row : n0 + row, r0 = (tall ? n0 : 0u) + col0;
        const uint32_t n_r = tall ? n0 + nn : m;
        const uint32_t cnt = (tall ? row < m : row < nn) && r0 < n_r ? min(32u, n_r - r0) : 0u;
        const uint64_t first = t.out_off + (uint64_t)r0 * t.out_stride + c;
        const float f = __fmul_rn(__fmul_rn(t.scale, inv_s), inv_s);
        put_result<32>(call.out, call.out_kind, first, t.out_stride, cnt, f, acc, call.lr, call.shrink);
    }
    if (!good) set_status(call.res, CO3_ERR_CUDA);
    if (a.ctas > 1) cluster_sync();  // what this block sent has been read
    else __syncthreads();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

template <typename T>
static int launch_small_type(SmallKernelArgs& a, uint32_t n_mats, cudaStream_t st) {
    static std::atomic<bool> ready[64];
    int dev = 0;
    CO3_CUDA(cudaGetDevice(&dev));
    if (dev >= 64 || !ready[dev].load(std::memory_order_relaxed)) {
        CO3_CUDA(cudaFuncSetAttribute(orth_small_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmallBytes));
        CO3_CUDA(cudaFuncSetAttribute(orth_small_kernel<T>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        if (dev < 64) ready[dev].store(true, std::memory_order_relaxed);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(n_mats * a.ctas);
    cfg.blockDim = dim3(kSmallThreads);
    cfg.dynamicSmemBytes = kSmallBytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = a.ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    CO3_CUDA(cudaLaunchKernelEx(&cfg, orth_small_kernel<T>, a));
    return CO3_OK;
}

int orth_small_run(const SmallBatch& batch, const SmallCall& call, int in_type, cudaStream_t st) {
    SmallKernelArgs a = {};
    a.call = call;
    for (uint32_t ctas = 1; ctas <= kSmallCluster; ctas *= 2) {
        uint32_t n = 0;
        for (uint32_t k = 0; k < batch.n_mats; ++k)
            if (small_ctas(batch.mat[k].rows, batch.mat[k].cols) == ctas) a.batch.mat[n++] = batch.mat[k];
        if (n == 0) continue;
        a.batch.n_mats = n;
        a.ctas = ctas;
        const int e = in_type == CO3_F32 ? launch_small_type<float>(a, n, st)
                      : in_type == CO3_F16 ? launch_small_type<__half>(a, n, st) : launch_small_type<__nv_bfloat16>(a, n, st);
        if (e != CO3_OK) return e;
        a.call.clear_result = 0;
    }
    return CO3_OK;
}

}  // namespace co3
