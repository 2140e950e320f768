// Gradients of a linear layer's weights and biases from the inputs that were kept in 8 bits, for each client into its own vector:
//     dW_u = sum over the client's rows r of dy[r]^T x[r],    db_u = sum of dy[r].
//
// The sum runs along the rows, along which the 8-bit blocks' scales differ, so the tensor cores cannot apply them: values are
// brought to bf16 on the way into shared memory, which is exact (four significant bits times a power of two).  dy is cut into parts
// of eight significant bits, one for bf16, two for fp16, three for fp32, so that nothing of it is lost: the products are exact and
// the sums fp32.  Tiles are 128 inputs (one block of columns: tensor memory's lanes, so that a warp writes neighbouring entries of
// dW) by 256 outputs; both operands lie in shared memory as they come, a row of the batch per row.
//
// Eight warps bring the rows in, 64 at a time, take the sums out after every 256 rows (the tensor core cuts what it adds
// towards zero) and add them up in registers; one thread issues the products.  Few tiles: the rows are divided, and a second
// launch adds the parts in order.
#include <algorithm>
#include <atomic>

#include "co3_f8.cuh"
#include "co3_launch.cuh"
#include "co3_orth.cuh"

namespace co3 {
namespace {

constexpr uint32_t kChunk = 64;              // rows of a stage
constexpr uint32_t kSumChunks = 4;           // chunks that tensor memory adds up
constexpr uint32_t kOuts = 256;              // outputs of a tile
constexpr uint32_t kAtom = kChunk * 128;     // bytes of 64 columns of a stage
constexpr uint32_t kPlaneX = 2 * kAtom, kPlaneDy = 4 * kAtom;
constexpr uint32_t kSmsAssumed = 148;        // how rows are divided does not depend on the device

struct WeightArgs {
    const void* dy;
    uint64_t dy_stride;
    const uint8_t *x, *x_scales;
    uint64_t x_rows;                         // rows of the packed inputs, padded
    uint64_t rows;                           // of a client
    uint32_t outs, ins, clients;
    uint32_t k_tiles, n_tiles, chunks, parts;
    float *dw, *db;
    uint64_t client_stride;
    int accumulate;
    float* partial;                          // parts x clients x outs x ins, then parts x clients x outs
    co3_result* res;
};

template <typename T>
struct Parts;
template <> struct Parts<float> { static constexpr int kParts = 3; static constexpr uint32_t kStages = 2; };
template <> struct Parts<__half> { static constexpr int kParts = 2; static constexpr uint32_t kStages = 2; };
template <> struct Parts<__nv_bfloat16> { static constexpr int kParts = 1; static constexpr uint32_t kStages = 4; };

struct WeightSmem {
    uint64_t full[4], empty[4], sum_full[2], sum_empty[2], done;
    uint32_t tmem, failed;
};
template <typename T>
constexpr uint32_t kStageBytesW = kPlaneX + Parts<T>::kParts * kPlaneDy;
template <typename T>
constexpr uint32_t kSmemW = 1024 + Parts<T>::kStages * kStageBytesW<T> + ((sizeof(WeightSmem) + 15) & ~15u);

// D fp32, A and B bf16, both with the sum along their rows
__host__ __device__ constexpr uint32_t weight_instr(uint32_t cols) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((cols / 8u) << 17) | (8u << 24);
}

// A tile, and the chunks of rows that it sums.
struct Place {
    uint32_t u, part, n0, kt, c0, c1;
};
__device__ __forceinline__ Place find_place(const WeightArgs& a, uint32_t t) {
    Place p;
    p.kt = t % a.k_tiles;
    t /= a.k_tiles;
    p.n0 = t % a.n_tiles * kOuts;
    t /= a.n_tiles;
    p.part = t % a.parts;
    p.u = t / a.parts;
    p.c0 = (uint32_t)((uint64_t)a.chunks * p.part / a.parts);
    p.c1 = (uint32_t)((uint64_t)a.chunks * (p.part + 1) / a.parts);
    return p;
}

// What a thread brings in of a chunk.  Its pieces of x: rows tid / 8 and 32 more, 16 columns each.  Of dy a warp has 32 columns
// and all rows, so that it has their sums by itself: at 16 bytes a time or more, a thread eight neighbouring columns of eight
// rows (rows four apart next to each other: fewer bank conflicts); at one element a time, one column of all rows.
template <typename T, bool kWide>
struct Piece {
    static constexpr int kParts = Parts<T>::kParts;
    static constexpr int kLoads = kWide ? (int)(sizeof(T) / 2) : 1;   // 16-byte loads of eight columns
    static constexpr int kSums = kWide ? 8 : 1;                       // columns of a thread
    uint4 x[2];
    uint32_t scale[2];
    uint4 wide[kWide ? 8 : 1][kLoads];
    T single[kWide ? 1 : kChunk];

    static __device__ __forceinline__ uint32_t column(uint32_t tid) { return kWide ? (tid >> 5) * 32u + (tid & 3u) * 8u : tid; }
    static __device__ __forceinline__ uint32_t row(uint32_t tid, int j) { return ((tid >> 3) & 3u) + (tid & 4u) + 8u * j; }

    __device__ __forceinline__ void fetch(const WeightArgs& a, const Place& p, uint32_t c, uint32_t tid) {
        const uint64_t row0 = p.u * a.rows + (uint64_t)c * kChunk;
        const uint32_t rows = (uint32_t)min((uint64_t)kChunk, a.rows - (uint64_t)c * kChunk);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t i = (tid >> 3) + 32u * j;
            x[j] = make_uint4(0, 0, 0, 0);
            scale[j] = 127u;
            if (i < rows) {
                const uint64_t row = row0 + i;
                x[j] = __ldg(reinterpret_cast<const uint4*>(a.x + f8_row(a.x_rows, p.kt, row) + ((tid & 7u) << 4)));
                scale[j] = __ldg(a.x_scales + ((p.kt >> 2) * (a.x_rows >> 7) + (row >> 7)) * kF8Scales + f8_scale_at((uint32_t)row & 127u, p.kt));
            }
        }
        const uint32_t col = column(tid);
        const T* from = static_cast<const T*>(a.dy) + row0 * a.dy_stride + p.n0 + col;
        if constexpr (kWide) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t i = row(tid, j);
#pragma unroll
                for (int l = 0; l < kLoads; ++l) {
                    wide[j][l] = make_uint4(0, 0, 0, 0);
                    // (eight columns of four bytes may end after the first load)
                    if (i < rows && p.n0 + col + l * (16 / sizeof(T)) < a.outs) wide[j][l] = __ldg(reinterpret_cast<const uint4*>(from + i * a.dy_stride) + l);
                }
            }
        } else {
#pragma unroll
            for (uint32_t i = 0; i < kChunk; ++i) single[i] = i < rows && p.n0 + col < a.outs ? from[i * a.dy_stride] : from_float<T>(0.0f);
        }
    }

    // The parts of a value, each exact in bf16, as the upper halves of fp32 patterns.
    static __device__ __forceinline__ void cut(float v, uint32_t (&part)[kParts]) {
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
            const uint32_t top = __float_as_uint(v) & 0xffff0000u;
            part[k] = top;
            // an infinity is its own first part
            if (k + 1 < kParts) v = f8_magnitude(v) == 0x7f800000u ? 0.0f : __fsub_rn(v, __uint_as_float(top));
        }
    }

    __device__ __forceinline__ void put(unsigned char* stage, uint32_t row_low, uint32_t tid, bool with_db, float (&db)[kSums]) const {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t i = (tid >> 3) + 32u * j;
            const uint32_t piece = (tid & 7u) ^ ((row_low + i) & 7u);  // 16 columns from 16 piece on
            const float s = __uint_as_float(scale[j] << 23);
            uint32_t w[8];
            const uint32_t q[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float2 v = f8_to2(q[k >> 1] >> (16 * (k & 1)));
                const __nv_bfloat162 b = __floats2bfloat162_rn(__fmul_rn(v.x, s), __fmul_rn(v.y, s));
                w[k] = *reinterpret_cast<const uint32_t*>(&b);
            }
            unsigned char* to = stage + (piece >> 2) * kAtom + i * 128u;
            const uint32_t unit = (piece & 3u) * 2u, odd = piece >> 2;  // the two halves in another order: fewer bank conflicts
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h) {
                const uint32_t k = h ^ odd;
                *reinterpret_cast<uint4*>(to + f8_piece(i, unit + k)) = k ? make_uint4(w[4], w[5], w[6], w[7]) : make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        const uint32_t col = column(tid);
        unsigned char* planes = stage + kPlaneX + (col >> 6) * kAtom;
        if constexpr (kWide) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t i = row(tid, j);
                unsigned char* to = planes + i * 128u + f8_piece(i, (col >> 3) & 7u);
                const T* e = reinterpret_cast<const T*>(wide[j]);
                if constexpr (kParts == 1) {
                    *reinterpret_cast<uint4*>(to) = wide[j][0];
                } else {
                    uint32_t w[kParts][4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint32_t lo[kParts], hi[kParts];
                        cut(to_float(e[2 * k]), lo);
                        cut(to_float(e[2 * k + 1]), hi);
#pragma unroll
                        for (int m = 0; m < kParts; ++m) w[m][k] = __byte_perm(lo[m], hi[m], 0x7632);
                    }
#pragma unroll
                    for (int m = 0; m < kParts; ++m) *reinterpret_cast<uint4*>(to + m * kPlaneDy) = make_uint4(w[m][0], w[m][1], w[m][2], w[m][3]);
                }
                if (with_db)
#pragma unroll
                    for (int k = 0; k < 8; ++k) db[k] = __fadd_rn(db[k], to_float(e[k]));
            }
        } else {
#pragma unroll
            for (uint32_t i = 0; i < kChunk; ++i) {
                unsigned char* to = planes + i * 128u + f8_piece(i, (col >> 3) & 7u) + (col & 7u) * 2u;
                const float v = to_float(single[i]);
                uint32_t part[kParts];
                cut(v, part);
#pragma unroll
                for (int m = 0; m < kParts; ++m) *reinterpret_cast<uint16_t*>(to + m * kPlaneDy) = (uint16_t)(part[m] >> 16);
                if (with_db) db[0] = __fadd_rn(db[0], v);
            }
        }
    }
};

template <typename T, bool kWide>
__global__ void __launch_bounds__(kF8Threads, 1) f8_weight_kernel(const __grid_constant__ WeightArgs a) {
    extern __shared__ unsigned char smem_raw[];
    constexpr int kParts = Parts<T>::kParts;
    constexpr uint32_t kStages = Parts<T>::kStages, kStageBytes = kStageBytesW<T>;
    unsigned char* ring = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    WeightSmem& sm = *reinterpret_cast<WeightSmem*>(ring + kStages * kStageBytes);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < kStages; ++i) { mbar_init(&sm.full[i], 8); mbar_init(&sm.empty[i], 1); }
        for (uint32_t i = 0; i < 2; ++i) { mbar_init(&sm.sum_full[i], 1); mbar_init(&sm.sum_empty[i], 8); }
        mbar_init(&sm.done, 1);
        sm.failed = 0;
    }
    if (warp == 0) {
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
    const uint32_t tiles = a.k_tiles * a.n_tiles * a.parts * a.clients;

    if (warp < 4) {
        few_registers();
        if (threadIdx.x == 0) {
            uint32_t st = 0, turn = 0, sum = 0, sum_turn = 0;
            bool ok = true;
            for (uint32_t t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
                const Place p = find_place(a, t);
                const uint32_t n = min(kOuts, (a.outs - p.n0 + 15u) & ~15u), instr = weight_instr(0) | ((n / 8u) << 17);
                for (uint32_t c = p.c0; c < p.c1; ++c) {
                    const uint32_t in_sum = (c - p.c0) % kSumChunks;
                    if (in_sum == 0 && sum_turn > 0 && !mbar_wait(&sm.sum_empty[sum], (sum_turn - 1) & 1u)) { ok = false; break; }
                    if (!mbar_wait(&sm.full[st], turn & 1u)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t d = tmem + sum * kOuts, at = smem_addr(ring + st * kStageBytes);
                    const uint64_t dx = smem_desc(at, true, kAtom);
#pragma unroll
                    for (int m = kParts - 1; m >= 0; --m) {
                        const uint64_t dd = smem_desc(at + kPlaneX + m * kPlaneDy, true, kAtom);
#pragma unroll
                        for (uint32_t e = 0; e < kChunk / 16u; ++e) tc_mma(d, dx + e * desc_step(true), dd + e * desc_step(true), instr, in_sum > 0 || m < kParts - 1 || e > 0);
                    }
                    tc_commit(&sm.empty[st]);
                    if (in_sum == kSumChunks - 1 || c + 1 == p.c1) {
                        tc_commit(&sm.sum_full[sum]);
                        if (++sum == 2) { sum = 0; ++sum_turn; }
                    }
                    if (++st == kStages) { st = 0; ++turn; }
                }
            }
            if (!ok) *failed = 1;
            tc_commit(&sm.done);
            mbar_wait(&sm.done, 0);
        }
    } else {
        many_registers();
        const uint32_t tid = threadIdx.x - 128u, quad = warp & 3u, half = (warp - 4u) >> 2, row = quad * 32u + lane;
        using P = Piece<T, kWide>;
        P piece;
        // what is brought in next, ahead of the sums that are taken out
        uint32_t in_t = blockIdx.x, in_c = 0, st = 0, turn = 0;
        Place in = {};
        bool more = in_t < tiles, ok = true;
        float db[P::kSums];
        auto begin = [&]() {
            in = find_place(a, in_t);
            in_c = in.c0;
#pragma unroll
            for (int k = 0; k < P::kSums; ++k) db[k] = 0.0f;
        };
        auto next = [&]() {  // one chunk
            if (turn > 0) {
                ok = lane != 0 || mbar_wait(&sm.empty[st], (turn - 1) & 1u);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) return;
            }
            const bool with_db = a.db != nullptr && in.kt == 0;
            piece.put(ring + st * kStageBytes, (uint32_t)(in.u * a.rows + (uint64_t)in_c * kChunk) & 7u, tid, with_db, db);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.full[st]);
            if (++st == kStages) { st = 0; ++turn; }
            if (++in_c == in.c1) {
                if (with_db) {
                    // the lanes of the same columns
                    if constexpr (kWide)
#pragma unroll
                        for (int k = 0; k < P::kSums; ++k)
#pragma unroll
                            for (int d = 4; d < 32; d *= 2) db[k] = __fadd_rn(db[k], __shfl_xor_sync(0xffffffffu, db[k], d));
                    const uint32_t o0 = in.n0 + P::column(tid);
                    if (!kWide || lane < 4) {
                        const uint64_t dw_all = (uint64_t)a.parts * a.clients * a.outs * a.ins;
                        float* to = (a.parts > 1 ? a.partial + dw_all + ((uint64_t)in.part * a.clients + in.u) * a.outs : a.db + in.u * a.client_stride) + o0;
#pragma unroll
                        for (int k = 0; k < P::kSums; ++k)
                            if (o0 + k < a.outs) to[k] = a.parts == 1 && a.accumulate ? __fadd_rn(to[k], db[k]) : db[k];
                    }
                }
                in_t += gridDim.x;
                more = in_t < tiles;
                if (more) begin();
            }
            if (more) piece.fetch(a, in, in_c, tid);
        };
        uint32_t brought = 0, taken = 0;  // chunks, all tiles together
        if (more) {
            begin();
            piece.fetch(a, in, in_c, tid);
        }
        uint32_t sum = 0, sum_turn = 0;
        for (uint32_t t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
            const Place p = find_place(a, t);
            float acc[kOuts / 2];
            for (uint32_t c = p.c0; c < p.c1; c += kSumChunks) {
                taken += min(kSumChunks, p.c1 - c);
                // the ring is filled before the sum is waited for
                while (ok && more && brought < taken + kStages) { next(); ++brought; }
                if (!ok) break;
                ok = lane != 0 || mbar_wait(&sm.sum_full[sum], sum_turn & 1u);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                const uint32_t from = tmem + ((quad * 32u) << 16) + sum * kOuts + half * (kOuts / 2);
                if (p.n0 + half * (kOuts / 2) < a.outs) {
                    if (c == p.c0) {
#pragma unroll
                        for (int h = 0; h < (int)kOuts / 2; h += 32) tc_load32(from + h, *reinterpret_cast<float(*)[32]>(acc + h));
                    } else {
#pragma unroll
                        for (int h = 0; h < (int)kOuts / 2; h += 32) {
                            float w[32];
                            tc_load32(from + h, w);
#pragma unroll
                            for (int i = 0; i < 32; ++i) acc[h + i] = __fadd_rn(acc[h + i], w[i]);
                        }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.sum_empty[sum]);
                if (++sum == 2) { sum = 0; ++sum_turn; }
            }
            if (!ok) break;
            const uint32_t k = p.kt * 128u + row, o0 = p.n0 + half * (kOuts / 2);
            if (k < a.ins && o0 < a.outs && (a.dw || a.parts > 1)) {
                const uint32_t count = min(kOuts / 2, a.outs - o0);
                const bool add = a.parts == 1 && a.accumulate;
                float* to = (a.parts > 1 ? a.partial + ((uint64_t)p.part * a.clients + p.u) * a.outs * a.ins : a.dw + p.u * a.client_stride) + (uint64_t)o0 * a.ins + k;
#pragma unroll
                for (int i0 = 0; i0 < (int)kOuts / 2; i0 += 16) {
                    if (add)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if ((uint32_t)(i0 + i) < count) acc[i0 + i] = __fadd_rn(to[(uint64_t)(i0 + i) * a.ins], acc[i0 + i]);
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if ((uint32_t)(i0 + i) < count) to[(uint64_t)(i0 + i) * a.ins] = acc[i0 + i];
                }
            }
        }
        if (!ok) *failed = 1;
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    if (threadIdx.x == 0 && *failed && a.res) atomicExch(&a.res->status, CO3_ERR_CUDA);
}

// to[u][i] (+)= sum over the parts of from[part][u][i], in order; with no parts: zeros.
struct JoinArgs {
    const float* from;
    float* to;
    uint64_t count, client_stride;
    uint32_t parts, clients;
    int accumulate;
};
__global__ void __launch_bounds__(256) f8_join_kernel(const __grid_constant__ JoinArgs a) {
    wait_for_previous_kernel();
    const uint64_t all = a.count * a.clients;
    for (uint64_t i = blockIdx.x * 256ull + threadIdx.x; i < all; i += gridDim.x * 256ull) {
        const uint64_t u = i / a.count;
        float* to = a.to + u * a.client_stride + (i - u * a.count);
        float v = a.accumulate ? *to : 0.0f;
        float s = 0.0f;
        for (uint32_t p = 0; p < a.parts; ++p) s = __fadd_rn(s, a.from[p * all + i]);
        *to = a.accumulate ? __fadd_rn(v, s) : s;
    }
}
int launch_join(const JoinArgs& a, cudaStream_t st) {
    if (!a.to || a.count == 0) return CO3_OK;
    const uint64_t blocks = (a.count * a.clients + 255u) / 256u;
    CO3_CUDA(launch_behind(f8_join_kernel, dim3((uint32_t)std::min<uint64_t>(blocks, 148 * 16)), dim3(256), 0, st, a));
    return CO3_OK;
}

// How many parts the rows of a client are divided into: the tiles alone leave multiprocessors idle, and each part has 128 rows.
uint32_t row_parts(uint64_t rows, uint32_t outs, uint32_t ins, uint32_t clients) {
    const uint64_t tiles = (uint64_t)((outs + kOuts - 1) / kOuts) * ((ins + 127u) / 128u) * clients;
    const uint64_t chunks = (rows + kChunk - 1) / kChunk;
    if (tiles == 0 || chunks == 0) return 1;
    return (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(kSmsAssumed / tiles, chunks / 2));
}

template <typename T, bool kWide>
int launch_weight(const WeightArgs& a, cudaStream_t st) {
    auto* kernel = f8_weight_kernel<T, kWide>;
    static std::atomic<int> sms[64];
    int dev = 0;
    CO3_CUDA(cudaGetDevice(&dev));
    int n = dev < 64 ? sms[dev].load(std::memory_order_relaxed) : 0;
    if (n == 0) {
        CO3_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemW<T>));
        CO3_CUDA(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev));
        if (dev < 64) sms[dev].store(n, std::memory_order_relaxed);
    }
    const uint32_t tiles = a.k_tiles * a.n_tiles * a.parts * a.clients;
    CO3_CUDA(launch_behind(kernel, dim3(std::min(tiles, (uint32_t)n)), dim3(kF8Threads), kSmemW<T>, st, a));
    return CO3_OK;
}

}  // namespace
}  // namespace co3

using namespace co3;

extern "C" {

int co3_f8_weight_gradient_workspace_bytes(uint64_t rows, uint32_t outs, uint32_t ins, uint32_t n_clients, size_t* out) {
    if (!out || n_clients == 0 || rows >= (1ull << 31) || outs >= (1u << 31) || ins >= (1u << 31)) return CO3_ERR_INVALID_ARG;
    const uint64_t parts = row_parts(rows, outs, ins, n_clients);
    const uint64_t bytes = parts > 1 ? parts * n_clients * ((uint64_t)outs * ins + outs) * 4 : 0;
    *out = (size_t)std::max<uint64_t>(256, (bytes + 255u) & ~(uint64_t)255u);
    return CO3_OK;
}

int co3_f8_weight_gradient(const void* dy, int type, uint64_t dy_row_stride, const void* x8, size_t x8_bytes, uint64_t rows, uint32_t outs, uint32_t ins,
                           float* dw, float* db, uint32_t n_clients, uint64_t client_stride_elems, int accumulate, void* workspace, size_t workspace_bytes,
                           co3_result* res, void* stream) {
    F8Layout l;
    if (type < CO3_F32 || type > CO3_BF16 || n_clients == 0 || rows >= (1ull << 31) || rows * n_clients >= (1ull << 31) ||
        !f8_layout(rows * n_clients, ins, CO3_F8_ROWS, &l) || (uint64_t)outs * ins >= (1ull << 40) || outs >= (1u << 31))
        return CO3_ERR_INVALID_ARG;
    if (outs == 0 || (!dw && !db)) return CO3_OK;
    if (!aligned(dw, 4) || !aligned(db, 4) || !aligned(res, 8) || client_stride_elems >= (1ull << 40) ||
        (n_clients > 1 && ((dw && client_stride_elems < (uint64_t)outs * ins) || (db && client_stride_elems < outs))))
        return CO3_ERR_INVALID_ARG;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows == 0) {  // no terms: zeros
        if (accumulate) return CO3_OK;
        const int e = launch_join({nullptr, dw, (uint64_t)outs * ins, client_stride_elems, 0, n_clients, 0}, st);
        return e != CO3_OK ? e : launch_join({nullptr, db, outs, client_stride_elems, 0, n_clients, 0}, st);
    }
    if (ins == 0) return CO3_ERR_INVALID_ARG;
    if (!dy || !aligned(dy, type_size(type)) || dy_row_stride < outs || dy_row_stride >= (1ull << 40) || !x8 || !aligned(x8, 256) || !workspace ||
        !aligned(workspace, 256))
        return CO3_ERR_INVALID_ARG;
    size_t need = 0;
    co3_f8_weight_gradient_workspace_bytes(rows, outs, ins, n_clients, &need);
    if (x8_bytes < l.bytes || workspace_bytes < need) return CO3_ERR_CAPACITY;
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
    a.k_tiles = l.kb;
    a.n_tiles = (outs + kOuts - 1) / kOuts;
    a.chunks = (uint32_t)((rows + kChunk - 1) / kChunk);
    a.parts = row_parts(rows, outs, ins, n_clients);
    a.dw = dw;
    a.db = db;
    a.client_stride = client_stride_elems;
    a.accumulate = accumulate;
    a.partial = static_cast<float*>(workspace);
    a.res = res;
    if ((uint64_t)a.k_tiles * a.n_tiles >= (1ull << 31) / n_clients / a.parts) return CO3_ERR_INVALID_ARG;
    const size_t s = type_size(type);
    const bool wide = aligned(dy, 16) && dy_row_stride * s % 16 == 0 && outs * s % 16 == 0;
    const int e = type == CO3_F32   ? (wide ? launch_weight<float, true>(a, st) : launch_weight<float, false>(a, st))
                  : type == CO3_F16 ? (wide ? launch_weight<__half, true>(a, st) : launch_weight<__half, false>(a, st))
                                    : (wide ? launch_weight<__nv_bfloat16, true>(a, st) : launch_weight<__nv_bfloat16, false>(a, st));
    if (e != CO3_OK || a.parts == 1) return e;
    const uint64_t dw_all = (uint64_t)a.parts * n_clients * outs * ins;
    const int f = launch_join({a.partial, dw, (uint64_t)outs * ins, client_stride_elems, a.parts, n_clients, accumulate}, st);
    return f != CO3_OK ? f : launch_join({a.partial + dw_all, db, outs, client_stride_elems, a.parts, n_clients, accumulate}, st);
}

}  // extern "C"
