// Values to 8-bit blocks and back, and the activation between two layers with its backward pass from what was kept.
//
// All of it is bound by memory: one pass, each thread takes 16 bytes at a time where rows allow it.  A warp takes a row's 512
// columns, four blocks, so that the four exponent bytes leave as one word; two rows at once keep enough loads in flight.  A
// square block is held in a thread block's registers until its largest magnitude is known.
#include <math.h>

#include <algorithm>

#include "co3_f8.cuh"
#include "co3_launch.cuh"

namespace co3 {
namespace {

constexpr int kWarps = 8;
constexpr int kRowsAtOnce = 2;
enum Way { kWide, kSingle };  // 16 bytes at a time, or one element at a time

// How a warp's lanes share 512 columns of a row: kChunks loads of kVals values.
template <typename T, Way kWay>
struct Lanes {
    static constexpr bool kPairs = kWay == kWide && sizeof(T) == 2;    // 16 lanes a block instead of 32
    static constexpr int kChunks = kPairs ? 2 : 4, kVals = kPairs ? 8 : 4;
    static constexpr uint32_t kChunkCols = 512 / kChunks;
    // block of this lane's values of chunk h among the four
    static __device__ __forceinline__ uint32_t block(int h, uint32_t lane) { return kPairs ? 2 * h + (lane >> 4) : h; }
    // first column of its values, and how far apart they are
    static __device__ __forceinline__ uint32_t column(int h, uint32_t lane) { return h * kChunkCols + (kWay == kSingle ? lane : lane * kVals); }

    // p: element at column(h, lane) of the row; `left`: columns from there to the row's end (none if <= 0)
    static __device__ __forceinline__ void load(const T* p, int64_t left, float (&v)[kVals]) {
        if constexpr (kWay == kWide) {
            uint4 raw = make_uint4(0, 0, 0, 0);
            if (left > 0) raw = __ldcs(reinterpret_cast<const uint4*>(p));
            const T* e = reinterpret_cast<const T*>(&raw);
#pragma unroll
            for (int i = 0; i < kVals; ++i) v[i] = to_float(e[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kVals; ++i) v[i] = (int64_t)(i * 32) < left ? to_float(p[i * 32]) : 0.0f;
        }
    }
    static __device__ __forceinline__ void store(T* p, int64_t left, const float (&v)[kVals]) {
        if constexpr (kWay == kWide) {
            uint4 raw;
            T* e = reinterpret_cast<T*>(&raw);
#pragma unroll
            for (int i = 0; i < kVals; ++i) e[i] = from_float<T>(v[i]);
            if (left > 0) *reinterpret_cast<uint4*>(p) = raw;
        } else {
#pragma unroll
            for (int i = 0; i < kVals; ++i)
                if ((int64_t)(i * 32) < left) p[i * 32] = from_float<T>(v[i]);
        }
    }

    // largest over the lanes that share a block
    static __device__ __forceinline__ uint32_t most(uint32_t m) {
        if constexpr (kPairs) {
#pragma unroll
            for (int d = 8; d > 0; d >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, d));
            return m;
        } else {
            return __reduce_max_sync(0xffffffffu, m);
        }
    }

    // Four lanes' words, of which byte c belongs to column 32 c + lane, into words of four neighbouring columns; its own inverse
    // as far as the columns go.
    static __device__ __forceinline__ uint32_t turn(uint32_t w, uint32_t lane) {
        const uint32_t q = lane & 3u;
        uint32_t r = ((w >> (8 * q)) & 0xffu) << (8 * q);
#pragma unroll
        for (uint32_t d = 1; d < 4; ++d) r |= ((__shfl_xor_sync(0xffffffffu, w, d) >> (8 * q)) & 0xffu) << (8 * (q ^ d));
        return r;
    }
    // offset of this lane's bytes in a block's 128
    static __device__ __forceinline__ uint32_t at(uint32_t lane, uint32_t row) {
        if constexpr (kPairs) return f8_piece(row, (lane & 15u) >> 1) + 8u * (lane & 1u);
        if constexpr (kWay == kWide) return f8_piece(row, lane >> 2) + 4u * (lane & 3u);
        return f8_piece(row, 2u * (lane & 3u) + (lane >> 4)) + 4u * ((lane >> 2) & 3u);
    }
    // whole warps, whether or not `valid`
    static __device__ __forceinline__ void put(uint8_t* p, bool valid, const float (&v)[kVals], float inverse, uint32_t lane) {
        uint32_t w[kVals / 4];
#pragma unroll
        for (int i = 0; i < kVals / 4; ++i)
            w[i] = f8_from4(__fmul_rn(v[4 * i], inverse), __fmul_rn(v[4 * i + 1], inverse), __fmul_rn(v[4 * i + 2], inverse), __fmul_rn(v[4 * i + 3], inverse));
        if constexpr (kWay == kSingle) w[0] = turn(w[0], lane);
        if (!valid) return;
        if constexpr (kPairs) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(p) = w[0];
    }
    static __device__ __forceinline__ void get(const uint8_t* p, bool valid, float scale, uint32_t lane, float (&v)[kVals]) {
        uint32_t w[2] = {0, 0};
        if (valid) {
            if constexpr (kPairs) {
                const uint2 two = __ldcs(reinterpret_cast<const uint2*>(p));
                w[0] = two.x; w[1] = two.y;
            } else {
                w[0] = __ldcs(reinterpret_cast<const uint32_t*>(p));
            }
        }
        if constexpr (kWay == kSingle) w[0] = turn(w[0], lane);
#pragma unroll
        for (int i = 0; i < kVals / 4; ++i) {
            const float2 a = f8_to2(w[i]), b = f8_to2(w[i] >> 16);
            v[4 * i] = __fmul_rn(a.x, scale);
            v[4 * i + 1] = __fmul_rn(a.y, scale);
            v[4 * i + 2] = __fmul_rn(b.x, scale);
            v[4 * i + 3] = __fmul_rn(b.y, scale);
        }
    }
};

// ------------------------------------------------------------------------------------------------
// Activations
// ------------------------------------------------------------------------------------------------
template <int kAct>
__device__ __forceinline__ float act(float x) {
    if constexpr (kAct == CO3_ACT_RELU) return x < 0.0f ? 0.0f : x;  // NaN stays
    if constexpr (kAct == CO3_ACT_GELU) return __fmul_rn(x, __fmul_rn(0.5f, erfcf(__fmul_rn(x, -0.70710678118654752f))));
    if constexpr (kAct == CO3_ACT_SILU) return __fdiv_rn(x, __fadd_rn(1.0f, expf(-x)));
    return x;
}
template <int kAct>
__device__ __forceinline__ float act_slope(float x) {
    if constexpr (kAct == CO3_ACT_RELU) return x > 0.0f ? 1.0f : x <= 0.0f ? 0.0f : x;  // NaN stays
    if constexpr (kAct == CO3_ACT_GELU) {
        const float below = __fmul_rn(0.5f, erfcf(__fmul_rn(x, -0.70710678118654752f)));
        return __fmaf_rn(x, __fmul_rn(0.39894228040143268f, expf(__fmul_rn(__fmul_rn(-0.5f, x), x))), below);
    }
    if constexpr (kAct == CO3_ACT_SILU) {
        const float p = __fdiv_rn(1.0f, __fadd_rn(1.0f, expf(-x)));
        return __fmul_rn(p, __fmaf_rn(x, __fsub_rn(1.0f, p), 1.0f));
    }
    return 1.0f;
}

// ------------------------------------------------------------------------------------------------
// Rows
// ------------------------------------------------------------------------------------------------
struct RowsArgs {
    const void* x;      // or dy
    void* y;            // or dx; nullable forward
    uint8_t *x8, *y8;   // nullable
    uint64_t rows, x_stride, y_stride;
    uint32_t cols, kb, groups;   // groups of four blocks
    uint64_t rows_padded, scales;
    uint32_t units;              // pairs of rows x groups
};

// Where a warp's unit lies.
struct Unit {
    uint64_t row;
    uint32_t group;
};
__device__ __forceinline__ bool find_unit(const RowsArgs& a, Unit& u) {
    const uint32_t unit = blockIdx.x * kWarps + (threadIdx.x >> 5);
    u.row = (uint64_t)(unit / a.groups) * kRowsAtOnce;
    u.group = unit % a.groups;
    return unit < a.units;
}
__device__ __forceinline__ uint64_t scale_word(const RowsArgs& a, uint64_t row, uint32_t group) {
    return a.scales + (group * (a.rows_padded >> 7) + (row >> 7)) * kF8Scales + f8_scale_at((uint32_t)row & 127u, 0);
}

// A row's four blocks into one buffer.
template <typename T, Way kWay>
__device__ __forceinline__ void put_row(const RowsArgs& a, uint8_t* to, uint64_t row, uint32_t group, uint32_t lane,
                                        float (&v)[Lanes<T, kWay>::kChunks][Lanes<T, kWay>::kVals]) {
    using L = Lanes<T, kWay>;
    uint32_t bytes[L::kChunks];
#pragma unroll
    for (int h = 0; h < L::kChunks; ++h) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < L::kVals; ++i) m = max(m, f8_magnitude(v[h][i]));
        m = L::most(m);
        int e = f8_exponent(m);
        if (__any_sync(0xffffffffu, m > kF8Rare)) {
            m = 0;
#pragma unroll
            for (int i = 0; i < L::kVals; ++i) m = max(m, f8_finite_magnitude(v[h][i]));
            e = f8_exponent(L::most(m));
#pragma unroll
            for (int i = 0; i < L::kVals; ++i) v[h][i] = f8_rare(v[h][i], e);
        }
        const uint32_t block = group * 4u + L::block(h, lane);
        L::put(to + f8_row(a.rows_padded, block, row) + L::at(lane, (uint32_t)row), block < a.kb, v[h], power_of_two(-e), lane);
        bytes[h] = (uint32_t)(e + 127);
    }
    uint32_t word;
    if constexpr (L::kPairs) {
        word = bytes[0] | (bytes[1] << 16);
        word |= __shfl_down_sync(0xffffffffu, word, 16) << 8;
    } else {
        word = bytes[0] | (bytes[1] << 8) | (bytes[2] << 16) | (bytes[3] << 24);
    }
    if (lane == 0) *reinterpret_cast<uint32_t*>(to + scale_word(a, row, group)) = word;
}

// x to x8 (if given), act(x) to y and to y8 (if given).  Rows up to a multiple of 16 are written, as zeros: the products read
// so many.
template <typename T, Way kWay, int kAct>
__global__ void __launch_bounds__(kWarps * 32) f8_rows_kernel(const __grid_constant__ RowsArgs a) {
    using L = Lanes<T, kWay>;
    wait_for_previous_kernel();
    Unit u;
    if (!find_unit(a, u)) return;
    const uint32_t lane = threadIdx.x & 31u;
    float v[kRowsAtOnce][L::kChunks][L::kVals];
    const T* x = static_cast<const T*>(a.x);
    T* y = static_cast<T*>(a.y);
#pragma unroll
    for (int r = 0; r < kRowsAtOnce; ++r)
#pragma unroll
        for (int h = 0; h < L::kChunks; ++h) {
            const uint64_t col = (uint64_t)u.group * 512u + L::column(h, lane);
            L::load(x + (u.row + r) * a.x_stride + col, u.row + r < a.rows ? (int64_t)a.cols - (int64_t)col : 0, v[r][h]);
        }
#pragma unroll
    for (int r = 0; r < kRowsAtOnce; ++r) {
        const uint64_t row = u.row + r;
        float t[L::kChunks][L::kVals];
        if constexpr (kAct != CO3_ACT_NONE) {
#pragma unroll
            for (int h = 0; h < L::kChunks; ++h)
#pragma unroll
                for (int i = 0; i < L::kVals; ++i) t[h][i] = act<kAct>(v[r][h][i]);
        } else {
#pragma unroll
            for (int h = 0; h < L::kChunks; ++h)
#pragma unroll
                for (int i = 0; i < L::kVals; ++i) t[h][i] = v[r][h][i];
        }
        if (y)
#pragma unroll
            for (int h = 0; h < L::kChunks; ++h) {
                const uint64_t col = (uint64_t)u.group * 512u + L::column(h, lane);
                L::store(y + row * a.y_stride + col, row < a.rows ? (int64_t)a.cols - (int64_t)col : 0, t[h]);
            }
        if (a.x8) put_row<T, kWay>(a, a.x8, row, u.group, lane, v[r]);
        if (a.y8) put_row<T, kWay>(a, a.y8, row, u.group, lane, t);
    }
}

// y <- the values of x8, or (kBackward) dx <- dy * act'(values of x8).
template <typename T, Way kWay, int kAct, bool kBackward>
__global__ void __launch_bounds__(kWarps * 32) f8_values_kernel(const __grid_constant__ RowsArgs a) {
    using L = Lanes<T, kWay>;
    wait_for_previous_kernel();
    Unit u;
    if (!find_unit(a, u)) return;
    const uint32_t lane = threadIdx.x & 31u;
    float v[kRowsAtOnce][L::kChunks][L::kVals], d[kRowsAtOnce][L::kChunks][L::kVals];
    const T* dy = static_cast<const T*>(a.x);
#pragma unroll
    for (int r = 0; r < kRowsAtOnce; ++r) {
        const uint64_t row = u.row + r;
        const uint32_t word = row < a.rows ? __ldg(reinterpret_cast<const uint32_t*>(a.x8 + scale_word(a, row, u.group))) : 0x7f7f7f7fu;
#pragma unroll
        for (int h = 0; h < L::kChunks; ++h) {
            const uint64_t col = (uint64_t)u.group * 512u + L::column(h, lane);
            if constexpr (kBackward) L::load(dy + row * a.x_stride + col, row < a.rows ? (int64_t)a.cols - (int64_t)col : 0, d[r][h]);
            const uint32_t block = u.group * 4u + L::block(h, lane);
            const float scale = __uint_as_float(((word >> (8u * L::block(h, lane))) & 0xffu) << 23);
            L::get(a.x8 + f8_row(a.rows_padded, block, row) + L::at(lane, (uint32_t)row), row < a.rows && block < a.kb, scale, lane, v[r][h]);
        }
    }
#pragma unroll
    for (int r = 0; r < kRowsAtOnce; ++r) {
        const uint64_t row = u.row + r;
#pragma unroll
        for (int h = 0; h < L::kChunks; ++h) {
            const uint64_t col = (uint64_t)u.group * 512u + L::column(h, lane);
            if constexpr (kBackward) {
#pragma unroll
                for (int i = 0; i < L::kVals; ++i) v[r][h][i] = __fmul_rn(d[r][h][i], act_slope<kAct>(v[r][h][i]));
            }
            L::store(static_cast<T*>(a.y) + row * a.y_stride + col, row < a.rows ? (int64_t)a.cols - (int64_t)col : 0, v[r][h]);
        }
    }
}

// ------------------------------------------------------------------------------------------------
// Square blocks: a thread block of 256 each, 16 rows a warp.
// ------------------------------------------------------------------------------------------------
struct SquareArgs {
    const void* x;
    uint8_t* out;
    uint64_t rows, x_stride, rows_padded, scales, scales_t;
    uint32_t cols, kb;
};

template <typename T, Way kWay>
__global__ void __launch_bounds__(256) f8_square_kernel(const __grid_constant__ SquareArgs a) {
    using L = Lanes<T, kWay>;
    constexpr int kRows = L::kPairs ? 2 : 1, kTurns = 16 / kRows;  // rows a warp's load covers
    __shared__ uint32_t part[kWarps];
    wait_for_previous_kernel();
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const uint32_t block = blockIdx.x % a.kb, tile = blockIdx.x / a.kb;
    const uint32_t row0 = warp * 16u + (L::kPairs ? lane >> 4 : 0u);
    const uint32_t in_block = kWay == kSingle ? lane : (lane & (L::kPairs ? 15u : 31u)) * L::kVals;
    const uint64_t col = (uint64_t)block * 128u + in_block;
    float v[kTurns][L::kVals];
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const uint64_t row = (uint64_t)tile * 128u + row0 + i * kRows;
        L::load(static_cast<const T*>(a.x) + row * a.x_stride + col, row < a.rows ? (int64_t)a.cols - (int64_t)col : 0, v[i]);
    }
    auto largest = [&](bool finite) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < kTurns; ++i)
#pragma unroll
            for (int k = 0; k < L::kVals; ++k) m = max(m, finite ? f8_finite_magnitude(v[i][k]) : f8_magnitude(v[i][k]));
        m = __reduce_max_sync(0xffffffffu, m);
        __syncthreads();
        if (lane == 0) part[warp] = m;
        __syncthreads();
        m = 0;
        for (int w = 0; w < kWarps; ++w) m = max(m, part[w]);
        return m;
    };
    const uint32_t m = largest(false);
    int e = f8_exponent(m);
    if (m > kF8Rare) {
        e = f8_exponent(largest(true));
#pragma unroll
        for (int i = 0; i < kTurns; ++i)
#pragma unroll
            for (int k = 0; k < L::kVals; ++k) v[i][k] = f8_rare(v[i][k], e);
    }
    const float inverse = power_of_two(-e);
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const uint32_t r = row0 + i * kRows;
        L::put(a.out + f8_row(a.rows_padded, block, (uint64_t)tile * 128u + r) + L::at(lane, r), true, v[i], inverse, lane);
    }
    const uint32_t t = threadIdx.x & 127u;
    const uint64_t at = threadIdx.x < 128 ? a.scales + ((block >> 2) * (a.rows_padded >> 7) + tile) * kF8Scales + f8_scale_at(t, block)
                                          : a.scales_t + ((uint64_t)(tile >> 2) * a.kb + block) * kF8Scales + f8_scale_at(t, tile);
    a.out[at] = (uint8_t)(e + 127);
}

// ------------------------------------------------------------------------------------------------
// Launches
// ------------------------------------------------------------------------------------------------
bool valid_rows(int type, const void* p, uint64_t stride, uint32_t cols) {
    return type >= CO3_F32 && type <= CO3_BF16 && p && aligned(p, type_size(type)) && stride >= cols && stride < (1ull << 40);
}
bool wide(int type, const void* p, uint64_t stride, uint32_t cols) {
    const size_t s = type_size(type);
    return !p || (aligned(p, 16) && stride * s % 16 == 0 && cols * s % 16 == 0);
}
bool valid_f8(const void* p) { return p && aligned(p, 256); }

void fill(RowsArgs& a, const F8Layout& l, uint64_t rows, uint32_t cols) {
    a.rows = rows;
    a.cols = cols;
    a.kb = l.kb;
    a.groups = (l.kb + 3u) / 4u;
    a.rows_padded = l.rows;
    a.scales = l.scales;
    a.units = (uint32_t)((rows + 15u) / 16u * (16u / kRowsAtOnce)) * a.groups;
}

template <typename T, Way kWay>
int launch_rows(const RowsArgs& a, int act, cudaStream_t st) {
    auto* kernel = act == CO3_ACT_RELU   ? f8_rows_kernel<T, kWay, CO3_ACT_RELU>
                   : act == CO3_ACT_GELU ? f8_rows_kernel<T, kWay, CO3_ACT_GELU>
                   : act == CO3_ACT_SILU ? f8_rows_kernel<T, kWay, CO3_ACT_SILU>
                                         : f8_rows_kernel<T, kWay, CO3_ACT_NONE>;
    CO3_CUDA(launch_behind(kernel, dim3((a.units + kWarps - 1) / kWarps), dim3(kWarps * 32), 0, st, a));
    return CO3_OK;
}
template <typename T, Way kWay>
int launch_values(const RowsArgs& a, int act, cudaStream_t st) {  // act < 0: the values themselves
    auto* kernel = act < 0               ? f8_values_kernel<T, kWay, CO3_ACT_NONE, false>
                   : act == CO3_ACT_RELU ? f8_values_kernel<T, kWay, CO3_ACT_RELU, true>
                   : act == CO3_ACT_GELU ? f8_values_kernel<T, kWay, CO3_ACT_GELU, true>
                   : act == CO3_ACT_SILU ? f8_values_kernel<T, kWay, CO3_ACT_SILU, true>
                                         : f8_values_kernel<T, kWay, CO3_ACT_NONE, true>;
    CO3_CUDA(launch_behind(kernel, dim3((a.units + kWarps - 1) / kWarps), dim3(kWarps * 32), 0, st, a));
    return CO3_OK;
}
template <typename T, Way kWay>
int launch_square(const SquareArgs& a, cudaStream_t st) {
    const uint32_t blocks = (uint32_t)(a.rows_padded / 128u * a.kb);
    CO3_CUDA(launch_behind(f8_square_kernel<T, kWay>, dim3(blocks), dim3(256), 0, st, a));
    return CO3_OK;
}

// f<T, kWay>() for the buffers' type and way
#define CO3_BY_TYPE(type, w, f, ...)                                                                        \
    ((type) == CO3_F32   ? ((w) ? f<float, kWide>(__VA_ARGS__) : f<float, kSingle>(__VA_ARGS__))            \
     : (type) == CO3_F16 ? ((w) ? f<__half, kWide>(__VA_ARGS__) : f<__half, kSingle>(__VA_ARGS__))          \
                         : ((w) ? f<__nv_bfloat16, kWide>(__VA_ARGS__) : f<__nv_bfloat16, kSingle>(__VA_ARGS__)))

}  // namespace
}  // namespace co3

using namespace co3;

extern "C" {

int co3_f8_bytes(uint64_t rows, uint32_t cols, int kind, size_t* out) {
    F8Layout l;
    if (!out || !f8_layout(rows, cols, kind, &l)) return CO3_ERR_INVALID_ARG;
    *out = (size_t)l.bytes;
    return CO3_OK;
}

int co3_f8_pack(const void* x, int type, uint64_t rows, uint32_t cols, uint64_t x_row_stride, int kind, void* out, size_t out_bytes, void* stream) {
    if (kind == CO3_F8_ROWS) return co3_f8_activation(x, type, rows, cols, x_row_stride, CO3_ACT_NONE, nullptr, 0, nullptr, out, out_bytes, stream);
    F8Layout l;
    if (type < CO3_F32 || type > CO3_BF16 || !f8_layout(rows, cols, kind, &l)) return CO3_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return CO3_OK;
    if (!valid_rows(type, x, x_row_stride, cols) || !valid_f8(out)) return CO3_ERR_INVALID_ARG;
    if (out_bytes < l.bytes) return CO3_ERR_CAPACITY;
    SquareArgs a = {x, static_cast<uint8_t*>(out), rows, x_row_stride, l.rows, l.scales, l.scales_t, cols, l.kb};
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return CO3_BY_TYPE(type, wide(type, x, x_row_stride, cols), launch_square, a, st);
}

int co3_f8_activation(const void* x, int type, uint64_t rows, uint32_t cols, uint64_t x_row_stride, int act, void* y, uint64_t y_row_stride,
                      void* y8, void* x8, size_t f8_bytes, void* stream) {
    F8Layout l;
    if (type < CO3_F32 || type > CO3_BF16 || act < CO3_ACT_NONE || act > CO3_ACT_SILU || !f8_layout(rows, cols, CO3_F8_ROWS, &l)) return CO3_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return CO3_OK;
    if (!valid_rows(type, x, x_row_stride, cols) || (y && !valid_rows(type, y, y_row_stride, cols)) || (y8 && !valid_f8(y8)) || (x8 && !valid_f8(x8)) ||
        (!y && !y8 && !x8) || (y8 && y8 == x8))
        return CO3_ERR_INVALID_ARG;
    if ((y8 || x8) && f8_bytes < l.bytes) return CO3_ERR_CAPACITY;
    RowsArgs a = {};
    a.x = x; a.y = y;
    a.x8 = static_cast<uint8_t*>(x8); a.y8 = static_cast<uint8_t*>(y8);
    a.x_stride = x_row_stride; a.y_stride = y_row_stride;
    fill(a, l, rows, cols);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return CO3_BY_TYPE(type, wide(type, x, x_row_stride, cols) && wide(type, y, y_row_stride, cols), launch_rows, a, act, st);
}

static int values(const void* dy, uint64_t dy_row_stride, const void* x8, size_t x8_bytes, int kind, int act, void* out, int type, uint64_t rows,
                  uint32_t cols, uint64_t out_row_stride, void* stream) {
    F8Layout l;
    if (type < CO3_F32 || type > CO3_BF16 || act > CO3_ACT_SILU || !f8_layout(rows, cols, kind, &l)) return CO3_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return CO3_OK;
    if (!valid_rows(type, out, out_row_stride, cols) || !valid_f8(x8) || (act >= 0 && !valid_rows(type, dy, dy_row_stride, cols))) return CO3_ERR_INVALID_ARG;
    if (x8_bytes < l.bytes) return CO3_ERR_CAPACITY;
    RowsArgs a = {};
    a.x = dy; a.y = out;
    a.x8 = static_cast<uint8_t*>(const_cast<void*>(x8));
    a.x_stride = dy_row_stride; a.y_stride = out_row_stride;
    fill(a, l, rows, cols);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return CO3_BY_TYPE(type, wide(type, act < 0 ? nullptr : dy, dy_row_stride, cols) && wide(type, out, out_row_stride, cols), launch_values, a, act, st);
}

int co3_f8_unpack(const void* in, size_t in_bytes, int kind, void* y, int type, uint64_t rows, uint32_t cols, uint64_t y_row_stride, void* stream) {
    return values(nullptr, 0, in, in_bytes, kind, -1, y, type, rows, cols, y_row_stride, stream);
}

int co3_f8_activation_backward(const void* dy, int type, uint64_t rows, uint32_t cols, uint64_t dy_row_stride, const void* x8, size_t x8_bytes, int act,
                               void* dx, uint64_t dx_row_stride, void* stream) {
    if (act < CO3_ACT_NONE) return CO3_ERR_INVALID_ARG;
    return values(dy, dy_row_stride, x8, x8_bytes, CO3_F8_ROWS, act, dx, type, rows, cols, dx_row_stride, stream);
}

}  // extern "C"
