// Values to 8-bit blocks and back, and the activation between two layers with its backward pass from what was kept.
//
// All of it is bound by memory: one pass, each thread takes 16 bytes at a time where rows allow it.  A warp takes a row's 512
// columns, four blocks, so that the four exponent bytes leave as one word.  A
// square block is held in a thread block's registers until its largest magnitude is known.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "co3_f8.cuh"
#include "co3_launch.cuh"

namespace co3 {
namespace {

constexpr int kWarps = 8;
// Rows that a warp has under way, and blocks of threads that an SM holds at least: two and three, but for GELU, whose arithmetic
// wants more warps (us: bf16 16384 x 8192 there and back 258 with four blocks, 274 with three; fp32 8192 x 8192 322, and 294 with one row
// and four blocks; fp32 values alone 111, and 125 with one row; SILU bf16 224, and 231 with four blocks).
template <typename T, int kAct>
constexpr int kRowsAtOnce = sizeof(T) == 4 && kAct == CO3_ACT_GELU ? 1 : 2;
template <int kAct>
constexpr int kBlocks = kAct == CO3_ACT_GELU ? 4 : 3;
enum Way { kWide, kSingle };  // 16 bytes at a time, or one element at a time

// Four fp32 or eight 16-bit values as 16 bytes.
template <typename T>
__device__ __forceinline__ uint4 rounded16(const float* v) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (std::is_same<T, float>::value) {
            w[i] = __float_as_uint(v[i]);
        } else if constexpr (std::is_same<T, __half>::value) {
            const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        } else {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// How a warp's lanes share 512 columns of a row: kChunks loads of kVals values.
template <typename T, Way kWay>
struct Lanes {
    static constexpr bool kPairs = kWay == kWide && sizeof(T) == 2;    // 16 lanes a block instead of 32
    static constexpr int kChunks = kPairs ? 2 : 4, kVals = kPairs ? 8 : 4, kBlocks = 4 / kChunks;
    static constexpr uint32_t kChunkCols = 512 / kChunks;
    struct Single { T v[4]; };
    using Raw = typename std::conditional<kWay == kWide, uint4, Single>::type;
    // block of this lane's values of the first chunk among the four (kBlocks further for each chunk)
    static __device__ __forceinline__ uint32_t block0(uint32_t lane) { return kPairs ? lane >> 4 : 0u; }
    // first column of its values; they are neighbours, or 32 columns apart
    static __device__ __forceinline__ uint32_t column0(uint32_t lane) { return kWay == kSingle ? lane : lane * kVals; }

    // p: element at column0 of the chunk; `left`: columns from there to the row's end (none if <= 0)
    static __device__ __forceinline__ Raw load(const T* p, int32_t left) {
        Raw raw;
        if constexpr (kWay == kWide) {
            raw = make_uint4(0, 0, 0, 0);
            if (left > 0) raw = __ldcs(reinterpret_cast<const uint4*>(p));
        } else {
#pragma unroll
            for (int i = 0; i < kVals; ++i) raw.v[i] = i * 32 < left ? p[i * 32] : from_float<T>(0.0f);
        }
        return raw;
    }
    static __device__ __forceinline__ float value(const Raw& raw, int i) {
        if constexpr (kWay == kSingle) {
            return to_float(raw.v[i]);
        } else {
            const uint32_t w = (&raw.x)[i * sizeof(T) / 4];
            if constexpr (sizeof(T) == 4) return __uint_as_float(w);
            else if constexpr (std::is_same<T, __nv_bfloat16>::value) return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
            else return __half2float(__ushort_as_half((unsigned short)(i & 1 ? w >> 16 : w & 0xffffu)));
        }
    }
    static __device__ __forceinline__ void store(T* p, int32_t left, const float (&v)[kVals]) {
        if constexpr (kWay == kWide) {
            if (left > 0) *reinterpret_cast<uint4*>(p) = rounded16<T>(v);
        } else {
#pragma unroll
            for (int i = 0; i < kVals; ++i)
                if (i * 32 < left) p[i * 32] = from_float<T>(v[i]);
        }
    }

    // Largest magnitude of each chunk's block, over the lanes that share it.  16-bit values are compared two at a time, and both
    // chunks' maxima travel together.
    static __device__ __forceinline__ void largest(const Raw (&raw)[kChunks], uint32_t (&m)[kChunks]) {
        if constexpr (kPairs) {
            uint32_t two[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                constexpr uint32_t kAbs = 0x7fff7fffu;
                const uint32_t w = __vmaxu2(__vmaxu2(raw[h].x & kAbs, raw[h].y & kAbs), __vmaxu2(raw[h].z & kAbs, raw[h].w & kAbs));
                two[h] = __vmaxu2(w, w >> 16);
            }
            uint32_t w = __byte_perm(two[0], two[1], 0x5410);
#pragma unroll
            for (int d = 8; d > 0; d >>= 1) w = __vmaxu2(w, __shfl_xor_sync(0xffffffffu, w, d));
            m[0] = __float_as_uint(value(make_uint4(w, 0, 0, 0), 0));
            m[1] = __float_as_uint(value(make_uint4(w, 0, 0, 0), 1));
        } else {
#pragma unroll
            for (int h = 0; h < kChunks; ++h) {
                uint32_t w = 0;
#pragma unroll
                for (int i = 0; i < kVals; ++i) w = max(w, f8_magnitude(value(raw[h], i)));
                m[h] = most(w);
            }
        }
    }
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
    // offset of this lane's bytes in a block's 128 of row 0; row r: XOR 16 (r % 8)
    static __device__ __forceinline__ uint32_t at(uint32_t lane) {
        if constexpr (kPairs) return (lane & 15u) * 8u;
        if constexpr (kWay == kWide) return lane * 4u;
        return 32u * (lane & 3u) + 4u * (lane >> 2);
    }
    // whole warps, whether or not `valid`
    static __device__ __forceinline__ void put(uint8_t* p, bool valid, const float (&v)[kVals], float inverse, uint32_t lane) {
        uint32_t w[kVals / 4];
#pragma unroll
        for (int i = 0; i < kVals / 4; ++i) {
            const F2 a = mul2({v[4 * i], v[4 * i + 1]}, f2_both(inverse)), b = mul2({v[4 * i + 2], v[4 * i + 3]}, f2_both(inverse));
            w[i] = f8_from4(a.x, a.y, b.x, b.y);
        }
        if constexpr (kWay == kSingle) w[0] = turn(w[0], lane);
        if (!valid) return;
        if constexpr (kPairs) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(p) = w[0];
    }
    // this lane's bytes of a block, and their values
    struct Bytes { uint32_t w[kVals / 4]; };
    static __device__ __forceinline__ Bytes get(const uint8_t* p, bool valid) {
        Bytes b = {};
        if (valid) {
            if constexpr (kPairs) {
                const uint2 two = __ldcs(reinterpret_cast<const uint2*>(p));
                b.w[0] = two.x; b.w[1] = two.y;
            } else {
                b.w[0] = __ldcs(reinterpret_cast<const uint32_t*>(p));
            }
        }
        return b;
    }
    static __device__ __forceinline__ void values(Bytes b, float scale, uint32_t lane, float (&v)[kVals]) {
        if constexpr (kWay == kSingle) b.w[0] = turn(b.w[0], lane);
#pragma unroll
        for (int i = 0; i < kVals / 4; ++i) {
            const float2 lo = f8_to2(b.w[i]), hi = f8_to2(b.w[i] >> 16);
            const F2 x = mul2({lo.x, lo.y}, f2_both(scale)), y = mul2({hi.x, hi.y}, f2_both(scale));
            v[4 * i] = x.x;
            v[4 * i + 1] = x.y;
            v[4 * i + 2] = y.x;
            v[4 * i + 3] = y.y;
        }
    }
};

// ------------------------------------------------------------------------------------------------
// Activations
// ------------------------------------------------------------------------------------------------
// For 16-bit results short forms take the place of the library's functions, two values at a time: with the library's, the kernels
// are bound by instructions (16384 x 8192 bf16, GELU: forward 299 and backward 338 us).
__device__ __forceinline__ float exp2_short(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float inverse_short(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float min_nan(float a, float b) {  // NaN stays
    float y;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
// Phi(-|x|), Phi the normal distribution function, is 1/2 erfc(z) with z = |x| / sqrt(2), and erfc(z) exp(z^2) = t P(t), t = 1 / (1 + 0.375 z).
// P is a polynomial of degree 6 fitted to the smallest relative error over 0 <= z <= 12 (1e-6); with the roundings 2e-6 for |x| <= 4
// and 6e-6 for |x| <= 10, far below half a step of 16 bits.  ax: |x|, 64 at most (where exp(-x^2 / 2) is zero); e: 2^16 exp(-x^2 / 2),
// so that the instruction, which takes what is below 2^-126 for zero, loses nothing that bf16 holds; the result is 2^-16 t P(t) / 2.
constexpr float kDown16 = 1.0f / 65536.0f;
__device__ __forceinline__ F2 normal_short(F2 ax, F2& e) {
    const F2 arg = fma2(mul2(ax, ax), f2_both(-0.72134752044448170f), f2_both(16.0f)), den = fma2(ax, f2_both(0.26516504294495533f), f2_both(1.0f));
    e = {exp2_short(arg.x), exp2_short(arg.y)};
    const F2 t = {inverse_short(den.x), inverse_short(den.y)};
    F2 p = fma2(f2_both(-0.0666150079f * kDown16), t, f2_both(0.19073585385f * kDown16));
    p = fma2(p, t, f2_both(-0.06032206705f * kDown16));
    p = fma2(p, t, f2_both(0.13837517965f * kDown16));
    p = fma2(p, t, f2_both(0.0845211864f * kDown16));
    p = fma2(p, t, f2_both(0.1076185385f * kDown16));
    p = fma2(p, t, f2_both(0.1056866174f * kDown16));
    return mul2(t, p);
}
// 1 / (1 + exp(-x)) as 2^-24 / (2^-24 + 2^-24 exp(-x)): the sum and its inverse are normal numbers down to x = -104.
constexpr float kDown24 = 1.0f / 16777216.0f;
__device__ __forceinline__ F2 logistic_short(F2 x) {
    const F2 arg = fma2(x, f2_both(-1.4426950408889634f), f2_both(-24.0f)), den = add2({exp2_short(arg.x), exp2_short(arg.y)}, f2_both(kDown24));
    return mul2({inverse_short(den.x), inverse_short(den.y)}, f2_both(kDown24));
}

// act(x), short forms if kShort.  Infinities give the limits (the bounds below lie where the other factor is zero), NaN stays.
template <int kAct, bool kShort>
__device__ __forceinline__ F2 act(F2 x) {
    if constexpr (kAct == CO3_ACT_GELU && kShort) {
        F2 e;  // x > 0: x - x Phi(-x);  x < 0: x Phi(x)
        const F2 ax = {min_nan(fabsf(x.x), 64.0f), min_nan(fabsf(x.y), 64.0f)}, q = normal_short(ax, e);
        return fma2(mul2(ax, f2_both(-1.0f)), mul2(e, q), {fmaxf(x.x, 0.0f), fmaxf(x.y, 0.0f)});
    } else if constexpr (kAct == CO3_ACT_SILU && kShort) {
        return mul2({fmaxf(x.x, -200.0f), fmaxf(x.y, -200.0f)}, logistic_short(x));
    } else {
        auto one = [](float v) {
            if constexpr (kAct == CO3_ACT_RELU) return v < 0.0f ? 0.0f : v;
            if constexpr (kAct == CO3_ACT_GELU) return __fmul_rn(fmaxf(v, -64.0f), __fmul_rn(0.5f, erfcf(__fmul_rn(v, -0.70710678118654752f))));
            if constexpr (kAct == CO3_ACT_SILU) {  // exp(-|x|), which stays in range
                const float e = expf(-fabsf(v));
                return __fdiv_rn(v < 0.0f ? __fmul_rn(fmaxf(v, -200.0f), e) : v, __fadd_rn(1.0f, e));
            }
            return v;
        };
        return {one(x.x), one(x.y)};
    }
}
template <int kAct, bool kShort>
__device__ __forceinline__ F2 act_slope(F2 x) {
    if constexpr (kAct == CO3_ACT_GELU && kShort) {
        F2 e;  // x < 0: g = Phi(x) + x phi(x);  x > 0: 1 - g(-x);  g(-|x|) = exp(-x^2 / 2) (t P / 2 - |x| / sqrt(2 pi)), the bracket times 2^-16
        const F2 ax = {min_nan(fabsf(x.x), 64.0f), min_nan(fabsf(x.y), 64.0f)}, q = normal_short(ax, e);
        const F2 g = mul2(e, fma2(ax, f2_both(-0.39894228040143268f * kDown16), q));
        auto flip = [](float v, float by) { return __uint_as_float(__float_as_uint(v) ^ (~__float_as_uint(by) & 0x80000000u)); };
        auto step = [](float v) { return (int)__float_as_uint(v) < 0 ? 0.0f : 1.0f; };
        return add2({step(x.x), step(x.y)}, {flip(g.x, x.x), flip(g.y, x.y)});
    } else if constexpr (kAct == CO3_ACT_SILU && kShort) {
        const F2 p = logistic_short(x);  // p (1 + x (1 - p))
        return mul2(p, fma2(x, fma2(p, f2_both(-1.0f), f2_both(1.0f)), f2_both(1.0f)));
    } else {
        auto one = [](float v) {
            if constexpr (kAct == CO3_ACT_RELU) return v > 0.0f ? 1.0f : v <= 0.0f ? 0.0f : v;
            if constexpr (kAct == CO3_ACT_GELU) {
                const float below = __fmul_rn(0.5f, erfcf(__fmul_rn(v, -0.70710678118654752f)));
                return __fmaf_rn(v, __fmul_rn(0.39894228040143268f, expf(__fmul_rn(__fmul_rn(-0.5f, v), v))), below);
            }
            if constexpr (kAct == CO3_ACT_SILU) {
                const float e = expf(-fabsf(v)), p = __fdiv_rn(v < 0.0f ? e : 1.0f, __fadd_rn(1.0f, e));
                return __fmul_rn(p, __fmaf_rn(v, __fsub_rn(1.0f, p), 1.0f));
            }
            return 1.0f;
        };
        return {one(x.x), one(x.y)};
    }
}

// ------------------------------------------------------------------------------------------------
// Rows: a warp takes unit_rows (8 or 2) rows of four blocks.
// ------------------------------------------------------------------------------------------------
struct RowsArgs {
    const void* x;      // or dy
    void* y;            // or dx; nullable forward
    uint8_t *x8, *y8;   // nullable
    uint64_t rows, x_stride, y_stride;
    uint32_t cols, kb, groups;   // groups of four blocks
    uint64_t rows_padded, scales;
    uint32_t units, unit_rows;   // row groups x groups of blocks
};

// Where a warp's unit lies, for this lane.
template <typename T, Way kWay>
struct Unit {
    using L = Lanes<T, kWay>;
    uint64_t row0;
    uint32_t group, lane;
    uint64_t col;           // column of its first chunk
    uint64_t f8, f8_chunk;  // offset of row0's 128 bytes of its first block, bytes from chunk to chunk
    uint64_t word;          // offset of row0's four exponent bytes
    uint32_t blocks;        // of this group, from the lane's first one on

    __device__ __forceinline__ Unit(const RowsArgs& a, uint32_t unit) {
        lane = threadIdx.x & 31u;
        const uint32_t r = unit / a.groups;
        group = unit - r * a.groups;
        row0 = (uint64_t)r * a.unit_rows;
        col = (uint64_t)group * 512u + L::column0(lane);
        f8 = f8_row(a.rows_padded, group * 4u + L::block0(lane), row0);
        f8_chunk = a.rows_padded * (128u * L::kBlocks);
        word = a.scales + (group * (a.rows_padded >> 7) + (row0 >> 7)) * kF8Scales + f8_scale_at((uint32_t)row0 & 127u, 0);
        blocks = min(4u, a.kb - group * 4u);
    }
    // columns from a chunk's first one of this lane to the row's end
    __device__ __forceinline__ int32_t left(const RowsArgs& a, int h) const { return (int32_t)(a.cols - min((uint64_t)a.cols, col + h * L::kChunkCols)); }
    __device__ __forceinline__ bool has(int h) const { return L::block0(lane) + h * L::kBlocks < blocks; }
    // offset of this lane's bytes of row row0 + r (rows of a unit lie in one atom of eight)
    __device__ __forceinline__ uint64_t bytes(uint32_t r, int h) const { return f8 + h * f8_chunk + r * 128u + (L::at(lane) ^ ((((uint32_t)row0 + r) & 7u) << 4)); }
};

// A row's four blocks into one buffer; m: their largest magnitudes.
template <typename T, Way kWay>
__device__ __forceinline__ void put_row(const Unit<T, kWay>& u, uint8_t* to, uint32_t r, float (&v)[Lanes<T, kWay>::kChunks][Lanes<T, kWay>::kVals],
                                        const uint32_t (&m)[Lanes<T, kWay>::kChunks]) {
    using L = Lanes<T, kWay>;
    int e[L::kChunks];
    bool rare = false;
#pragma unroll
    for (int h = 0; h < L::kChunks; ++h) {
        e[h] = f8_exponent(m[h]);
        rare |= m[h] > kF8Rare;
    }
    if (__any_sync(0xffffffffu, rare)) {
#pragma unroll
        for (int h = 0; h < L::kChunks; ++h) {
            uint32_t finite = 0;
#pragma unroll
            for (int i = 0; i < L::kVals; ++i) finite = max(finite, f8_finite_magnitude(v[h][i]));
            e[h] = f8_exponent(L::most(finite));
#pragma unroll
            for (int i = 0; i < L::kVals; ++i) v[h][i] = f8_rare(v[h][i], e[h]);
        }
    }
#pragma unroll
    for (int h = 0; h < L::kChunks; ++h) L::put(to + u.bytes(r, h), u.has(h), v[h], power_of_two(-e[h]), u.lane);
    uint32_t word = 0;
#pragma unroll
    for (int h = 0; h < L::kChunks; ++h) word |= (uint32_t)(e[h] + 127) << (8 * L::kBlocks * h);
    if constexpr (L::kPairs) word |= __shfl_down_sync(0xffffffffu, word, 16) << 8;
    if (u.lane == 0) *reinterpret_cast<uint32_t*>(to + u.word + r * 16u) = word;
}

// x to x8 (if given), act(x) to y and to y8 (if given).  Rows up to a multiple of 16 are written, as zeros: the products read
// so many.
template <typename T, Way kWay, int kAct>
__global__ void __launch_bounds__(kWarps * 32, kBlocks<kAct>) f8_rows_kernel(const __grid_constant__ RowsArgs a) {
    using L = Lanes<T, kWay>;
    wait_for_previous_kernel();
    const uint32_t unit = blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (unit >= a.units) return;
    const Unit<T, kWay> u(a, unit);
    const T* x = static_cast<const T*>(a.x) + u.row0 * a.x_stride + u.col;
    T* y = static_cast<T*>(a.y) + u.row0 * a.y_stride + u.col;
    const uint32_t rows = (uint32_t)min((uint64_t)a.unit_rows, a.rows - min(a.rows, u.row0));
    int32_t left[L::kChunks];
#pragma unroll
    for (int h = 0; h < L::kChunks; ++h) left[h] = u.left(a, h);
    typename L::Raw raw[kRowsAtOnce<T, kAct>][L::kChunks];
    auto fetch = [&](uint32_t r0) {
#pragma unroll
        for (int r = 0; r < kRowsAtOnce<T, kAct>; ++r) {
#pragma unroll
            for (int h = 0; h < L::kChunks; ++h) raw[r][h] = L::load(x + h * L::kChunkCols, r0 + r < rows ? left[h] : 0);
            x += a.x_stride;
        }
    };
#pragma unroll 1
    for (uint32_t r0 = 0; r0 < a.unit_rows; r0 += kRowsAtOnce<T, kAct>) {
        fetch(r0);
#pragma unroll
        for (int r = 0; r < kRowsAtOnce<T, kAct>; ++r) {
            float v[L::kChunks][L::kVals];
#pragma unroll
            for (int h = 0; h < L::kChunks; ++h)
#pragma unroll
                for (int i = 0; i < L::kVals; ++i) v[h][i] = L::value(raw[r][h], i);
            uint32_t m[L::kChunks];
            if (a.x8) {
                L::largest(raw[r], m);
                if constexpr (kAct == CO3_ACT_NONE) {
                    put_row<T, kWay>(u, a.x8, r0 + r, v, m);
                } else {  // (the rare way changes them)
                    float t[L::kChunks][L::kVals];
#pragma unroll
                    for (int h = 0; h < L::kChunks; ++h)
#pragma unroll
                        for (int i = 0; i < L::kVals; ++i) t[h][i] = v[h][i];
                    put_row<T, kWay>(u, a.x8, r0 + r, t, m);
                }
            }
            if (a.y || a.y8) {
                if constexpr (kAct == CO3_ACT_NONE) {
#pragma unroll
                    for (int h = 0; h < L::kChunks; ++h)
#pragma unroll
                        for (int i = 0; i < L::kVals; ++i) v[h][i] = L::value(raw[r][h], i);
                } else {
#pragma unroll
                    for (int h = 0; h < L::kChunks; ++h)
#pragma unroll
                        for (int i = 0; i < L::kVals; i += 2) {
                            const F2 t = act<kAct, sizeof(T) == 2>({v[h][i], v[h][i + 1]});
                            v[h][i] = t.x;
                            v[h][i + 1] = t.y;
                        }
                }
                if (a.y)
#pragma unroll
                    for (int h = 0; h < L::kChunks; ++h) L::store(y + h * L::kChunkCols, r0 + r < rows ? left[h] : 0, v[h]);
                if (a.y8) {
#pragma unroll
                    for (int h = 0; h < L::kChunks; ++h) {
                        uint32_t w = 0;
#pragma unroll
                        for (int i = 0; i < L::kVals; ++i) w = max(w, f8_magnitude(v[h][i]));
                        m[h] = L::most(w);
                    }
                    put_row<T, kWay>(u, a.y8, r0 + r, v, m);
                }
            }
            y += a.y_stride;
        }
    }
}

// y <- the values of x8, or (kBackward) dx <- dy * act'(values of x8).
template <typename T, Way kWay, int kAct, bool kBackward>
__global__ void __launch_bounds__(kWarps * 32, kBlocks<kAct>) f8_values_kernel(const __grid_constant__ RowsArgs a) {
    using L = Lanes<T, kWay>;
    wait_for_previous_kernel();
    const uint32_t unit = blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (unit >= a.units) return;
    const Unit<T, kWay> u(a, unit);
    const T* dy = static_cast<const T*>(a.x) + u.row0 * a.x_stride + u.col;
    T* y = static_cast<T*>(a.y) + u.row0 * a.y_stride + u.col;
    const uint32_t rows = (uint32_t)min((uint64_t)a.unit_rows, a.rows - min(a.rows, u.row0));
    int32_t left[L::kChunks];
#pragma unroll
    for (int h = 0; h < L::kChunks; ++h) left[h] = u.left(a, h);
    struct {
        uint32_t word;
        typename L::Bytes f8[L::kChunks];
        typename L::Raw dy[kBackward ? L::kChunks : 1];
    } in[kRowsAtOnce<T, kAct>];
    auto fetch = [&](uint32_t r0) {
#pragma unroll
        for (int r = 0; r < kRowsAtOnce<T, kAct>; ++r) {
            const bool valid = r0 + r < rows;
            in[r].word = valid ? *reinterpret_cast<const uint32_t*>(a.x8 + u.word + (r0 + r) * 16u) : 0x7f7f7f7fu;
#pragma unroll
            for (int h = 0; h < L::kChunks; ++h) {
                in[r].f8[h] = L::get(a.x8 + u.bytes(r0 + r, h), valid && u.has(h));
                if constexpr (kBackward) in[r].dy[h] = L::load(dy + h * L::kChunkCols, valid ? left[h] : 0);
            }
            if constexpr (kBackward) dy += a.x_stride;
        }
    };
#pragma unroll 1
    for (uint32_t r0 = 0; r0 < rows; r0 += kRowsAtOnce<T, kAct>) {
        fetch(r0);
#pragma unroll
        for (int r = 0; r < kRowsAtOnce<T, kAct>; ++r) {
            const auto& now = in[r];
            const uint32_t word = now.word >> (8u * L::block0(u.lane));
#pragma unroll
            for (int h = 0; h < L::kChunks; ++h) {
                float v[L::kVals];
                L::values(now.f8[h], __uint_as_float(((word >> (8 * L::kBlocks * h)) & 0xffu) << 23), u.lane, v);
                if constexpr (kBackward) {
#pragma unroll
                    for (int i = 0; i < L::kVals; i += 2) {
                        const F2 d = mul2({L::value(now.dy[h], i), L::value(now.dy[h], i + 1)}, act_slope<kAct, sizeof(T) == 2>({v[i], v[i + 1]}));
                        v[i] = d.x;
                        v[i + 1] = d.y;
                    }
                }
                L::store(y + h * L::kChunkCols, r0 + r < rows ? left[h] : 0, v);
            }
            y += a.y_stride;
        }
    }
}

// ------------------------------------------------------------------------------------------------
// Square blocks: a thread block of 256 each, 16 rows a warp.  Two blocks an SM, so that one stores while the other loads (4096 x 4096
// fp32 there and back 29 us; one block of up to 217 registers a thread 34).
// ------------------------------------------------------------------------------------------------
struct SquareArgs {
    const void* x;
    uint8_t* out;
    uint64_t rows, x_stride, rows_padded, scales, scales_t;
    uint32_t cols, kb;
};

template <typename T, Way kWay>
__global__ void __launch_bounds__(256, kWay == kWide ? 2 : 3) f8_square_kernel(const __grid_constant__ SquareArgs a) {
    using L = Lanes<T, kWay>;
    constexpr int kRows = L::kPairs ? 2 : 1, kTurns = 16 / kRows;  // rows a warp's load covers
    __shared__ uint32_t part[kWarps];
    wait_for_previous_kernel();
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const uint32_t block = blockIdx.x % a.kb, tile = blockIdx.x / a.kb;
    const uint32_t row0 = warp * 16u + L::block0(lane);
    const uint64_t col = (uint64_t)block * 128u + (kWay == kSingle ? lane : (lane & (L::kPairs ? 15u : 31u)) * L::kVals);
    const int32_t left = (int32_t)(a.cols - min((uint64_t)a.cols, col));
    float v[kTurns][L::kVals];
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const uint64_t row = (uint64_t)tile * 128u + row0 + i * kRows;
        const typename L::Raw raw = L::load(static_cast<const T*>(a.x) + row * a.x_stride + col, row < a.rows ? left : 0);
#pragma unroll
        for (int k = 0; k < L::kVals; ++k) v[i][k] = L::value(raw, k);
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
        L::put(a.out + f8_row(a.rows_padded, block, (uint64_t)tile * 128u + r) + (L::at(lane) ^ ((r & 7u) << 4)), true, v[i], inverse, lane);
    }
    const uint32_t t = threadIdx.x & 127u;
    const uint64_t at = threadIdx.x < 128 ? a.scales + ((block >> 2) * (a.rows_padded >> 7) + tile) * kF8Scales + f8_scale_at(t, block)
                                          : a.scales_t + ((uint64_t)(tile >> 2) * a.kb + block) * kF8Scales + f8_scale_at(t, tile);
    a.out[at] = (uint8_t)(e + 127);
}

// ------------------------------------------------------------------------------------------------
// Launches
// ------------------------------------------------------------------------------------------------
bool wide(int type, const void* p, uint64_t stride, uint32_t cols) {
    const size_t s = type_size(type);
    return !p || (aligned(p, 16) && stride * s % 16 == 0 && cols * s % 16 == 0);
}
void fill(RowsArgs& a, const F8Layout& l, uint64_t rows, uint32_t cols) {
    a.rows = rows;
    a.cols = cols;
    a.kb = l.kb;
    a.groups = (l.kb + 3u) / 4u;
    a.rows_padded = l.rows;
    a.scales = l.scales;
    // eight rows a warp where that still gives every multiprocessor eight warps (148 of them), two otherwise
    const uint64_t padded = (rows + 15u) / 16u * 16u;
    a.unit_rows = padded / 8u * a.groups >= 148u * 8u ? 8 : 2;
    a.units = (uint32_t)(padded / a.unit_rows * a.groups);
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

// Rows over themselves under another stride: some would be written before they are read.
bool crossed(const void* x, uint64_t x_stride, const void* y, uint64_t y_stride, uint64_t rows) { return x == y && x_stride != y_stride && rows > 1; }
bool overlapping(const void* a, const void* b, uint64_t bytes) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
    return a && b && (p < q ? q - p : p - q) < bytes;
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
    if (!f8_valid_rows(type, x, x_row_stride, cols) || !f8_valid(out)) return CO3_ERR_INVALID_ARG;
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
    if (!f8_valid_rows(type, x, x_row_stride, cols) || (y && !f8_valid_rows(type, y, y_row_stride, cols)) || (y8 && !f8_valid(y8)) || (x8 && !f8_valid(x8)) ||
        (!y && !y8 && !x8) || overlapping(x8, y8, l.bytes) || crossed(x, x_row_stride, y, y_row_stride, rows))
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
    if (!f8_valid_rows(type, out, out_row_stride, cols) || !f8_valid(x8) ||
        (act >= 0 && (!f8_valid_rows(type, dy, dy_row_stride, cols) || crossed(dy, dy_row_stride, out, out_row_stride, rows))))
        return CO3_ERR_INVALID_ARG;
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
