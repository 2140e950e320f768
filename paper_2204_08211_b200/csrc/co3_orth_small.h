// Interface of the kernel for small matrices (co3_orth_small.cu) to the entry points (co3_orth.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "co3.h"

namespace co3 {

constexpr uint32_t kSmallMats = 64;     // matrices of one call
constexpr uint32_t kSmallCluster = 16;  // blocks of a matrix at most

struct SmallMat {
    uint64_t in_off, in_stride, out_off, out_stride;
    uint32_t rows, cols;
    float scale;
    uint32_t index;  // in the caller's list
};

struct SmallBatch {
    SmallMat mat[kSmallMats];
    uint32_t n_mats;
};

struct SmallCall {
    const void* in;
    float* momentum;  // null: orthogonalize only
    void* out;
    int out_kind;     // OrthOut
    float mu, lr, shrink;
    int nesterov;
    int clear_result;  // the first launch starts the result
    co3_ns ns;
    co3_result* res;
};

// Blocks (a power of two) that hold a matrix, 0 if it is too large.
inline uint32_t small_ctas(uint32_t rows, uint32_t cols) {
    const uint32_t m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    if (m > 128u || n > 128u * kSmallCluster) return 0;
    uint32_t c = 1;
    while (c * 128u < n) c *= 2;
    return c;
}

// Enqueues the whole call for these matrices, each of which small_ctas accepts.
int orth_small_run(const SmallBatch& batch, const SmallCall& call, int in_type, cudaStream_t st);

}  // namespace co3
