// Sums over rows of partial sums, as the kernels that end a backward pass take them.
#pragma once
#include "operators_internal.h"

namespace lf {
namespace ops {

// 32 columns a block, 32 threads a column, each over every 32nd row with eight loads under way.  No rows: zeros.
constexpr int kFinishCols = 32, kFinishWays = 32, kFinishThreads = kFinishCols * kFinishWays;
inline unsigned finish_blocks(const ColumnSums& a) { return a.out ? (unsigned)((a.cols + kFinishCols - 1) / kFinishCols) : 0; }
__device__ __forceinline__ void finish_columns(const ColumnSums& a, unsigned block) {
    __shared__ float ways[kFinishWays][kFinishCols];
    const int c = threadIdx.x % kFinishCols, way = threadIdx.x / kFinishCols;
    const int col = block * kFinishCols + c;
    float v = 0.0f;
    if (col < a.cols) {
#pragma unroll 8
        for (int p = way; p < a.partials; p += kFinishWays) v += a.partial[(size_t)p * a.cols + col];
    }
    ways[way][c] = v;
    __syncthreads();
    if (way == 0 && col < a.cols) {
#pragma unroll
        for (int i = 1; i < kFinishWays; ++i) v += ways[i][c];
        a.out[col] = v;
    }
}

}  // namespace ops
}  // namespace lf
