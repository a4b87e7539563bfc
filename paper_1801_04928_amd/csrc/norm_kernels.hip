// The row-wise operators of residual blocks: the root-mean-square norm with the residual's addition and its backward pass,
// activations into 8 bits and back, the gradient before an activation, and sums over rows.  All of them are bound by memory:
// every value is read once, held in registers, and written once.
#include "activation.h"
#include "chunks.h"

#include <algorithm>

namespace lf {
namespace ops {
namespace {

constexpr int kThreads = 256;
constexpr int kMostGroups = 1 << 20;      // a grid has fewer than 2^32 threads

__host__ __device__ constexpr int ceil_div(int a, int b) { return a / b + (a % b != 0); }
__host__ __device__ constexpr int whole_groups(int cols) { return ceil_div(cols, kGroup) * kGroup; }

// Sum over the TPR threads that hold one row (all of the block if TPR > 64), in a fixed order; every thread gets it.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* shared) {
    v = wave_sum(v);
    if constexpr (TPR > kWave) {
        __syncthreads();                          // the previous row's sum has been read
        if (threadIdx.x % kWave == 0) shared[threadIdx.x / kWave] = v;
        __syncthreads();
        v = shared[0];
#pragma unroll
        for (int i = 1; i < TPR / kWave; ++i) v += shared[i];
    }
    return v;
}

// ================================================================================================
// norm, forward
// ================================================================================================
struct NormForward {
    int rows, cols;
    Mat x, branch, sum, y;
    const float* gain;
    float* rstd;
    float eps;
};

__device__ __forceinline__ void load_gain(const float* gain, int col, int n, float (&g)[8]) {
    if (gain) {
        load_values(gain + col, n, g);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = 1.0f;
    }
}

// TPR threads hold a row, NCH chunks of eight values each: a row is read once.  AGAIN: rows wider than TPR * NCH chunks are
// read a second time for the outputs.
template <int T, int OUT, int TPR, int NCH, bool AGAIN>
__global__ __launch_bounds__(TPR > kThreads ? TPR : kThreads) void k_norm_forward(const NormForward a) {
    constexpr int kRows = TPR > kThreads ? 1 : kThreads / TPR;
    __shared__ float shared[TPR > kWave ? TPR / kWave : 1];
    const int t = threadIdx.x % TPR;
    const bool more = a.branch.p != nullptr;
    long long row;

    auto load = [&](int chunk, float (&v)[8]) {
        const int col = chunk * kChunk, n = a.cols - col;
        load_chunk<T>(a.x, row, col, n, v);
        if (more) {
            float u[8];
            load_chunk<T>(a.branch, row, col, n, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += u[i];
        }
    };
    auto store = [&](int chunk, const float (&v)[8], float rstd) {
        const int col = chunk * kChunk, n = a.cols - col;
        if (a.sum.p) store_chunk<T>(a.sum, row, col, n, v, n > 0);
        float g[8], y[8];
        load_gain(a.gain, col, n, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = i < n ? v[i] * rstd * g[i] : 0.0f;
        store_chunk<OUT>(a.y, row, col, n, y, col < whole_groups(a.cols));
    };

    const int turns = AGAIN ? ceil_div(a.cols, kChunk * TPR * NCH) : 1;
    // (the grid has a block for every kRows rows, up to kMostGroups of them)
    for (row = (long long)blockIdx.x * kRows + threadIdx.x / TPR; row < a.rows; row += (long long)gridDim.x * kRows) {
        float v[NCH][8], square = 0.0f;
        for (int turn = 0; turn < turns; ++turn) {
#pragma unroll
            for (int j = 0; j < NCH; ++j) load((turn * NCH + j) * TPR + t, v[j]);
#pragma unroll
            for (int j = 0; j < NCH; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) square = fmaf(v[j][i], v[j][i], square);
        }
        const float rstd = 1.0f / sqrtf(row_sum<TPR>(square, shared) / (float)a.cols + a.eps);
        if (a.rstd && t == 0) a.rstd[row] = rstd;
        for (int turn = 0; turn < turns; ++turn) {
            if constexpr (AGAIN) {
#pragma unroll
                for (int j = 0; j < NCH; ++j) load((turn * NCH + j) * TPR + t, v[j]);
            }
#pragma unroll
            for (int j = 0; j < NCH; ++j) store((turn * NCH + j) * TPR + t, v[j], rstd);
        }
    }
}

// ================================================================================================
// norm, backward
// ================================================================================================
struct NormBackward {
    int rows, cols;
    Mat dy, sum, dsum, dx;
    const float* gain;
    const float* rstd;
    float* partial;      // [gridDim.x][cols], or null
};

// A block takes rows blockIdx.x, + gridDim.x, ...: the sums of dy h over its rows stay in registers, a row of partial sums
// per block is all that the gain's gradient costs in memory.  AGAIN as in the forward pass (the gain's gradient is then
// a kernel of its own, k_gain_gradient).
template <int T, int S, int TPR, int NCH, bool AGAIN>
__global__ __launch_bounds__(TPR > kThreads ? TPR : kThreads) void k_norm_backward(const NormBackward a) {
    constexpr int kBlock = TPR > kThreads ? TPR : kThreads, kRows = kBlock / TPR;
    __shared__ float shared[TPR > kWave ? TPR / kWave : 1];
    const int t = threadIdx.x % TPR, mine = threadIdx.x / TPR;
    float total[AGAIN ? 1 : NCH][8];
    if constexpr (!AGAIN) {
#pragma unroll
        for (int j = 0; j < NCH; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) total[j][i] = 0.0f;
    }
    for (long long row = (long long)blockIdx.x * kRows + mine; row < a.rows; row += (long long)gridDim.x * kRows) {
        const float rstd = a.rstd[row];
        float dy[NCH][8], h[NCH][8], along = 0.0f;
        const int turns = AGAIN ? ceil_div(a.cols, kChunk * TPR * NCH) : 1;
        for (int turn = 0; turn < turns; ++turn) {
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                const int col = ((turn * NCH + j) * TPR + t) * kChunk, n = a.cols - col;
                load_chunk<T>(a.dy, row, col, n, dy[j]);
                load_chunk<S>(a.sum, row, col, n, h[j]);
            }
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                const int col = ((turn * NCH + j) * TPR + t) * kChunk, n = a.cols - col;
                float g[8];
                load_gain(a.gain, col, n, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    h[j][i] *= rstd;
                    if constexpr (!AGAIN) total[j][i] = fmaf(dy[j][i], h[j][i], total[j][i]);
                    dy[j][i] *= g[i];
                    along = fmaf(dy[j][i], h[j][i], along);
                }
            }
        }
        const float mean = row_sum<TPR>(along, shared) / (float)a.cols;
        for (int turn = 0; turn < turns; ++turn) {
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                const int col = ((turn * NCH + j) * TPR + t) * kChunk, n = a.cols - col;
                if constexpr (AGAIN) {
                    float g[8];
                    load_chunk<T>(a.dy, row, col, n, dy[j]);
                    load_chunk<S>(a.sum, row, col, n, h[j]);
                    load_gain(a.gain, col, n, g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) { h[j][i] *= rstd; dy[j][i] *= g[i]; }
                }
                float d[8];
                if (a.dsum.p) {
                    load_chunk<T>(a.dsum, row, col, n, d);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[i] = 0.0f;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] = fmaf(rstd, dy[j][i] - h[j][i] * mean, d[i]);
                store_chunk<T>(a.dx, row, col, n, d, n > 0);
            }
        }
    }
    if constexpr (!AGAIN) {
        if (!a.partial) return;
        float* out = a.partial + (size_t)blockIdx.x * a.cols;
        if constexpr (kRows == 1) {
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                const int col = (j * TPR + t) * kChunk;
                if (col < a.cols) store_values(out + col, a.cols - col, total[j]);
            }
        } else {
            __shared__ float rows_total[kRows - 1][NCH * TPR * kChunk];
            if (mine > 0) {
#pragma unroll
                for (int j = 0; j < NCH; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) rows_total[mine - 1][(j * TPR + t) * kChunk + i] = total[j][i];
            }
            __syncthreads();
            if (mine == 0) {
#pragma unroll
                for (int j = 0; j < NCH; ++j) {
                    const int col = (j * TPR + t) * kChunk;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int r = 0; r < kRows - 1; ++r) total[j][i] += rows_total[r][col + i];
                    if (col < a.cols) store_values(out + col, a.cols - col, total[j]);
                }
            }
        }
    }
}

// Walks of a block over rows of a strip of 64 chunks: what the column sums of dy h (wide norms) and of dz have in common.
// Four threads share a chunk column and take every fourth row.
constexpr int kStripChunks = 64, kStripRows = kThreads / kStripChunks;

__device__ __forceinline__ void strip_finish(float (&total)[8], float* partial, int cols) {
    __shared__ float others[kStripRows - 1][kStripChunks * kChunk];
    const int t = threadIdx.x % kStripChunks, mine = threadIdx.x / kStripChunks;
    if (mine > 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) others[mine - 1][t * kChunk + i] = total[i];
    }
    __syncthreads();
    const int col = (blockIdx.x * kStripChunks + t) * kChunk;
    if (mine == 0 && col < cols) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int r = 0; r < kStripRows - 1; ++r) total[i] += others[r][t * kChunk + i];
        store_values(partial + (size_t)blockIdx.y * cols + col, cols - col, total);
    }
}

template <int T, int S>
__global__ __launch_bounds__(kThreads) void k_gain_gradient(const NormBackward a, int rows_per_block) {
    const int col = (blockIdx.x * kStripChunks + threadIdx.x % kStripChunks) * kChunk, n = a.cols - col;
    const int first = blockIdx.y * rows_per_block, end = min(a.rows, first + rows_per_block);
    float total[8] = {};
    for (int row = first + threadIdx.x / kStripChunks; row < end; row += kStripRows) {
        float dy[8], h[8];
        load_chunk<T>(a.dy, row, col, n, dy);
        load_chunk<S>(a.sum, row, col, n, h);
        const float rstd = a.rstd[row];
#pragma unroll
        for (int i = 0; i < 8; ++i) total[i] = fmaf(dy[i], h[i] * rstd, total[i]);
    }
    strip_finish(total, a.partial, a.cols);
}

// ================================================================================================
// the gradient before an activation, and its sums over rows
// ================================================================================================
struct Slope {
    int rows, cols, act;
    Mat dy, z, dz;
    float* partial;      // [gridDim.y][cols], or null
};
template <int T, int Z>
__global__ __launch_bounds__(kThreads) void k_slope(const Slope a, int rows_per_block) {
    const int col = (blockIdx.x * kStripChunks + threadIdx.x % kStripChunks) * kChunk, n = a.cols - col;
    const int first = blockIdx.y * rows_per_block, end = min(a.rows, first + rows_per_block);
    float total[8] = {};
    for (int row = first + threadIdx.x / kStripChunks; row < end; row += kStripRows) {
        float d[8];
        load_chunk<T>(a.dy, row, col, n, d);
        if (a.act != NONE) {
            float z[8];
            load_chunk<Z>(a.z, row, col, n, z);
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] *= slope(a.act, z[i]);
        }
        if (a.dz.p) store_chunk<T>(a.dz, row, col, n, d, n > 0);
#pragma unroll
        for (int i = 0; i < 8; ++i) total[i] += d[i];
    }
    if (a.partial) strip_finish(total, a.partial, a.cols);
}

// Sums of partial rows: 64 columns a block, 16 threads a column, each over every sixteenth row.
constexpr int kFinishCols = 64, kFinishWays = 16;
__global__ __launch_bounds__(kFinishCols * kFinishWays) void k_column_finish(const float* partial, int partials, int cols,
                                                                             float* out) {
    __shared__ float ways[kFinishWays][kFinishCols];
    const int c = threadIdx.x % kFinishCols, way = threadIdx.x / kFinishCols;
    const int col = blockIdx.x * kFinishCols + c;
    float v = 0.0f;
    if (col < cols)
        for (int p = way; p < partials; p += kFinishWays) v += partial[(size_t)p * cols + col];
    ways[way][c] = v;
    __syncthreads();
    if (way == 0 && col < cols) {
#pragma unroll
        for (int i = 1; i < kFinishWays; ++i) v += ways[i][c];
        out[col] = v;
    }
}

// ================================================================================================
// 8 bits
// ================================================================================================
// A block is TX chunks wide (a power of two, at least a group's four) and kThreads / TX rows high, and takes kSteps such
// pieces below each other: the loads of all of them are under way at once.
constexpr int kSteps = 4;
struct Copy {
    int rows, cols;
    int tx_bits, blocks_x;
    Mat from, to;
};
template <int FROM, int TO>
__global__ __launch_bounds__(kThreads) void k_copy(const Copy a) {
    const int tx = 1 << a.tx_bits, ty = kThreads >> a.tx_bits;
    const unsigned bx = blockIdx.x % (unsigned)a.blocks_x, by = blockIdx.x / (unsigned)a.blocks_x;
    const int col = (int)((bx << a.tx_bits) + (threadIdx.x & (tx - 1))) * kChunk, n = a.cols - col;
    const long long row0 = (long long)by * ty * kSteps + (threadIdx.x >> a.tx_bits);
    float v[kSteps][8];
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        const long long row = row0 + u * ty;
        load_chunk<FROM>(a.from, row, col, row < a.rows ? n : 0, v[u]);
    }
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        const long long row = row0 + u * ty;
        store_chunk<TO>(a.to, row, col, n, v[u], row < a.rows && col < whole_groups(a.cols));
    }
}

template <int FROM, int TO>
hipError_t copy(int rows, int cols, const Mat& from, const Mat& to, hipStream_t s) {
    if (rows == 0) return hipSuccess;
    Copy a{rows, cols, 2, 1, from, to};
    const int chunks = whole_groups(cols) / kChunk;
    while ((1 << a.tx_bits) < chunks && (1 << a.tx_bits) < kThreads) ++a.tx_bits;
    a.blocks_x = ceil_div(chunks, 1 << a.tx_bits);
    const long long blocks_y = ((long long)rows + (kThreads >> a.tx_bits) * kSteps - 1) / ((kThreads >> a.tx_bits) * kSteps);
    k_copy<FROM, TO><<<dim3((unsigned)(blocks_y * a.blocks_x)), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

// Threads and chunks a row takes: the fewest chunks a thread that hold it, waves of their own up to 2048 columns.
template <class F> hipError_t by_width(int cols, F&& f) {
    using std::integral_constant;
    if (cols <= 512) return f(integral_constant<int, 64>(), integral_constant<int, 1>(), std::false_type());
    if (cols <= 1024) return f(integral_constant<int, 64>(), integral_constant<int, 2>(), std::false_type());
    if (cols <= 2048) return f(integral_constant<int, 64>(), integral_constant<int, 4>(), std::false_type());
    if (cols <= 4096) return f(integral_constant<int, 256>(), integral_constant<int, 2>(), std::false_type());
    if (cols <= 8192) return f(integral_constant<int, 256>(), integral_constant<int, 4>(), std::false_type());
    if (cols <= 16384) return f(integral_constant<int, 512>(), integral_constant<int, 4>(), std::false_type());
    return f(integral_constant<int, 512>(), integral_constant<int, 4>(), std::true_type());
}
constexpr int kHeldCols = 16384;
int rows_per_block(int cols) { return cols <= 2048 ? 4 : 1; }

template <int T, int OUT>
hipError_t norm_forward(const NormForward& a, hipStream_t s) {
    return by_width(a.cols, [&](auto tpr, auto nch, auto again) {
        constexpr int block = tpr() > kThreads ? tpr() : kThreads;
        k_norm_forward<T, OUT, tpr(), nch(), again()><<<dim3(std::min(ceil_div(a.rows, block / tpr()), kMostGroups)),
                                                            block, 0, s>>>(a);
        return hipGetLastError();
    });
}
template <int T, int S>
hipError_t norm_backward(const NormBackward& a, hipStream_t s) {
    return by_width(a.cols, [&](auto tpr, auto nch, auto again) {
        constexpr int block = tpr() > kThreads ? tpr() : kThreads;
        const int groups = again() ? std::min(a.rows, kMostGroups) : norm_partials(a.rows, a.cols);
        k_norm_backward<T, S, tpr(), nch(), again()><<<dim3(groups), block, 0, s>>>(a);
        if (again() && a.partial) {
            const int parts = norm_partials(a.rows, a.cols);
            k_gain_gradient<T, S><<<dim3(ceil_div(a.cols, kStripChunks * kChunk), parts), kThreads, 0, s>>>(
                a, ceil_div(a.rows, parts));
        }
        return hipGetLastError();
    });
}
template <int T, int Z>
hipError_t slopes(const Slope& a, int parts, hipStream_t s) {
    k_slope<T, Z><<<dim3(ceil_div(a.cols, kStripChunks * kChunk), parts), kThreads, 0, s>>>(a, ceil_div(a.rows, parts));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_save(int rows, int cols, const Mat& x, const Mat& out, hipStream_t s) {
    return x.kind == F32 ? copy<F32, E4M3>(rows, cols, x, out, s) : copy<BF16, E4M3>(rows, cols, x, out, s);
}
hipError_t launch_load(int rows, int cols, const Mat& in, const Mat& out, hipStream_t s) {
    return out.kind == F32 ? copy<E4M3, F32>(rows, cols, in, out, s) : copy<E4M3, BF16>(rows, cols, in, out, s);
}

hipError_t launch_norm_forward(int rows, int cols, const Mat& x, const Mat& branch, const float* gain, float eps,
                               const Mat& sum, const Mat& y, float* rstd, hipStream_t s) {
    if (rows == 0) return hipSuccess;
    const NormForward a{rows, cols, x, branch, sum, y, gain, rstd, eps};
    if (x.kind == F32) return y.kind == E4M3 ? norm_forward<F32, E4M3>(a, s) : norm_forward<F32, F32>(a, s);
    return y.kind == E4M3 ? norm_forward<BF16, E4M3>(a, s) : norm_forward<BF16, BF16>(a, s);
}

int norm_partials(int rows, int cols) {
    if (rows == 0) return 0;
    if (cols > kHeldCols) return std::min(ceil_div(rows, 16), 64);
    return std::min(ceil_div(rows, rows_per_block(cols)), 512);
}

hipError_t launch_norm_backward(int rows, int cols, const Mat& dy, const Mat& sum, const float* gain, const float* rstd,
                                const Mat& dsum, const Mat& dx, float* dgain, float* partial, hipStream_t s) {
    if (rows > 0) {
        const NormBackward a{rows, cols, dy, sum, dsum, dx, gain, rstd, dgain ? partial : nullptr};
        hipError_t e;
        if (dy.kind == F32) e = sum.kind == E4M3 ? norm_backward<F32, E4M3>(a, s) : norm_backward<F32, F32>(a, s);
        else e = sum.kind == E4M3 ? norm_backward<BF16, E4M3>(a, s) : norm_backward<BF16, BF16>(a, s);
        if (e != hipSuccess) return e;
    }
    return dgain ? launch_column_finish(partial, norm_partials(rows, cols), cols, dgain, s) : hipSuccess;
}

hipError_t launch_column_finish(const float* partial, int partials, int cols, float* out, hipStream_t s) {
    k_column_finish<<<dim3(ceil_div(cols, kFinishCols)), kFinishCols * kFinishWays, 0, s>>>(partial, partials, cols, out);
    return hipGetLastError();
}

int slope_partials(int rows, int cols) {
    if (rows == 0) return 0;
    const int strips = ceil_div(cols, kStripChunks * kChunk);
    return std::max(1, std::min(ceil_div(rows, 4 * kStripRows), std::max(1, 2048 / strips)));
}

hipError_t launch_slope(int rows, int cols, const Mat& dy, const Mat& z, int act, const Mat& dz, float* partial,
                        hipStream_t s) {
    if (rows == 0) return hipSuccess;
    const Slope a{rows, cols, act, dy, z, dz, partial};
    const int parts = slope_partials(rows, cols);
    if (dy.kind == F32) return act != NONE && z.kind == E4M3 ? slopes<F32, E4M3>(a, parts, s) : slopes<F32, F32>(a, parts, s);
    return act != NONE && z.kind == E4M3 ? slopes<BF16, E4M3>(a, parts, s) : slopes<BF16, BF16>(a, parts, s);
}

}  // namespace ops
}  // namespace lf
