// The row-wise operators of residual blocks: the root-mean-square norm with the residual's addition and its backward pass,
// activations into 8 bits and back, the gradient before an activation, and sums over rows.  All of them are bound by memory:
// every value is read once, held in registers, and written once.
#include "activation.h"
#include "chunks.h"
#include "column_sums.h"

#include <algorithm>
#include <type_traits>

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

// 1 / sqrt(m) to half an ulp: the instruction's value (good to one) and a Newton step whose remainder 1 - m r^2 keeps what m r
// loses in rounding.  A row's values share it, and those kept in 8 bits next to a rounding border show its last bit.
__device__ __forceinline__ float inverse_root(float m) {
    if (!(m > 0x1p-100f && m < 0x1p+120f)) return 1.0f / sqrtf(m);
    const float r = __builtin_amdgcn_rsqf(m), t = m * r;
    const float rest = fmaf(-t, r, 1.0f) - fmaf(m, r, -t) * r;
    return fmaf(0.5f * r, rest, r);
}

// Bound by memory: 16384 x 8192 bf16 with y in 8 bits 167 us = 5.65 TB/s, fp32 385 us = 5.6.  TPR threads hold a row, NCH chunks of eight values
// each: a row is read once.  AGAIN: rows wider than TPR * NCH chunks are
// read a second time for the outputs.
template <int T, int OUT, int TPR, int NCH, bool AGAIN, bool NARROW>
__global__ __launch_bounds__(TPR > kThreads ? TPR : kThreads) void k_norm_forward(const NormForward a) {
    constexpr int kRows = TPR > kThreads ? 1 : kThreads / TPR;
    __shared__ float shared[TPR > kWave ? TPR / kWave : 1];
    const int t = threadIdx.x % TPR;
    const bool more = a.branch.p != nullptr;
    const int turns = AGAIN ? ceil_div(a.cols, kChunk * TPR * NCH) : 1;
    long long row;

    auto load = [&](int turn, float (&v)[NCH][8]) {
        Chunk<T> x[NCH], branch[NCH];
#pragma unroll
        for (int j = 0; j < NCH; ++j)
            fetch_chunk<T, NARROW>(x[j], a.x, row, ((turn * NCH + j) * TPR + t) * kChunk, a.cols);
        if (more) {
#pragma unroll
            for (int j = 0; j < NCH; ++j)
                fetch_chunk<T, NARROW>(branch[j], a.branch, row, ((turn * NCH + j) * TPR + t) * kChunk, a.cols);
        }
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int n = a.cols - ((turn * NCH + j) * TPR + t) * kChunk;
            take_chunk<T, NARROW>(x[j], n, v[j]);
            if (more) {
                float u[8];
                take_chunk<T, NARROW>(branch[j], n, u);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[j][i] += u[i];
            }
        }
    };
    // (the grid has a block for every kRows rows, up to kMostGroups of them)
    for (row = (long long)blockIdx.x * kRows + (kRows == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / TPR)); row < a.rows; row += (long long)gridDim.x * kRows) {
        float v[NCH][8], square = 0.0f;
        for (int turn = 0; turn < turns; ++turn) {
            load(turn, v);
#pragma unroll
            for (int j = 0; j < NCH; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) square = fmaf(v[j][i], v[j][i], square);
        }
        const float rstd = inverse_root(row_sum<TPR>(square, shared) / (float)a.cols + a.eps);
        if (a.rstd && t == 0) a.rstd[row] = rstd;
        for (int turn = 0; turn < turns; ++turn) {
            if constexpr (AGAIN) load(turn, v);
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                const int col = ((turn * NCH + j) * TPR + t) * kChunk, n = a.cols - col;
                if (a.sum.p) store_chunk<T>(a.sum, row, col, n, v[j], n > 0);
                float g[8], y[8];
                load_gain(a.gain, col, n, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = i < n ? v[j][i] * rstd * g[i] : 0.0f;
                store_chunk<OUT>(a.y, row, col, n, y, col < whole_groups(a.cols));
            }
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
// per block is all that the gain's gradient costs in memory.  The next row is under way, as it lies in memory, while one is
// worked on (16384 x 8192 bf16, s in 8 bits: 314 -> 171 us = 5.5 TB/s; fp32 397 us = 5.4).  Rows of 8193 to 16384 columns take 1024
// threads of at most 128 registers, which do not hold all that: 18 (bf16), 31 (from 8 bits), 151 (fp32) and 156 (from 8 bits) are
// spilled, and 16384 x 16384 bf16 takes 512 us = 4.2 TB/s, 8192 x 16384 fp32 671 us = 3.2.  AGAIN as in the forward pass (the gain's
// gradient is then a kernel of its own, k_gain_gradient).
template <int T, int S, int TPR, int NCH, bool AGAIN, bool NARROW>
__global__ __launch_bounds__(TPR > kThreads ? TPR : kThreads) void k_norm_backward(const NormBackward a) {
    constexpr int kBlock = TPR > kThreads ? TPR : kThreads, kRows = kBlock / TPR;
    __shared__ float shared[TPR > kWave ? TPR / kWave : 1];
    // (the row is the same for a whole wave: its addresses are scalars)
    const int t = threadIdx.x % TPR, mine = kRows == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    const bool more = a.dsum.p != nullptr;
    const long long step = (long long)gridDim.x * kRows;
    const auto col_of = [&](int turn, int j) { return ((turn * NCH + j) * TPR + t) * kChunk; };
    float total[AGAIN ? 1 : NCH][8], gain[AGAIN ? 1 : NCH][8];
    Chunk<T> dy_raw[NCH], dsum_raw[NCH];
    Chunk<S> s_raw[NCH];
    float rstd_raw = 0.0f;
    auto request = [&](long long row, int turn) {
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            fetch_chunk<T, NARROW>(dy_raw[j], a.dy, row, col_of(turn, j), a.cols);
            fetch_chunk<S, NARROW>(s_raw[j], a.sum, row, col_of(turn, j), a.cols);
        }
        rstd_raw = a.rstd[row];
    };
    auto request_dsum = [&](long long row, int turn) {
#pragma unroll
        for (int j = 0; j < NCH; ++j) fetch_chunk<T, NARROW>(dsum_raw[j], a.dsum, row, col_of(turn, j), a.cols);
    };
    // t = dy gain and h = sum rstd of chunk j
    auto take = [&](int turn, int j, float rstd, float (&dy)[8], float (&h)[8]) {
        const int n = a.cols - col_of(turn, j);
        take_chunk<T, NARROW>(dy_raw[j], n, dy);
        take_chunk<S, NARROW>(s_raw[j], n, h);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] *= rstd;
    };
    if constexpr (!AGAIN) {
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            load_gain(a.gain, col_of(0, j), a.cols - col_of(0, j), gain[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) total[j][i] = 0.0f;
        }
    }
    long long row = (long long)blockIdx.x * kRows + mine;
    if constexpr (!AGAIN) {
        if (row < a.rows) request(row, 0);
    }
    for (; row < a.rows; row += step) {
        float dy[NCH][8], h[NCH][8], along = 0.0f;
        const int turns = AGAIN ? ceil_div(a.cols, kChunk * TPR * NCH) : 1;
        if constexpr (AGAIN) {
            for (int turn = 0; turn < turns; ++turn) {
                request(row, turn);
#pragma unroll
                for (int j = 0; j < NCH; ++j) {
                    float g[8];
                    take(turn, j, rstd_raw, dy[j], h[j]);
                    load_gain(a.gain, col_of(turn, j), a.cols - col_of(turn, j), g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) along = fmaf(dy[j][i] * g[i], h[j][i], along);
                }
            }
        } else {
            if (more) request_dsum(row, 0);
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                take(0, j, rstd_raw, dy[j], h[j]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    total[j][i] = fmaf(dy[j][i], h[j][i], total[j][i]);
                    dy[j][i] *= gain[j][i];
                    along = fmaf(dy[j][i], h[j][i], along);
                }
            }
        }
        const float rstd = rstd_raw;
        // (past the last row the last one again: no branch around the loads)
        if constexpr (!AGAIN) request(min(row + step, (long long)a.rows - 1), 0);
        const float mean = row_sum<TPR>(along, shared) / (float)a.cols;
        for (int turn = 0; turn < turns; ++turn) {
            if constexpr (AGAIN) {
                request(row, turn);
                if (more) request_dsum(row, turn);
            }
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                const int col = col_of(turn, j), n = a.cols - col;
                if constexpr (AGAIN) {
                    float g[8];
                    take(turn, j, rstd, dy[j], h[j]);
                    load_gain(a.gain, col, n, g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) dy[j][i] *= g[i];
                }
                float d[8] = {};
                if (more) take_chunk<T, NARROW>(dsum_raw[j], n, d);
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
            for (int j = 0; j < NCH; ++j)
                if (col_of(0, j) < a.cols) store_values(out + col_of(0, j), a.cols - col_of(0, j), total[j]);
        } else {
            __shared__ float rows_total[kRows - 1][NCH * TPR * kChunk];
            if (mine > 0) {
#pragma unroll
                for (int j = 0; j < NCH; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) rows_total[mine - 1][col_of(0, j) + i] = total[j][i];
            }
            __syncthreads();
            if (mine == 0) {
#pragma unroll
                for (int j = 0; j < NCH; ++j) {
                    const int col = col_of(0, j);
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

template <int ACT>
__device__ __forceinline__ void times_slope(float (&d)[8], const float (&z)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) d[i] *= slope(ACT, z[i]);
}

// ================================================================================================
// the gradient before an activation, and its sums over rows
// ================================================================================================
// A block is W chunks wide and kThreads / W rows high and walks down a part of the rows, kSlopeSteps of its heights at once.  Four
// chunks where one part holds all rows (its sums are db itself): of few values, the more threads the less each
// computes.  16 chunks, whole lines, where memory counts: 4096 x 8192 bf16, z in 8 bits, gelu 45 us = 3.7 TB/s, half of
// which the slope's arithmetic takes.
constexpr int kSlopeSteps = 2, kNarrowStrip = 4, kWideStrip = 16;
struct Slope {
    int rows, cols, act;
    Mat dy, z, dz;
    float* partial;      // [gridDim.y][cols], or null
};
template <int T, int Z, int W>
__global__ __launch_bounds__(kThreads) void k_slope(const Slope a, int rows_per_block) {
    constexpr int kHigh = kThreads / W;
    const int t = threadIdx.x % W, mine = threadIdx.x / W;
    const int col = (blockIdx.x * W + t) * kChunk, n = a.cols - col;
    const int first = blockIdx.y * rows_per_block, end = min(a.rows, first + rows_per_block);
    float total[8] = {};
    for (int row0 = first + mine; row0 < end; row0 += kHigh * kSlopeSteps) {
        float d[kSlopeSteps][8], z[kSlopeSteps][8];
#pragma unroll
        for (int u = 0; u < kSlopeSteps; ++u) {
            const int row = row0 + u * kHigh, there = row < end ? n : 0;
            load_chunk<T>(a.dy, row, col, there, d[u]);
            if (a.act != NONE) load_chunk<Z>(a.z, row, col, there, z[u]);
        }
#pragma unroll
        for (int u = 0; u < kSlopeSteps; ++u) {
            const int row = row0 + u * kHigh;
            if (row >= end) continue;
            switch (a.act) {
                case SIGMOID: times_slope<SIGMOID>(d[u], z[u]); break;
                case RELU: times_slope<RELU>(d[u], z[u]); break;
                case SILU: times_slope<SILU>(d[u], z[u]); break;
                case GELU: times_slope<GELU>(d[u], z[u]); break;
                default: break;
            }
            if (a.dz.p) store_chunk<T>(a.dz, row, col, n, d[u], n > 0);
#pragma unroll
            for (int i = 0; i < 8; ++i) total[i] += d[u][i];
        }
    }
    if (!a.partial) return;
    __shared__ float others[kHigh][W * kChunk + 1];
#pragma unroll
    for (int i = 0; i < 8; ++i) others[mine][t * kChunk + i] = total[i];
    __syncthreads();
    const int c = threadIdx.x, out = blockIdx.x * W * kChunk + c;
    if (c < W * kChunk && out < a.cols) {
        float v = others[0][c];
#pragma unroll 8
        for (int r = 1; r < kHigh; ++r) v += others[r][c];
        a.partial[(size_t)blockIdx.y * a.cols + out] = v;
    }
}

__global__ __launch_bounds__(kFinishThreads) void k_column_finish(const ColumnSums a) { finish_columns(a, blockIdx.x); }

// ================================================================================================
// 8 bits
// ================================================================================================
// A block is TX chunks wide (a power of two, at least a group's four) and kThreads / TX rows high, and takes kSteps such
// pieces below each other: the loads of all of them are under way at once.  16384 x 8192 bf16 there and back: 153 us =
// 5.3 TB/s.
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

// Threads that hold a row, each NCH chunks of it.  Waves of their own up to 1024 columns: no barrier.
template <class F> hipError_t by_width(int cols, F&& f) {
    using std::integral_constant;
    const std::false_type no;
    const std::true_type yes;
    const integral_constant<int, 2> two;
    if (cols < kChunk) return f(integral_constant<int, 64>(), integral_constant<int, 1>(), no, yes);
    if (cols <= 512) return f(integral_constant<int, 64>(), integral_constant<int, 1>(), no, no);
    if (cols <= 1024) return f(integral_constant<int, 64>(), two, no, no);
    if (cols <= 4096) return f(integral_constant<int, 256>(), two, no, no);
    if (cols <= 8192) return f(integral_constant<int, 512>(), two, no, no);
    if (cols <= 16384) return f(integral_constant<int, 1024>(), two, no, no);
    return f(integral_constant<int, 1024>(), two, yes, no);
}
constexpr int kHeldCols = 16384;
int rows_per_block(int cols) { return cols <= 1024 ? 4 : 1; }

template <int T, int OUT>
hipError_t norm_forward(const NormForward& a, hipStream_t s) {
    return by_width(a.cols, [&](auto tpr, auto nch, auto again, auto narrow) {
        constexpr int block = tpr() > kThreads ? tpr() : kThreads;
        k_norm_forward<T, OUT, tpr(), nch(), again(), narrow()><<<dim3(std::min(ceil_div(a.rows, block / tpr()), kMostGroups)),
                                                            block, 0, s>>>(a);
        return hipGetLastError();
    });
}
template <int T, int S>
hipError_t norm_backward(const NormBackward& a, hipStream_t s) {
    return by_width(a.cols, [&](auto tpr, auto nch, auto again, auto narrow) {
        constexpr int block = tpr() > kThreads ? tpr() : kThreads;
        const int groups = again() ? std::min(a.rows, kMostGroups) : norm_partials(a.rows, a.cols);
        k_norm_backward<T, S, tpr(), nch(), again(), narrow()><<<dim3(groups), block, 0, s>>>(a);
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
    const int rows = ceil_div(a.rows, parts);
    if (parts == 1) k_slope<T, Z, kNarrowStrip><<<dim3(ceil_div(a.cols, kNarrowStrip * kChunk)), kThreads, 0, s>>>(a, rows);
    else k_slope<T, Z, kWideStrip><<<dim3(ceil_div(a.cols, kWideStrip * kChunk), parts), kThreads, 0, s>>>(a, rows);
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
    const int blocks = ceil_div(rows, rows_per_block(cols));
    // few values: one block, whose sums are dgain itself, takes less than a second launch
    if (blocks <= 8 && (long long)rows * cols <= 32768) return 1;
    return std::min(blocks, 512);
}

hipError_t launch_norm_backward(int rows, int cols, const Mat& dy, const Mat& sum, const float* gain, const float* rstd,
                                const Mat& dsum, const Mat& dx, float* dgain, float* partial, hipStream_t s) {
    const bool direct = norm_partials(rows, cols) == 1;
    if (rows > 0) {
        const NormBackward a{rows, cols, dy, sum, dsum, dx, gain, rstd, !dgain ? nullptr : direct ? dgain : partial};
        hipError_t e;
        if (dy.kind == F32) e = sum.kind == E4M3 ? norm_backward<F32, E4M3>(a, s) : norm_backward<F32, F32>(a, s);
        else e = sum.kind == E4M3 ? norm_backward<BF16, E4M3>(a, s) : norm_backward<BF16, BF16>(a, s);
        if (e != hipSuccess) return e;
    }
    return dgain && !direct ? launch_column_finish(ColumnSums{partial, norm_partials(rows, cols), cols, dgain}, s) : hipSuccess;
}

hipError_t launch_column_finish(const ColumnSums& a, hipStream_t s) {
    if (!a.out) return hipSuccess;
    k_column_finish<<<dim3(finish_blocks(a)), kFinishThreads, 0, s>>>(a);
    return hipGetLastError();
}

// Parts of the rows: one as long as a block's walk down all of them costs less than a second launch, then as many as give the
// chip eight blocks a compute unit (4096 x 8192: four take 1.5 us more).
int slope_partials(int rows, int cols) {
    if (rows == 0) return 0;
    const int strips = ceil_div(cols, kWideStrip * kChunk), step = kThreads / kWideStrip * kSlopeSteps;
    if (rows <= 256) return 1;
    return std::max(1, std::min(ceil_div(rows, step), std::max(1, 2048 / strips)));
}

ColumnSums slope_sums(int rows, int cols, float* db, float* partial) {
    const int parts = slope_partials(rows, cols);
    return ColumnSums{partial, parts, cols, parts == 1 ? nullptr : db};
}

hipError_t launch_slope(int rows, int cols, const Mat& dy, const Mat& z, int act, const Mat& dz, float* db, float* partial,
                        hipStream_t s) {
    if (rows == 0) return hipSuccess;
    const int parts = slope_partials(rows, cols);
    const Slope a{rows, cols, act, dy, z, dz, !db ? nullptr : parts == 1 ? db : partial};
    if (dy.kind == F32) return act != NONE && z.kind == E4M3 ? slopes<F32, E4M3>(a, parts, s) : slopes<F32, F32>(a, parts, s);
    return act != NONE && z.kind == E4M3 ? slopes<BF16, E4M3>(a, parts, s) : slopes<BF16, BF16>(a, parts, s);
}

}  // namespace ops
}  // namespace lf
