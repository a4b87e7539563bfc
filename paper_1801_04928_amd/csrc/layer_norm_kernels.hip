// The layer norm with the residual's addition, and its backward pass.  Bound by memory: every value is read once, held in registers,
// and written once.  16384 x 8192 bf16, four matrices of it: forward 190 us, 5.7 TB/s, backward 200 us, 5.4 TB/s (fp32 406 and 405), where a copy of 1
// GiB reaches 5.1 and kernels that only read or only write 6.3 and 5.7; small ones take the call's time on the host (1 x 1024 9 us, the kernel 3.4 of it).
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
__host__ __device__ constexpr int whole(int cols, int group) { return ceil_div(cols, group) * group; }

// Sums over the TPR threads that hold one row (all of the block if TPR > 64), in a fixed order; every thread gets them.  Calls take
// turns with two places in `shared`, so that one barrier a call is enough: a place is written again only after the next call's.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (&shared)[2][N][TPR > kWave ? TPR / kWave : 1], int& turn) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = wave_sum(v[k]);
    if constexpr (TPR > kWave) {
        if (threadIdx.x % kWave == 0) {
#pragma unroll
            for (int k = 0; k < N; ++k) shared[turn][k][threadIdx.x / kWave] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = shared[turn][k][0];
#pragma unroll
            for (int i = 1; i < TPR / kWave; ++i) v[k] += shared[turn][k][i];
        }
        turn ^= 1;
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

__device__ __forceinline__ void load_vector_of(const float* p, float otherwise, int col, int n, float (&g)[8]) {
    if (p) {
        load_values(p + col, n, g);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = otherwise;
    }
}

// ================================================================================================
// forward
// ================================================================================================
struct Forward {
    int rows, cols;
    Mat x, branch, sum, y;
    const float* gain;
    const float* shift;
    float* mean;
    float* rstd;
    float eps;
};

// TPR threads hold a row, NCH chunks of eight values each: a row is read once.  The mean square is taken of differences from the
// mean, a second sum over what is in registers: E(s^2) - mean^2 would lose the digits of a row whose mean is far from 0.  AGAIN: rows
// wider than TPR * NCH chunks are read three times.
template <int T, int OUT, int TPR, int NCH, bool AGAIN, bool NARROW>
__global__ __launch_bounds__(TPR > kThreads ? TPR : kThreads) void k_layer_forward(const Forward a) {
    constexpr int kRows = TPR > kThreads ? 1 : kThreads / TPR, kOutGroup = OUT == E4M3_128 ? kBlock : kGroup;
    __shared__ float shared[2][1][TPR > kWave ? TPR / kWave : 1];
    int place = 0;
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
    for (row = (long long)blockIdx.x * kRows + (kRows == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / TPR)); row < a.rows;
         row += (long long)gridDim.x * kRows) {
        float v[NCH][8], total[1] = {0.0f}, square[1] = {0.0f};
        for (int turn = 0; turn < turns; ++turn) {
            load(turn, v);
#pragma unroll
            for (int j = 0; j < NCH; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) total[0] += v[j][i];
        }
        row_sums<TPR>(total, shared, place);
        const float mean = total[0] / (float)a.cols;
        for (int turn = 0; turn < turns; ++turn) {
            if constexpr (AGAIN) load(turn, v);
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                const int n = a.cols - ((turn * NCH + j) * TPR + t) * kChunk;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float off = i < n ? v[j][i] - mean : 0.0f;
                    square[0] = fmaf(off, off, square[0]);
                }
            }
        }
        row_sums<TPR>(square, shared, place);
        const float rstd = inverse_root(square[0] / (float)a.cols + a.eps);
        if (t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        for (int turn = 0; turn < turns; ++turn) {
            if constexpr (AGAIN) load(turn, v);
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                const int col = ((turn * NCH + j) * TPR + t) * kChunk, n = a.cols - col;
                if (a.sum.p) store_chunk<T>(a.sum, row, col, n, v[j], n > 0);
                float g[8], b[8], y[8];
                load_vector_of(a.gain, 1.0f, col, n, g);
                load_vector_of(a.shift, 0.0f, col, n, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = i < n ? fmaf((v[j][i] - mean) * rstd, g[i], b[i]) : 0.0f;
                store_chunk<OUT>(a.y, row, col, n, y, col < whole(a.cols, kOutGroup));
            }
        }
    }
}

// ================================================================================================
// backward
// ================================================================================================
struct Backward {
    int rows, cols;
    Mat dy, sum, dsum, dx;
    const float* gain;
    const float* mean;
    const float* rstd;
    float* partial;      // [gridDim.x][2][cols], or null
};

// The gradients of gain and shift for 64 columns, over all rows, by a whole block of THREADS: eight threads hold the columns' chunks, and every
// THREADS / 8-th row is a thread's.  For few rows, whose dy and s are read once more for it: that costs less than another launch.
constexpr int kStripCols = 64;
template <int T, int S, int THREADS, bool NARROW>
__device__ __forceinline__ void strip_gradients(const Backward& a, float* dgain, float* dshift, int strip) {
    constexpr int kWays = THREADS / 8, kWaves = THREADS / kWave, kSome = 4;
    __shared__ float sums[kWaves][2][kStripCols];
    const int col = strip * kStripCols + threadIdx.x % 8 * kChunk, n = min(max(a.cols - col, 0), kChunk);
    float total[2][8] = {};
#pragma unroll 1
    for (int row0 = threadIdx.x / 8; row0 < a.rows; row0 += kWays * kSome) {
        // (past the last row it is loaded again: a branch would have each load waited for by itself)
        Chunk<T> dy_raw[kSome];
        Chunk<S> s_raw[kSome];
        float rstd[kSome], mean[kSome];
#pragma unroll
        for (int u = 0; u < kSome; ++u) {
            const int row = min(row0 + u * kWays, a.rows - 1);
            fetch_chunk<T, NARROW>(dy_raw[u], a.dy, row, col, a.cols);
            fetch_chunk<S, NARROW>(s_raw[u], a.sum, row, col, a.cols);
            rstd[u] = a.rstd[row];
            mean[u] = a.mean[row];
        }
#pragma unroll
        for (int u = 0; u < kSome; ++u) {
            const int there = row0 + u * kWays < a.rows ? n : 0;
            float dy[8], h[8];
            take_chunk<T, NARROW>(dy_raw[u], there, dy);
            take_chunk<S, NARROW>(s_raw[u], there, h);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // (what is not there has no part in it, whatever lies in the statistics that were read for it)
                total[0][i] = fmaf(dy[i], i < there ? (h[i] - mean[u]) * rstd[u] : 0.0f, total[0][i]);
                total[1][i] += dy[i];
            }
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float v = total[k][i];
            v += __shfl_xor(v, 8);
            v += __shfl_xor(v, 16);
            v += __shfl_xor(v, 32);
            if (threadIdx.x % kWave < 8) sums[threadIdx.x / kWave][k][threadIdx.x % 8 * kChunk + i] = v;
        }
    __syncthreads();
    if (threadIdx.x >= 2 * kStripCols) return;
    const int k = threadIdx.x / kStripCols, c = threadIdx.x % kStripCols, at = strip * kStripCols + c;
    float v = sums[0][k][c];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v += sums[w][k][c];
    float* const out = k == 0 ? dgain : dshift;
    if (out && at < a.cols) out[at] = v;
}

// A few rows: a row at a time and no sums over them, which blocks of their own take at the same time (strip_gradients).  333 x 4100 fp32 9.4 us,
// 6.3 without the strips; with partial sums and a launch that ends them 17.
template <int T, int S, int TPR, int NCH, bool NARROW>
__global__ __launch_bounds__(TPR > kThreads ? TPR : kThreads) void k_layer_backward_few(const Backward a, int strips, float* dgain, float* dshift) {
    constexpr int kBlockThreads = TPR > kThreads ? TPR : kThreads, kRows = kBlockThreads / TPR;
    if ((int)blockIdx.x < strips) {                        // (they take longer than the rows)
        strip_gradients<T, S, kBlockThreads, NARROW>(a, dgain, dshift, (int)blockIdx.x);
        return;
    }
    __shared__ float shared[2][2][TPR > kWave ? TPR / kWave : 1];
    int place = 0;
    const int t = threadIdx.x % TPR, mine = kRows == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    const long long row = (long long)((int)blockIdx.x - strips) * kRows + mine;
    if (row >= a.rows) return;                              // (with several rows a block there is no barrier)
    const bool more = a.dsum.p != nullptr;
    const auto col_of = [&](int j) { return (j * TPR + t) * kChunk; };
    Chunk<T> dy_raw[NCH], dsum_raw[NCH];
    Chunk<S> s_raw[NCH];
    const float rstd = a.rstd[row], mean = a.mean[row];
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        fetch_chunk<T, NARROW>(dy_raw[j], a.dy, row, col_of(j), a.cols);
        fetch_chunk<S, NARROW>(s_raw[j], a.sum, row, col_of(j), a.cols);
        if (more) fetch_chunk<T, NARROW>(dsum_raw[j], a.dsum, row, col_of(j), a.cols);
    }
    float dy[NCH][8], h[NCH][8], along[2] = {0.0f, 0.0f};      // sums of t h and of t
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        const int n = a.cols - col_of(j);
        float g[8];
        load_vector_of(a.gain, 1.0f, col_of(j), n, g);
        take_chunk<T, NARROW>(dy_raw[j], n, dy[j]);
        take_chunk<S, NARROW>(s_raw[j], n, h[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[j][i] = i < n ? (h[j][i] - mean) * rstd : 0.0f;
            dy[j][i] *= g[i];
            along[0] = fmaf(dy[j][i], h[j][i], along[0]);
            along[1] += dy[j][i];
        }
    }
    row_sums<TPR>(along, shared, place);
    const float by = along[0] / (float)a.cols, level = along[1] / (float)a.cols;
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        const int n = a.cols - col_of(j);
        float d[8] = {};
        if (more) take_chunk<T, NARROW>(dsum_raw[j], n, d);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = fmaf(rstd, (dy[j][i] - level) - h[j][i] * by, d[i]);
        store_chunk<T>(a.dx, row, col_of(j), n, d, n > 0);
    }
}

// A block takes rows blockIdx.x, + gridDim.x, ...: the sums of dy h and of dy over its rows stay in registers, two rows of partial
// sums a block are all that both gradients cost in memory.  The next row is under way, as it lies in memory, while one is worked
// on.  AGAIN as in the forward pass (the two gradients are then a kernel of their own, k_layer_gradients).
template <int T, int S, int TPR, int NCH, bool AGAIN, bool NARROW>
__global__ __launch_bounds__(TPR > kThreads ? TPR : kThreads) void k_layer_backward(const Backward a) {
    constexpr int kBlockThreads = TPR > kThreads ? TPR : kThreads, kRows = kBlockThreads / TPR;
    __shared__ float shared[2][2][TPR > kWave ? TPR / kWave : 1];
    int place = 0;
    // (the row is the same for a whole wave: its addresses are scalars)
    const int t = threadIdx.x % TPR, mine = kRows == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    const bool more = a.dsum.p != nullptr;
    const long long step = (long long)gridDim.x * kRows;
    const auto col_of = [&](int turn, int j) { return ((turn * NCH + j) * TPR + t) * kChunk; };
    float by_h[AGAIN ? 1 : NCH][8], by_one[AGAIN ? 1 : NCH][8], gain[AGAIN ? 1 : NCH][8];
    Chunk<T> dy_raw[NCH], dsum_raw[NCH];
    Chunk<S> s_raw[NCH];
    float rstd_raw = 0.0f, mean_raw = 0.0f;
    auto request = [&](long long row, int turn) {
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            fetch_chunk<T, NARROW>(dy_raw[j], a.dy, row, col_of(turn, j), a.cols);
            fetch_chunk<S, NARROW>(s_raw[j], a.sum, row, col_of(turn, j), a.cols);
        }
        rstd_raw = a.rstd[row];
        mean_raw = a.mean[row];
    };
    auto request_dsum = [&](long long row, int turn) {
#pragma unroll
        for (int j = 0; j < NCH; ++j) fetch_chunk<T, NARROW>(dsum_raw[j], a.dsum, row, col_of(turn, j), a.cols);
    };
    // dy and h = (sum - mean) rstd of chunk j, zeros past the row's end
    auto take = [&](int turn, int j, float mean, float rstd, float (&dy)[8], float (&h)[8]) {
        const int n = a.cols - col_of(turn, j);
        take_chunk<T, NARROW>(dy_raw[j], n, dy);
        take_chunk<S, NARROW>(s_raw[j], n, h);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = i < n ? (h[i] - mean) * rstd : 0.0f;
    };
    if constexpr (!AGAIN) {
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            load_vector_of(a.gain, 1.0f, col_of(0, j), a.cols - col_of(0, j), gain[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) by_h[j][i] = by_one[j][i] = 0.0f;
        }
    }
    long long row = (long long)blockIdx.x * kRows + mine;
    if constexpr (!AGAIN) {
        if (row < a.rows) request(row, 0);
    }
    for (; row < a.rows; row += step) {
        float dy[NCH][8], h[NCH][8], along[2] = {0.0f, 0.0f};      // sums of t h and of t
        const int turns = AGAIN ? ceil_div(a.cols, kChunk * TPR * NCH) : 1;
        if constexpr (AGAIN) {
            for (int turn = 0; turn < turns; ++turn) {
                request(row, turn);
#pragma unroll
                for (int j = 0; j < NCH; ++j) {
                    float g[8];
                    take(turn, j, mean_raw, rstd_raw, dy[j], h[j]);
                    load_vector_of(a.gain, 1.0f, col_of(turn, j), a.cols - col_of(turn, j), g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        along[0] = fmaf(dy[j][i] * g[i], h[j][i], along[0]);
                        along[1] = fmaf(dy[j][i], g[i], along[1]);
                    }
                }
            }
        } else {
            if (more) request_dsum(row, 0);
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                take(0, j, mean_raw, rstd_raw, dy[j], h[j]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    by_h[j][i] = fmaf(dy[j][i], h[j][i], by_h[j][i]);
                    by_one[j][i] += dy[j][i];
                    dy[j][i] *= gain[j][i];
                    along[0] = fmaf(dy[j][i], h[j][i], along[0]);
                    along[1] += dy[j][i];
                }
            }
        }
        const float rstd = rstd_raw, mean = mean_raw;
        // (past the last row the last one again: no branch around the loads)
        if constexpr (!AGAIN) request(min(row + step, (long long)a.rows - 1), 0);
        row_sums<TPR>(along, shared, place);
        const float by = along[0] / (float)a.cols, level = along[1] / (float)a.cols;
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
                    take(turn, j, mean, rstd, dy[j], h[j]);
                    load_vector_of(a.gain, 1.0f, col, n, g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) dy[j][i] *= g[i];
                }
                float d[8] = {};
                if (more) take_chunk<T, NARROW>(dsum_raw[j], n, d);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] = fmaf(rstd, (dy[j][i] - level) - h[j][i] * by, d[i]);
                store_chunk<T>(a.dx, row, col, n, d, n > 0);
            }
        }
    }
    if constexpr (!AGAIN) {
        if (!a.partial) return;
        float* out = a.partial + (size_t)blockIdx.x * 2 * a.cols;
        if constexpr (kRows == 1) {
#pragma unroll
            for (int j = 0; j < NCH; ++j)
                if (col_of(0, j) < a.cols) {
                    store_values(out + col_of(0, j), a.cols - col_of(0, j), by_h[j]);
                    store_values(out + a.cols + col_of(0, j), a.cols - col_of(0, j), by_one[j]);
                }
        } else {
            __shared__ float others[kRows - 1][2][NCH * TPR * kChunk];
            if (mine > 0) {
#pragma unroll
                for (int j = 0; j < NCH; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        others[mine - 1][0][col_of(0, j) + i] = by_h[j][i];
                        others[mine - 1][1][col_of(0, j) + i] = by_one[j][i];
                    }
            }
            __syncthreads();
            if (mine == 0) {
#pragma unroll
                for (int j = 0; j < NCH; ++j) {
                    const int col = col_of(0, j);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int r = 0; r < kRows - 1; ++r) {
                            by_h[j][i] += others[r][0][col + i];
                            by_one[j][i] += others[r][1][col + i];
                        }
                    if (col < a.cols) {
                        store_values(out + col, a.cols - col, by_h[j]);
                        store_values(out + a.cols + col, a.cols - col, by_one[j]);
                    }
                }
            }
        }
    }
}

// The two gradients of rows too wide for that: a block walks down a part of the rows of a strip of 64 chunks, four threads a column of
// chunks.
constexpr int kStripChunks = 64, kStripRows = kThreads / kStripChunks;
template <int T, int S>
__global__ __launch_bounds__(kThreads) void k_layer_gradients(const Backward a, int rows_per_block) {
    __shared__ float others[kStripRows - 1][2][kStripChunks * kChunk];
    const int t = threadIdx.x % kStripChunks, mine = threadIdx.x / kStripChunks;
    const int col = (blockIdx.x * kStripChunks + t) * kChunk, n = a.cols - col;
    const int first = blockIdx.y * rows_per_block, end = min(a.rows, first + rows_per_block);
    float total[2][8] = {};
    for (int row = first + mine; row < end; row += kStripRows) {
        Chunk<T> dy_raw;
        Chunk<S> s_raw;
        float dy[8], h[8];
        fetch_chunk<T, false>(dy_raw, a.dy, row, col, a.cols);      // (rows of many columns)
        fetch_chunk<S, false>(s_raw, a.sum, row, col, a.cols);
        const float rstd = a.rstd[row], mean = a.mean[row];
        take_chunk<T, false>(dy_raw, n, dy);
        take_chunk<S, false>(s_raw, n, h);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            total[0][i] = fmaf(dy[i], i < n ? (h[i] - mean) * rstd : 0.0f, total[0][i]);
            total[1][i] += dy[i];
        }
    }
    if (mine > 0) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) others[mine - 1][k][t * kChunk + i] = total[k][i];
    }
    __syncthreads();
    if (mine == 0 && col < a.cols) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int r = 0; r < kStripRows - 1; ++r) total[k][i] += others[r][k][t * kChunk + i];
            store_values(a.partial + ((size_t)blockIdx.y * 2 + k) * a.cols + col, n, total[k]);
        }
    }
}

// Sums over the partial sums: 32 columns a block, 32 threads a column.  No rows: zeros.
__global__ __launch_bounds__(kFinishThreads) void k_layer_finish(const float* partial, int partials, int cols, float* dgain, float* dshift) {
    __shared__ float ways[kFinishWays][kFinishCols];
    const int blocks = ceil_div(cols, kFinishCols), k = blockIdx.x / blocks;
    const int c = threadIdx.x % kFinishCols, way = threadIdx.x / kFinishCols, col = (blockIdx.x % blocks) * kFinishCols + c;
    float* out = k == 0 ? dgain : dshift;
    if (!out) return;
    float v = 0.0f;
    if (col < cols) {
#pragma unroll 8
        for (int p = way; p < partials; p += kFinishWays) v += partial[((size_t)p * 2 + k) * cols + col];
    }
    ways[way][c] = v;
    __syncthreads();
    if (way == 0 && col < cols) {
#pragma unroll
        for (int i = 1; i < kFinishWays; ++i) v += ways[i][c];
        out[col] = v;
    }
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
hipError_t forward(const Forward& a, hipStream_t s) {
    return by_width(a.cols, [&](auto tpr, auto nch, auto again, auto narrow) {
        constexpr int block = tpr() > kThreads ? tpr() : kThreads;
        k_layer_forward<T, OUT, tpr(), nch(), again(), narrow()>
            <<<dim3(std::min(ceil_div(a.rows, block / tpr()), kMostGroups)), block, 0, s>>>(a);
        return hipGetLastError();
    });
}
template <int T>
hipError_t forward_of(const Forward& a, hipStream_t s) {
    return a.y.kind == E4M3 ? forward<T, E4M3>(a, s) : a.y.kind == E4M3_128 ? forward<T, E4M3_128>(a, s) : forward<T, T>(a, s);
}
// 1024 threads have 128 registers each, which do not hold a row's two gradients beside the next row: of such rows the gradients are a
// kernel of their own.  (16384 x 16384 bf16 in one, with 156 registers spilled: 1054 us.)
constexpr int kThreadsWithSums = 512, kColsWithSums = 8192;
// A few rows: the second reading of dy and s, of matrices that lie in the caches, costs less than the launch that ends partial sums (us, this
// way | with partial sums: 256 x 1000 fp32 8 | 11.4, 500 x 8192 bf16 10.2 | 22.5, 1000 x 8192 fp32 30 | 42, 1000 x 4096 19 | 20; but 1000 x 1000 16 | 11).
bool few(int rows, int cols) { return cols <= kHeldCols && rows <= (cols >= 4096 && cols <= kColsWithSums ? 1024 : 512); }

template <int T, int S>
hipError_t backward_few(const Backward& a, float* dgain, float* dshift, hipStream_t s) {
    return by_width(a.cols, [&](auto tpr, auto nch, auto again, auto narrow) {
        if constexpr (!again()) {
            constexpr int block = tpr() > kThreads ? tpr() : kThreads;
            const int rows = ceil_div(a.rows, block / tpr()), strips = dgain || dshift ? ceil_div(a.cols, kStripCols) : 0;
            k_layer_backward_few<T, S, tpr(), nch(), narrow()><<<dim3(strips + rows), block, 0, s>>>(a, strips, dgain, dshift);
        }
        return hipGetLastError();
    });
}
// `rows` rows from `first` on.
Mat rows_of(Mat m, long long first) {
    if (m.p) m.p = (uint8_t*)m.p + first * m.ld * (m.kind == F32 ? 4 : m.kind == BF16 ? 2 : 1);
    if (m.scales) m.scales += first * m.scale_ld;
    return m;
}
Backward rows_of(const Backward& a, int first, int rows) {
    return Backward{rows, a.cols, rows_of(a.dy, first), rows_of(a.sum, first), rows_of(a.dsum, first), rows_of(a.dx, first),
                    a.gain, a.mean + first, a.rstd + first, a.partial};
}
template <int T, int S>
hipError_t backward(const Backward& a, hipStream_t s) {
    return by_width(a.cols, [&](auto tpr, auto nch, auto again, auto narrow) {
        constexpr int block = tpr() > kThreads ? tpr() : kThreads;
        const int parts = layer_norm_partials(a.rows, a.cols);
        if constexpr (again()) {
            k_layer_backward<T, S, tpr(), nch(), true, narrow()><<<dim3(std::min(a.rows, kMostGroups)), block, 0, s>>>(a);
        } else if constexpr (tpr() > kThreadsWithSums) {
            for (int first = 0; first < a.rows; first += kMostGroups) {      // (a workgroup a row)
                const Backward part = rows_of(a, first, std::min(a.rows - first, kMostGroups));
                k_layer_backward_few<T, S, tpr(), nch(), narrow()><<<dim3(part.rows), block, 0, s>>>(part, 0, nullptr, nullptr);
                const hipError_t e = hipGetLastError();
                if (e != hipSuccess) return e;
            }
        } else {
            k_layer_backward<T, S, tpr(), nch(), false, narrow()><<<dim3(parts), block, 0, s>>>(a);
        }
        if (tpr() > kThreadsWithSums && a.partial)
            k_layer_gradients<T, S><<<dim3(ceil_div(a.cols, kStripChunks * kChunk), parts), kThreads, 0, s>>>(a, ceil_div(a.rows, parts));
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_layer_norm_forward(int rows, int cols, const Mat& x, const Mat& branch, const float* gain, const float* shift,
                                     float eps, const Mat& sum, const Mat& y, float* mean, float* rstd, hipStream_t s) {
    if (rows == 0) return hipSuccess;
    const Forward a{rows, cols, x, branch, sum, y, gain, shift, mean, rstd, eps};
    return x.kind == F32 ? forward_of<F32>(a, s) : forward_of<BF16>(a, s);
}

int layer_norm_partials(int rows, int cols) {
    if (rows == 0 || few(rows, cols)) return 0;
    if (cols > kColsWithSums) return std::min(ceil_div(rows, 16), 64);
    return std::min(ceil_div(rows, rows_per_block(cols)), 512);
}

hipError_t launch_layer_norm_backward(int rows, int cols, const Mat& dy, const Mat& sum, const float* gain, const float* mean,
                                      const float* rstd, const Mat& dsum, const Mat& dx, float* dgain, float* dshift,
                                      float* partial, hipStream_t s) {
    if (rows > 0) {
        const Backward a{rows, cols, dy, sum, dsum, dx, gain, mean, rstd, dgain || dshift ? partial : nullptr};
        hipError_t e;
        if (few(rows, cols)) {
            if (dy.kind == F32) return sum.kind == E4M3 ? backward_few<F32, E4M3>(a, dgain, dshift, s) : backward_few<F32, F32>(a, dgain, dshift, s);
            return sum.kind == E4M3 ? backward_few<BF16, E4M3>(a, dgain, dshift, s) : backward_few<BF16, BF16>(a, dgain, dshift, s);
        }
        if (dy.kind == F32) e = sum.kind == E4M3 ? backward<F32, E4M3>(a, s) : backward<F32, F32>(a, s);
        else e = sum.kind == E4M3 ? backward<BF16, E4M3>(a, s) : backward<BF16, BF16>(a, s);
        if (e != hipSuccess) return e;
    }
    if (!dgain && !dshift) return hipSuccess;
    k_layer_finish<<<dim3(2 * ceil_div(cols, kFinishCols)), kFinishThreads, 0, s>>>(partial, layer_norm_partials(rows, cols), cols, dgain, dshift);
    return hipGetLastError();
}

}  // namespace ops
}  // namespace lf
