// Internal interface between the entry points of the residual blocks' operators (operators_api.hip) and their kernels.
// Every launcher only enqueues work on `s` and returns the launch status; arguments have been checked.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace lf {
namespace ops {

enum Kind { F32 = 0, BF16 = 1, E4M3 = 2, E4M3_128 = 3, E4M3_TILES = 4 };      // lf_matrix_type

// A matrix as kernels take it.  p == nullptr: not there.
struct Mat {
    void* p;
    long long ld;
    uint8_t* scales;
    long long scale_ld;
    int kind;
};

enum Act { NONE = 0, SIGMOID = 1, RELU = 2, SILU = 3, GELU = 4 };   // lf_activation

// ---- norm_kernels.hip ----------------------------------------------------------------------------------------------
hipError_t launch_save(int rows, int cols, const Mat& x, const Mat& out, hipStream_t s);
hipError_t launch_load(int rows, int cols, const Mat& in, const Mat& out, hipStream_t s);
hipError_t launch_norm_forward(int rows, int cols, const Mat& x, const Mat& branch, const float* gain, float eps,
                               const Mat& sum, const Mat& y, float* rstd, hipStream_t s);
// partial: [norm_partials(rows, cols)][cols] fp32, needed with dgain
int norm_partials(int rows, int cols);
hipError_t launch_norm_backward(int rows, int cols, const Mat& dy, const Mat& sum, const float* gain, const float* rstd,
                                const Mat& dsum, const Mat& dx, float* dgain, float* partial, hipStream_t s);
// out[c] = sum over p of partial[p][c], p in order of a tree that `partials` alone decides; nothing to do if out is null
struct ColumnSums {
    const float* partial;
    int partials, cols;
    float* out;
};
hipError_t launch_column_finish(const ColumnSums& a, hipStream_t s);
// dz = dy act'(z) into dz (may be absent), and partial sums over its rows for db (may be null; partial: [slope_partials(rows,
// cols)][cols]); what is left to do for db is slope_sums
int slope_partials(int rows, int cols);
ColumnSums slope_sums(int rows, int cols, float* db, float* partial);
hipError_t launch_slope(int rows, int cols, const Mat& dy, const Mat& z, int act, const Mat& dz, float* db, float* partial,
                        hipStream_t s);

// ---- product_kernels.hip -------------------------------------------------------------------------------------------
// What is done with a finished element C[m][n] of a product: bias, z kept, activation, residual, y.
struct Finish {
    const float* bias;      // [N] or null
    int act;
    Mat residual, z, y;     // y is always there
};
// C[m][n] = sum_q P(m,q) Q(n,q), m < M, n < N, q < K.  An operand is contiguous along q (element (i,q) at p[i*ld + q]) or, if
// *_along_own, along its own index (p[q*ld + i]).  raw: fp32 scratch for partial sums, product_scratch_bytes(...) of it.
struct Product {
    Mat P, Q;
    bool P_along_own, Q_along_own;
    int M, N, K;
    Finish f;
    float* raw;
};
size_t product_scratch_bytes(int M, int N, int K, bool bf16);
hipError_t launch_product(const Product& g, hipStream_t s);
// The two products of a backward pass, each with scratch of its own, and what is left to do for db.
hipError_t launch_backward(const Product& dx, const Product& dw, const ColumnSums& db, hipStream_t s);

// ---- layer_norm_kernels.hip ------------------------------------------------------------------------------------------
hipError_t launch_layer_norm_forward(int rows, int cols, const Mat& x, const Mat& branch, const float* gain, const float* shift,
                                     float eps, const Mat& sum, const Mat& y, float* mean, float* rstd, hipStream_t s);
// partial: [layer_norm_partials(rows, cols)][2][cols] fp32, needed with dgain or dshift
int layer_norm_partials(int rows, int cols);
hipError_t launch_layer_norm_backward(int rows, int cols, const Mat& dy, const Mat& sum, const float* gain, const float* mean,
                                      const float* rstd, const Mat& dsum, const Mat& dx, float* dgain, float* dshift,
                                      float* partial, hipStream_t s);

// ---- block_kernels.hip ---------------------------------------------------------------------------------------------
// d = x act'(z), or x (z absent), into 8 bits with blocks of 128 as it lies (out) and transposed (out_t), either may be absent; and
// sums over each 128 of its rows into partial ([block_partials(rows)][cols], may be null)
struct BlockSave {
    int rows, cols, act;
    Mat x, z, out, out_t;
    float* partial;
};
int block_partials(int rows);
hipError_t launch_block_save(const BlockSave& a, hipStream_t s);
hipError_t launch_block_load(int rows, int cols, const Mat& in, const Mat& out, hipStream_t s);

// ---- block_product_kernels.hip -----------------------------------------------------------------------------------------
// C[m][n] = sum_q P(m,q) Q(n,q), both contiguous along q in 8 bits with blocks of 128; P may be dense for the products of a few rows
// (block_product_takes_dense).  raw: fp32 scratch, block_product_scratch_bytes(...) of it.
struct BlockProduct {
    Mat P, Q;
    int M, N, K;
    Finish f;
    float* raw;
};
size_t block_product_scratch_bytes(int M, int N, int K);
bool block_product_takes_dense(int M, int N, int K, const Mat& y, const Mat& z);
hipError_t launch_block_product(const BlockProduct& g, hipStream_t s);
// The two products of a backward pass, each with scratch of its own.
hipError_t launch_block_backward(const BlockProduct& dx, const BlockProduct& dw, const ColumnSums& db, hipStream_t s);

// ---- distil_kernels.hip --------------------------------------------------------------------------------------------
constexpr int kMostTop = 1024;
struct Distil {
    int rows, classes, top;
    Mat logits, top_logits, dlogits;
    const int* top_classes;
    long long top_classes_ld;
    float temperature;
    const float* weight;
    float* loss;
};
hipError_t launch_distil(const Distil& a, hipStream_t s);

}  // namespace ops
}  // namespace lf
