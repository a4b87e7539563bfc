// C ABI of the residual blocks' operators (see include/lf_operators.h): argument checks, workspace layout, and the order of the
// kernels.  Nothing here allocates, waits or throws.
#include "../../include/lf_operators.h"
#include "operators_internal.h"

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

using lf::ops::Mat;

namespace {

constexpr size_t kAlign = 256;
constexpr int kMostRows = 1 << 28;                // grids stay below 2^32 threads
constexpr long long kMostRowBytes = 8 << 20;      // offsets inside a tile stay below 2^32 bytes
constexpr int kMostCols = (int)(kMostRowBytes / 4);

thread_local char g_error[256] = "no error";

lf_status fail(lf_status st, const char* format, ...) {
    va_list args;
    va_start(args, format);
    vsnprintf(g_error, sizeof(g_error), format, args);
    va_end(args);
    return st;
}
lf_status done(const char* call, hipError_t e) {
    return e == hipSuccess ? LF_OK : fail(LF_EHIP, "%s: %s", call, hipGetErrorString(e));
}

size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
bool is_eight(int type) { return type >= LF_MATRIX_E4M3; }
bool in_blocks(int type) { return type == LF_MATRIX_E4M3_128 || type == LF_MATRIX_E4M3_TILES; }
// Groups of a row in 8 bits of this type, and bytes that a row of their scales has in memory.
long long groups_of(int type, int cols) { return in_blocks(type) ? ((long long)cols + 127) / 128 : ((long long)cols + 31) / 32; }
long long scale_bytes(int type, int cols) {
    const long long groups = groups_of(type, cols);
    return in_blocks(type) ? (groups + 3) / 4 * 4 : groups;
}

lf_status check_size(const char* call, const char* what, int n, int least, int most) {
    if (n < least) return fail(LF_EINVAL, "%s: %s = %d, at least %d are needed", call, what, n, least);
    if (n > most) return fail(LF_EUNSUPPORTED, "%s: %s = %d, at most %d are supported", call, what, n, most);
    return LF_OK;
}

// Bits of the types an argument may have.
enum { kF32 = 1 << LF_MATRIX_F32, kBF16 = 1 << LF_MATRIX_BF16, kE4M3 = 1 << LF_MATRIX_E4M3, kE4M3_128 = 1 << LF_MATRIX_E4M3_128,
       kTiles = 1 << LF_MATRIX_E4M3_TILES };

lf_status take(const char* call, const char* what, const lf_matrix* m, int rows, int cols, int types, Mat* out) {
    *out = Mat{nullptr, 0, nullptr, 0, 0};
    if (!m) return fail(LF_EINVAL, "%s: %s is NULL", call, what);
    const int type = (int)m->type;
    if (type < LF_MATRIX_F32 || type > LF_MATRIX_E4M3_TILES || !(types >> type & 1))
        return fail(LF_EINVAL, "%s: type %d of %s is not one this call takes there", call, type, what);
    const int bytes = type == LF_MATRIX_F32 ? 4 : type == LF_MATRIX_BF16 ? 2 : 1, group = in_blocks(type) ? 128 : 32;
    const long long least = is_eight(type) ? groups_of(type, cols) * group : cols;
    if (m->ld < least) return fail(LF_EINVAL, "%s: ld = %lld of %s, rows have %lld elements", call, m->ld, what, least);
    if (m->ld > kMostRowBytes / bytes)
        return fail(LF_EUNSUPPORTED, "%s: ld = %lld of %s, a row is at most %lld bytes", call, m->ld, what, kMostRowBytes);
    if (!m->data && rows > 0) return fail(LF_EINVAL, "%s: data of %s is NULL", call, what);
    if (!aligned(m->data, is_eight(type) ? 16 : (size_t)bytes)) return fail(LF_EINVAL, "%s: data of %s is misaligned", call, what);
    if (is_eight(type)) {
        if (m->ld % group != 0) return fail(LF_EINVAL, "%s: ld = %lld of %s, its 8 bits need a multiple of %d", call, m->ld, what, group);
        if (!m->scales && rows > 0) return fail(LF_EINVAL, "%s: scales of %s are NULL", call, what);
        if (m->scale_ld < scale_bytes(type, cols) || m->scale_ld > kMostRowBytes)
            return fail(LF_EINVAL, "%s: scale_ld = %lld of %s, rows have %lld scales", call, m->scale_ld, what, scale_bytes(type, cols));
        if (in_blocks(type) && (m->scale_ld % 4 != 0 || !aligned(m->scales, 4)))
            return fail(LF_EINVAL, "%s: scales of %s are misaligned (scale_ld = %lld), blocks of 128 need multiples of 4", call, what, m->scale_ld);
    }
    *out = Mat{m->data, m->ld, is_eight(type) ? m->scales : nullptr, is_eight(type) ? m->scale_ld : 0, type};
    return LF_OK;
}
// The same for one that may be absent.
lf_status take_optional(const char* call, const char* what, const lf_matrix* m, int rows, int cols, int types, Mat* out) {
    if (m) return take(call, what, m, rows, cols, types, out);
    *out = Mat{nullptr, 0, nullptr, 0, 0};
    return LF_OK;
}
lf_status check_vector(const char* call, const char* what, const float* p, bool needed) {
    if (!p) return needed ? fail(LF_EINVAL, "%s: %s is NULL", call, what) : LF_OK;
    return aligned(p, 4) ? LF_OK : fail(LF_EINVAL, "%s: %s is misaligned", call, what);
}
lf_status check_workspace(const char* call, const void* p, size_t bytes, size_t needed) {
    if (needed == 0) return LF_OK;
    if (!p || !aligned(p, kAlign)) return fail(LF_EINVAL, "%s: workspace is NULL or not 256-byte aligned", call);
    if (bytes < needed) return fail(LF_EINVAL, "%s: workspace of %zu bytes, %zu are needed", call, bytes, needed);
    return LF_OK;
}

#define LF_TRY(expr)                        \
    do {                                    \
        const lf_status st_ = (expr);       \
        if (st_ != LF_OK) return st_;       \
    } while (0)

int storage(const Mat& m) { return 1 << m.kind; }
const Mat kAbsent{nullptr, 0, nullptr, 0, 0};

// Scratch of a product's backward pass: dz, and the partial sums of db and of the products.
struct Backward {
    long long dz_ld;
    size_t dz_off, db_off, raw_x_off, raw_w_off, total;
};
Backward backward_layout(int rows, int outputs, int inputs, bool bf16) {
    Backward w;
    w.dz_ld = ((long long)outputs + 7) / 8 * 8;      // whole vectors, whatever dy's rows are
    w.dz_off = 0;
    w.db_off = w.dz_off + align_up((size_t)rows * w.dz_ld * (bf16 ? 2 : 4));
    w.raw_x_off = w.db_off + align_up((size_t)lf::ops::slope_partials(rows, outputs) * outputs * sizeof(float));
    w.raw_w_off = w.raw_x_off + align_up(lf::ops::product_scratch_bytes(rows, inputs, outputs, bf16));
    w.total = w.raw_w_off + align_up(lf::ops::product_scratch_bytes(outputs, inputs, rows, bf16));
    return w;
}
// Scratch of a product of operands with blocks of 128: x in 8 bits, and partial sums.
struct BlockForward {
    long long x_ld, x_scale_ld;
    size_t x_off, x_scales_off, raw_off, total;
};
long long block_ld(int cols) { return groups_of(LF_MATRIX_E4M3_128, cols) * 128; }
BlockForward block_forward_layout(int rows, int outputs, int inputs) {
    BlockForward w;
    w.x_ld = block_ld(inputs);
    w.x_scale_ld = scale_bytes(LF_MATRIX_E4M3_128, inputs);
    w.x_off = 0;
    w.x_scales_off = w.x_off + align_up((size_t)rows * w.x_ld);
    w.raw_off = w.x_scales_off + align_up((size_t)rows * w.x_scale_ld);
    w.total = w.raw_off + align_up(lf::ops::block_product_scratch_bytes(rows, outputs, inputs));
    return w;
}
// Scratch of its backward pass: dz in 8 bits both ways, and the partial sums of db and of the products.
struct BlockBackward {
    long long dz_ld, dz_scale_ld, dz_t_ld, dz_t_scale_ld;
    size_t dz_off, dz_scales_off, dz_t_off, dz_t_scales_off, db_off, raw_x_off, raw_w_off, total;
};
BlockBackward block_backward_layout(int rows, int outputs, int inputs) {
    BlockBackward w;
    w.dz_ld = block_ld(outputs);
    w.dz_scale_ld = scale_bytes(LF_MATRIX_E4M3_128, outputs);
    w.dz_t_ld = block_ld(rows);
    w.dz_t_scale_ld = scale_bytes(LF_MATRIX_E4M3_128, rows);
    w.dz_off = 0;
    w.dz_scales_off = w.dz_off + align_up((size_t)rows * w.dz_ld);
    w.dz_t_off = w.dz_scales_off + align_up((size_t)rows * w.dz_scale_ld);
    w.dz_t_scales_off = w.dz_t_off + align_up((size_t)outputs * w.dz_t_ld);
    w.db_off = w.dz_t_scales_off + align_up((size_t)outputs * w.dz_t_scale_ld);
    w.raw_x_off = w.db_off + align_up((size_t)lf::ops::block_partials(rows) * outputs * sizeof(float));
    w.raw_w_off = w.raw_x_off + align_up(lf::ops::block_product_scratch_bytes(rows, inputs, outputs));
    w.total = w.raw_w_off + align_up(lf::ops::block_product_scratch_bytes(outputs, inputs, rows));
    return w;
}
// Rows of a product with blocks of 128: they lie along a row of the transposed matrices.
constexpr int kMostBlockRows = (int)kMostRowBytes;
bool block_sizes(int rows, int outputs, int inputs) {
    return rows >= 0 && rows <= kMostBlockRows && outputs >= 1 && outputs <= kMostCols && inputs >= 1 && inputs <= kMostCols;
}
bool product_sizes(int rows, int outputs, int inputs, lf_dtype dt) {
    return rows >= 0 && rows <= kMostRows && outputs >= 1 && outputs <= kMostCols && inputs >= 1 && inputs <= kMostCols &&
           (dt == LF_F32 || dt == LF_BF16);
}

}  // namespace

extern "C" {

const char* lf_operator_error(void) { return g_error; }

lf_status lf_checkpoint_save(int rows, int cols, const lf_matrix* x, const lf_matrix* out, void* hip_stream) {
    const char* call = "lf_checkpoint_save";
    Mat from, to;
    LF_TRY(check_size(call, "rows", rows, 0, kMostRows));
    LF_TRY(check_size(call, "cols", cols, 1, kMostCols));
    LF_TRY(take(call, "x", x, rows, cols, kF32 | kBF16, &from));
    LF_TRY(take(call, "out", out, rows, cols, kE4M3, &to));
    return done(call, lf::ops::launch_save(rows, cols, from, to, (hipStream_t)hip_stream));
}

lf_status lf_checkpoint_load(int rows, int cols, const lf_matrix* in, const lf_matrix* out, void* hip_stream) {
    const char* call = "lf_checkpoint_load";
    Mat from, to;
    LF_TRY(check_size(call, "rows", rows, 0, kMostRows));
    LF_TRY(check_size(call, "cols", cols, 1, kMostCols));
    LF_TRY(take(call, "in", in, rows, cols, kE4M3, &from));
    LF_TRY(take(call, "out", out, rows, cols, kF32 | kBF16, &to));
    return done(call, lf::ops::launch_load(rows, cols, from, to, (hipStream_t)hip_stream));
}

lf_status lf_norm_forward(int rows, int cols, const lf_matrix* x, const lf_matrix* branch, const float* gain, float eps,
                          const lf_matrix* sum, const lf_matrix* y, float* rstd, void* hip_stream) {
    const char* call = "lf_norm_forward";
    Mat mx, mb, ms, my;
    LF_TRY(check_size(call, "rows", rows, 0, kMostRows));
    LF_TRY(check_size(call, "cols", cols, 1, kMostCols));
    if (!(eps >= 0.0f) || std::isinf(eps)) return fail(LF_EINVAL, "%s: eps = %g is not finite and >= 0", call, (double)eps);
    LF_TRY(take(call, "x", x, rows, cols, kF32 | kBF16, &mx));
    LF_TRY(take_optional(call, "branch", branch, rows, cols, storage(mx), &mb));
    LF_TRY(check_vector(call, "gain", gain, false));
    LF_TRY(take_optional(call, "sum", sum, rows, cols, storage(mx), &ms));
    LF_TRY(take(call, "y", y, rows, cols, storage(mx) | kE4M3, &my));
    LF_TRY(check_vector(call, "rstd", rstd, false));
    return done(call, lf::ops::launch_norm_forward(rows, cols, mx, mb, gain, eps, ms, my, rstd, (hipStream_t)hip_stream));
}

size_t lf_norm_workspace_bytes(int rows, int cols) {
    if (rows < 0 || rows > kMostRows || cols < 1 || cols > kMostCols) return 0;
    return align_up((size_t)lf::ops::norm_partials(rows, cols) * cols * sizeof(float));
}

lf_status lf_norm_backward(int rows, int cols, const lf_matrix* dy, const lf_matrix* sum, const float* gain,
                           const float* rstd, const lf_matrix* dsum, const lf_matrix* dx, float* dgain,
                           void* workspace, size_t workspace_bytes, void* hip_stream) {
    const char* call = "lf_norm_backward";
    Mat mdy, ms, mds, mdx;
    LF_TRY(check_size(call, "rows", rows, 0, kMostRows));
    LF_TRY(check_size(call, "cols", cols, 1, kMostCols));
    LF_TRY(take(call, "dy", dy, rows, cols, kF32 | kBF16, &mdy));
    LF_TRY(take(call, "sum", sum, rows, cols, storage(mdy) | kE4M3, &ms));
    LF_TRY(check_vector(call, "gain", gain, false));
    LF_TRY(check_vector(call, "rstd", rstd, rows > 0));
    LF_TRY(take_optional(call, "dsum", dsum, rows, cols, storage(mdy), &mds));
    LF_TRY(take(call, "dx", dx, rows, cols, storage(mdy), &mdx));
    LF_TRY(check_vector(call, "dgain", dgain, false));
    LF_TRY(check_workspace(call, workspace, workspace_bytes, dgain ? lf_norm_workspace_bytes(rows, cols) : 0));
    return done(call, lf::ops::launch_norm_backward(rows, cols, mdy, ms, gain, rstd, mds, mdx, dgain, (float*)workspace,
                                                    (hipStream_t)hip_stream));
}

size_t lf_linear_workspace_bytes(int rows, int outputs, int inputs, lf_dtype dt) {
    if (!product_sizes(rows, outputs, inputs, dt)) return 0;
    return align_up(lf::ops::product_scratch_bytes(rows, outputs, inputs, dt == LF_BF16));
}

lf_status lf_linear_forward(int rows, int outputs, int inputs, const lf_matrix* x, const lf_matrix* w, const float* bias,
                            lf_activation act, const lf_matrix* residual, const lf_matrix* y, const lf_matrix* z,
                            void* workspace, size_t workspace_bytes, void* hip_stream) {
    const char* call = "lf_linear_forward";
    Mat mx, mw, mr, my, mz;
    LF_TRY(check_size(call, "rows", rows, 0, kMostRows));
    LF_TRY(check_size(call, "outputs", outputs, 1, kMostCols));
    LF_TRY(check_size(call, "inputs", inputs, 1, kMostCols));
    if ((int)act < LF_ACT_NONE || (int)act > LF_ACT_GELU) return fail(LF_EINVAL, "%s: activation %d", call, (int)act);
    LF_TRY(take(call, "w", w, outputs, inputs, kF32 | kBF16, &mw));
    LF_TRY(take(call, "x", x, rows, inputs, storage(mw) | kE4M3, &mx));
    LF_TRY(check_vector(call, "bias", bias, false));
    LF_TRY(take_optional(call, "residual", residual, rows, outputs, storage(mw), &mr));
    LF_TRY(take(call, "y", y, rows, outputs, storage(mw) | kE4M3, &my));
    LF_TRY(take_optional(call, "z", z, rows, outputs, storage(mw) | kE4M3, &mz));
    const lf_dtype dt = mw.kind == LF_MATRIX_BF16 ? LF_BF16 : LF_F32;
    LF_TRY(check_workspace(call, workspace, workspace_bytes, lf_linear_workspace_bytes(rows, outputs, inputs, dt)));
    if (rows == 0) return LF_OK;
    const lf::ops::Product g{mx, mw, false, false, rows, outputs, inputs, {bias, (int)act, mr, mz, my}, (float*)workspace};
    return done(call, lf::ops::launch_product(g, (hipStream_t)hip_stream));
}

size_t lf_linear_backward_workspace_bytes(int rows, int outputs, int inputs, lf_dtype dt) {
    if (!product_sizes(rows, outputs, inputs, dt)) return 0;
    return backward_layout(rows, outputs, inputs, dt == LF_BF16).total;
}

lf_status lf_linear_backward(int rows, int outputs, int inputs, const lf_matrix* dy, const lf_matrix* z,
                             lf_activation act, const lf_matrix* x, const lf_matrix* w, const lf_matrix* dx,
                             const lf_matrix* dw, float* db, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const char* call = "lf_linear_backward";
    Mat mdy, mz, mx, mw, mdx, mdw;
    LF_TRY(check_size(call, "rows", rows, 0, kMostRows));
    LF_TRY(check_size(call, "outputs", outputs, 1, kMostCols));
    LF_TRY(check_size(call, "inputs", inputs, 1, kMostCols));
    if ((int)act < LF_ACT_NONE || (int)act > LF_ACT_GELU) return fail(LF_EINVAL, "%s: activation %d", call, (int)act);
    LF_TRY(take(call, "dy", dy, rows, outputs, kF32 | kBF16, &mdy));
    const int same = storage(mdy);
    LF_TRY(act == LF_ACT_NONE ? take_optional(call, "z", nullptr, rows, outputs, same, &mz)
                              : take(call, "z", z, rows, outputs, same | kE4M3, &mz));
    LF_TRY(take_optional(call, "dx", dx, rows, inputs, same, &mdx));
    LF_TRY(take_optional(call, "dw", dw, outputs, inputs, same | kF32, &mdw));
    LF_TRY(check_vector(call, "db", db, false));
    // (an operand whose product is not asked for is not looked at)
    LF_TRY(dw ? take(call, "x", x, rows, inputs, same | kE4M3, &mx) : take_optional(call, "x", nullptr, 0, 1, same, &mx));
    LF_TRY(dx ? take(call, "w", w, outputs, inputs, same, &mw) : take_optional(call, "w", nullptr, 0, 1, same, &mw));
    const bool bf16 = mdy.kind == LF_MATRIX_BF16;
    const Backward at = backward_layout(rows, outputs, inputs, bf16);
    LF_TRY(check_workspace(call, workspace, workspace_bytes, at.total));
    const hipStream_t s = (hipStream_t)hip_stream;
    uint8_t* const scratch = (uint8_t*)workspace;

    // The gradient before the activation: made once, both products read it.  Of bf16 operands it is rounded to bf16, one rounding more
    // than the outputs': the matrix instructions take both operands in one type, and fp32 ones run at a tenth of the rate.
    const bool products = mdx.p || mdw.p;
    Mat dz = mdy;
    if (act != LF_ACT_NONE && products) dz = Mat{scratch + at.dz_off, at.dz_ld, nullptr, 0, mdy.kind};
    const Mat made = act != LF_ACT_NONE && products ? dz : Mat{nullptr, 0, nullptr, 0, 0};
    if (made.p || db)
        LF_TRY(done(call, lf::ops::launch_slope(rows, outputs, mdy, mz, (int)act, made, db, (float*)(scratch + at.db_off), s)));
    const Mat none{nullptr, 0, nullptr, 0, 0};
    float* const raw_x = (float*)(scratch + at.raw_x_off);
    float* const raw_w = (float*)(scratch + at.raw_w_off);
    const lf::ops::Product gx{dz, mw, false, true, rows, inputs, outputs, {nullptr, LF_ACT_NONE, none, none, mdx}, raw_x};
    const lf::ops::Product gw{dz, mx, true, true, outputs, inputs, rows, {nullptr, LF_ACT_NONE, none, none, mdw}, raw_w};
    const lf::ops::ColumnSums sums = lf::ops::slope_sums(rows, outputs, db, (float*)(scratch + at.db_off));
    if (mdx.p && mdw.p && rows > 0) return done(call, lf::ops::launch_backward(gx, gw, sums, s));
    LF_TRY(done(call, lf::ops::launch_column_finish(sums, s)));
    if (mdx.p && rows > 0) return done(call, lf::ops::launch_product(gx, s));
    if (mdw.p) return done(call, lf::ops::launch_product(gw, s));
    return LF_OK;
}

lf_status lf_layer_norm_forward(int rows, int cols, const lf_matrix* x, const lf_matrix* branch, const float* gain,
                                const float* shift, float eps, const lf_matrix* sum, const lf_matrix* y, float* mean,
                                float* rstd, void* hip_stream) {
    const char* call = "lf_layer_norm_forward";
    Mat mx, mb, ms, my;
    LF_TRY(check_size(call, "rows", rows, 0, kMostRows));
    LF_TRY(check_size(call, "cols", cols, 1, kMostCols));
    if (!(eps >= 0.0f) || std::isinf(eps)) return fail(LF_EINVAL, "%s: eps = %g is not finite and >= 0", call, (double)eps);
    LF_TRY(take(call, "x", x, rows, cols, kF32 | kBF16, &mx));
    LF_TRY(take_optional(call, "branch", branch, rows, cols, storage(mx), &mb));
    LF_TRY(check_vector(call, "gain", gain, false));
    LF_TRY(check_vector(call, "shift", shift, false));
    LF_TRY(take_optional(call, "sum", sum, rows, cols, storage(mx), &ms));
    LF_TRY(take(call, "y", y, rows, cols, storage(mx) | kE4M3 | kE4M3_128, &my));
    LF_TRY(check_vector(call, "mean", mean, false));
    LF_TRY(check_vector(call, "rstd", rstd, false));
    return done(call, lf::ops::launch_layer_norm_forward(rows, cols, mx, mb, gain, shift, eps, ms, my, mean, rstd, (hipStream_t)hip_stream));
}

size_t lf_layer_norm_workspace_bytes(int rows, int cols) {
    if (rows < 0 || rows > kMostRows || cols < 1 || cols > kMostCols) return 0;
    return align_up((size_t)lf::ops::layer_norm_partials(rows, cols) * 2 * cols * sizeof(float));
}

lf_status lf_layer_norm_backward(int rows, int cols, const lf_matrix* dy, const lf_matrix* sum, const float* gain,
                                 const float* mean, const float* rstd, const lf_matrix* dsum, const lf_matrix* dx,
                                 float* dgain, float* dshift, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const char* call = "lf_layer_norm_backward";
    Mat mdy, ms, mds, mdx;
    LF_TRY(check_size(call, "rows", rows, 0, kMostRows));
    LF_TRY(check_size(call, "cols", cols, 1, kMostCols));
    LF_TRY(take(call, "dy", dy, rows, cols, kF32 | kBF16, &mdy));
    LF_TRY(take(call, "sum", sum, rows, cols, storage(mdy) | kE4M3, &ms));
    LF_TRY(check_vector(call, "gain", gain, false));
    LF_TRY(check_vector(call, "mean", mean, rows > 0));
    LF_TRY(check_vector(call, "rstd", rstd, rows > 0));
    LF_TRY(take_optional(call, "dsum", dsum, rows, cols, storage(mdy), &mds));
    LF_TRY(take(call, "dx", dx, rows, cols, storage(mdy), &mdx));
    LF_TRY(check_vector(call, "dgain", dgain, false));
    LF_TRY(check_vector(call, "dshift", dshift, false));
    LF_TRY(check_workspace(call, workspace, workspace_bytes, dgain || dshift ? lf_layer_norm_workspace_bytes(rows, cols) : 0));
    return done(call, lf::ops::launch_layer_norm_backward(rows, cols, mdy, ms, gain, mean, rstd, mds, mdx, dgain, dshift,
                                                          (float*)workspace, (hipStream_t)hip_stream));
}

lf_status lf_block_save(int rows, int cols, const lf_matrix* x, const lf_matrix* out, const lf_matrix* out_t, void* hip_stream) {
    const char* call = "lf_block_save";
    Mat from, to, to_t;
    LF_TRY(check_size(call, "rows", rows, 0, kMostBlockRows));
    LF_TRY(check_size(call, "cols", cols, 1, kMostCols));
    LF_TRY(take(call, "x", x, rows, cols, kF32 | kBF16, &from));
    if (!out && !out_t) return fail(LF_EINVAL, "%s: out and out_t are NULL", call);
    LF_TRY(take_optional(call, "out", out, rows, cols, kE4M3_128 | kTiles, &to));
    // (a matrix of rows without elements is nothing to write)
    LF_TRY(take_optional(call, "out_t", out_t, rows > 0 ? cols : 0, rows, out ? storage(to) : kE4M3_128 | kTiles, &to_t));
    return done(call, lf::ops::launch_block_save(lf::ops::BlockSave{rows, cols, LF_ACT_NONE, from, kAbsent, to, to_t, nullptr},
                                                 (hipStream_t)hip_stream));
}

lf_status lf_block_load(int rows, int cols, const lf_matrix* in, const lf_matrix* out, void* hip_stream) {
    const char* call = "lf_block_load";
    Mat from, to;
    LF_TRY(check_size(call, "rows", rows, 0, kMostRows));
    LF_TRY(check_size(call, "cols", cols, 1, kMostCols));
    LF_TRY(take(call, "in", in, rows, cols, kE4M3_128 | kTiles, &from));
    LF_TRY(take(call, "out", out, rows, cols, kF32 | kBF16, &to));
    return done(call, lf::ops::launch_block_load(rows, cols, from, to, (hipStream_t)hip_stream));
}

size_t lf_block_linear_workspace_bytes(int rows, int outputs, int inputs) {
    return block_sizes(rows, outputs, inputs) ? block_forward_layout(rows, outputs, inputs).total : 0;
}

lf_status lf_block_linear_forward(int rows, int outputs, int inputs, const lf_matrix* x, const lf_matrix* w, const float* bias,
                                  lf_activation act, const lf_matrix* residual, const lf_matrix* y, const lf_matrix* z,
                                  const lf_matrix* x_t, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const char* call = "lf_block_linear_forward";
    Mat mx, mw, mr, my, mz, mxt;
    LF_TRY(check_size(call, "rows", rows, 0, kMostBlockRows));
    LF_TRY(check_size(call, "outputs", outputs, 1, kMostCols));
    LF_TRY(check_size(call, "inputs", inputs, 1, kMostCols));
    if ((int)act < LF_ACT_NONE || (int)act > LF_ACT_GELU) return fail(LF_EINVAL, "%s: activation %d", call, (int)act);
    LF_TRY(take(call, "x", x, rows, inputs, kF32 | kBF16 | kE4M3_128, &mx));
    // the storage type of all that is not in 8 bits: x's, or the first's that has one
    const bool dense = !is_eight(mx.kind);
    int same = dense ? storage(mx) : kF32 | kBF16;
    LF_TRY(take(call, "w", w, outputs, inputs, kTiles | kE4M3_128, &mw));
    LF_TRY(check_vector(call, "bias", bias, false));
    LF_TRY(take(call, "y", y, rows, outputs, same | kE4M3_128, &my));
    if (!is_eight(my.kind)) same = storage(my);
    LF_TRY(take_optional(call, "residual", residual, rows, outputs, same, &mr));
    if (mr.p) same = storage(mr);
    LF_TRY(take_optional(call, "z", z, rows, outputs, same | kE4M3_128, &mz));
    if (x_t && !dense) return fail(LF_EINVAL, "%s: x_t is made of x in fp32 or bf16", call);
    LF_TRY(take_optional(call, "x_t", x_t, rows > 0 ? inputs : 0, rows, kE4M3_128, &mxt));
    const BlockForward at = block_forward_layout(rows, outputs, inputs);
    LF_TRY(check_workspace(call, workspace, workspace_bytes, at.total));
    if (rows == 0) return LF_OK;
    const hipStream_t s = (hipStream_t)hip_stream;
    uint8_t* const scratch = (uint8_t*)workspace;
    Mat p = mx;
    // (the products of a few rows take x as it is, and keep it in 8 bits in registers)
    const bool made = dense && !lf::ops::block_product_takes_dense(rows, outputs, inputs, my, mz);
    if (made) p = Mat{scratch + at.x_off, at.x_ld, scratch + at.x_scales_off, at.x_scale_ld, LF_MATRIX_E4M3_128};
    if (made || mxt.p)
        LF_TRY(done(call, lf::ops::launch_block_save(lf::ops::BlockSave{rows, inputs, LF_ACT_NONE, mx, kAbsent, made ? p : kAbsent, mxt, nullptr}, s)));
    const lf::ops::BlockProduct g{p, mw, rows, outputs, inputs, {bias, (int)act, mr, mz, my}, (float*)(scratch + at.raw_off)};
    return done(call, lf::ops::launch_block_product(g, s));
}

size_t lf_block_linear_backward_workspace_bytes(int rows, int outputs, int inputs) {
    return block_sizes(rows, outputs, inputs) ? block_backward_layout(rows, outputs, inputs).total : 0;
}

lf_status lf_block_linear_backward(int rows, int outputs, int inputs, const lf_matrix* dy, const lf_matrix* z,
                                   lf_activation act, const lf_matrix* x_t, const lf_matrix* w_t, const lf_matrix* dx,
                                   const lf_matrix* dw, float* db, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const char* call = "lf_block_linear_backward";
    Mat mdy, mz, mx, mw, mdx, mdw;
    LF_TRY(check_size(call, "rows", rows, 0, kMostBlockRows));
    LF_TRY(check_size(call, "outputs", outputs, 1, kMostCols));
    LF_TRY(check_size(call, "inputs", inputs, 1, kMostCols));
    if ((int)act < LF_ACT_NONE || (int)act > LF_ACT_GELU) return fail(LF_EINVAL, "%s: activation %d", call, (int)act);
    LF_TRY(take(call, "dy", dy, rows, outputs, kF32 | kBF16, &mdy));
    const int same = storage(mdy);
    LF_TRY(act == LF_ACT_NONE ? take_optional(call, "z", nullptr, rows, outputs, same, &mz)
                              : take(call, "z", z, rows, outputs, same | kE4M3_128, &mz));
    LF_TRY(take_optional(call, "dx", dx, rows, inputs, same, &mdx));
    LF_TRY(take_optional(call, "dw", dw, outputs, inputs, same | kF32, &mdw));
    LF_TRY(check_vector(call, "db", db, false));
    // (an operand whose product is not asked for is not looked at)
    LF_TRY(take_optional(call, "x_t", nullptr, 0, 1, same, &mx));
    LF_TRY(take_optional(call, "w_t", nullptr, 0, 1, same, &mw));
    if (dw) LF_TRY(take(call, "x_t", x_t, rows > 0 ? inputs : 0, rows, kE4M3_128, &mx));
    if (dx) LF_TRY(take(call, "w_t", w_t, inputs, outputs, kTiles | kE4M3_128, &mw));
    const BlockBackward at = block_backward_layout(rows, outputs, inputs);
    LF_TRY(check_workspace(call, workspace, workspace_bytes, at.total));
    const hipStream_t s = (hipStream_t)hip_stream;
    uint8_t* const scratch = (uint8_t*)workspace;
    const Mat dz{scratch + at.dz_off, at.dz_ld, scratch + at.dz_scales_off, at.dz_scale_ld, LF_MATRIX_E4M3_128};
    const Mat dz_t{scratch + at.dz_t_off, at.dz_t_ld, scratch + at.dz_t_scales_off, at.dz_t_scale_ld, LF_MATRIX_E4M3_128};
    float* const partial = (float*)(scratch + at.db_off);
    const int parts = lf::ops::block_partials(rows);
    const lf::ops::BlockSave save{rows, outputs, (int)act, mdy, mz, mdx.p ? dz : kAbsent, mdw.p ? dz_t : kAbsent,
                                  !db ? nullptr : parts == 1 ? db : partial};
    if (save.out.p || save.out_t.p || db) LF_TRY(done(call, lf::ops::launch_block_save(save, s)));
    const lf::ops::ColumnSums sums{partial, parts, outputs, parts == 1 ? nullptr : db};
    const lf::ops::BlockProduct gx{dz, mw, rows, inputs, outputs, {nullptr, LF_ACT_NONE, kAbsent, kAbsent, mdx}, (float*)(scratch + at.raw_x_off)};
    const lf::ops::BlockProduct gw{dz_t, mx, outputs, inputs, rows, {nullptr, LF_ACT_NONE, kAbsent, kAbsent, mdw}, (float*)(scratch + at.raw_w_off)};
    return done(call, lf::ops::launch_block_backward(gx, gw, sums, s));
}

lf_status lf_distil(int rows, int classes, int top, const lf_matrix* logits, const lf_matrix* top_logits,
                    const int* top_classes, long long top_classes_ld, float temperature, const float* weight, float* loss,
                    const lf_matrix* dlogits, void* hip_stream) {
    const char* call = "lf_distil";
    lf::ops::Distil a{};
    LF_TRY(check_size(call, "rows", rows, 0, kMostRows));
    LF_TRY(check_size(call, "classes", classes, 1, kMostCols));
    LF_TRY(check_size(call, "top", top, 1, lf::ops::kMostTop));
    LF_TRY(take(call, "logits", logits, rows, classes, kF32 | kBF16, &a.logits));
    LF_TRY(take(call, "top_logits", top_logits, rows, top, kF32 | kBF16, &a.top_logits));
    if (!top_classes && rows > 0) return fail(LF_EINVAL, "%s: top_classes is NULL", call);
    if (!aligned(top_classes, 4)) return fail(LF_EINVAL, "%s: top_classes is misaligned", call);
    if (top_classes_ld < top) return fail(LF_EINVAL, "%s: top_classes_ld = %lld, rows have %d entries", call, top_classes_ld, top);
    if (top_classes_ld > kMostCols) return fail(LF_EUNSUPPORTED, "%s: top_classes_ld = %lld, at most %d is supported", call, top_classes_ld, kMostCols);
    if (!(temperature >= 0x1p-20f && temperature <= 0x1p20f))
        return fail(LF_EINVAL, "%s: temperature = %g is not between 2^-20 and 2^20", call, (double)temperature);
    LF_TRY(check_vector(call, "weight", weight, false));
    LF_TRY(check_vector(call, "loss", loss, false));
    LF_TRY(take_optional(call, "dlogits", dlogits, rows, classes, storage(a.logits), &a.dlogits));
    if (!loss && !dlogits) return fail(LF_EINVAL, "%s: loss and dlogits are NULL", call);
    a.rows = rows; a.classes = classes; a.top = top;
    a.top_classes = top_classes; a.top_classes_ld = top_classes_ld;
    a.temperature = temperature; a.weight = weight; a.loss = loss;
    return done(call, lf::ops::launch_distil(a, (hipStream_t)hip_stream));
}

}  // extern "C"
