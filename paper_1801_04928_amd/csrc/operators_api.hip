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
long long groups_of(int cols) { return ((long long)cols + 31) / 32; }

lf_status check_size(const char* call, const char* what, int n, int least, int most) {
    if (n < least) return fail(LF_EINVAL, "%s: %s = %d, at least %d are needed", call, what, n, least);
    if (n > most) return fail(LF_EUNSUPPORTED, "%s: %s = %d, at most %d are supported", call, what, n, most);
    return LF_OK;
}

// Bits of the types an argument may have.
enum { kF32 = 1 << LF_MATRIX_F32, kBF16 = 1 << LF_MATRIX_BF16, kE4M3 = 1 << LF_MATRIX_E4M3 };

lf_status take(const char* call, const char* what, const lf_matrix* m, int rows, int cols, int types, Mat* out) {
    *out = Mat{nullptr, 0, nullptr, 0, 0};
    if (!m) return fail(LF_EINVAL, "%s: %s is NULL", call, what);
    const int type = (int)m->type;
    if (type < LF_MATRIX_F32 || type > LF_MATRIX_E4M3 || !(types >> type & 1))
        return fail(LF_EINVAL, "%s: type %d of %s is not one this call takes there", call, type, what);
    const int bytes = type == LF_MATRIX_F32 ? 4 : type == LF_MATRIX_BF16 ? 2 : 1;
    const long long least = type == LF_MATRIX_E4M3 ? groups_of(cols) * 32 : cols;
    if (m->ld < least) return fail(LF_EINVAL, "%s: ld = %lld of %s, rows have %lld elements", call, m->ld, what, least);
    if (m->ld > kMostRowBytes / bytes)
        return fail(LF_EUNSUPPORTED, "%s: ld = %lld of %s, a row is at most %lld bytes", call, m->ld, what, kMostRowBytes);
    if (!m->data && rows > 0) return fail(LF_EINVAL, "%s: data of %s is NULL", call, what);
    if (!aligned(m->data, type == LF_MATRIX_E4M3 ? 16 : (size_t)bytes))
        return fail(LF_EINVAL, "%s: data of %s is misaligned", call, what);
    if (type == LF_MATRIX_E4M3) {
        if (m->ld % 32 != 0) return fail(LF_EINVAL, "%s: ld = %lld of %s, 8 bits need a multiple of 32", call, m->ld, what);
        if (!m->scales && rows > 0) return fail(LF_EINVAL, "%s: scales of %s are NULL", call, what);
        if (m->scale_ld < groups_of(cols) || m->scale_ld > kMostRowBytes)
            return fail(LF_EINVAL, "%s: scale_ld = %lld of %s, rows have %lld scales", call, m->scale_ld, what, groups_of(cols));
    }
    *out = Mat{m->data, m->ld, type == LF_MATRIX_E4M3 ? m->scales : nullptr,
               type == LF_MATRIX_E4M3 ? m->scale_ld : 0, type};
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

}  // extern "C"
