// vp_fp8_api.cpp -- host side of the 8-bit operators declared in include/vp.h:
// argument checks, then one launcher each.  No function throws: messages are
// formatted into a buffer of their own, and nothing here allocates.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <cstring>

#include "vp.h"
#include "vp_fp8.h"

namespace {

using vp::Fp8View;

__attribute__((format(printf, 2, 3)))
int32_t fail(int32_t status, const char* format, ...) {
    char text[256];
    va_list ap;
    va_start(ap, format);
    std::vsnprintf(text, sizeof text, format, ap);
    va_end(ap);
    return vp::set_error(status, text);
}

int32_t done(int err, const char* what) {
    if (err != 0)
        return fail(VP_ERR_HIP, "%s: %s", what, hipGetErrorString(static_cast<hipError_t>(err)));
    vp::set_error(VP_OK, "");
    return VP_OK;
}

bool misaligned(const void* p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

bool dims_ok(int64_t v) { return v >= 0 && v <= VP_MAX_DIM; }

// The conversions that work on tiles of 128 x 128 number them in 32 bits.
int32_t check_tiles(int64_t rows, int64_t cols) {
    if ((rows + 127) / 128 * ((cols + 127) / 128) > int64_t(UINT32_MAX))
        return fail(VP_ERR_DIMS, "a matrix of more than 2^32 tiles of 128 x 128");
    return VP_OK;
}

int32_t check_dtype(int32_t dtype) {
    if (dtype != VP_OUT_F32 && dtype != VP_OUT_BF16)
        return fail(VP_ERR_ARG, "the element type must be VP_OUT_F32 or VP_OUT_BF16");
    return VP_OK;
}

// A dense matrix argument: `optional` ones may be NULL; one without elements
// is never read.
int32_t check_dense(const void* p, const char* name, int32_t dtype, int64_t rows, int64_t cols,
                    int64_t ld, bool optional = false) {
    if (p == nullptr) {
        if (optional || rows == 0 || cols == 0) return VP_OK;
        return fail(VP_ERR_NULL, "%s is NULL", name);
    }
    const int64_t size = dtype == VP_OUT_BF16 ? 2 : 4;
    if (misaligned(p, size)) return fail(VP_ERR_ARG, "%s must be aligned to its element", name);
    if (ld < cols)
        return fail(VP_ERR_ARG, "%s: rows of %lld elements are %lld apart", name,
                    static_cast<long long>(cols), static_cast<long long>(ld));
    if (ld > INT64_MAX / 8 / (rows > 0 ? rows : 1))
        return fail(VP_ERR_ARG, "%s: rows too far apart", name);
    return VP_OK;
}

// A vp_fp8 argument into `v`; rows, cols < 0: any size.
int32_t check_fp8(const vp_fp8* f, const char* name, int64_t rows, int64_t cols, Fp8View* v) {
    if (f == nullptr) return fail(VP_ERR_NULL, "%s is NULL", name);
    if (f->block != 1 && f->block != 128)
        return fail(VP_ERR_ARG, "%s: block must be 1 or 128", name);
    if (f->reserved != 0) return fail(VP_ERR_ARG, "%s: reserved must be 0", name);
    if (!dims_ok(f->rows) || !dims_ok(f->cols))
        return fail(VP_ERR_DIMS, "%s: rows and cols must lie in [0, VP_MAX_DIM]", name);
    if ((rows >= 0 && f->rows != rows) || (cols >= 0 && f->cols != cols))
        return fail(VP_ERR_DIMS, "%s is [%lld][%lld], and [%lld][%lld] is needed", name,
                    static_cast<long long>(f->rows), static_cast<long long>(f->cols),
                    static_cast<long long>(rows >= 0 ? rows : f->rows),
                    static_cast<long long>(cols >= 0 ? cols : f->cols));
    if (f->rows > 0 && f->cols > 0) {
        if (f->q == nullptr || f->scale == nullptr)
            return fail(VP_ERR_NULL, "%s: q or scale is NULL", name);
        if (misaligned(f->q, 16)) return fail(VP_ERR_ARG, "%s: q must be 16-byte aligned", name);
        if (misaligned(f->scale, 4))
            return fail(VP_ERR_ARG, "%s: scale must be 4-byte aligned", name);
    }
    v->q = static_cast<uint8_t*>(f->q);
    v->scale = f->scale;
    v->rows = static_cast<int32_t>(f->rows);
    v->cols = static_cast<int32_t>(f->cols);
    v->block = f->block;
    v->ld = vp::q_ld(f->cols);
    v->sld = vp::scale_ld(f->cols);
    return VP_OK;
}

int32_t check_workspace(const void* p, int64_t have, int64_t need) {
    if (need == 0) return VP_OK;
    if (p == nullptr) return fail(VP_ERR_NULL, "workspace is NULL");
    if (misaligned(p, 16)) return fail(VP_ERR_ARG, "workspace must be 16-byte aligned");
    if (have < need)
        return fail(VP_ERR_CAPACITY, "workspace holds %lld of %lld bytes",
                    static_cast<long long>(have), static_cast<long long>(need));
    return VP_OK;
}

}  // namespace

#define VP_TRY(call)                     \
    do {                                 \
        const int32_t st_ = (call);      \
        if (st_ != VP_OK) return st_;    \
    } while (0)

extern "C" {

int32_t vp_fp8_layout(int64_t rows, int64_t cols, int32_t block, int64_t* q_bytes,
                      int64_t* scale_bytes) {
    if (block != 1 && block != 128) return fail(VP_ERR_ARG, "block must be 1 or 128");
    if (!dims_ok(rows) || !dims_ok(cols))
        return fail(VP_ERR_DIMS, "rows and cols must lie in [0, VP_MAX_DIM]");
    if (q_bytes != nullptr) *q_bytes = rows * vp::q_ld(cols);
    if (scale_bytes != nullptr) *scale_bytes = (rows + block - 1) / block * vp::scale_ld(cols);
    vp::set_error(VP_OK, "");
    return VP_OK;
}

int32_t vp_fp8_quantize(const void* x, int32_t x_dtype, int64_t rows, int64_t cols, int64_t ld,
                        const vp_fp8* by_rows, const vp_fp8* by_cols, hipStream_t stream) {
    if (by_rows == nullptr && by_cols == nullptr)
        return fail(VP_ERR_NULL, "by_rows and by_cols are both NULL");
    VP_TRY(check_dtype(x_dtype));
    if (!dims_ok(rows) || !dims_ok(cols))
        return fail(VP_ERR_DIMS, "rows and cols must lie in [0, VP_MAX_DIM]");
    VP_TRY(check_dense(x, "x", x_dtype, rows, cols, ld));
    vp::QuantizeArgs a{};
    a.x = x;
    a.type = x_dtype == VP_OUT_BF16 ? vp::In::bf16 : vp::In::f32;
    a.ld = ld;
    a.rows = static_cast<int32_t>(rows);
    a.cols = static_cast<int32_t>(cols);
    if (by_rows != nullptr) VP_TRY(check_fp8(by_rows, "by_rows", rows, cols, &a.by_rows));
    if (by_cols != nullptr) VP_TRY(check_fp8(by_cols, "by_cols", cols, rows, &a.by_cols));
    if (by_rows != nullptr && by_cols != nullptr && by_rows->block != by_cols->block)
        return fail(VP_ERR_ARG, "by_rows and by_cols must have one block");
    if (by_cols != nullptr || by_rows->block != 1) VP_TRY(check_tiles(rows, cols));
    if (rows == 0 || cols == 0) return done(0, "");
    return done(vp::launch_quantize(a, stream), "quantize launch");
}

int32_t vp_fp8_transpose(const vp_fp8* in, const vp_fp8* out, hipStream_t stream) {
    vp::QuantizeArgs a{};
    VP_TRY(check_fp8(in, "in", -1, -1, &a.in));
    VP_TRY(check_fp8(out, "out", in->cols, in->rows, &a.by_cols));
    if (in->block != out->block) return fail(VP_ERR_ARG, "in and out must have one block");
    VP_TRY(check_tiles(in->rows, in->cols));
    a.type = vp::In::fp8;
    a.rows = a.in.rows;
    a.cols = a.in.cols;
    if (a.rows == 0 || a.cols == 0) return done(0, "");
    return done(vp::launch_quantize(a, stream), "transpose launch");
}

int32_t vp_fp8_dequantize(const vp_fp8* in, void* out, int32_t out_dtype, int64_t ld,
                          hipStream_t stream) {
    Fp8View v{};
    VP_TRY(check_dtype(out_dtype));
    VP_TRY(check_fp8(in, "in", -1, -1, &v));
    VP_TRY(check_dense(out, "out", out_dtype, in->rows, in->cols, ld));
    if (v.rows == 0 || v.cols == 0) return done(0, "");
    return done(vp::launch_dequantize(v, out, out_dtype == VP_OUT_BF16, ld, stream),
                "dequantize launch");
}

int32_t vp_fp8_matmul_workspace(int64_t m, int64_t n, int64_t k, int32_t out_dtype,
                                int64_t* workspace_bytes) {
    if (workspace_bytes == nullptr) return fail(VP_ERR_NULL, "workspace_bytes is NULL");
    VP_TRY(check_dtype(out_dtype));
    if (!dims_ok(m) || !dims_ok(n) || !dims_ok(k))
        return fail(VP_ERR_DIMS, "m, n and k must lie in [0, VP_MAX_DIM]");
    if (k > VP_MAX_SUM) return fail(VP_ERR_DIMS, "k must be at most VP_MAX_SUM");
    const int64_t need = vp::matmul_workspace(m, n, k, out_dtype == VP_OUT_BF16);
    if (need < 0) return fail(VP_ERR_DIMS, "a result of more tiles than a launch takes");
    *workspace_bytes = need;
    vp::set_error(VP_OK, "");
    return VP_OK;
}

int32_t vp_fp8_matmul(const vp_fp8* a, const vp_fp8* b, void* out, int32_t out_dtype, int64_t ld,
                      void* workspace, int64_t workspace_bytes, hipStream_t stream) {
    vp::MatmulArgs m{};
    VP_TRY(check_dtype(out_dtype));
    VP_TRY(check_fp8(a, "a", -1, -1, &m.a));
    VP_TRY(check_fp8(b, "b", -1, a->cols, &m.b));
    if (a->cols > VP_MAX_SUM)
        return fail(VP_ERR_DIMS, "a sum of %lld products, at most %lld", static_cast<long long>(a->cols),
                    static_cast<long long>(VP_MAX_SUM));
    m.bf16 = out_dtype == VP_OUT_BF16;
    const int64_t need = vp::matmul_workspace(a->rows, b->rows, a->cols, m.bf16);
    if (need < 0) return fail(VP_ERR_DIMS, "a result of more tiles than a launch takes");
    VP_TRY(check_dense(out, "out", out_dtype, a->rows, b->rows, ld));
    m.out = out;
    m.ld = ld;
    m.partial = static_cast<float*>(workspace);
    VP_TRY(check_workspace(workspace, workspace_bytes, need));
    if (a->rows == 0 || b->rows == 0) return done(0, "");
    return done(vp::launch_matmul(m, stream), "matmul launch");
}

int32_t vp_fp8_matmul_kernels(int64_t m, int64_t n, int64_t k, int32_t out_dtype, int64_t ld, int32_t* launches,
                              int32_t capacity, int32_t* n_launches) {
    if (n_launches == nullptr) return fail(VP_ERR_NULL, "n_launches is NULL");
    if (capacity < 0 || (launches == nullptr && capacity > 0))
        return fail(VP_ERR_ARG, "launches must hold capacity rows of 4 int32");
    int64_t need;
    VP_TRY(vp_fp8_matmul_workspace(m, n, k, out_dtype, &need));
    if (ld < n)
        return fail(VP_ERR_ARG, "rows of %lld elements are %lld apart", static_cast<long long>(n),
                    static_cast<long long>(ld));
    int32_t rows[2][4];
    const int count = vp::describe_matmul(m, n, k, ld, out_dtype == VP_OUT_BF16, rows);
    for (int i = 0; i < count && i < capacity; ++i) std::memcpy(launches + 4 * i, rows[i], sizeof rows[i]);
    *n_launches = count;
    return VP_OK;
}

int32_t vp_rms_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr,
                    const void* weight, int32_t dtype, int64_t rows, int64_t cols, float eps,
                    void* h, int64_t ldh, void* out, int64_t ldo, const vp_fp8* out8, float* rstd,
                    hipStream_t stream) {
    vp::NormArgs a{};
    VP_TRY(check_dtype(dtype));
    if (out == nullptr && out8 == nullptr) return fail(VP_ERR_NULL, "out and out8 are both NULL");
    if (!dims_ok(rows) || !dims_ok(cols) || cols < 1)
        return fail(VP_ERR_DIMS, "rows must lie in [0, VP_MAX_DIM], cols in [1, VP_MAX_DIM]");
    if (!(eps >= 0.0f) || !std::isfinite(eps))
        return fail(VP_ERR_ARG, "eps must be finite and not negative");
    VP_TRY(check_dense(x, "x", dtype, rows, cols, ldx));
    VP_TRY(check_dense(residual, "residual", dtype, rows, cols, ldr, true));
    VP_TRY(check_dense(weight, "weight", dtype, 1, cols, cols));
    VP_TRY(check_dense(h, "h", dtype, rows, cols, ldh, true));
    VP_TRY(check_dense(out, "out", dtype, rows, cols, ldo, true));
    if (out8 != nullptr) {
        VP_TRY(check_fp8(out8, "out8", rows, cols, &a.out8));
        if (out8->block != 1) return fail(VP_ERR_ARG, "out8: block must be 1");
    }
    if (misaligned(rstd, 4)) return fail(VP_ERR_ARG, "rstd must be 4-byte aligned");
    a.x = x;
    a.residual = residual;
    a.weight = weight;
    a.h = h;
    a.out = out;
    a.rstd = rstd;
    a.ldx = ldx;
    a.ldr = ldr;
    a.ldh = ldh;
    a.ldo = ldo;
    a.rows = static_cast<int32_t>(rows);
    a.cols = static_cast<int32_t>(cols);
    a.eps = eps;
    if (rows == 0) return done(0, "");
    return done(vp::launch_norm(a, dtype == VP_OUT_BF16, stream), "norm launch");
}

int32_t vp_rms_norm_backward_workspace(int64_t rows, int64_t cols, int64_t* workspace_bytes) {
    if (workspace_bytes == nullptr) return fail(VP_ERR_NULL, "workspace_bytes is NULL");
    if (!dims_ok(rows) || !dims_ok(cols) || cols < 1)
        return fail(VP_ERR_DIMS, "rows must lie in [0, VP_MAX_DIM], cols in [1, VP_MAX_DIM]");
    *workspace_bytes = int64_t(vp::norm_backward_groups(rows, cols)) * cols * 4;
    vp::set_error(VP_OK, "");
    return VP_OK;
}

int32_t vp_rms_norm_backward(const void* dy, int64_t ldy, const void* h, int64_t ldh,
                             const void* weight, const float* rstd, const void* dh, int64_t lddh,
                             int32_t dtype, int64_t rows, int64_t cols, void* dx, int64_t lddx,
                             float* dweight, void* workspace, int64_t workspace_bytes,
                             hipStream_t stream) {
    vp::NormBackwardArgs a{};
    VP_TRY(check_dtype(dtype));
    if (!dims_ok(rows) || !dims_ok(cols) || cols < 1)
        return fail(VP_ERR_DIMS, "rows must lie in [0, VP_MAX_DIM], cols in [1, VP_MAX_DIM]");
    VP_TRY(check_dense(dy, "dy", dtype, rows, cols, ldy));
    VP_TRY(check_dense(h, "h", dtype, rows, cols, ldh));
    VP_TRY(check_dense(weight, "weight", dtype, 1, cols, cols));
    VP_TRY(check_dense(rstd, "rstd", VP_OUT_F32, rows, 1, 1));
    VP_TRY(check_dense(dh, "dh", dtype, rows, cols, lddh, true));
    VP_TRY(check_dense(dx, "dx", dtype, rows, cols, lddx));
    if (misaligned(dweight, 4)) return fail(VP_ERR_ARG, "dweight must be 4-byte aligned");
    if (dweight != nullptr)
        VP_TRY(check_workspace(workspace, workspace_bytes,
                               int64_t(vp::norm_backward_groups(rows, cols)) * cols * 4));
    a.dy = dy;
    a.h = h;
    a.weight = weight;
    a.dh = dh;
    a.rstd = rstd;
    a.dx = dx;
    a.dweight = dweight;
    a.partial = dweight != nullptr ? static_cast<float*>(workspace) : nullptr;
    a.ldy = ldy;
    a.ldh = ldh;
    a.lddh = lddh;
    a.lddx = lddx;
    a.rows = static_cast<int32_t>(rows);
    a.cols = static_cast<int32_t>(cols);
    if (rows == 0 && dweight == nullptr) return done(0, "");
    return done(vp::launch_norm_backward(a, dtype == VP_OUT_BF16, stream), "norm backward launch");
}

}  // extern "C"
