// libqamw device entry points of served layers (8-bit products, routed experts): argument validation on the host, then dispatch.
#include "qamw.h"
#include "qamw_product.hpp"

namespace {

bool misaligned(const void *q, size_t a) { return (reinterpret_cast<uintptr_t>(q) & (a - 1)) != 0; }
bool float_dtype(int t) { return t == QAMW_DTYPE_F32 || t == QAMW_DTYPE_BF16; }
size_t round16(size_t n) { return (n + 15) & ~(size_t)15; }
int status_of(hipError_t e) { return e == hipSuccess ? QAMW_OK : e == hipErrorNotSupported ? QAMW_ERR_UNSUPPORTED : QAMW_ERR_DEVICE; }

// The element type's own alignment: the kernels load and store whole elements.
bool off_type(const void *q, int dtype) { return misaligned(q, dtype == QAMW_DTYPE_F32 ? 4 : dtype == QAMW_DTYPE_BF16 ? 2 : 1); }

}  // namespace

extern "C" {

int qamw_int8_quantize(const void *X, int dtype, int m, int d, int64_t ldx, const float *col_scale, int8_t *codes, int64_t ldc,
                       float *scales, void *stream) {
    if (m < 0 || m > QAMW_INT8_MAX_ROWS || d < 1 || !float_dtype(dtype)) return QAMW_ERR_INVALID_ARG;
    if (m > 0 && (!X || !codes || !scales)) return QAMW_ERR_INVALID_ARG;
    if (off_type(X, dtype) || misaligned(scales, 4) || misaligned(col_scale, 4)) return QAMW_ERR_INVALID_ARG;
    if (ldx < d || ldc < d) return QAMW_ERR_SHAPE;
    return status_of(qamw::launch_int8_quantize(X, dtype, m, d, ldx, col_scale, codes, ldc, scales, (hipStream_t)stream));
}

// In the workspace: the codes, rows of whole 16 bytes, their scales, then what the product needs.
static size_t codes_bytes(int x_dtype, int m, int d_in) {
    return x_dtype == QAMW_DTYPE_I8 ? 0 : (size_t)m * round16((size_t)d_in) + round16((size_t)m * 4);
}

int qamw_int8_matmul_workspace_bytes(int x_dtype, int m, int d_out, int d_in, int gated, size_t *bytes_out) {
    if (!bytes_out || m < 0 || m > QAMW_INT8_MAX_ROWS || d_in < 1 || d_in > QAMW_INT8_MAX_D_IN || d_out < 1 ||
        d_out > QAMW_PRODUCT_MAX_D_OUT || gated < 0 || gated > 1)
        return QAMW_ERR_INVALID_ARG;
    if (!float_dtype(x_dtype) && x_dtype != QAMW_DTYPE_I8) return QAMW_ERR_INVALID_ARG;
    *bytes_out = codes_bytes(x_dtype, m, d_in) + qamw::product_scratch_bytes(m, d_out, d_in, gated != 0);
    return QAMW_OK;
}

int qamw_int8_matmul(const void *X, int x_dtype, const float *x_scales, const float *col_scale, int m, int64_t ldx, const int8_t *W,
                     const float *w_scales, int64_t ldw, int d_out, int d_in, int gated, void *Y, int y_dtype, int64_t ldy,
                     void *workspace, size_t workspace_bytes, void *stream) {
    size_t need = 0;
    const int rc = qamw_int8_matmul_workspace_bytes(x_dtype, m, d_out, d_in, gated, &need);
    if (rc != QAMW_OK) return rc;
    if (!float_dtype(y_dtype)) return QAMW_ERR_INVALID_ARG;
    const bool codes = x_dtype == QAMW_DTYPE_I8;
    if (m > 0 && (!X || !W || !w_scales || !Y || (codes && !x_scales))) return QAMW_ERR_INVALID_ARG;
    if (codes ? col_scale != nullptr : x_scales != nullptr) return QAMW_ERR_INVALID_ARG;
    if (off_type(X, x_dtype) || off_type(Y, y_dtype) || misaligned(x_scales, 4) || misaligned(w_scales, 4) || misaligned(col_scale, 4))
        return QAMW_ERR_INVALID_ARG;
    if (ldx < d_in || ldw < d_in || ldy < d_out) return QAMW_ERR_SHAPE;
    if (m == 0) return QAMW_OK;
    qamw::Product p;
    p.W = W;
    p.ldw = ldw;
    p.w_scales = w_scales;
    p.Y = Y;
    p.ldy = ldy;
    p.m = p.x_rows = m;
    p.d_out = d_out;
    p.d_in = d_in;
    p.i8 = true;
    p.gated = gated != 0;
    p.y_bf16 = y_dtype == QAMW_DTYPE_BF16;
    p.stream = (hipStream_t)stream;
    p.ldx = codes ? ldx : (int64_t)round16((size_t)d_in);
    if (!codes && qamw::product_wide_supported(p) && qamw::product_from_floats_supported(p, X, x_dtype, ldx, col_scale))
        return status_of(qamw::launch_product_from_floats(p, X, x_dtype, ldx, col_scale));
    if (need && (!workspace || workspace_bytes < need || misaligned(workspace, 16))) return QAMW_ERR_INVALID_ARG;
    const size_t before = codes_bytes(x_dtype, m, d_in);
    if (need > before) p.scratch = static_cast<char *>(workspace) + before;
    if (codes) {
        p.X = X;
        p.x_scales = x_scales;
    } else {
        float *scales = reinterpret_cast<float *>(static_cast<char *>(workspace) + (size_t)m * (size_t)p.ldx);
        p.X = workspace;
        p.x_scales = scales;
        const hipError_t e = qamw::launch_int8_quantize(X, x_dtype, m, d_in, ldx, col_scale, static_cast<int8_t *>(workspace), p.ldx,
                                                        scales, (hipStream_t)stream);
        if (e != hipSuccess) return status_of(e);
    }
    return status_of(qamw::launch_product(p));
}

int qamw_grouped_matmul(const void *X, int dtype, const float *x_scales, int x_rows, int64_t ldx, const int32_t *rows, const void *W,
                        const float *w_scales, int64_t ldw, int64_t expert_stride, const int32_t *offsets, int n_experts, int m,
                        int d_out, int d_in, int gated, void *Y, int y_dtype, int64_t ldy, void *stream) {
    if (dtype != QAMW_DTYPE_BF16 && dtype != QAMW_DTYPE_I8) return QAMW_ERR_INVALID_ARG;
    if (m < 0 || m > QAMW_INT8_MAX_ROWS || x_rows < 0 || x_rows > QAMW_INT8_MAX_ROWS || n_experts < 1 ||
        n_experts > QAMW_MAX_EXPERTS || d_in < 1 || d_in > QAMW_INT8_MAX_D_IN || d_out < 1 || d_out > QAMW_PRODUCT_MAX_D_OUT ||
        !float_dtype(y_dtype) || gated < 0 || gated > 1)
        return QAMW_ERR_INVALID_ARG;
    const bool codes = dtype == QAMW_DTYPE_I8;
    if (m > 0 && (!X || !W || !offsets || !Y || (codes && (!x_scales || !w_scales)))) return QAMW_ERR_INVALID_ARG;
    if (!codes && (x_scales || w_scales)) return QAMW_ERR_INVALID_ARG;
    if (off_type(X, dtype) || off_type(W, dtype) || off_type(Y, y_dtype) || misaligned(x_scales, 4) || misaligned(w_scales, 4) ||
        misaligned(rows, 4) || misaligned(offsets, 4))
        return QAMW_ERR_INVALID_ARG;
    if (ldx < d_in || ldw < d_in || ldy < d_out || expert_stride < 0) return QAMW_ERR_SHAPE;
    if (m > 0 && (rows ? x_rows < 1 : x_rows < m)) return QAMW_ERR_SHAPE;
    qamw::Product p;
    p.X = X;
    p.ldx = ldx;
    p.x_scales = x_scales;
    p.rows = rows;
    p.x_rows = x_rows;
    p.W = W;
    p.ldw = ldw;
    p.expert_stride = expert_stride;
    p.w_scales = w_scales;
    p.offsets = offsets;
    p.n_experts = n_experts;
    p.Y = Y;
    p.ldy = ldy;
    p.m = m;
    p.d_out = d_out;
    p.d_in = d_in;
    p.i8 = codes;
    p.gated = gated != 0;
    p.y_bf16 = y_dtype == QAMW_DTYPE_BF16;
    p.stream = (hipStream_t)stream;
    return status_of(qamw::launch_product(p));
}

int qamw_product_plan(int dtype, int m, int n_experts, int d_out, int d_in, int gated, int plan_out[3]) {
    if (!plan_out || m < 1 || m > QAMW_INT8_MAX_ROWS || n_experts < 0 || n_experts > QAMW_MAX_EXPERTS || d_in < 1 ||
        d_in > QAMW_INT8_MAX_D_IN || d_out < 1 || d_out > QAMW_PRODUCT_MAX_D_OUT || gated < 0 || gated > 1)
        return QAMW_ERR_INVALID_ARG;
    if (dtype != QAMW_DTYPE_I8 && (dtype != QAMW_DTYPE_BF16 || n_experts == 0)) return QAMW_ERR_INVALID_ARG;
    int plan[3];
    qamw::product_plan(m, n_experts, n_experts > 0, d_out, d_in, gated != 0, dtype == QAMW_DTYPE_I8, n_experts == 0, plan);
    for (int i = 0; i < 3; ++i) plan_out[i] = plan[i];
    return QAMW_OK;
}

static int route_check(int m, int n_experts, int k) {
    if (m < 0 || m > QAMW_INT8_MAX_ROWS || n_experts < 1 || n_experts > QAMW_MAX_EXPERTS || k < 1 || k > QAMW_MAX_CHOICES || k > n_experts)
        return QAMW_ERR_INVALID_ARG;
    return QAMW_OK;
}

int qamw_route_workspace_bytes(int m, int n_experts, int k, size_t *bytes_out) {
    if (!bytes_out) return QAMW_ERR_INVALID_ARG;
    const int rc = route_check(m, n_experts, k);
    if (rc == QAMW_OK) *bytes_out = qamw::route_workspace_bytes(m, n_experts, k);
    return rc;
}

int qamw_route(const void *logits, int dtype, int m, int n_experts, int64_t ld, int k, int renormalise, int32_t *experts,
               float *weights, int32_t *offsets, int32_t *rows, int32_t *positions, void *workspace, size_t workspace_bytes,
               void *stream) {
    size_t need = 0;
    const int rc = qamw_route_workspace_bytes(m, n_experts, k, &need);
    if (rc != QAMW_OK) return rc;
    if (!float_dtype(dtype) || renormalise < 0 || renormalise > 1 || !offsets) return QAMW_ERR_INVALID_ARG;
    if (m > 0 && (!logits || !experts || !weights || !rows || !positions)) return QAMW_ERR_INVALID_ARG;
    if (workspace_bytes < need || (need && (!workspace || misaligned(workspace, 16)))) return QAMW_ERR_INVALID_ARG;
    if (off_type(logits, dtype) || misaligned(experts, 4) || misaligned(weights, 4) || misaligned(offsets, 4) || misaligned(rows, 4) ||
        misaligned(positions, 4))
        return QAMW_ERR_INVALID_ARG;
    if (ld < n_experts) return QAMW_ERR_SHAPE;
    qamw::RouteProblem q;
    q.logits = logits;
    q.dtype = dtype;
    q.m = m;
    q.n_experts = n_experts;
    q.k = k;
    q.ld = ld;
    q.renormalise = renormalise != 0;
    q.experts = experts;
    q.weights = weights;
    q.offsets = offsets;
    q.rows = rows;
    q.positions = positions;
    q.counts = static_cast<uint8_t *>(workspace);
    q.stream = (hipStream_t)stream;
    return status_of(qamw::launch_route(q));
}

int qamw_combine(const void *Y, int dtype, int y_rows, int64_t ldy, const int32_t *positions, const float *weights, int m, int k, int d,
                 void *out, int out_dtype, int64_t ldo, void *stream) {
    if (m < 0 || m > QAMW_INT8_MAX_ROWS || y_rows < 0 || k < 1 || k > QAMW_MAX_CHOICES || d < 1 || !float_dtype(dtype) ||
        !float_dtype(out_dtype))
        return QAMW_ERR_INVALID_ARG;
    if (m > 0 && ((!Y && y_rows > 0) || !positions || !weights || !out)) return QAMW_ERR_INVALID_ARG;
    if (off_type(Y, dtype) || off_type(out, out_dtype) || misaligned(positions, 4) || misaligned(weights, 4)) return QAMW_ERR_INVALID_ARG;
    if (ldy < d || ldo < d) return QAMW_ERR_SHAPE;
    return status_of(qamw::launch_combine(Y, dtype, y_rows, ldy, positions, weights, m, k, d, out, out_dtype, ldo, (hipStream_t)stream));
}

}  // extern "C"
