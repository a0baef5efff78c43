// C ABI of the microscaled 4-bit linears and of the layer norm: argument validation on the host, workspace carving, launch sequencing.
#include <math.h>

#include "mx_common.h"

namespace mq {

static inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
static inline bool type_ok(int dtype) { return dtype == MQ_F16 || dtype == MQ_BF16; }

// A matrix of 16-bit values with `cols` columns: rows may lie apart, and need not start on any boundary but their own type's.
// (Without rows there is nothing to point to.)
static int check_matrix(const void* p, int rows, long ld, int cols) {
    if (ld < cols) return MQ_ERR_BAD_SHAPE;
    if (rows > 0 && (!p || !aligned(p, 2))) return MQ_ERR_BAD_ARG;
    return MQ_OK;
}
// Whether two matrices of M rows share no value: one lies behind the other, or the rows of one between those of the other.
static bool apart(const void* a, long lda, int ca, const void* b, long ldb, int cb, int M) {
    const uintptr_t p = (uintptr_t)a, q = (uintptr_t)b;
    if (q >= p + ((size_t)(M - 1) * lda + ca) * 2 || p >= q + ((size_t)(M - 1) * ldb + cb) * 2) return true;
    if (M == 1 || lda != ldb) return false;
    const size_t row = (size_t)lda * 2, behind = q >= p ? (q - p) % row : (row - (p - q) % row) % row;  // of b's first value in a row of a's
    return behind >= (size_t)ca * 2 && behind + (size_t)cb * 2 <= row;
}
// An output that is written while others still read an operand: the operand itself (a thread reads its values before it writes them) or apart from it.
static bool itself_or_apart(const void* out, long ldo, const void* in, long ldi, int cols, int M) {
    return !in || (out == in && (ldo == ldi || M == 1)) || apart(out, ldo, cols, in, ldi, cols, M);
}
static bool mx_size_ok(int rows, int K) { return rows >= 0 && rows <= (1 << 28) && K > 0 && K % 32 == 0 && K <= (1 << 21); }
static int check_mx(const void* p, int rows, int K) {
    if (!mx_size_ok(rows, K)) return MQ_ERR_BAD_SHAPE;
    if (rows > 0 && (!p || !aligned(p, 256))) return MQ_ERR_BAD_ARG;
    return MQ_OK;
}

static int check_product(int M, int N, int K, const void* w, const void* bias, const void* y, long ldy, int dtype, const void* residual, long ldr) {
    if (!type_ok(dtype)) return MQ_ERR_BAD_ARG;
    if (M < 0 || N <= 0 || N > (1 << 22)) return MQ_ERR_BAD_SHAPE;
    int rc;
    if ((rc = check_mx(w, N, K))) return rc;
    if (!aligned(bias, 2)) return MQ_ERR_BAD_ARG;
    if ((rc = check_matrix(y, M, ldy, N))) return rc;
    if (residual && (rc = check_matrix(residual, M, ldr, N))) return rc;
    return MQ_OK;
}

static MxGemm product(int M, int K, const void* w, int N, const void* bias, void* y, long ldy, int dtype, const void* residual, long ldr) {
    MxGemm g = {};
    g.w = mx_view(w, N, K);
    g.M = M;
    g.N = N;
    g.K = K;
    g.bias = (const uint16_t*)bias;
    g.y = (uint16_t*)y;
    g.ldy = ldy;
    g.res = (const uint16_t*)residual;
    g.ldr = ldr;
    g.dtype = dtype;
    return g;
}
static int run(MxGemm& g, const void* a, hipStream_t st) {
    g.a = mx_view(a, g.M, g.K);
    return mx_rows_takes(g.M, g.N) ? launch_mx_rows(g, nullptr, 0, st) : launch_mx_gemm(g, st);
}

static int check_norm(const void* x, int M, int C, long ldx, const void* weight, const void* bias, int param_dtype, int dtype) {
    if (!type_ok(dtype)) return MQ_ERR_BAD_ARG;
    if ((weight || bias) && !type_ok(param_dtype) && param_dtype != MQ_F32) return MQ_ERR_BAD_ARG;
    if (!aligned(weight, param_dtype == MQ_F32 ? 4 : 2) || !aligned(bias, param_dtype == MQ_F32 ? 4 : 2)) return MQ_ERR_BAD_ARG;
    if (M < 0 || C <= 0 || C > 16384) return MQ_ERR_BAD_SHAPE;
    return check_matrix(x, M, ldx, C);
}

}  // namespace mq

using namespace mq;

extern "C" {

size_t mq_mx_bytes(int rows, int K) { return mx_size_ok(rows, K) ? mx_bytes(rows, K) : 0; }

int mq_mx_quantize(const void* x, int M, int K, long ldx, int dtype, void* mx, void* stream) {
    if (!type_ok(dtype)) return MQ_ERR_BAD_ARG;
    int rc;
    if ((rc = check_mx(mx, M, K)) || (rc = check_matrix(x, M, ldx, K))) return rc;
    return M == 0 ? MQ_OK : launch_mx_quantize(x, M, K, ldx, dtype, mx, (hipStream_t)stream);
}

int mq_mx_dequantize(const void* mx, int M, int K, int dtype, void* y, long ldy, void* stream) {
    if (!type_ok(dtype)) return MQ_ERR_BAD_ARG;
    int rc;
    if ((rc = check_mx(mx, M, K)) || (rc = check_matrix(y, M, ldy, K))) return rc;
    return M == 0 ? MQ_OK : launch_mx_dequantize(mx, M, K, dtype, y, ldy, (hipStream_t)stream);
}

int mq_mx_pack(const uint8_t* codes, const uint8_t* scales, int M, int K, void* mx, void* stream) {
    int rc;
    if ((rc = check_mx(mx, M, K))) return rc;
    if (M > 0 && (!codes || !scales)) return MQ_ERR_BAD_ARG;
    return M == 0 ? MQ_OK : launch_mx_pack(codes, scales, M, K, mx, (hipStream_t)stream);
}

int mq_mx_unpack(const void* mx, int M, int K, uint8_t* codes, uint8_t* scales, void* stream) {
    int rc;
    if ((rc = check_mx(mx, M, K))) return rc;
    if (M > 0 && (!codes || !scales)) return MQ_ERR_BAD_ARG;
    return M == 0 ? MQ_OK : launch_mx_unpack(mx, M, K, codes, scales, (hipStream_t)stream);
}

int mq_mx_column_top(const void* mx, int rows, int K, uint8_t* top, void* stream) {
    int rc;
    if ((rc = check_mx(mx, rows, K))) return rc;
    if (!top) return MQ_ERR_BAD_ARG;
    return launch_mx_column_top(mx, rows, K, top, (hipStream_t)stream);
}

size_t mq_mx_linear_workspace_bytes(int M, int N, int K) {
    return M <= 0 || N <= 0 || K <= 0 || K % 32 != 0 || mx_rows_quantizes(M, N, K) ? 0 : up256(mx_bytes(M, K));
}

int mq_mx_linear(const void* x, int M, int K, long ldx, const void* w, int N, const void* bias, void* y, long ldy, int dtype, const void* residual,
                 long ldr, void* ws, size_t ws_bytes, void* stream) {
    int rc;
    if ((rc = check_product(M, N, K, w, bias, y, ldy, dtype, residual, ldr)) || (rc = check_matrix(x, M, ldx, K))) return rc;
    if (M == 0) return MQ_OK;
    if (!itself_or_apart(y, ldy, residual, ldr, N, M)) return MQ_ERR_BAD_ARG;
    MxGemm g = product(M, K, w, N, bias, y, ldy, dtype, residual, ldr);
    // (one launch reads activations while others of its workgroups store results)
    if (mx_rows_quantizes(M, N, K) && apart(x, ldx, K, y, ldy, N, M)) return launch_mx_rows(g, x, ldx, (hipStream_t)stream);
    if (!ws || !aligned(ws, 256)) return MQ_ERR_BAD_ARG;
    if (ws_bytes < up256(mx_bytes(M, K))) return MQ_ERR_WORKSPACE_TOO_SMALL;
    if ((rc = launch_mx_quantize(x, M, K, ldx, dtype, ws, (hipStream_t)stream))) return rc;
    return run(g, ws, (hipStream_t)stream);
}

int mq_mx_linear_codes(const void* a, int M, int K, const void* w, int N, const void* bias, void* y, long ldy, int dtype, const void* residual, long ldr,
                       void* stream) {
    int rc;
    if ((rc = check_product(M, N, K, w, bias, y, ldy, dtype, residual, ldr)) || (rc = check_mx(a, M, K))) return rc;
    if (M == 0) return MQ_OK;
    if (!itself_or_apart(y, ldy, residual, ldr, N, M)) return MQ_ERR_BAD_ARG;
    MxGemm g = product(M, K, w, N, bias, y, ldy, dtype, residual, ldr);
    return run(g, a, (hipStream_t)stream);
}

size_t mq_mx_linear_grad_workspace_bytes(int M, int N, int K) { return M <= 0 || N <= 0 || K <= 0 || K % 32 != 0 ? 0 : up256(mx_grad_workspace_bytes(M, N, K)); }

int mq_mx_linear_grad(const void* dy, int M, int N, long lddy, const void* w, const uint8_t* top, int K, void* dx, long lddx, int dtype, void* ws,
                      size_t ws_bytes, void* stream) {
    if (!type_ok(dtype) || !top) return MQ_ERR_BAD_ARG;
    if (M < 0 || N <= 0 || N > (1 << 22)) return MQ_ERR_BAD_SHAPE;
    int rc;
    if ((rc = check_mx(w, N, K)) || (rc = check_matrix(dy, M, lddy, N)) || (rc = check_matrix(dx, M, lddx, K))) return rc;
    if (M == 0) return MQ_OK;
    const size_t need = mq_mx_linear_grad_workspace_bytes(M, N, K);
    if (need > 0 && (!ws || !aligned(ws, 256))) return MQ_ERR_BAD_ARG;
    if (ws_bytes < need) return MQ_ERR_WORKSPACE_TOO_SMALL;
    if (!apart(dx, lddx, K, dy, lddy, N, M)) return MQ_ERR_BAD_ARG;
    return launch_mx_grad(dy, M, N, lddy, w, top, K, dx, lddx, dtype, ws, (hipStream_t)stream);
}

int mq_layer_norm(const void* x, int M, int C, long ldx, const void* weight, const void* bias, int param_dtype, float eps, void* y, long ldy, int dtype,
                  float* mean, float* rstd, void* stream) {
    int rc;
    if ((rc = check_norm(x, M, C, ldx, weight, bias, param_dtype, dtype)) || (rc = check_matrix(y, M, ldy, C))) return rc;
    if (!(eps >= 0.0f) || !aligned(mean, 4) || !aligned(rstd, 4)) return MQ_ERR_BAD_ARG;
    if (M == 0) return MQ_OK;
    if (!itself_or_apart(y, ldy, x, ldx, C, M)) return MQ_ERR_BAD_ARG;
    NormArgs a = {};
    a.x = (const uint16_t*)x, a.ldx = ldx, a.M = M, a.C = C, a.weight = weight, a.bias = bias, a.param_dtype = param_dtype, a.eps = eps;
    a.dtype = dtype, a.mean = mean, a.rstd = rstd, a.y = (uint16_t*)y, a.ldy = ldy;
    return launch_layer_norm(a, (hipStream_t)stream);
}

int mq_layer_norm_mx(const void* x, int M, int C, long ldx, const void* weight, const void* bias, int param_dtype, float eps, void* mx, int dtype,
                     float* mean, float* rstd, void* stream) {
    int rc;
    if ((rc = check_norm(x, M, C, ldx, weight, bias, param_dtype, dtype)) || (rc = check_mx(mx, M, C))) return rc;
    if (!(eps >= 0.0f) || !aligned(mean, 4) || !aligned(rstd, 4)) return MQ_ERR_BAD_ARG;
    if (M == 0) return MQ_OK;
    NormArgs a = {};
    a.x = (const uint16_t*)x, a.ldx = ldx, a.M = M, a.C = C, a.weight = weight, a.bias = bias, a.param_dtype = param_dtype, a.eps = eps;
    a.dtype = dtype, a.mean = mean, a.rstd = rstd, a.mx = mx;
    return launch_layer_norm_mx(a, (hipStream_t)stream);
}

size_t mq_layer_norm_grad_workspace_bytes(int M, int C) { return M < 0 || C <= 0 ? 0 : up256(layer_norm_grad_workspace_bytes(M, C)); }

int mq_layer_norm_grad(const void* dy, long lddy, const void* x, long ldx, int M, int C, const void* weight, int param_dtype, const float* mean,
                       const float* rstd, const void* residual, long ldr, void* dx, long lddx, int dtype, float* dweight, float* dbias, void* ws,
                       size_t ws_bytes, void* stream) {
    int rc;
    if ((rc = check_norm(x, M, C, ldx, weight, nullptr, param_dtype, dtype)) || (rc = check_matrix(dy, M, lddy, C)) || (rc = check_matrix(dx, M, lddx, C)))
        return rc;
    if (residual && (rc = check_matrix(residual, M, ldr, C))) return rc;
    if (M > 0 && (!mean || !rstd || !ws || !aligned(ws, 256))) return MQ_ERR_BAD_ARG;
    if (!aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dweight, 4) || !aligned(dbias, 4)) return MQ_ERR_BAD_ARG;
    if (ws_bytes < mq_layer_norm_grad_workspace_bytes(M, C)) return MQ_ERR_WORKSPACE_TOO_SMALL;
    if (M > 0 && !(itself_or_apart(dx, lddx, dy, lddy, C, M) && itself_or_apart(dx, lddx, x, ldx, C, M) && itself_or_apart(dx, lddx, residual, ldr, C, M)))
        return MQ_ERR_BAD_ARG;
    NormArgs a = {};
    a.x = (const uint16_t*)x, a.ldx = ldx, a.M = M, a.C = C, a.weight = weight, a.param_dtype = param_dtype, a.dtype = dtype;
    a.mean = (float*)mean, a.rstd = (float*)rstd, a.dy = (const uint16_t*)dy, a.lddy = lddy, a.res = (const uint16_t*)residual, a.ldr = ldr;
    a.dx = (uint16_t*)dx, a.lddx = lddx, a.dweight = dweight, a.dbias = dbias, a.partial = (float*)ws;
    return launch_layer_norm_grad(a, (hipStream_t)stream);
}

}  // extern "C"
