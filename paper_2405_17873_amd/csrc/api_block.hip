// C ABI of what a transformer block has around its microscaled linears: argument validation on the host, workspace carving, launch sequencing.
#include <math.h>

#include "api_checks.h"

namespace mq {

static int check_heads(const void* x, int M, int q, int k, int D, long ldx, const void* qw, const void* kw, int param_dtype, float eps, int norm, const void* table,
                       int pairs, const void* pos, int pos_bytes, int axes, long ldpos, int dtype) {
    if (!type_ok(dtype)) return MQ_ERR_BAD_ARG;
    if (M < 0 || M > (1 << 28) || q < 0 || k < 0 || q > 4096 || k > 4096 || q + k == 0 || D <= 0 || D % 8 != 0 || D > 512) return MQ_ERR_BAD_SHAPE;
    if (pairs < 0 || pairs % 4 != 0 || 2 * pairs > D || (long)M * (q + k) > 0x7FFFFFFFL) return MQ_ERR_BAD_SHAPE;
    if (norm ? !(eps >= 0.0f) : (qw || kw)) return MQ_ERR_BAD_ARG;
    if ((qw || kw) && !type_ok(param_dtype) && param_dtype != MQ_F32) return MQ_ERR_BAD_ARG;
    if (!aligned(qw, param_dtype == MQ_F32 ? 4 : 2) || !aligned(kw, param_dtype == MQ_F32 ? 4 : 2)) return MQ_ERR_BAD_ARG;
    if (pairs > 0) {
        if (axes < 1 || axes > 4 || ldpos < axes) return MQ_ERR_BAD_SHAPE;
        if ((pos_bytes != 4 && pos_bytes != 8) || !table || !aligned(table, 16) || (M > 0 && !pos) || !aligned(pos, pos_bytes)) return MQ_ERR_BAD_ARG;
    }
    return check_matrix(x, M, ldx, (q + k) * D);
}
static HeadArgs head_args(const void* x, int M, int q, int k, int D, long ldx, const void* qw, const void* kw, int param_dtype, float eps, int norm, const void* table,
                          int pairs, int interleaved, const void* pos, int pos_bytes, int axes, long ldpos, int dtype) {
    HeadArgs a = {};
    a.x = (const uint16_t*)x, a.ldx = ldx, a.M = M, a.q = q, a.k = k, a.D = D, a.qw = qw, a.kw = kw, a.param_dtype = param_dtype, a.eps = eps, a.norm = norm != 0;
    a.table = (const uint4v*)table, a.pairs = pairs, a.interleaved = interleaved != 0, a.pos = pos, a.pos_bytes = pos_bytes, a.axes = pairs > 0 ? axes : 0;
    a.ldpos = ldpos, a.dtype = dtype;
    return a;
}

// What a product with an activation or a gate (N rows of weights for N / 2 columns of Y) has beside one without.
static int check_act(int M, int N, int act, int gated, const void* y, long ldy, const void* residual, const void* pre, long ldpre) {
    if (act < MQ_ACT_NONE || act > MQ_ACT_SILU || (gated && (act == MQ_ACT_NONE || residual))) return MQ_ERR_BAD_ARG;
    if (gated && N % 64 != 0) return MQ_ERR_BAD_SHAPE;
    if (pre)
        if (const int rc = check_matrix(pre, M, ldpre, N)) return rc;
    if (M > 0 && pre && !apart(pre, ldpre, N, y, ldy, gated ? N / 2 : N, M)) return MQ_ERR_BAD_ARG;
    return MQ_OK;
}
// (offsets of a gate's weights behind its values' are 32-bit)
static bool gate_fits(int N, int K) { return (long)N * K <= 1L << 32; }
static int check_product_act(int M, int N, int K, const void* w, const void* bias, int act, int gated, const void* y, long ldy, int dtype, const void* residual,
                             long ldr, const void* pre, long ldpre) {
    int rc;
    if (N <= 0 || N > (1 << 22) || (gated && (N % 64 != 0 || !gate_fits(N, K)))) return MQ_ERR_BAD_SHAPE;
    const int outs = gated ? N / 2 : N;
    if ((rc = check_product(M, outs, K, w, bias, y, ldy, dtype, residual, ldr)) || (rc = check_mx(w, N, K)) ||
        (rc = check_act(M, N, act, gated, y, ldy, residual, pre, ldpre)))
        return rc;
    if (M > 0 && !itself_or_apart(y, ldy, residual, ldr, outs, M)) return MQ_ERR_BAD_ARG;
    if (M > 0 && pre && residual && !apart(pre, ldpre, N, residual, ldr, N, M)) return MQ_ERR_BAD_ARG;
    return MQ_OK;
}
static MxGemm product_act(int M, int K, const void* w, int N, const void* bias, int act, void* y, long ldy, int dtype, const void* residual, long ldr, void* pre,
                          long ldpre) {
    MxGemm g = product(M, K, w, N, bias, y, ldy, dtype, residual, ldr);
    g.act = act, g.pre = (uint16_t*)pre, g.ldpre = ldpre;
    return g;
}
static int run_act(MxGemm& g, int gated, const void* a, hipStream_t st) {
    g.a = mx_view(a, g.M, g.K);
    return mx_rows_takes(g.M, g.N) ? launch_mx_rows_act(g, gated, st) : launch_mx_gemm_act(g, gated, st);
}
// Weights of `experts` experts, N rows of each, one behind the other in one matrix.
static int check_experts(const void* w, int N, int K, int experts, const int* offsets, int M) {
    if (experts <= 0 || experts > 4096 || N <= 0 || N > (1 << 22) || N % 32 != 0 || (long)N * experts > 1 << 28 || M > (1 << 28)) return MQ_ERR_BAD_SHAPE;
    if (!offsets || !aligned(offsets, 4)) return MQ_ERR_BAD_ARG;
    return check_mx(w, N * experts, K);
}

}  // namespace mq

using namespace mq;

extern "C" {

int mq_rotary_table(const double* freq_host, const int* axis_host, int pairs, uint32_t* table_host) {
    if (pairs < 0) return MQ_ERR_BAD_SHAPE;
    if (pairs > 0 && (!freq_host || !axis_host || !table_host)) return MQ_ERR_BAD_ARG;
    const long double two_pi = 6.283185307179586476925286766559005768L;
    for (int i = 0; i < pairs; ++i) {
        if (!isfinite(freq_host[i]) || axis_host[i] < 0 || axis_host[i] > 3) return MQ_ERR_BAD_ARG;
        long double turn = fabsl((long double)freq_host[i]) / two_pi;
        turn -= floorl(turn);
        const long double units = roundl(ldexpl(turn, 64));
        uint64_t f = units >= 18446744073709551616.0L ? 0 : (uint64_t)units;
        if (freq_host[i] < 0) f = 0 - f;
        table_host[4 * i] = (uint32_t)f;
        table_host[4 * i + 1] = (uint32_t)(f >> 32);
        table_host[4 * i + 2] = (uint32_t)axis_host[i];
        table_host[4 * i + 3] = 0;
    }
    return MQ_OK;
}

int mq_qk_norm_rope(const void* x, int M, int q_heads, int k_heads, int head_dim, long ldx, const void* q_weight, const void* k_weight, int param_dtype, float eps,
                    int norm, const void* table, int pairs, int interleaved, const void* positions, int position_bytes, int axes, long ldpos, void* y, long ldy,
                    int dtype, void* stream) {
    int rc;
    if ((rc = check_heads(x, M, q_heads, k_heads, head_dim, ldx, q_weight, k_weight, param_dtype, eps, norm, table, pairs, positions, position_bytes, axes, ldpos,
                          dtype)))
        return rc;
    const int cols = (q_heads + k_heads) * head_dim;
    if ((rc = check_matrix(y, M, ldy, cols))) return rc;
    if (M == 0) return MQ_OK;
    if (!itself_or_apart(y, ldy, x, ldx, cols, M)) return MQ_ERR_BAD_ARG;
    HeadArgs a = head_args(x, M, q_heads, k_heads, head_dim, ldx, q_weight, k_weight, param_dtype, eps, norm, table, pairs, interleaved, positions, position_bytes,
                           axes, ldpos, dtype);
    a.y = (uint16_t*)y, a.ldy = ldy;
    return launch_heads(a, false, (hipStream_t)stream);
}

size_t mq_qk_norm_rope_grad_workspace_bytes(int M, int q_heads, int k_heads, int head_dim) {
    if (M <= 0 || q_heads < 0 || k_heads < 0 || q_heads > 4096 || k_heads > 4096 || head_dim <= 0 || head_dim > 512) return 0;
    return up256(heads_grad_workspace_bytes(M, q_heads + k_heads, head_dim));
}

int mq_qk_norm_rope_grad(const void* dy, long lddy, const void* x, int M, int q_heads, int k_heads, int head_dim, long ldx, const void* q_weight,
                         const void* k_weight, int param_dtype, float eps, int norm, const void* table, int pairs, int interleaved, const void* positions,
                         int position_bytes, int axes, long ldpos, void* dx, long lddx, int dtype, float* dq_weight, float* dk_weight, void* ws, size_t ws_bytes,
                         void* stream) {
    int rc;
    if ((rc = check_heads(norm ? x : dy, M, q_heads, k_heads, head_dim, norm ? ldx : lddy, q_weight, k_weight, param_dtype, eps, norm, table, pairs, positions,
                          position_bytes, axes, ldpos, dtype)))
        return rc;
    const int cols = (q_heads + k_heads) * head_dim;
    if ((rc = check_matrix(dy, M, lddy, cols)) || (rc = check_matrix(dx, M, lddx, cols))) return rc;
    if (!aligned(dq_weight, 4) || !aligned(dk_weight, 4) || (!norm && (dq_weight || dk_weight))) return MQ_ERR_BAD_ARG;
    if (dq_weight || dk_weight) {
        const size_t need = mq_qk_norm_rope_grad_workspace_bytes(M, q_heads, k_heads, head_dim);
        if (need > 0 && (!ws || !aligned(ws, 256))) return MQ_ERR_BAD_ARG;
        if (ws_bytes < need) return MQ_ERR_WORKSPACE_TOO_SMALL;
    }
    if (M > 0 && !(itself_or_apart(dx, lddx, dy, lddy, cols, M) && (!norm || itself_or_apart(dx, lddx, x, ldx, cols, M)))) return MQ_ERR_BAD_ARG;
    HeadArgs a = head_args(x, M, q_heads, k_heads, head_dim, ldx, q_weight, k_weight, param_dtype, eps, norm, table, pairs, interleaved, positions, position_bytes,
                           axes, ldpos, dtype);
    a.dy = (const uint16_t*)dy, a.lddy = lddy, a.dx = (uint16_t*)dx, a.lddx = lddx, a.dq_weight = dq_weight, a.dk_weight = dk_weight, a.partial = (float*)ws;
    return launch_heads(a, true, (hipStream_t)stream);
}

int mq_mx_linear_act(const void* x, int M, int K, long ldx, const void* w, int N, const void* bias, int act, int gated, void* y, long ldy, int dtype,
                     const void* residual, long ldr, void* pre, long ldpre, void* ws, size_t ws_bytes, void* stream) {
    int rc;
    if ((rc = check_product_act(M, N, K, w, bias, act, gated, y, ldy, dtype, residual, ldr, pre, ldpre)) || (rc = check_matrix(x, M, ldx, K))) return rc;
    if (M == 0) return MQ_OK;
    MxGemm g = product_act(M, K, w, N, bias, act, y, ldy, dtype, residual, ldr, pre, ldpre);
    // (one launch reads activations while others of its workgroups store results)
    if (mx_few_rows_takes(M, N, K) && apart(x, ldx, K, y, ldy, gated ? N / 2 : N, M) && (!pre || apart(x, ldx, K, pre, ldpre, N, M)))
        return launch_mx_few_rows(g, gated, x, ldx, (hipStream_t)stream);
    if (!ws || !aligned(ws, 256)) return MQ_ERR_BAD_ARG;
    if (ws_bytes < up256(mx_bytes(M, K))) return MQ_ERR_WORKSPACE_TOO_SMALL;
    if ((rc = launch_mx_quantize(x, M, K, ldx, dtype, ws, (hipStream_t)stream))) return rc;
    return run_act(g, gated, ws, (hipStream_t)stream);
}

int mq_mx_linear_act_codes(const void* a, int M, int K, const void* w, int N, const void* bias, int act, int gated, void* y, long ldy, int dtype,
                           const void* residual, long ldr, void* pre, long ldpre, void* stream) {
    int rc;
    if ((rc = check_product_act(M, N, K, w, bias, act, gated, y, ldy, dtype, residual, ldr, pre, ldpre)) || (rc = check_mx(a, M, K))) return rc;
    if (M == 0) return MQ_OK;
    MxGemm g = product_act(M, K, w, N, bias, act, y, ldy, dtype, residual, ldr, pre, ldpre);
    return run_act(g, gated, a, (hipStream_t)stream);
}

size_t mq_act_grad_workspace_bytes(int M, int N, int gated) { return M <= 0 || N <= 0 ? 0 : up256(act_grad_workspace_bytes(M, N, gated)); }

int mq_act_grad(const void* dy, int M, int N, long lddy, const void* pre, long ldpre, int act, int gated, void* da, long ldda, int dtype, float* dbias, void* ws,
                size_t ws_bytes, void* stream) {
    if (!type_ok(dtype) || act <= MQ_ACT_NONE || act > MQ_ACT_SILU) return MQ_ERR_BAD_ARG;
    if (M < 0 || M > (1 << 28) || N <= 0 || N > (1 << 22) || (gated && N % 2 != 0)) return MQ_ERR_BAD_SHAPE;
    const int outs = gated ? N / 2 : N;
    int rc;
    if ((rc = check_matrix(dy, M, lddy, outs)) || (rc = check_matrix(pre, M, ldpre, N)) || (rc = check_matrix(da, M, ldda, N))) return rc;
    if (!aligned(dbias, 4)) return MQ_ERR_BAD_ARG;
    if (dbias) {
        const size_t need = mq_act_grad_workspace_bytes(M, N, gated);
        if (need > 0 && (!ws || !aligned(ws, 256))) return MQ_ERR_BAD_ARG;
        if (ws_bytes < need) return MQ_ERR_WORKSPACE_TOO_SMALL;
    }
    if (M > 0 && !(itself_or_apart(da, ldda, pre, ldpre, N, M) && (gated ? apart(da, ldda, N, dy, lddy, outs, M) : itself_or_apart(da, ldda, dy, lddy, N, M))))
        return MQ_ERR_BAD_ARG;
    ActGrad a = {};
    a.dy = (const uint16_t*)dy, a.lddy = lddy, a.pre = (const uint16_t*)pre, a.ldpre = ldpre, a.M = M, a.N = N, a.act = act, a.gated = gated != 0;
    a.da = (uint16_t*)da, a.ldda = ldda, a.dtype = dtype, a.dbias = dbias, a.partial = (float*)ws;
    return launch_act_grad(a, (hipStream_t)stream);
}

int mq_mx_experts_column_top(const void* mx, int experts, int N, int K, uint8_t* top, void* stream) {
    int rc;
    if (experts <= 0 || experts > 4096 || N <= 0 || N % 32 != 0 || (long)N * experts > 1 << 28) return MQ_ERR_BAD_SHAPE;
    if ((rc = check_mx(mx, N * experts, K))) return rc;
    if (!top) return MQ_ERR_BAD_ARG;
    return launch_mx_experts_column_top(mx, experts, N, K, top, (hipStream_t)stream);
}

size_t mq_mx_linear_grouped_workspace_bytes(int M, int N, int K, int experts) {
    return M <= 0 || N <= 0 || K <= 0 || K % 32 != 0 || experts <= 0 ? 0 : up256(mx_experts_workspace_bytes(M, N, K, experts));
}

int mq_mx_linear_grouped(const void* x, int M, int K, long ldx, const void* w, int N, int experts, const int* offsets, const void* bias, int act, int gated,
                         void* y, long ldy, int dtype, void* pre, long ldpre, void* ws, size_t ws_bytes, void* stream) {
    if (!type_ok(dtype)) return MQ_ERR_BAD_ARG;
    if (M < 0) return MQ_ERR_BAD_SHAPE;
    int rc;
    if ((rc = check_experts(w, N, K, experts, offsets, M)) || (rc = check_matrix(x, M, ldx, K))) return rc;
    if (gated && (N % 64 != 0 || !gate_fits(N, K))) return MQ_ERR_BAD_SHAPE;
    const int outs = gated ? N / 2 : N;
    if ((rc = check_matrix(y, M, ldy, outs)) || (rc = check_act(M, N, act, gated, y, ldy, nullptr, pre, ldpre))) return rc;
    if (!aligned(bias, 2)) return MQ_ERR_BAD_ARG;
    if (M == 0) return MQ_OK;
    if (!apart(x, ldx, K, y, ldy, outs, M) || (pre && !apart(x, ldx, K, pre, ldpre, N, M))) return MQ_ERR_BAD_ARG;
    const size_t need = mq_mx_linear_grouped_workspace_bytes(M, N, K, experts);
    if (need > 0 && (!ws || !aligned(ws, 256))) return MQ_ERR_BAD_ARG;
    if (ws_bytes < need) return MQ_ERR_WORKSPACE_TOO_SMALL;
    MxGemm g = product_act(M, K, w, N, bias, act, y, ldy, dtype, nullptr, 0, pre, ldpre);
    g.w.scales = g.w.codes + (size_t)experts * g.w.groups * g.w.kc * 1024;
    g.offsets = offsets, g.experts = experts;
    return launch_mx_experts(g, gated, x, ldx, ws, (hipStream_t)stream);
}

int mq_mx_linear_grouped_grad(const void* dy, int M, int N, long lddy, const void* w, const uint8_t* top, int K, int experts, const int* offsets, void* dx,
                              long lddx, int dtype, void* stream) {
    if (!type_ok(dtype) || !top) return MQ_ERR_BAD_ARG;
    if (M < 0) return MQ_ERR_BAD_SHAPE;
    int rc;
    if ((rc = check_experts(w, N, K, experts, offsets, M)) || (rc = check_matrix(dy, M, lddy, N)) || (rc = check_matrix(dx, M, lddx, K))) return rc;
    if (M == 0) return MQ_OK;
    if (!apart(dx, lddx, K, dy, lddy, N, M)) return MQ_ERR_BAD_ARG;
    return launch_mx_experts_grad(dy, M, N, lddy, w, top, K, experts, offsets, dx, lddx, dtype, (hipStream_t)stream);
}

}  // extern "C"
