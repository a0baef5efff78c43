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

}  // namespace mq

using namespace mq;

extern "C" {

int mq_rotary_table(const double* freq_host, const int* axis_host, int pairs, uint32_t* table_host) {
    if (pairs < 0) return MQ_ERR_BAD_SHAPE;
    if (pairs > 0 && (!freq_host || !axis_host || !table_host)) return MQ_ERR_BAD_ARG;
    const long double two_pi = 6.283185307179586476925286766559005768L;
    for (int i = 0; i < pairs; ++i) {
        if (!isfinite(freq_host[i]) || axis_host[i] < 0 || axis_host[i] > 3) return MQ_ERR_BAD_ARG;
        long double turn = (long double)freq_host[i] / two_pi;
        turn -= floorl(turn);
        const long double units = roundl(ldexpl(turn, 64));
        const uint64_t f = units >= 18446744073709551616.0L ? 0 : (uint64_t)units;
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

}  // extern "C"
