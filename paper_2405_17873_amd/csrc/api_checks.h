// What the entry points of the microscaled linears, the norms and what stands around them check of their arguments.
#pragma once
#include "mx_common.h"

namespace mq {

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
inline bool type_ok(int dtype) { return dtype == MQ_F16 || dtype == MQ_BF16; }

// A matrix of 16-bit values with `cols` columns: rows may lie apart, and need not start on any boundary but their own type's.
// (Without rows there is nothing to point to.)
inline int check_matrix(const void* p, int rows, long ld, int cols) {
    if (ld < cols) return MQ_ERR_BAD_SHAPE;
    if (rows > 0 && (!p || !aligned(p, 2))) return MQ_ERR_BAD_ARG;
    return MQ_OK;
}
// Whether two matrices of M rows share no value: one lies behind the other, or the rows of one between those of the other.
inline bool apart(const void* a, long lda, int ca, const void* b, long ldb, int cb, int M) {
    const uintptr_t p = (uintptr_t)a, q = (uintptr_t)b;
    if (q >= p + ((size_t)(M - 1) * lda + ca) * 2 || p >= q + ((size_t)(M - 1) * ldb + cb) * 2) return true;
    if (M == 1 || lda != ldb) return false;
    const size_t row = (size_t)lda * 2, behind = q >= p ? (q - p) % row : (row - (p - q) % row) % row;  // of b's first value in a row of a's
    return behind >= (size_t)ca * 2 && behind + (size_t)cb * 2 <= row;
}
// An output that is written while others still read an operand: the operand itself (a thread reads its values before it writes them) or apart from it.
inline bool itself_or_apart(const void* out, long ldo, const void* in, long ldi, int cols, int M) {
    return !in || (out == in && (ldo == ldi || M == 1)) || apart(out, ldo, cols, in, ldi, cols, M);
}
inline bool mx_size_ok(int rows, int K) { return rows >= 0 && rows <= (1 << 28) && K > 0 && K % 32 == 0 && K <= (1 << 21); }
inline int check_mx(const void* p, int rows, int K) {
    if (!mx_size_ok(rows, K)) return MQ_ERR_BAD_SHAPE;
    if (rows > 0 && (!p || !aligned(p, 256))) return MQ_ERR_BAD_ARG;
    return MQ_OK;
}

inline int check_product(int M, int N, int K, const void* w, const void* bias, const void* y, long ldy, int dtype, const void* residual, long ldr) {
    if (!type_ok(dtype)) return MQ_ERR_BAD_ARG;
    if (M < 0 || N <= 0 || N > (1 << 22)) return MQ_ERR_BAD_SHAPE;
    int rc;
    if ((rc = check_mx(w, N, K))) return rc;
    if (!aligned(bias, 2)) return MQ_ERR_BAD_ARG;
    if ((rc = check_matrix(y, M, ldy, N))) return rc;
    if (residual && (rc = check_matrix(residual, M, ldr, N))) return rc;
    return MQ_OK;
}

inline MxGemm product(int M, int K, const void* w, int N, const void* bias, void* y, long ldy, int dtype, const void* residual, long ldr) {
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

}  // namespace mq
