// C ABI of the 8-bit matrices with a scale for each block of 128: quantiser and product.
#include <hip/hip_runtime.h>

#include "fp8.h"
#include "host_util.h"

using namespace tsr;

namespace {

constexpr int MOST_K = 1 << 22;              // 256 rows of it lie within 31-bit offsets
constexpr int MOST_ROWS = 1 << 30;           // a row's number and what is added to it stay within an int
constexpr long long MOST_GROUPS = 1 << 24;   // workgroups of a launch: times 256 threads, 2^32

bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
int blocks(int n, int of) { return (int)(((long long)n + of - 1) / of); }
bool is_fp8(int d) { return d == TSR_E4M3 || d == TSR_E5M2; }
int format(int d) { return d == TSR_E4M3 ? 0 : 1; }

// An 8-bit matrix of rows x cols and its scales.
int check_fp8(const void* q, long long ld, const void* scale, long long ld_scale, int cols) {
    if (!q || !scale) return TSR_INVALID_ARG;
    if (ld < cols || ld_scale < blocks(cols, 128)) return TSR_BAD_SHAPE;
    if (!aligned(q, 16) || ld % 16 || !aligned(scale, 4) || ld_scale % 4) return TSR_INVALID_ARG;
    if (ld > (1ll << 40) || ld_scale > (1ll << 40)) return TSR_BAD_SHAPE;
    return TSR_OK;
}

int check_operand(const tsr_fp8_matrix* x, int k) {
    if (!x) return TSR_INVALID_ARG;
    if (!is_fp8(x->dtype)) return TSR_BAD_DTYPE;
    if (x->block_rows != 1 && x->block_rows != 128) return TSR_BAD_SHAPE;
    TSR_TRY(check_fp8(x->q, x->ld, x->scale, x->ld_scale, k));
    if (x->ld > MOST_K || x->ld_scale > MOST_K) return TSR_BAD_SHAPE;
    return TSR_OK;
}

Fp8Operand operand(const tsr_fp8_matrix* x, int rows) {
    return Fp8Operand{(const unsigned char*)x->q, x->scale, x->ld, x->ld_scale, rows, x->block_rows == 128 ? 7 : 0};
}

}  // namespace

extern "C" {

int tsr_fp8_quantize(const void* X, int x_dtype, int m, int n, long long ldx, int block_rows, int q_dtype,
                     void* Q, long long ldq, unsigned char* S, long long lds,
                     void* Qt, long long ldqt, unsigned char* St, long long ldst, void* stream) {
    if (m <= 0 || n <= 0 || m > MOST_ROWS || n > MOST_ROWS || ldx < n || (block_rows != 1 && block_rows != 128)) return TSR_BAD_SHAPE;
    if ((x_dtype != TSR_F32 && x_dtype != TSR_BF16) || !is_fp8(q_dtype)) return TSR_BAD_DTYPE;
    if (!X || !aligned(X, x_dtype == TSR_F32 ? 4 : 2) || (!Q && !Qt)) return TSR_INVALID_ARG;
    if ((long long)blocks(m, 128) * blocks(n, 128) >= MOST_GROUPS) return TSR_BAD_SHAPE;
    if (Q) TSR_TRY(check_fp8(Q, ldq, S, lds, n));
    if (Qt) TSR_TRY(check_fp8(Qt, ldqt, St, ldst, m));
    QuantizeArgs a{X, ldx, x_dtype == TSR_BF16, m, n, (unsigned char*)Q, ldq, S, lds, (unsigned char*)Qt, ldqt, St, ldst};
    TSR_HIP(launch_fp8_quantize(a, format(q_dtype), block_rows, (hipStream_t)stream));
    return TSR_OK;
}

size_t tsr_fp8_matmul_workspace_bytes(int m, int n, int k) {
    if (m <= 0 || n <= 0 || k <= 0 || m > MOST_ROWS || n > MOST_ROWS || k > MOST_K) return 0;
    const Fp8Plan p = fp8_plan(m, n, k);
    return p.pieces > 1 ? align_up((size_t)p.pieces * m * p.ldp * sizeof(float)) : 0;
}

int tsr_fp8_matmul(const tsr_fp8_matrix* A, const tsr_fp8_matrix* B, int m, int n, int k,
                   void* C, long long ldc, void* ws, size_t ws_bytes, void* stream) {
    if (m <= 0 || n <= 0 || k <= 0 || k > MOST_K || ldc < n) return TSR_BAD_SHAPE;
    TSR_TRY(check_operand(A, k));
    TSR_TRY(check_operand(B, k));
    if (!C || !aligned(C, 2)) return TSR_INVALID_ARG;
    // 2^40 elements are beyond any card; a result of few rows or columns takes a workgroup for every 16 of the others
    if (m > MOST_ROWS || n > MOST_ROWS || (long long)m * n > (1ll << 40)) return TSR_BAD_SHAPE;
    if ((m <= 32 || n <= 32) && (m > 16 * (MOST_GROUPS - 1) || n > 16 * (MOST_GROUPS - 1))) return TSR_BAD_SHAPE;
    Fp8Args a{};
    a.a = operand(A, m); a.b = operand(B, n);
    a.k = k; a.C = C; a.ldc = ldc;
    Fp8Plan p = fp8_plan(m, n, k);
    if (p.pieces > 1) {                      // as many pieces as the workspace holds
        const size_t piece = (size_t)m * p.ldp * sizeof(float), fit = ws ? ws_bytes / piece : 0;
        if ((size_t)p.pieces > fit) p = fp8_plan(m, n, k, fit < 1 ? 1 : (int)fit);
        if (p.pieces > 1 && (uintptr_t)ws % ALIGN) return TSR_INVALID_ARG;
        a.partial = (float*)ws;
    }
    TSR_HIP(launch_fp8_matmul(a, p, format(A->dtype), format(B->dtype), (hipStream_t)stream));
    return TSR_OK;
}

}  // extern "C"
