// 8-bit matrices with a scale for each block of 128: how they are made and multiplied (internal interface).
#pragma once
#include <hip/hip_runtime.h>

namespace tsr {

struct QuantizeArgs {
    const void* X; long long ldx; int x_bf16;
    int m, n;
    unsigned char* Q; long long ldq; unsigned char* S; long long lds;            // as stored, or null
    unsigned char* Qt; long long ldqt; unsigned char* St; long long ldst;        // transposed, or null
};
hipError_t launch_fp8_quantize(const QuantizeArgs& a, int fmt, int block_rows, hipStream_t stream);

// One operand: rows x k bytes, and a scale byte for each 128 of them and 1 << shift rows.
struct Fp8Operand {
    const unsigned char* q; const unsigned char* scale;
    long long ld, ld_scale;
    int rows, shift;
};
struct Fp8Args {
    Fp8Operand a, b;            // C is a.rows x b.rows
    int k;
    void* C; long long ldc;     // bf16
    // set by the launch
    float* partial; long long ldp;       // pieces of the contraction: fp32 sums of each, rows of ldp
    int chunk;                           // of k in a piece, a multiple of 512 where there are several
    int groups_n;                        // of 16 rows of B
};

// How a product is done, by its sizes alone.
enum { FP8_DIRECT = 0, FP8_TILES = 1, FP8_WIDE = 2 };
struct Fp8Plan { int kind, pieces, chunk; long long ldp; };      // pieces of chunk along k, the last of what is left
constexpr int FP8_PIECES = 16;
Fp8Plan fp8_plan(int m, int n, int k, int most = FP8_PIECES);    // with `most` pieces at most
hipError_t launch_fp8_matmul(const Fp8Args& a, const Fp8Plan& p, int fmt_a, int fmt_b, hipStream_t stream);

}  // namespace tsr
