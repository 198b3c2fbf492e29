// 8-bit floating point with a power of two as the scale of each block of 128: the quantiser, and C = A B^T on the scaled
// matrix instructions of gfx950.
#include "fp8.h"
#include "fp8_format.h"

namespace tsr {

typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;
// vectors of a matrix whose rows begin anywhere
typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4_any;
typedef __attribute__((ext_vector_type(8), aligned(2))) unsigned short u16x8_any;

// ------------------------------------------------------------------ quantiser
// A workgroup takes 128 x 128 elements of X, a thread 8 rows x 8 columns of them: X is read once, whichever outputs are
// wanted.  Blocks of one row: the largest of a row of the tile is found among the 16 threads of a row (moves within 16
// lanes), that of a column among the threads of a column (two moves across the wave, then LDS).  The transposed tile goes
// through LDS, whose rows are padded by 8 bytes.
template <int FMT> __device__ inline unsigned fp8_encode4(const float* x) {        // nearest, |x| at most the largest value
    int w = 0;
    if constexpr (FMT == FP8_E4M3) {
        w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], w, false); w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
    } else {
        w = __builtin_amdgcn_cvt_pk_bf8_f32(x[0], x[1], w, false); w = __builtin_amdgcn_cvt_pk_bf8_f32(x[2], x[3], w, true);
    }
    return (unsigned)w;
}
__device__ inline unsigned finite_abs_bits(float x) {
    const unsigned a = __builtin_bit_cast(unsigned, x) & 0x7fffffffu;
    return a < 0x7f800000u ? a : 0u;
}
__device__ inline unsigned row16_max(unsigned x) {              // over the 16 lanes of a row of lanes, in all of them
#define TSR_MAX_DPP(ctrl) x = max(x, (unsigned)__builtin_amdgcn_update_dpp((int)x, (int)x, ctrl, 0xf, 0xf, false))
    TSR_MAX_DPP(0x121); TSR_MAX_DPP(0x122); TSR_MAX_DPP(0x124); TSR_MAX_DPP(0x128);   // row_ror 1, 2, 4, 8
#undef TSR_MAX_DPP
    return x;
}

template <int FMT, int ROWS, bool X16>
__global__ __launch_bounds__(256) void fp8_quantize_kernel(const QuantizeArgs a) {
    constexpr int PITCH = 136;
    __shared__ __attribute__((aligned(16))) unsigned char turned[128 * PITCH];
    __shared__ unsigned col_max[4][128];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row0 = blockIdx.y * 128, col0 = blockIdx.x * 128;
    const int r0 = row0 + (tid >> 4) * 8, c0 = col0 + (tid & 15) * 8;
    float x[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool row_in = r0 + i < a.m;
        const long long at = (long long)(r0 + i) * a.ldx + c0;
        if (row_in && c0 + 8 <= a.n) {
            if constexpr (X16) {
                const u16x8_any h = *(const u16x8_any*)((const unsigned short*)a.X + at);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[i][j] = __builtin_bit_cast(float, (unsigned)h[j] << 16);
            } else {
                const f32x4_any lo = *(const f32x4_any*)((const float*)a.X + at), hi = *(const f32x4_any*)((const float*)a.X + at + 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) { x[i][j] = lo[j]; x[i][4 + j] = hi[j]; }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[i][j] = 0.0f;
                if (row_in && c0 + j < a.n)
                    x[i][j] = X16 ? __builtin_bit_cast(float, (unsigned)((const unsigned short*)a.X)[at + j] << 16) : ((const float*)a.X)[at + j];
            }
        }
    }
    // the largest of each row and column of the thread's 8 x 8
    unsigned rmax[8], cmax[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) cmax[j] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        rmax[i] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned b = finite_abs_bits(x[i][j]);
            rmax[i] = max(rmax[i], b); cmax[j] = max(cmax[j], b);
        }
    }
    int tile_byte = 0;
    if constexpr (ROWS == 128) {
        unsigned t = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) t = max(t, rmax[i]);
        t = wave_max(t);
        if (lane == 0) col_max[0][wave] = t;
        __syncthreads();
        tile_byte = fp8_scale_byte<FMT>(max(max(col_max[0][0], col_max[0][1]), max(col_max[0][2], col_max[0][3])));
    } else if (a.Qt) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            cmax[j] = max(cmax[j], (unsigned)__shfl_xor((int)cmax[j], 16));
            cmax[j] = max(cmax[j], (unsigned)__shfl_xor((int)cmax[j], 32));
            if (lane < 16) col_max[wave][lane * 8 + j] = cmax[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = (tid & 15) * 8 + j;
            cmax[j] = max(max(col_max[0][c], col_max[1][c]), max(col_max[2][c], col_max[3][c]));
        }
    }
    if (a.Q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int b = ROWS == 128 ? tile_byte : fp8_scale_byte<FMT>(row16_max(rmax[i]));
            const float inv = fp8_inverse(b);
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = x[i][j] * inv;
            const u32x2 q = {fp8_encode4<FMT>(y), fp8_encode4<FMT>(y + 4)};
            if (r0 + i < a.m) {
                unsigned char* to = a.Q + (long long)(r0 + i) * a.ldq + c0;
                if (c0 + 8 <= a.n) *(u32x2*)to = q;
                else
#pragma unroll
                    for (int j = 0; j < 8; ++j) if (c0 + j < a.n) to[j] = (unsigned char)(q[j >> 2] >> (8 * (j & 3)));
                if (ROWS == 1 && (tid & 15) == 0) a.S[(long long)(r0 + i) * a.lds + blockIdx.x] = (unsigned char)b;
            }
        }
    }
    if (ROWS == 128 && tid == 0) {
        if (a.Q) a.S[(long long)blockIdx.y * a.lds + blockIdx.x] = (unsigned char)tile_byte;
        if (a.Qt) a.St[(long long)blockIdx.x * a.ldst + blockIdx.y] = (unsigned char)tile_byte;
    }
    if (!a.Qt) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int b = ROWS == 128 ? tile_byte : fp8_scale_byte<FMT>(cmax[j]);
        const float inv = fp8_inverse(b);
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i][j] * inv;
        const u32x2 q = {fp8_encode4<FMT>(y), fp8_encode4<FMT>(y + 4)};
        *(u32x2*)(turned + ((tid & 15) * 8 + j) * PITCH + (tid >> 4) * 8) = q;
        if (ROWS == 1 && tid < 16 && c0 + j < a.n) a.St[(long long)(c0 + j) * a.ldst + blockIdx.y] = (unsigned char)b;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 8; ++u) {                               // 16 threads a row of 128 bytes
        const int c = u * 16 + (tid >> 4), r = (tid & 15) * 8;
        if (col0 + c >= a.n) continue;
        const u32x2 q = *(const u32x2*)(turned + c * PITCH + r);
        unsigned char* to = a.Qt + (long long)(col0 + c) * a.ldqt + row0 + r;
        if (row0 + r + 8 <= a.m) *(u32x2*)to = q;
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) if (row0 + r + j < a.m) to[j] = (unsigned char)(q[j >> 2] >> (8 * (j & 3)));
    }
}

hipError_t launch_fp8_quantize(const QuantizeArgs& a, int fmt, int block_rows, hipStream_t stream) {
    const dim3 grid((unsigned)((a.n + 127) / 128), (unsigned)((a.m + 127) / 128));
#define TSR_Q(F, R, X) hipLaunchKernelGGL((fp8_quantize_kernel<F, R, X>), grid, dim3(256), 0, stream, a)
    const int v = (fmt == FP8_E5M2 ? 4 : 0) + (block_rows == 128 ? 2 : 0) + (a.x_bf16 ? 1 : 0);
    switch (v) {
        case 0: TSR_Q(FP8_E4M3, 1, false); break;
        case 1: TSR_Q(FP8_E4M3, 1, true); break;
        case 2: TSR_Q(FP8_E4M3, 128, false); break;
        case 3: TSR_Q(FP8_E4M3, 128, true); break;
        case 4: TSR_Q(FP8_E5M2, 1, false); break;
        case 5: TSR_Q(FP8_E5M2, 1, true); break;
        case 6: TSR_Q(FP8_E5M2, 128, false); break;
        default: TSR_Q(FP8_E5M2, 128, true); break;
    }
#undef TSR_Q
    return hipGetLastError();
}

// ------------------------------------------------------------------ product
// The scaled matrix instruction multiplies 16 x 128 by 128 x 16 and takes a scale byte for each row and column, so a block of
// 128 along the contraction is one instruction and its scales cost nothing.  The rows of B are the instruction's rows and
// those of A its columns: a lane then holds four neighbouring elements of a row of C.
typedef __amdgpu_buffer_rsrc_t rsrc_t;
__device__ inline rsrc_t make_rsrc(const void* p, long long bytes) {
    const int n = (bytes > 0x7fffffffLL) ? 0x7fffffff : (int)bytes;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, n, 0x00020000);
}

// zeros for the bytes at and beyond `valid` of 32
__device__ inline i32x8 keep_bytes(i32x8 x, int valid) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int left = valid - 4 * j;
        const unsigned mask = left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
        x[j] &= (int)mask;
    }
    return x;
}

// Fragments straight from memory: 16 rows of B and 16 FM of A for a workgroup, whose four waves share the blocks of the
// contraction among them and add up through LDS in a fixed order.
template <int FA, int FB, int FM>
__global__ __launch_bounds__(256) void fp8_direct_kernel(const Fp8Args g) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int l16 = lane & 15, quad = lane >> 4;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * (16 * FM);
    const int k16 = (g.k + 15) & ~15, blocks = (g.k + 127) >> 7;
    const int brow = min(n0 + l16, g.b.rows - 1);
    const rsrc_t rb = make_rsrc(g.b.q + n0 * g.b.ld, (long long)(min(16, g.b.rows - n0) - 1) * g.b.ld + k16);
    const rsrc_t ra = make_rsrc(g.a.q + m0 * g.a.ld, (long long)(min(16 * FM, g.a.rows - m0) - 1) * g.a.ld + k16);
    const unsigned char* sb = g.b.scale + (long long)(brow >> g.b.shift) * g.b.ld_scale;
    const unsigned ob = (unsigned)((brow - n0) * g.b.ld) + quad * 32;
    unsigned oa[FM];
    const unsigned char* sa[FM];
#pragma unroll
    for (int f = 0; f < FM; ++f) {
        const int r = min(m0 + f * 16 + l16, g.a.rows - 1);
        oa[f] = (unsigned)((r - m0) * g.a.ld) + quad * 32;
        sa[f] = g.a.scale + (long long)(r >> g.a.shift) * g.a.ld_scale;
    }
    auto fetch = [](rsrc_t r, unsigned at) -> i32x8 {
        const u32x4 lo = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)at, 0, 0));
        const u32x4 hi = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)(at + 16), 0, 0));
        return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
    };
    f32x4 acc[FM];
#pragma unroll
    for (int f = 0; f < FM; ++f) acc[f] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int kb = wave; kb < blocks; kb += 4) {
        const unsigned k0 = (unsigned)kb * 128;
        i32x8 b = fetch(rb, ob + k0), x[FM];
        const int scale_b = sb[kb];
        int scale_a[FM];
#pragma unroll
        for (int f = 0; f < FM; ++f) { x[f] = fetch(ra, oa[f] + k0); scale_a[f] = sa[f][kb]; }
        const int valid = g.k - (int)k0 - quad * 32;
        if (g.k - (int)k0 < 128) {
            b = keep_bytes(b, valid);
#pragma unroll
            for (int f = 0; f < FM; ++f) x[f] = keep_bytes(x[f], valid);
        }
#pragma unroll
        for (int f = 0; f < FM; ++f)
            acc[f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, x[f], acc[f], FB, FA, 0, scale_b, 0, scale_a[f]);
    }
    __shared__ __attribute__((aligned(16))) f32x4 part[4][FM][64];
#pragma unroll
    for (int f = 0; f < FM; ++f) part[wave][f][lane] = acc[f];
    __syncthreads();
    for (int f = wave; f < FM; f += 4) {
        const f32x4 c = (part[0][f][lane] + part[1][f][lane]) + (part[2][f][lane] + part[3][f][lane]);
        const int m = m0 + f * 16 + l16, n = n0 + quad * 4;
        if (m >= g.a.rows) continue;
        const long long at = (long long)m * g.ldc + n;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (n + i >= g.b.rows) continue;
            ((__bf16*)g.C)[at + i] = (__bf16)c[i];
        }
    }
}

hipError_t launch_fp8_matmul(const Fp8Args& a, int fmt_a, int fmt_b, hipStream_t stream) {
    const dim3 grid((unsigned)((a.b.rows + 15) / 16), (unsigned)((a.a.rows + 63) / 64));
    if (fmt_a == FP8_E4M3 && fmt_b == FP8_E4M3) hipLaunchKernelGGL((fp8_direct_kernel<0, 0, 4>), grid, dim3(256), 0, stream, a);
    else if (fmt_a == FP8_E4M3) hipLaunchKernelGGL((fp8_direct_kernel<0, 1, 4>), grid, dim3(256), 0, stream, a);
    else if (fmt_b == FP8_E4M3) hipLaunchKernelGGL((fp8_direct_kernel<1, 0, 4>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((fp8_direct_kernel<1, 1, 4>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace tsr
