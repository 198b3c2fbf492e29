// 8-bit floating point with a power of two as the scale of each block of 128: the quantiser, and C = A B^T on the scaled
// matrix instructions of gfx950.
#include <type_traits>

#include "device_lds.h"
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
typedef __attribute__((ext_vector_type(4), aligned(2))) unsigned int u32x4_any;

// ------------------------------------------------------------------ quantiser
// A workgroup takes 128 x 128 elements of X, a thread 8 rows x 8 columns of them: X is read once, whichever outputs are
// wanted.  Blocks of one row: the largest of a row of the tile is found among the 16 threads of a row (moves within 16
// lanes), that of a column among the threads of a column (two moves across the wave, then LDS).  The transposed tile goes
// through LDS, whose rows are padded by 8 bytes.
// Bound by memory: 16384 x 8192 bf16 both ways 120 us, 4.5 TB/s (a copy: 5.1), fp32 160 us, 5.0 TB/s; 16384 x 2048 bf16 31 us,
// 4.3 TB/s.  All loads of a thread are in flight before the first is looked at.
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
    const int tiles_n = (a.n + 127) >> 7, tile_m = blockIdx.x / tiles_n, tile_n = blockIdx.x - tile_m * tiles_n;
    const int row0 = tile_m * 128, col0 = tile_n * 128;
    const int r0 = row0 + (tid >> 4) * 8, c0 = col0 + (tid & 15) * 8;
    // bf16 values stay as they came, in 32 registers and not 64: three waves on a SIMD and not two (16384 x 2048 both ways: 36 -> 31 us)
    u32x4 raw[8];
    float x[X16 ? 1 : 8][8];
    auto value = [&](int i, int j) -> float {
        if constexpr (X16) {
            const unsigned w = raw[i][j >> 1];
            return __builtin_bit_cast(float, j & 1 ? w & 0xffff0000u : w << 16);
        } else {
            return x[i][j];
        }
    };
    auto forget = [&]() {                                    // values widened for what came before are not kept for what follows
        if constexpr (X16)
#pragma unroll
            for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(raw[i]));
    };
    if (X16 && row0 + 128 <= a.m && col0 + 128 <= a.n) {     // all loads in flight before the first is looked at
#pragma unroll
        for (int i = 0; i < 8; ++i) raw[i] = *(const u32x4_any*)((const unsigned short*)a.X + (long long)(r0 + i) * a.ldx + c0);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool row_in = r0 + i < a.m;
            const long long at = (long long)(r0 + i) * a.ldx + c0;
            if constexpr (X16) {
                const unsigned short* from = (const unsigned short*)a.X + at;
                raw[i] = u32x4{0, 0, 0, 0};
                if (row_in && c0 + 8 <= a.n) raw[i] = *(const u32x4_any*)from;
                else
#pragma unroll
                    for (int j = 0; j < 8; ++j) if (row_in && c0 + j < a.n) raw[i][j >> 1] |= (unsigned)from[j] << (16 * (j & 1));
            } else {
                const float* from = (const float*)a.X + at;
                if (row_in && c0 + 8 <= a.n) {
                    const f32x4_any lo = *(const f32x4_any*)from, hi = *(const f32x4_any*)(from + 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) { x[i][j] = lo[j]; x[i][4 + j] = hi[j]; }
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        x[i][j] = 0.0f;
                        if (row_in && c0 + j < a.n) x[i][j] = from[j];
                    }
                }
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
            const unsigned b = finite_abs_bits(value(i, j));
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
    forget();
    if (a.Q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int b = ROWS == 128 ? tile_byte : fp8_scale_byte<FMT>(row16_max(rmax[i]));
            const float inv = fp8_inverse(b);
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = value(i, j) * inv;
            const u32x2 q = {fp8_encode4<FMT>(y), fp8_encode4<FMT>(y + 4)};
            if (r0 + i < a.m) {
                unsigned char* to = a.Q + (long long)(r0 + i) * a.ldq + c0;
                if (c0 + 8 <= a.n) *(u32x2*)to = q;
                else
#pragma unroll
                    for (int j = 0; j < 8; ++j) if (c0 + j < a.n) to[j] = (unsigned char)(q[j >> 2] >> (8 * (j & 3)));
                if (ROWS == 1 && (tid & 15) == 0) a.S[(long long)(r0 + i) * a.lds + tile_n] = (unsigned char)b;
            }
        }
    }
    if (ROWS == 128 && tid == 0) {
        if (a.Q) a.S[(long long)tile_m * a.lds + tile_n] = (unsigned char)tile_byte;
        if (a.Qt) a.St[(long long)tile_n * a.ldst + tile_m] = (unsigned char)tile_byte;
    }
    if (!a.Qt) return;
    forget();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int b = ROWS == 128 ? tile_byte : fp8_scale_byte<FMT>(cmax[j]);
        const float inv = fp8_inverse(b);
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = value(i, j) * inv;
        const u32x2 q = {fp8_encode4<FMT>(y), fp8_encode4<FMT>(y + 4)};
        *(u32x2*)(turned + ((tid & 15) * 8 + j) * PITCH + (tid >> 4) * 8) = q;
        if (ROWS == 1 && tid < 16 && c0 + j < a.n) a.St[(long long)(c0 + j) * a.ldst + tile_m] = (unsigned char)b;
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
    const dim3 grid((unsigned)(((a.n + 127ll) / 128) * ((a.m + 127ll) / 128)));
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
// contraction among them and add up through LDS in a fixed order.  For few rows (or columns) of one operand: bound by reading the
// other, which nobody shares.  1 x 5461 x 2048: 4.6 us, of which the 11 MB of B take 2.2 at the rate of a copy, the rest is the
// launch and the first access; 32 rows: 8.8 us.
template <int FA, int FB, int FM>
__global__ __launch_bounds__(256) void fp8_direct_kernel(const Fp8Args g) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int l16 = lane & 15, quad = lane >> 4;
    const int n0 = blockIdx.x % g.groups_n * 16, m0 = blockIdx.x / g.groups_n * (16 * FM);
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
    // N blocks of this wave from kb on: all loads first, so that a few hundred rows of B keep the memory busy
    auto blocks_from = [&](int kb, auto number) {
        constexpr int N = decltype(number)::value;
        i32x8 b[N], x[N][FM];
        int scale_b[N], scale_a[N][FM];
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const unsigned k0 = (unsigned)(kb + 4 * u) * 128;
            b[u] = fetch(rb, ob + k0);
            scale_b[u] = sb[kb + 4 * u];
#pragma unroll
            for (int f = 0; f < FM; ++f) { x[u][f] = fetch(ra, oa[f] + k0); scale_a[u][f] = sa[f][kb + 4 * u]; }
        }
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int left = g.k - (kb + 4 * u) * 128;
            if (left < 128) {
                b[u] = keep_bytes(b[u], left - quad * 32);
#pragma unroll
                for (int f = 0; f < FM; ++f) x[u][f] = keep_bytes(x[u][f], left - quad * 32);
            }
#pragma unroll
            for (int f = 0; f < FM; ++f)
                acc[f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[u], x[u][f], acc[f], FB, FA, 0, scale_b[u], 0, scale_a[u][f]);
        }
    };
    constexpr int AHEAD = FM == 1 ? 4 : 2;
    int kb = wave;
    for (; kb + 4 * (AHEAD - 1) < blocks; kb += 4 * AHEAD) blocks_from(kb, std::integral_constant<int, AHEAD>{});
    for (; kb < blocks; kb += 4) blocks_from(kb, std::integral_constant<int, 1>{});
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

// ------------------------------------------------------------------ product, tiles through LDS
// A workgroup of four waves (2 x 2) computes 128 x 128 elements of C, each wave 2 x 2 tiles of 32 x 32, in blocks of 128 along
// the contraction (two instructions deep); two workgroups a compute unit.  Rows of A and B go from memory straight into LDS, no
// registers between, 128 bytes of a row at a time: whole cache lines (in steps of 64 bytes every line came twice, its first half
// long gone when the second was asked for).  Two buffers: block p + 2 is asked for in the second step of block p, when all
// fragments of p are in registers, and is needed in the second step of p + 1.
// LDS rows are 128 bytes, eight chunks of 16; chunk c of row r sits at c ^ ((r >> 1) & 7), which keeps the fragment reads (16
// lanes at a time) free of bank conflicts.  The 32 rows of B of a tile are kept in the order in which the instruction hands its
// results out, so that a lane ends up with 16 neighbouring elements of a row of C: row 8 j + 4 h + i of the instruction is row
// 16 h + 4 j + i of B.
// Scale bytes go through LDS too: for every block the word that holds its byte, again for each of its four blocks, so that
// the loop is free of branches: the compiler moves matrix instructions across those.
// Bound by the path from memory to LDS: a unit takes some 53 bytes a cycle there, and a tile of this size wants 32 KB for every
// 512 cycles of its matrix instructions.  2736 x 1024 x 12345 in two pieces: 73 us, 0.95 PFLOP/s, and 6 for their sum (176 tiles
// would leave 80 units idle); 2048 x 2048 x 2048: 14 us, 1.2 PFLOP/s.  Waves of 4 x 4 tiles of 16 x 16, which read a whole block's
// fragments before they multiply, need fewer instructions but do not read beside the multiplication: 17 us.
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;

__device__ inline i32x4 lds_rsrc(const void* p, long long bytes) {
    const unsigned long long a = (unsigned long long)p;
    return i32x4{(int)(unsigned)a, (int)((unsigned)(a >> 32) & 0xffffu), (int)(bytes > 0x7fffffffLL ? 0x7fffffffLL : bytes), 0x00020000};
}
// 16 (or 4) bytes a lane from `rsrc` + voff to LDS at `to` + 16 (or 4) times the lane.  Not known to the compiler's counting
// of loads in flight: whoever reads the place waits by wait_loads and a barrier.  m0 is set where it is used and read one wait
// state later (s_nop).  It is a reserved register, which the compiler lets nobody declare as overwritten; it keeps nothing there for
// itself, but sets it before each instruction of its own that reads it, and this file has none (no index into registers, no message,
// no load into LDS by a builtin).
__device__ inline void load_lds16(i32x4 rsrc, unsigned voff, unsigned to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(voff), "s"(rsrc) : "memory");
}
__device__ inline void load_lds4(i32x4 rsrc, unsigned voff, unsigned to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(to), "v"(voff), "s"(rsrc) : "memory");
}
template <int N> __device__ inline void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
#define TSR_PIN __builtin_amdgcn_sched_barrier(0)

struct TileLds {
    static constexpr int ROWS = 256, BUF = ROWS * 128;
    static constexpr int SCALES = 2 * BUF, BYTES = SCALES + 2 * ROWS * 4;
};

// With more than one piece (blockIdx.y) of the contraction each writes its fp32 sums, and fp8_join_kernel adds them up.
template <int FA, int FB>
__global__ __launch_bounds__(256, 2) void fp8_tile_kernel(const Fp8Args whole_k) {
    Fp8Args g = whole_k;
    const long long k_from = (long long)blockIdx.y * g.chunk;
    g.a.q += k_from; g.b.q += k_from;
    g.a.scale += k_from >> 7; g.b.scale += k_from >> 7;
    g.k = (int)min((long long)g.chunk, g.k - k_from);
    using L = TileLds;
    constexpr int FM = 2, FN = 2, TM = 64 * FM, TN = 64 * FN, NF = FM + FN, NM = FM * FN;
    constexpr unsigned OUT = 0x80000000u;                    // an offset beyond every operand: no access
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, h = lane >> 5, wm = wave >> 1, wn = wave & 1;

    // The tile.  Workgroups go round the 8 XCDs; each XCD takes a run of neighbouring tiles, in bands of 8 rows of tiles, so that
    // the tiles at work together share rows of A and B in its L2.
    const int tiles_m = (g.a.rows + TM - 1) / TM, tiles_n = (g.b.rows + TN - 1) / TN, tiles = tiles_m * tiles_n;
    const int xcd = blockIdx.x & 7, per = tiles >> 3, more = tiles & 7;
    const int at = xcd * per + min(xcd, more) + (int)(blockIdx.x >> 3);
    const int band = at / (8 * tiles_n), in_band = at - band * 8 * tiles_n, band_rows = min(8, tiles_m - band * 8);
    const int m0 = (band * 8 + in_band % band_rows) * TM, n0 = in_band / band_rows * TN;

    const int k16 = (g.k + 15) & ~15, np = (g.k + 127) >> 7;
    const int ma = min(TM, g.a.rows - m0) - 1, nb = min(TN, g.b.rows - n0) - 1;      // last row of each operand's tile
    const i32x4 ra = lds_rsrc(g.a.q + m0 * g.a.ld, ma * g.a.ld + k16);
    const i32x4 rb = lds_rsrc(g.b.q + n0 * g.b.ld, nb * g.b.ld + k16);
    const int sk = ((g.k + 511) >> 9) * 4;                   // scale bytes of a row in whole words, which the row's pitch holds
    const int sa0 = m0 >> g.a.shift, sb0 = n0 >> g.b.shift;
    const i32x4 rsa = lds_rsrc(g.a.scale + sa0 * g.a.ld_scale, (((m0 + ma) >> g.a.shift) - sa0) * g.a.ld_scale + sk);
    const i32x4 rsb = lds_rsrc(g.b.scale + sb0 * g.b.ld_scale, (((n0 + nb) >> g.b.shift) - sb0) * g.b.ld_scale + sk);

    // Loads of a block: wave w brings rows 16 FM w .. of A and 16 FN w .. of B, 8 rows an instruction.  Rows beyond the operand
    // repeat its last one; nothing of them is stored.
    auto n_of = [](int r) { return (r & ~31) + ((r & 4) << 2) + ((r >> 3) & 3) * 4 + (r & 3); };
    unsigned off[2 * NF];
#pragma unroll
    for (int x = 0; x < 2 * NF; ++x) {
        const int r = (x < 2 * FM ? wave * 16 * FM + x * 8 : wave * 16 * FN + (x - 2 * FM) * 8) + (lane >> 3);
        const int c = ((lane & 7) ^ ((r >> 1) & 7)) * 16;
        off[x] = (x < 2 * FM ? (unsigned)(min(r, ma) * g.a.ld) : (unsigned)(min(n_of(r), nb) * g.b.ld)) + c;
    }
    const unsigned base = (unsigned)(unsigned long long)(__attribute__((address_space(3))) unsigned char*)lds;
    auto load_one = [&](int p, int x) {                      // part x of block p into its buffer
        const unsigned to = base + (p & 1) * L::BUF + (x < 2 * FM ? wave * 16 * FM + x * 8 : TM + wave * 16 * FN + (x - 2 * FM) * 8) * 128;
        load_lds16(x < 2 * FM ? ra : rb, p < np ? off[x] + (unsigned)p * 128 : OUT, to);
    };
    // Scales of block p: a word for each row of the tile's A rows, then of its B rows; wave w brings 64 SL of them.
    constexpr int SL = (L::ROWS + 255) / 256;
    static_assert(L::ROWS % 256 == 0 && TM % 64 == 0, "all lanes of an instruction on one side");
    unsigned soff[SL];
#pragma unroll
    for (int x = 0; x < SL; ++x) {
        const int r = (wave * SL + x) * 64 + lane;
        soff[x] = r < TM ? (unsigned)((((m0 + min(r, ma)) >> g.a.shift) - sa0) * g.a.ld_scale)
                         : (unsigned)((((n0 + min(n_of(r - TM), nb)) >> g.b.shift) - sb0) * g.b.ld_scale);
    }
    auto load_scales = [&](int p) {
#pragma unroll
        for (int x = 0; x < SL; ++x) {
            const int r = (wave * SL + x) * 64;
            const unsigned to = base + L::SCALES + ((p & 1) * L::ROWS + r) * 4;
            load_lds4(r < TM ? rsa : rsb, p < np ? soff[x] + (p & ~3) : OUT, to);
        }
    };

    f32x16 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    i32x8 F[2][NF];
    unsigned sn[NF];
    int s[NF];
    // where this lane's two chunks of fragment f of step slot lie in a buffer: 4 slot + 2 h and the next, by the key of its row
    const int key = (l32 >> 1) & 7;
    const int fa = (wm * FM * 32 + l32) * 128, fb = (TM + wn * FN * 32 + l32) * 128;
    const int c0 = ((2 * h) ^ key) * 16, c1 = ((2 * h + 1) ^ key) * 16;
    auto read = [&](int slot, int p, int f) {
        const unsigned char* from = lds + (p & 1) * L::BUF + (f < FM ? fa + f * 4096 : fb + (f - FM) * 4096);
        F[slot][f] = __builtin_shufflevector(*(const i32x4*)(from + (c0 ^ slot * 64)), *(const i32x4*)(from + (c1 ^ slot * 64)), 0, 1, 2, 3, 4, 5, 6, 7);
    };
    auto read_scale = [&](int p, int f) {
        const int r = f < FM ? wm * FM * 32 + f * 32 + l32 : TM + wn * FN * 32 + (f - FM) * 32 + l32;
        sn[f] = *(const unsigned*)(lds + L::SCALES + ((p & 1) * L::ROWS + r) * 4);
    };

#pragma unroll
    for (int p = 0; p < 2; ++p) {
        load_scales(p);
#pragma unroll
        for (int x = 0; x < 2 * NF; ++x) load_one(p, x);
    }
    wait_loads<2 * NF + SL>();                               // block 0
    __builtin_amdgcn_s_barrier();
    TSR_PIN;
#pragma unroll
    for (int f = 0; f < NF; ++f) { read(0, 0, f); read_scale(0, f); }

    // Both steps of block p.  TAIL: what lies beyond k is not part of the sum.
    auto block = [&](int p, auto tail) {
        constexpr bool TAIL = decltype(tail)::value;
#pragma unroll
        for (int slot = 0; slot < 2; ++slot) {
            if (slot == 0) {
#pragma unroll
                for (int f = 0; f < NF; ++f) s[f] = (int)(sn[f] >> ((p & 3) * 8));
            } else {
                // block p + 1 has landed, everybody's, and everybody has the fragments of block p
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                wait_loads<0>();
                __builtin_amdgcn_s_barrier();
                TSR_PIN;
                load_scales(p + 2);
            }
            if constexpr (TAIL) {
#pragma unroll
                for (int f = 0; f < NF; ++f) F[slot][f] = keep_bytes(F[slot][f], g.k - p * 128 - slot * 64 - h * 32);
            }
            TSR_PIN;
#pragma unroll
            for (int q = 0; q < NM; ++q) {
                const int i = q / FN, j = q % FN;
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(F[slot][FM + j], F[slot][i], acc[i][j], FB, FA, 0, s[FM + j], 0, s[i]);
                TSR_PIN;
                // beside the multiplication: the fragments of the next step, and in the second step the loads of block p + 2
                // and the scales of block p + 1
#pragma unroll
                for (int f = q * NF / NM; f < (q + 1) * NF / NM; ++f) {
                    if (slot == 0) read(1, p, f);
                    else { read(0, p + 1, f); read_scale(p + 1, f); }
                }
                if (slot == 1) {
#pragma unroll
                    for (int x = q * 2 * NF / NM; x < (q + 1) * 2 * NF / NM; ++x) load_one(p + 2, x);
                }
                TSR_PIN;
            }
        }
    };
    const int whole = g.k >> 7;
    for (int p = 0; p < whole; ++p) block(p, std::false_type{});
    if (g.k & 127) block(whole, std::true_type{});
    wait_loads<0>();                                         // nothing may land after this workgroup's LDS is another's

    if (g.partial) {
        float* part = g.partial + (long long)blockIdx.y * g.a.rows * g.ldp;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int m = m0 + wm * FM * 32 + i * 32 + l32;
            if (m >= g.a.rows) continue;
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const int n = n0 + wn * FN * 32 + j * 32 + h * 16 + e;
                    if (n < g.b.rows) *(f32x4*)(part + (long long)m * g.ldp + n) = f32x4{acc[i][j][e], acc[i][j][e + 1], acc[i][j][e + 2], acc[i][j][e + 3]};
                }
        }
        return;
    }
    const bool vec = ((unsigned long long)g.C & 15) == 0 && (g.ldc & 7) == 0;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int m = m0 + wm * FM * 32 + i * 32 + l32;
        if (m >= g.a.rows) continue;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int n = n0 + wn * FN * 32 + j * 32 + h * 16;
            __bf16* to = (__bf16*)g.C + (long long)m * g.ldc + n;
            typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
            if (vec && n + 16 <= g.b.rows) {
                bf16x8 lo, hi;
#pragma unroll
                for (int e = 0; e < 8; ++e) { lo[e] = (__bf16)acc[i][j][e]; hi[e] = (__bf16)acc[i][j][8 + e]; }
                *(bf16x8*)to = lo;
                *(bf16x8*)(to + 8) = hi;
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) if (n + e < g.b.rows) to[e] = (__bf16)acc[i][j][e];
            }
        }
    }
}

// ------------------------------------------------------------------ product, two groups of waves in turn
// 256 x 256 elements of C by eight waves, 128 x 64 each, in blocks of 128 along the contraction, one workgroup a compute unit
// that walks its share of the tiles.  Each SIMD holds a wave of either group, and the groups take turns, a barrier between the
// phases: while one multiplies (32 instructions of 16 x 16 x 128, 1024 cycles) the other moves its fragments of the next
// block from LDS into registers, so the matrix unit always has a wave that does nothing else.
//   phase 2 q      group 0 reads block q,        group 1 multiplies block q - 1
//   phase 2 q + 1  group 0 multiplies block q,   group 1 reads block q
// In phase 2 q block q + 1 is asked for (A by group 0, B by group 1) into the buffer that block q - 1 has left; it is needed two
// phases later.  Blocks are counted across tiles: the first block of the next tile is on its way while the last one of this
// tile is multiplied, and a group begins to write its part of C while the other multiplies (the wait for its next loads is one for
// these stores too).
// LDS rows are 128 bytes (whole cache lines), eight chunks of 16; chunk c of row r sits at c ^ ((r >> 1) & 7): 16 lanes that
// read the same chunk of 16 rows meet no bank twice.  The 64 rows of B of a wave are kept in the order in which the instruction
// hands its results out: a lane ends up with 16 neighbouring elements of a row of C, 16 lanes apart with a whole line of it.
// Scale bytes go through LDS as the words that hold them, one for every row, once in four blocks: a wave keeps its words in
// registers and shifts them on.
// Bound by power: 8192 x 32000 x 2048 takes 497 us, 2.16 PFLOP/s; 8192^3 414 us, 2.65 PFLOP/s.  Of two kernels whose blocks take
// 1100 and 1500 cycles the shorter ran at 1.7 GHz and the longer at 2.1, in the same time.  C costs 7 us a tile beside the 16
// blocks of k = 2048.  Other forms, 8192^3: four waves of 128 x 128 each with their sums in the accumulation registers 440 us, with
// loads spread over the block 437; four waves of 32 x 32 x 64 instructions 489.
struct WideLds {
    static constexpr int BUF = 512 * 128, SCALES = 2 * BUF, BYTES = SCALES + 2 * 512 * 4;
};

template <int FA, int FB>
__global__ __launch_bounds__(512, 2) void fp8_wide_kernel(const Fp8Args g) {
    using L = WideLds;
    constexpr unsigned OUT = 0x80000000u;                    // an offset beyond every operand: no access
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int group = wave >> 2, w4 = wave & 3;

    // Tiles: round r of the workgroups takes a run of neighbouring tiles, each XCD (workgroups go round the eight) a run within
    // it, in bands of 8 rows of tiles, so that the tiles at work on an XCD share rows of A and B in its L2.
    const int tiles_m = (g.a.rows + 255) >> 8, tiles_n = (g.b.rows + 255) >> 8, tiles = tiles_m * tiles_n;
    const int first = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
    if (first >= tiles) return;
    auto place = [&](int at, int& m0, int& n0) {
        const int band = at / (8 * tiles_n), in_band = at - band * 8 * tiles_n, rows = min(8, tiles_m - band * 8);
        m0 = (band * 8 + in_band % rows) << 8;
        n0 = (in_band / rows) << 8;
    };
    const int k16 = (g.k + 15) & ~15, np = (g.k + 127) >> 7, sk = ((g.k + 511) >> 9) * 4;
    const int tail = (g.k & 127) ? np - 1 : -1;
    const unsigned base = (unsigned)(unsigned long long)(__attribute__((address_space(3))) unsigned char*)lds;

    // ---- the loader of a group: its operand's 256 rows of the block after the last one it brought, 8 instructions a wave of 8
    // rows each, and their scales.  Rows beyond the operand repeat its last one; nothing of them is stored.
    const Fp8Operand& x = group ? g.b : g.a;
    auto n_of = [](int r) { return (r & ~63) + ((r >> 2) & 3) * 16 + ((r >> 4) & 3) * 4 + (r & 3); };
    auto again = [](int v) { asm volatile("" : "+v"(v)); return v; };        // what follows from v is not kept in registers
    auto chunk_of = [&](int lane) { return ((lane & 7) ^ (((w4 * 8 + (lane >> 3)) >> 1) & 7)) * 16; };
    const int lr = w4 * 8 + (lane >> 3);
    const unsigned row_off = (unsigned)((group ? n_of(lr) : lr) * x.ld) + chunk_of(lane);
    const unsigned step0 = (unsigned)x.ld * (group ? 8 : 32), step1 = (unsigned)x.ld * 64;      // from part 2 u to 2 u + 1, to 2 u + 2
    int l_at = first, l_p = 0, l_buf = 0;
    i32x4 l_rsrc, l_srsrc;
    unsigned l_lim, l_soff;
    auto open_tile = [&]() {
        int m0, n0;
        place(min(l_at, tiles - 1), m0, n0);
        const int x0 = group ? n0 : m0, last = min(256, x.rows - x0) - 1, s0 = x0 >> x.shift;
        l_rsrc = lds_rsrc(x.q + x0 * x.ld, last * x.ld + k16);
        const int ln = again(lane), sr = group ? n_of(w4 * 64 + ln) : w4 * 64 + ln;
        l_lim = (unsigned)(last * x.ld) + chunk_of(ln);
        l_srsrc = lds_rsrc(x.scale + s0 * x.ld_scale, (((x0 + last) >> x.shift) - s0) * x.ld_scale + sk);
        l_soff = (unsigned)((((x0 + min(sr, last)) >> x.shift) - s0) * x.ld_scale);
    };
    auto load_part = [&](int u) {                            // u < 8: rows; 8: scales
        const bool live = l_at < tiles;
        if (u < 8) {
            const unsigned r = min((unsigned)again((int)row_off) + (unsigned)(u >> 1) * step1 + (unsigned)(u & 1) * step0, l_lim);
            load_lds16(l_rsrc, live ? r + (unsigned)l_p * 128 : OUT, base + l_buf * L::BUF + (group * 256 + u * 32 + w4 * 8) * 128);
        } else {
            load_lds4(l_srsrc, live && (l_p & 3) == 0 ? l_soff + l_p : OUT, base + L::SCALES + (l_buf * 512 + group * 256 + w4 * 64) * 4);
        }
    };
    auto next_block = [&]() {
        l_buf ^= 1;
        if (++l_p == np) { l_p = 0; l_at += gridDim.x; open_tile(); }
    };

    // ---- fragments: 32 bytes a lane, chunks 2 quad and 2 quad + 1 of its row
    i32x8 A[8], B[4];
    int sa[8], sb[4];                                        // scales: this block's byte lowest, those of the word's later blocks above
    auto read = [&](int buf, int p) {
        const int ln = again(lane), row = ln & 15, row_a = group * 128 + row, row_b = 256 + w4 * 64 + row;
        const int c0 = ((2 * (ln >> 4)) ^ ((row >> 1) & 7)) * 16, c1 = c0 ^ 16;
        const unsigned char* at = lds + buf * L::BUF;
        auto fetch = [&](const unsigned char* from) {
            return __builtin_shufflevector(*(const i32x4*)(from + c0), *(const i32x4*)(from + c1), 0, 1, 2, 3, 4, 5, 6, 7);
        };
        if ((p & 3) == 0) {
            const unsigned char* sc = lds + L::SCALES + buf * 2048;
#pragma unroll
            for (int j = 0; j < 4; ++j) sb[j] = *(const int*)(sc + (row_b + j * 16) * 4);
#pragma unroll
            for (int i = 0; i < 8; ++i) sa[i] = *(const int*)(sc + (row_a + i * 16) * 4);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) sb[j] = (int)((unsigned)sb[j] >> 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) sa[i] = (int)((unsigned)sa[i] >> 8);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) B[j] = fetch(at + (row_b + j * 16) * 128);
#pragma unroll
        for (int i = 0; i < 8; ++i) A[i] = fetch(at + (row_a + i * 16) * 128);
        if (p == tail) {                                     // what lies beyond k is not part of the sum
            const int valid = g.k - p * 128 - (ln >> 4) * 32;
#pragma unroll
            for (int j = 0; j < 4; ++j) B[j] = keep_bytes(B[j], valid);
#pragma unroll
            for (int i = 0; i < 8; ++i) A[i] = keep_bytes(A[i], valid);
        }
    };
    auto wait_reads = []() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };
    f32x4 acc[8][4];
    auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    };
    auto phase_end = [&]() { TSR_PIN; __builtin_amdgcn_s_barrier(); TSR_PIN; };
    // the 32 products of a block, with a group's loads among them (LOADS) or not
    auto multiply = [&](auto loads) {
        constexpr bool LOADS = decltype(loads)::value;
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(B[j], A[i], acc[i][j], FB, FA, 0, sb[j], 0, sa[i]);
            TSR_PIN;
            if constexpr (LOADS) {
                load_part(i);
                if (i == 3) load_part(8);
                TSR_PIN;
            }
        }
        __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int i = 0; i < 8; ++i)                          // the products are done here, not where the compiler would move them
            asm volatile("" : "+v"(acc[i][0]), "+v"(acc[i][1]), "+v"(acc[i][2]), "+v"(acc[i][3]));
    };
    // A result that the 256 MB of the last cache cannot hold is written past the caches (8192 x 32000 x 2048: 495 -> 482 us); a
    // smaller one is left there for whoever reads it next (8192 x 8192 x 2048: 124 us, and 136 past the caches).
    const bool large = (long long)g.a.rows * g.b.rows > (128ll << 20);
    const bool vec = ((unsigned long long)g.C & 15) == 0 && (g.ldc & 7) == 0;
    auto store = [&](int at) {
        int m0, n0;
        place(at, m0, n0);
        const int ln = again(lane), n = n0 + w4 * 64 + (ln >> 4) * 16;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int m = m0 + group * 128 + i * 16 + (ln & 15);
            typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
            bf16x8 lo, hi;
#pragma unroll
            for (int e = 0; e < 8; ++e) { lo[e] = (__bf16)acc[i][e >> 2][e & 3]; hi[e] = (__bf16)acc[i][2 + (e >> 2)][e & 3]; }
            if (m >= g.a.rows) continue;
            __bf16* to = (__bf16*)g.C + (long long)m * g.ldc + n;
            if (vec && n + 16 <= g.b.rows) {
                if (large) {
                    __builtin_nontemporal_store(lo, (bf16x8*)to);
                    __builtin_nontemporal_store(hi, (bf16x8*)(to + 8));
                } else {
                    *(bf16x8*)to = lo;
                    *(bf16x8*)(to + 8) = hi;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) if (n + e < g.b.rows) to[e] = e < 8 ? lo[e & 7] : hi[e & 7];
            }
        }
    };
    open_tile();
#pragma unroll
    for (int u = 0; u < 9; ++u) load_part(u);
    wait_loads<0>();
    phase_end();
    next_block();
    int buf = 0;
    clear();
    if (group == 0) {
        for (int at = first; at < tiles; at += gridDim.x) {
            for (int p = 0; p < np; ++p) {
                read(buf, p);
                TSR_PIN;
#pragma unroll
                for (int u = 0; u < 9; ++u) load_part(u);
                next_block();
                buf ^= 1;
                wait_reads();
                phase_end();
                multiply(std::false_type{});
                wait_loads<0>();
                phase_end();
            }
            store(at);
            clear();
        }
        phase_end();                                         // group 1 is a phase behind
    } else {
#pragma unroll
        for (int u = 0; u < 9; ++u) load_part(u);
        next_block();
        phase_end();
        for (int at = first; at < tiles; at += gridDim.x) {
            for (int p = 0; p < np; ++p) {
                read(buf, p);
                buf ^= 1;
                wait_reads();
                wait_loads<0>();
                phase_end();
                multiply(std::true_type{});
                next_block();
                phase_end();
            }
            store(at);
            clear();
        }
        wait_loads<0>();                                     // nothing may land after this workgroup's LDS is another's
    }
}

// The sum of the pieces, in their order, as bf16.
__global__ __launch_bounds__(256) void fp8_join_kernel(const Fp8Args g, int pieces) {
    const long long quads = g.ldp >> 2, at = (long long)blockIdx.x * 256 + threadIdx.x;
    if (at >= quads * g.a.rows) return;
    const long long m = at / quads;
    const int n = (int)(at - m * quads) * 4;
    const float* from = g.partial + m * g.ldp + n;
    f32x4 sum = *(const f32x4*)from;
    for (int p = 1; p < pieces; ++p) sum += *(const f32x4*)(from + (long long)p * g.a.rows * g.ldp);
    __bf16* to = (__bf16*)g.C + m * g.ldc + n;
#pragma unroll
    for (int e = 0; e < 4; ++e) if (n + e < g.b.rows) to[e] = (__bf16)sum[e];
}

namespace {
long long tiles_of(int m, int n, int t) { return ((m + t - 1ll) / t) * ((n + t - 1ll) / t); }
int direct_rows(int m) { return m <= 16 ? 16 : m <= 32 ? 32 : 64; }       // rows of A of a workgroup without tiles
}

// Tiles of 128 x 128 with the contraction in `most` pieces at most, each a multiple of 512 along k (where a word of scale bytes
// begins) but for the last; which number of them is best, and its time in us beside what every form costs.  As measured on 583
// sizes drawn at random up to 16384 x 16384 and k up to 60000, each in all its numbers of pieces: 4.5 ns for every step along k
// while the tiles have a unit each, 1.2 times that for more than 256 of them and in proportion from 420 on; several pieces cost a
// second launch, 2 us, and their sums written and read at 4 TB/s.  The choice is on average 2.5 % slower than the best one, 1.32
// times at worst (on 273 other sizes 3.0 %, 1.39 times).  512 x 512 x 8192: 31 us whole, 18 in eight pieces; 2736 x 1024 x 12345:
// 82 and 74 in two; 2048 x 2048 x 2048: 13.5 and 35 in two.
static double fp8_cut(Fp8Plan& p, int m, int n, int k, int most) {
    const double tiles = (double)tiles_of(m, n, 128);
    double least = 0.0;
    for (int s = 1; s <= most && (s - 1) * 512 < k; ++s) {
        const int chunk = s == 1 ? k : ((k + s - 1) / s + 511) / 512 * 512, pieces = (k + chunk - 1) / chunk;
        const double groups = tiles * pieces, share = groups <= 256.0 ? 1.0 : groups <= 420.0 ? 1.2 : groups / 350.0;
        const double us = chunk * 0.0045 * share + (pieces == 1 ? 0.0 : 2.0 + pieces * ((double)m * n * 8.0 / 4e6));
        if (s == 1 || us < least) { least = us; p.pieces = pieces; p.chunk = chunk; }
    }
    return least;
}

Fp8Plan fp8_plan(int m, int n, int k, int most) {
    Fp8Plan p{};
    p.pieces = 1;
    p.chunk = k;
    p.ldp = (n + 3) & ~3ll;
    // Few rows or columns: bound by reading the other operand, straight from memory (32 x 5461 x 2048: 8.8 us, in tiles 10.4; 64
    // rows: 13.8 and 11.5), unless the contraction is so long that its pieces in tiles gain more than the 4 us that they take
    // longer to begin and to join: a step along k takes 0.8 to 2.4 ns while the workgroups have a unit each, twice that at least
    // beyond (16 x 16 x 131072: 166 us, in tiles 35; 32 x 5461 x 8192: 34 and 17; 1 x 2048 x 8192: 9.6 and 10.3).  On 255 sizes drawn
    // at random the choice is 0.9 % slower than the better one on average, 1.43 times at worst (100 others: 0.6 %, 1.32 times).
    if (m <= 32 || n <= 32) {
        const int rows = direct_rows(m);
        const double groups = (double)(((n + 15ll) / 16) * ((m + rows - 1) / rows));
        const double us = k * (rows == 16 ? 0.0008 : rows == 32 ? 0.0011 : 0.0024) * (groups <= 256.0 ? 1.0 : groups <= 512.0 ? 2.0 : groups / 256.0);
        Fp8Plan tiles = p;
        tiles.kind = FP8_TILES;
        if (us > 4.0 + fp8_cut(tiles, m, n, k, most)) return tiles;
        p.kind = FP8_DIRECT;
        return p;
    }
    // 160 tiles of 256 x 256 keep enough compute units busy (2048 x 5461 x 16384, 176 tiles: 224 us, in 128 x 128 241 us; 2048 x
    // 4096 x 2048, 128 tiles: 31 and 23 us), unless half of every tile or more is empty (64 x 41000 x 2048: 27 us, in 128 x 128 18;
    // 128 x 65536 x 2048: 33 and 26; 129 x 65536 x 2048: 33 and 38)
    if (m > 128 && n > 128 && tiles_of(m, n, 256) >= 160) { p.kind = FP8_WIDE; return p; }
    p.kind = FP8_TILES;
    fp8_cut(p, m, n, k, most);
    return p;
}

template <int FA, int FB> hipError_t launch_kind(Fp8Args a, const Fp8Plan& p, hipStream_t stream) {
    if (p.kind == FP8_DIRECT) {
        const int fm = direct_rows(a.a.rows) / 16;
        a.groups_n = (int)((a.b.rows + 15ll) / 16);
        const dim3 grid((unsigned)((long long)a.groups_n * ((a.a.rows + 16 * fm - 1) / (16 * fm))));
        if (fm == 1) hipLaunchKernelGGL((fp8_direct_kernel<FA, FB, 1>), grid, dim3(256), 0, stream, a);
        else if (fm == 2) hipLaunchKernelGGL((fp8_direct_kernel<FA, FB, 2>), grid, dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((fp8_direct_kernel<FA, FB, 4>), grid, dim3(256), 0, stream, a);
        return hipGetLastError();
    }
    if (p.kind == FP8_WIDE) {
        const long long tiles = tiles_of(a.a.rows, a.b.rows, 256);
        const hipError_t e = allow_lds((const void*)fp8_wide_kernel<FA, FB>, WideLds::BYTES);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((fp8_wide_kernel<FA, FB>), dim3((unsigned)(tiles < 256 ? (tiles + 7) / 8 * 8 : 256)), dim3(512), WideLds::BYTES, stream, a);
        return hipGetLastError();
    }
    const hipError_t e = allow_lds((const void*)fp8_tile_kernel<FA, FB>, TileLds::BYTES);
    if (e != hipSuccess) return e;
    a.chunk = p.chunk;
    a.ldp = p.ldp;
    if (p.pieces == 1) a.partial = nullptr;
    hipLaunchKernelGGL((fp8_tile_kernel<FA, FB>), dim3((unsigned)tiles_of(a.a.rows, a.b.rows, 128), (unsigned)p.pieces), dim3(256), TileLds::BYTES, stream, a);
    if (p.pieces > 1)
        hipLaunchKernelGGL(fp8_join_kernel, dim3((unsigned)(((long long)a.a.rows * (a.ldp >> 2) + 255) / 256)), dim3(256), 0, stream, a, p.pieces);
    return hipGetLastError();
}

hipError_t launch_fp8_matmul(const Fp8Args& a, const Fp8Plan& p, int fmt_a, int fmt_b, hipStream_t stream) {
    if (fmt_a == FP8_E4M3 && fmt_b == FP8_E4M3) return launch_kind<0, 0>(a, p, stream);
    if (fmt_a == FP8_E4M3) return launch_kind<0, 1>(a, p, stream);
    if (fmt_b == FP8_E4M3) return launch_kind<1, 0>(a, p, stream);
    return launch_kind<1, 1>(a, p, stream);
}

}  // namespace tsr
