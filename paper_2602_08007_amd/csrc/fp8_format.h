// 8-bit floating point in blocks with a power of two as their scale (internal, device code).
//   e4m3 (OCP): 3 fraction bits, largest 448 = 1.75 * 2^8, no infinities
//   e5m2 (OCP): 2 fraction bits, largest 57344 = 1.75 * 2^15
// A block's scale 2^(b - 127) is the least one that brings its largest finite value to the type's largest at most; b is
// held as a byte, which is also the form that the matrix instructions of this GPU take a scale in.  A power of two costs
// these types nothing (they are floating), scaling by it is exact, and the choice of b turns on bits alone: 1.75 is the
// largest fraction of both types.
#pragma once
#include <hip/hip_runtime.h>

namespace tsr {

enum { FP8_E4M3 = 0, FP8_E5M2 = 1 };     // as the matrix instructions number them

typedef __attribute__((ext_vector_type(2))) float fp8_f32x2;
typedef __attribute__((ext_vector_type(4))) float fp8_f32x4;

// amax: bits of the largest finite absolute value.  127 (a scale of 1) for a block without one; 1 at least, so that
// scale and inverse are normal numbers.
template <int FMT> __device__ inline int fp8_scale_byte(unsigned amax) {
    constexpr int TOP = FMT == FP8_E4M3 ? 8 : 15;
    const int b = (int)(amax >> 23) - TOP + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
    return amax == 0 ? 127 : max(b, 1);
}
// 2^(127 - b) for b from fp8_scale_byte (at most 254 - 8 + 1)
__device__ inline float fp8_inverse(int b) { return __builtin_bit_cast(float, (unsigned)(254 - b) << 23); }

template <int FMT> __device__ inline fp8_f32x4 fp8_decode4(unsigned x) {
    fp8_f32x2 lo, hi;
    if constexpr (FMT == FP8_E4M3) {
        lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false); hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
    } else {
        lo = __builtin_amdgcn_cvt_pk_f32_bf8((int)x, false); hi = __builtin_amdgcn_cvt_pk_f32_bf8((int)x, true);
    }
    return fp8_f32x4{lo[0], lo[1], hi[0], hi[1]};
}

// The largest of 64 lanes' values, the same in every lane: four moves within rows of 16 lanes, two across rows.
__device__ inline unsigned wave_max(unsigned x) {
#define TSR_MAX_DPP(ctrl) x = max(x, (unsigned)__builtin_amdgcn_update_dpp((int)x, (int)x, ctrl, 0xf, 0xf, false))
    TSR_MAX_DPP(0x111); TSR_MAX_DPP(0x112); TSR_MAX_DPP(0x114); TSR_MAX_DPP(0x118);   // row_shr 1, 2, 4, 8
    TSR_MAX_DPP(0x142); TSR_MAX_DPP(0x143);                                           // row_bcast 15, 31
#undef TSR_MAX_DPP
    return (unsigned)__builtin_amdgcn_readlane((int)x, 63);
}

}  // namespace tsr
