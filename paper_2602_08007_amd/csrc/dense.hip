// Parameters that are kept dense: AdamW over many tensors at once, with states in 32 or 8 bits, and the norm of all
// gradients that stands before it.
#include "dense.h"
#include "fp8_format.h"

namespace tsr {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned short u16x4;
// the same at any address of their element: the memory path takes vectors that straddle their boundary (60 tensors packed one
// behind the other, 332 MB: 112 us element by element)
typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4_any;
typedef __attribute__((ext_vector_type(4), aligned(2))) unsigned short u16x4_any;
typedef __attribute__((aligned(1))) unsigned u8x4_any;

constexpr int GROUPS = DENSE_CHUNK / 1024;               // groups of 256 elements of one wave (of four)
static_assert(DENSE_CHUNK % 1024 == 0 && STATE_BLOCK == 256, "a wave takes whole blocks of states");

// ------------------------------------------------------------------ four elements of a tensor
// WHOLE: all four exist; else element by element, those at or beyond n as zero.  Every value is touched once, so past the caches
// (the 109 tensors of the 130M model: 451 -> 400 us).
template <typename T, bool WHOLE> __device__ inline f32x4 load4(const void* base, long long i, long long n) {
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (sizeof(T) == 4) {
        const float* p = (const float*)base + i;
        if constexpr (WHOLE) return __builtin_nontemporal_load((const f32x4_any*)p);
#pragma unroll
        for (int j = 0; j < 4; ++j) if (i + j < n) x[j] = p[j];
    } else {
        const unsigned short* p = (const unsigned short*)base + i;
        u16x4 h = {0, 0, 0, 0};
        if constexpr (WHOLE) {
            h = __builtin_nontemporal_load((const u16x4_any*)p);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) if (i + j < n) h[j] = p[j];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = __builtin_bit_cast(float, (unsigned)h[j] << 16);
    }
    return x;
}
template <bool WHOLE> __device__ inline void store4(float* base, long long i, long long n, f32x4 x) {
    if constexpr (WHOLE) { __builtin_nontemporal_store(x, (f32x4_any*)(base + i)); return; }
#pragma unroll
    for (int j = 0; j < 4; ++j) if (i + j < n) base[i + j] = x[j];
}
template <bool WHOLE> __device__ inline void store4(unsigned short* base, long long i, long long n, u16x4 x) {
    if constexpr (WHOLE) { __builtin_nontemporal_store(x, (u16x4_any*)(base + i)); return; }
#pragma unroll
    for (int j = 0; j < 4; ++j) if (i + j < n) base[i + j] = x[j];
}
template <bool WHOLE> __device__ inline unsigned load4b(const void* base, long long i, long long n) {
    const unsigned char* p = (const unsigned char*)base + i;
    if constexpr (WHOLE) return __builtin_nontemporal_load((const u8x4_any*)p);
    unsigned x = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) if (i + j < n) x |= (unsigned)p[j] << (8 * j);
    return x;
}
template <bool WHOLE> __device__ inline void store4b(void* base, long long i, long long n, unsigned x) {
    unsigned char* p = (unsigned char*)base + i;
    if constexpr (WHOLE) { __builtin_nontemporal_store(x, (u8x4_any*)p); return; }
#pragma unroll
    for (int j = 0; j < 4; ++j) if (i + j < n) p[j] = (unsigned char)(x >> (8 * j));
}

// ------------------------------------------------------------------ random bits
// 32 bits for element i of a tensor: the finalizer of MurmurHash3 (A. Appleby, public domain) on index and key.
__device__ inline unsigned mix32(unsigned h) {
    h ^= h >> 16; h *= 0x85EBCA6Bu;
    h ^= h >> 13; h *= 0xC2B2AE35u;
    return h ^ (h >> 16);
}
__device__ inline unsigned random_bits(unsigned key, long long i) {
    return mix32((unsigned)i * 0x9E3779B1u + key + (unsigned)(i >> 32) * 0x7FEB352Du);
}

// Stochastic rounding of a block's values: x * 2^-e, e from the block's largest finite value (fp8_format.h), to the
// value of the type below or above with 16 random bits.  To the nearest value the states would stand still: with
// beta2 = 0.999 a step moves v by a thousandth, while half a step of e5m2 is an eighth; rounded so, the expected value of
// what is stored is what was computed, but for what 16 bits cannot tell: the probability is cut to a multiple of 2^-16, so a
// magnitude loses 2^-17 of its type's step on average.  Of a v that remembers 1 / (1 - beta2) steps that is 0.1 to 0.2 % at 0.999
// (1 to 2 % at 0.9999).  A million elements beside 32-bit states, beta2 = 0.999: after 400 and 8000 steps v 0.00 and 0.15 % low on
// average with a scatter of 28 %, m with one of 9 % of the gradient, p moved 2.5 and 3.0 % further.  A positive v is kept at the
// least positive value at least: v = 0 beside m != 0 would divide by eps.
template <int FMT> __device__ inline unsigned state_code(float x, float inv, unsigned r16) {
    const unsigned bits = __builtin_bit_cast(unsigned, x * inv);
    const unsigned a = bits & 0x7fffffffu;
    const float y = __builtin_bit_cast(float, a);
    unsigned code;
    if constexpr (FMT == FP8_E4M3) {
        code = (y < 0x1p-6f) ? (unsigned)(y * 0x1p9f + (float)r16 * 0x1p-16f) : ((a + (r16 << 4)) >> 20) - (120u << 3);
        if (a >= 0x7f800000u) code = 0x7f;                                   // no infinities in this type
    } else {
        code = (y < 0x1p-14f) ? (unsigned)(y * 0x1p16f + (float)r16 * 0x1p-16f) : ((a + (r16 << 5)) >> 21) - (112u << 2);
        if (a != 0 && code < 1) code = 1;
        if (a >= 0x7f800000u) code = a == 0x7f800000u ? 0x7c : 0x7f;
    }
    return code | ((bits >> 24) & 0x80u);
}
__device__ inline unsigned finite_bits(float x) {                           // |x| as an integer that orders like it; 0 if not finite
    const unsigned a = __builtin_bit_cast(unsigned, x) & 0x7fffffffu;
    return a < 0x7f800000u ? a : 0u;
}

// m / (sqrt(v) + eps) by the units' own root and reciprocal, off by a step of fp32 each, where the states hold 3 bits: beside
// 8-bit states the correctly rounded root and quotient are what bounds the step (two tables of 32000 x 2048: 351 -> 305 us).
// The root takes no subnormal numbers: those are multiplied by 2^24 before it and their root by 2^-12 after it, both exact.
// The reciprocal neither takes nor gives them: r is at least 2^-75 or 0 without eps, and the caller sees to an eps of 0 or
// between 2^-126 and DENSE_EPS8_MOST = 2^100.
__device__ inline float quick_ratio(float m, float v, float eps) {
    const bool tiny = v < 0x1p-126f;
    const float root = __builtin_amdgcn_sqrtf(v * (tiny ? 0x1p24f : 1.0f));
    const float r = __builtin_fmaf(root, tiny ? 0x1p-12f : 1.0f, eps);
    return __builtin_amdgcn_div_fixupf(m * __builtin_amdgcn_rcpf(r), r, m);       // zeros, infinities and the like as a quotient has them
}

// ------------------------------------------------------------------ AdamW
// m <- b1 m + (1 - b1) g ; v <- b2 v + (1 - b2) g^2 ; p <- (1 - lr wd) p - lr scale (m c1) / (sqrt(v c2) + eps).
// Bound by memory: every stream is read and written once, 28 bytes an element with 32-bit states and an fp32 gradient,
// 14 with 8-bit states and a bf16 gradient, 10 with bf16 parameters too.  All loads of a thread's GROUPS groups are in
// flight before the first is used.
// The blocks of the 130M model with a bf16 copy, 28 bytes an element: 400 us, 6.0 TB/s.  Two tables of 32000 x 2048 with 8-bit
// states: 304 us, 6.0 TB/s.  101 M bf16 parameters with 8-bit states: 219 us, 4.6 TB/s, where hash, rounding and root take
// the units as long as the memory takes.
// The products and sums are rounded one by one (no contraction): the results then do not depend on how a compiler
// pairs them, and stochastic rounding, which turns on single bits, gives the same states wherever the formula is evaluated so.
// `base`: the wave's first element; N groups of 256 from there.
template <typename P, typename G, bool S8, bool WHOLE, int N>
__device__ inline void adamw_groups(const DenseItem& d, const AdamScalars& s, float step, float gs, long long base) {
#pragma clang fp contract(off)
    const int lane = threadIdx.x & 63;
    const long long n = d.count;
    const float omb1 = 1.0f - s.beta1, omb2 = 1.0f - s.beta2;
    f32x4 p[N], g[N], m[N], v[N];
    unsigned mc[N], vc[N];
    int mb[N], vb[N];
    const long long at = base + lane * 4;
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const long long i = at + u * 256;
        g[u] = load4<G, WHOLE>(d.g, i, n);
        p[u] = load4<P, WHOLE>(d.p, i, n);
        if constexpr (S8) {
            mc[u] = load4b<WHOLE>(d.m, i, n); vc[u] = load4b<WHOLE>(d.v, i, n);
            mb[u] = d.m_scale[(base >> 8) + u]; vb[u] = d.v_scale[(base >> 8) + u];
        } else {
            m[u] = load4<float, WHOLE>(d.m, i, n);
            v[u] = load4<float, WHOLE>(d.v, i, n);
        }
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const long long i = at + u * 256;
        if constexpr (S8) {
            m[u] = fp8_decode4<FP8_E4M3>(mc[u]); v[u] = fp8_decode4<FP8_E5M2>(vc[u]);
#pragma unroll
            for (int j = 0; j < 4; ++j) { m[u][j] = ldexpf(m[u][j], mb[u] - 127); v[u][j] = ldexpf(v[u][j], vb[u] - 127); }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float gj = g[u][j] * gs;
            const float mj = m[u][j] * s.beta1 + gj * omb1;
            const float vj = v[u][j] * s.beta2 + (gj * gj) * omb2;
            const float dj = S8 ? quick_ratio(mj * s.inv_c1, vj * s.inv_c2, s.eps) : (mj * s.inv_c1) / (sqrtf(vj * s.inv_c2) + s.eps);
            p[u][j] = p[u][j] * d.decay - dj * step;
            m[u][j] = mj; v[u][j] = vj;
        }
        unsigned h[4];
        if constexpr (S8 || sizeof(P) == 2) {
#pragma unroll
            for (int j = 0; j < 4; ++j) h[j] = random_bits(d.key, i + j);
        }
        if constexpr (sizeof(P) == 4) {
            store4<WHOLE>((float*)d.p, i, n, p[u]);
            if (d.p16) {                                                     // nearest: the fp32 value is kept beside it
                u16x4 c;
#pragma unroll
                for (int j = 0; j < 4; ++j) c[j] = __builtin_bit_cast(unsigned short, (__bf16)p[u][j]);
                store4<WHOLE>(d.p16, i, n, c);
            }
        } else {                                                             // a step of lr is below half a step of bf16: stochastic
            u16x4 c;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float pj = p[u][j];                                    // (a cast of the element itself would take the vector's first)
                const unsigned b = __builtin_bit_cast(unsigned, pj);
                const bool nan = (b & 0x7fffffffu) > 0x7f800000u;            // infinity stays as it is below 16 more bits
                c[j] = (unsigned short)((nan ? b | 0x400000u : b + ((h[j] * 0x9E3779B1u) >> 16)) >> 16);
            }
            store4<WHOLE>((unsigned short*)d.p, i, n, c);
        }
        if constexpr (S8) {
            unsigned am = 0, av = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) { am = max(am, finite_bits(m[u][j])); av = max(av, finite_bits(v[u][j])); }
            am = wave_max(am); av = wave_max(av);
            const int bm = fp8_scale_byte<FP8_E4M3>(am), bv = fp8_scale_byte<FP8_E5M2>(av);
            const float im = fp8_inverse(bm), iv = fp8_inverse(bv);
            unsigned cm = 0, cv = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                cm |= state_code<FP8_E4M3>(m[u][j], im, h[j] & 0xffffu) << (8 * j);
                cv |= state_code<FP8_E5M2>(v[u][j], iv, h[j] >> 16) << (8 * j);
            }
            store4b<WHOLE>(d.m, i, n, cm); store4b<WHOLE>(d.v, i, n, cv);
            if (lane == 0) { d.m_scale[(base >> 8) + u] = (unsigned char)bm; d.v_scale[(base >> 8) + u] = (unsigned char)bv; }
        } else {
            store4<WHOLE>((float*)d.m, i, n, m[u]);
            store4<WHOLE>((float*)d.v, i, n, v[u]);
        }
    }
}

template <typename P, typename G, bool S8>
__device__ inline void adamw_item(const DenseItem& d, const AdamScalars& s, float step, float gs, long long base) {
    base += __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * (GROUPS * 256);
    const long long end = min(d.count, base + GROUPS * 256);
    if (base + GROUPS * 256 <= end) { adamw_groups<P, G, S8, true, GROUPS>(d, s, step, gs, base); return; }
#pragma unroll 1
    for (; base + 256 <= end; base += 256) adamw_groups<P, G, S8, true, 1>(d, s, step, gs, base);
    if (base < end) adamw_groups<P, G, S8, false, 1>(d, s, step, gs, base);
}

__global__ __launch_bounds__(256) void adamw_kernel(const DenseArgs a) {
    const int lane = threadIdx.x & 63;
    // the tensor of this workgroup: one load and one ballot instead of a search
    const bool below = lane < a.count && a.first[lane < DENSE_ITEMS ? lane : 0] <= blockIdx.x;
    const int k = __builtin_amdgcn_readfirstlane((int)__popcll(__ballot(below)) - 1);
    const DenseItem d = a.item[k];
    float gs = 1.0f;
    if (a.g_scale) {
        gs = *a.g_scale;
        if (!(fabsf(gs) <= 3.402823466e38f)) return;       // not finite: the step is left out
    }
    const long long base = (long long)(blockIdx.x - a.first[k]) * DENSE_CHUNK;
    switch (d.flags & (DENSE_P16 | DENSE_G16 | DENSE_STATE8)) {
        case 0: adamw_item<float, float, false>(d, a.s, a.step, gs, base); break;
        case DENSE_P16: adamw_item<__bf16, float, false>(d, a.s, a.step, gs, base); break;
        case DENSE_G16: adamw_item<float, __bf16, false>(d, a.s, a.step, gs, base); break;
        case DENSE_P16 | DENSE_G16: adamw_item<__bf16, __bf16, false>(d, a.s, a.step, gs, base); break;
        case DENSE_STATE8: adamw_item<float, float, true>(d, a.s, a.step, gs, base); break;
        case DENSE_STATE8 | DENSE_P16: adamw_item<__bf16, float, true>(d, a.s, a.step, gs, base); break;
        case DENSE_STATE8 | DENSE_G16: adamw_item<float, __bf16, true>(d, a.s, a.step, gs, base); break;
        default: adamw_item<__bf16, __bf16, true>(d, a.s, a.step, gs, base); break;
    }
}

hipError_t launch_adamw(const DenseArgs& a, unsigned workgroups, hipStream_t stream) {
    static_assert(sizeof(DenseArgs) <= 3584, "arguments of a launch");
    hipLaunchKernelGGL(adamw_kernel, dim3(workgroups), dim3(256), 0, stream, a);
    return hipGetLastError();
}

// ------------------------------------------------------------------ norm of all gradients
// norm = sqrt(sum g^2).  Squares and sums in fp64: no square overflows or vanishes, and the order of the sums, which is
// fixed, does not show in the fp32 result.  Bound by reading the gradients; an element costs a conversion and an fp64 FMA, a
// tenth of what the units do in the time of its four bytes.  300 M bf16 values: 94 us, 6.4 TB/s.
__device__ inline double square_sum4(f32x4 x, double acc) {
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_fma((double)x[j], (double)x[j], acc);
    return acc;
}
// elements [begin, end) of a gradient by `threads` threads, begin a multiple of 4
template <typename G> __device__ inline double square_sum(const void* g, long long begin, long long end, int thread, int threads) {
    double a0 = 0.0, a1 = 0.0;
    long long i = begin + thread * 4;
    const long long stride = threads * 4;
    for (; i + 3 * stride + 4 <= end; i += 4 * stride) {
        f32x4 x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = load4<G, true>(g, i + u * stride, end);
        a0 = square_sum4(x[0], a0); a1 = square_sum4(x[1], a1);
        a0 = square_sum4(x[2], a0); a1 = square_sum4(x[3], a1);
    }
    for (; i + 4 <= end; i += stride) a0 = square_sum4(load4<G, true>(g, i, end), a0);
    for (; i < end; i += stride) a1 = square_sum4(load4<G, false>(g, i, end), a1);
    return a0 + a1;
}
__device__ inline double wave_sum(double x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    return x;
}
__device__ inline void norm_out(double sum, float max_norm, float* norm, float* coef) {
    const double r = sqrt(sum);
    *norm = (float)r;
    if (coef) *coef = !(r <= 1.7976931348623157e308) ? __builtin_nanf("") : r > max_norm ? (float)(max_norm / r) : 1.0f;
}

__global__ __launch_bounds__(256) void norm_parts_kernel(const NormArgs a) {
    const int tid = threadIdx.x, lane = tid & 63;
    int k = -1;
#pragma unroll
    for (int h = 0; h < NORM_ITEMS; h += 64) {
        const int l = h + lane;
        k += (int)__popcll(__ballot(l < a.count && a.item[l < NORM_ITEMS ? l : 0].first <= blockIdx.x));
    }
    k = __builtin_amdgcn_readfirstlane(k);
    const NormItem& d = a.item[k];
    const long long begin = (long long)(blockIdx.x - d.first) * a.chunk, end = min(d.count, begin + a.chunk);
    double x = (d.flags & DENSE_G16) ? square_sum<__bf16>(d.g, begin, end, tid, 256) : square_sum<float>(d.g, begin, end, tid, 256);
    x = wave_sum(x);
    __shared__ double part[4];
    if (lane == 0) part[tid >> 6] = x;
    __syncthreads();
    if (tid == 0) a.partial[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

__global__ __launch_bounds__(1024) void norm_total_kernel(const double* partial, int parts, float max_norm, float* norm, float* coef) {
    const int tid = threadIdx.x;
    double x = 0.0;
    for (int i = tid; i < parts; i += 1024) x += partial[i];
    x = wave_sum(x);
    __shared__ double part[16];
    if ((tid & 63) == 0) part[tid >> 6] = x;
    __syncthreads();
    if (tid < 64) {
        x = wave_sum(tid < 16 ? part[tid] : 0.0);
        if (tid == 0) norm_out(x, max_norm, norm, coef);
    }
}

// A few small gradients: one workgroup, whose waves take stretches of NORM_STRETCH elements in turn, all loads of a stretch in
// flight at once: a wave reads no more than the others, however the elements are spread over the tensors.
__global__ __launch_bounds__(1024) void norm_one_kernel(const NormArgs a) {
    const int tid = threadIdx.x, lane = tid & 63;
    double x = 0.0;
    static_assert(NORM_ITEMS <= 128, "two tensors a lane");
    const unsigned first0 = lane < a.count ? a.item[lane].first : ~0u, first1 = lane + 64 < a.count ? a.item[lane + 64].first : ~0u;
    for (unsigned s = __builtin_amdgcn_readfirstlane(tid >> 6); s < a.stretches; s += 16) {
        const int k = __builtin_amdgcn_readfirstlane((int)(__popcll(__ballot(first0 <= s)) + __popcll(__ballot(first1 <= s))) - 1);
        const NormItem& d = a.item[k];
        const long long begin = (long long)(s - d.first) * NORM_STRETCH, end = min(d.count, begin + NORM_STRETCH);
        x += (d.flags & DENSE_G16) ? square_sum<__bf16>(d.g, begin, end, lane, 64) : square_sum<float>(d.g, begin, end, lane, 64);
    }
    x = wave_sum(x);
    __shared__ double part[16];
    if (lane == 0) part[tid >> 6] = x;
    __syncthreads();
    if (tid < 64) {
        x = wave_sum(tid < 16 ? part[tid] : 0.0);
        if (tid == 0) norm_out(x, a.max_norm, a.norm, a.coef);
    }
}

hipError_t launch_norm_parts(const NormArgs& a, unsigned workgroups, hipStream_t stream) {
    static_assert(sizeof(NormArgs) <= 3584, "arguments of a launch");
    hipLaunchKernelGGL(norm_parts_kernel, dim3(workgroups), dim3(256), 0, stream, a);
    return hipGetLastError();
}
hipError_t launch_norm_total(const double* partial, int parts, float max_norm, float* norm, float* coef, hipStream_t stream) {
    hipLaunchKernelGGL(norm_total_kernel, dim3(1), dim3(1024), 0, stream, partial, parts, max_norm, norm, coef);
    return hipGetLastError();
}
hipError_t launch_norm_one(const NormArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL(norm_one_kernel, dim3(1), dim3(1024), 0, stream, a);
    return hipGetLastError();
}

}  // namespace tsr
