// AdamW over many tensors and the norm of many gradients (internal interface).
#pragma once
#include <hip/hip_runtime.h>

#include "small.h"

namespace tsr {

// One tensor of the step as the kernel takes it.  The tables travel in the kernel's arguments: nothing is uploaded,
// no workspace holds them, and a recorded launch keeps its own copy.
struct DenseItem {
    void* p; const void* g; void* m; void* v;
    unsigned char* m_scale; unsigned char* v_scale;     // 8-bit states: a byte for each STATE_BLOCK elements
    unsigned short* p16;                                // optional bf16 copy
    long long count;
    float decay;                                        // 1 - lr wd
    unsigned key;                                       // of this tensor's random bits in this step
    unsigned flags;
};
enum : unsigned { DENSE_P16 = 1, DENSE_G16 = 2, DENSE_STATE8 = 4 };

constexpr int STATE_BLOCK = 256;
constexpr float DENSE_EPS8_LEAST = 0x1p-126f, DENSE_EPS8_MOST = 0x1p100f;     // of an eps beside 8-bit states that is not 0
constexpr int DENSE_CHUNK = 4096;        // elements of one workgroup (8192: 431 us where these take 400)
constexpr int DENSE_ITEMS = 40;          // tensors of one launch: 84 bytes each, under the 4 KB that a launch's arguments may take

struct DenseArgs {
    AdamScalars s;
    float step;                          // lr * scale
    const float* g_scale;                // device scalar that multiplies the gradients, or null
    int count;
    unsigned first[DENSE_ITEMS];         // first workgroup of each tensor
    DenseItem item[DENSE_ITEMS];
};
hipError_t launch_adamw(const DenseArgs& a, unsigned workgroups, hipStream_t stream);

// Sums of squares: partial[workgroup] for every launch of a call, then the norm of all of them.
constexpr int NORM_ITEMS = 120;
constexpr int NORM_PARTS = 4096;         // partial sums of a call, one more at most for each tensor
constexpr int NORM_CHUNK = 8192;         // least elements of one workgroup, and what its chunks are multiples of
constexpr long long NORM_ONE = 1 << 15;  // up to so many elements in all, one workgroup does the whole call,
constexpr int NORM_STRETCH = 1024;       // its waves so many at a time
constexpr int NORM_STRETCHES = 64;       // and in so many stretches at most

struct NormItem { const void* g; long long count; unsigned first; unsigned flags; };     // first workgroup, or stretch
struct NormArgs {
    double* partial;                     // of this launch's first workgroup
    long long chunk;
    float max_norm; float* norm; float* coef;        // the call in one workgroup only
    int count;
    unsigned stretches;                  // in one workgroup only
    NormItem item[NORM_ITEMS];
};
hipError_t launch_norm_parts(const NormArgs& a, unsigned workgroups, hipStream_t stream);
hipError_t launch_norm_total(const double* partial, int parts, float max_norm, float* norm, float* coef, hipStream_t stream);
hipError_t launch_norm_one(const NormArgs& a, hipStream_t stream);

}  // namespace tsr
