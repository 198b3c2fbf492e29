// C ABI of the parameters that are kept dense: AdamW over many tensors, the norm of many gradients.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "dense.h"
#include "host_util.h"

using namespace tsr;

namespace {

constexpr long long MOST = 1ll << 35;        // elements of a tensor
constexpr unsigned MOST_GROUPS = 1u << 23;   // of one launch: times 256 threads, under 2^32
static_assert(MOST / DENSE_CHUNK <= MOST_GROUPS, "a tensor fits one launch");

bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
bool is_float(int d) { return d == TSR_F32 || d == TSR_BF16; }
size_t size_of(int d) { return d == TSR_F32 ? 4 : 2; }

int check_gradient(const tsr_tensor_desc& d) {
    if (d.count < 0 || d.count > MOST) return TSR_BAD_SHAPE;
    if (!is_float(d.g_dtype)) return TSR_BAD_DTYPE;
    if (d.count && (!d.g || !aligned(d.g, size_of(d.g_dtype)))) return TSR_INVALID_ARG;
    return TSR_OK;
}

int check_tensor(const tsr_tensor_desc& d) {
    TSR_TRY(check_gradient(d));
    if (!is_float(d.p_dtype)) return TSR_BAD_DTYPE;
    if (d.state != TSR_STATE_F32 && d.state != TSR_STATE_8BIT) return TSR_BAD_DTYPE;
    if (!std::isfinite(d.wd_scale)) return TSR_INVALID_ARG;
    if (!d.count) return TSR_OK;
    if (!d.p || !d.m || !d.v || !aligned(d.p, size_of(d.p_dtype))) return TSR_INVALID_ARG;
    if (d.state == TSR_STATE_F32 ? !aligned(d.m, 4) || !aligned(d.v, 4) : !d.m_scale || !d.v_scale) return TSR_INVALID_ARG;
    if (d.p16 && (d.p_dtype != TSR_F32 || !aligned(d.p16, 2))) return TSR_INVALID_ARG;
    return TSR_OK;
}

struct Range { uintptr_t begin, end; };

// The ranges that the call writes: whether two of them meet, or one of them something that is read only.
int check_ranges(const tsr_tensor_desc* t, int count, const float* g_scale) {
    std::unique_ptr<Range[]> r(new (std::nothrow) Range[6 * (size_t)count]);
    if (!r) return TSR_OUT_OF_HOST_MEMORY;
    size_t k = 0;
    auto add = [&](const void* p, long long bytes) { r[k++] = {(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes}; };
    for (int i = 0; i < count; ++i) {
        const tsr_tensor_desc& d = t[i];
        if (!d.count) continue;
        const int state = d.state == TSR_STATE_F32 ? 4 : 1;
        add(d.p, d.count * (long long)size_of(d.p_dtype));
        add(d.m, d.count * state);
        add(d.v, d.count * state);
        if (d.state == TSR_STATE_8BIT) {
            const long long blocks = (d.count + STATE_BLOCK - 1) / STATE_BLOCK;
            add(d.m_scale, blocks);
            add(d.v_scale, blocks);
        }
        if (d.p16) add(d.p16, d.count * 2);
    }
    std::sort(r.get(), r.get() + k, [](const Range& a, const Range& b) { return a.begin < b.begin; });
    for (size_t i = 1; i < k; ++i)
        if (r[i].begin < r[i - 1].end) return TSR_INVALID_ARG;
    // of the written ranges, which lie apart, the last that begins before what is read ends reaches furthest
    auto written = [&](const void* p, long long bytes) {
        const Range x{(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes};
        const Range* at = std::lower_bound(r.get(), r.get() + k, x.end, [](const Range& a, uintptr_t end) { return a.begin < end; });
        return at != r.get() && at[-1].end > x.begin;
    };
    for (int i = 0; i < count; ++i)
        if (t[i].count && written(t[i].g, t[i].count * (long long)size_of(t[i].g_dtype))) return TSR_INVALID_ARG;
    if (g_scale && written(g_scale, 4)) return TSR_INVALID_ARG;
    return TSR_OK;
}

unsigned mix32(unsigned h) {                 // as the kernel's
    h ^= h >> 16; h *= 0x85EBCA6Bu;
    h ^= h >> 13; h *= 0xC2B2AE35u;
    return h ^ (h >> 16);
}

float decay_of(const tsr_tensor_desc& d, const tsr_hyper& h) {
    return (float)(1.0 - (double)h.lr * (double)h.wd * (double)d.wd_scale);
}

DenseItem item_of(const tsr_tensor_desc& d, const tsr_hyper& h, unsigned key) {
    DenseItem it{};
    it.p = d.p; it.g = d.g; it.m = d.m; it.v = d.v;
    it.m_scale = d.m_scale; it.v_scale = d.v_scale;
    it.p16 = (unsigned short*)d.p16;
    it.count = d.count;
    it.decay = decay_of(d, h);
    it.key = key;
    const size_t ps = size_of(d.p_dtype), gs = size_of(d.g_dtype);
    const bool s8 = d.state == TSR_STATE_8BIT;
    it.flags = (ps == 2 ? DENSE_P16 : 0) | (gs == 2 ? DENSE_G16 : 0) | (s8 ? DENSE_STATE8 : 0);
    return it;
}

// How the gradients of a norm are cut: `chunk` elements a workgroup, `parts` workgroups in all.
struct NormCut { long long chunk, total, parts; };
int cut_norm(const tsr_tensor_desc* t, int count, NormCut& c) {
    c = {};
    for (int i = 0; i < count; ++i) {
        TSR_TRY(check_gradient(t[i]));
        c.total += t[i].count;               // at most 2^31 tensors of 2^35; no sum overflows before the check
        if (c.total > (1ll << 60)) return TSR_BAD_SHAPE;
    }
    const long long even = (c.total + NORM_PARTS - 1) / NORM_PARTS;
    c.chunk = (even + NORM_CHUNK - 1) / NORM_CHUNK * NORM_CHUNK;
    if (c.chunk < NORM_CHUNK) c.chunk = NORM_CHUNK;
    for (int i = 0; i < count; ++i) c.parts += (t[i].count + c.chunk - 1) / c.chunk;
    return TSR_OK;
}

}  // namespace

extern "C" {

int tsr_adamw_batched(const tsr_tensor_desc* tensors, int count, int t, const tsr_hyper* h, unsigned long long seed,
                      const float* g_scale, void* stream) {
    if (!tensors || !h) return TSR_INVALID_ARG;
    if (count <= 0) return TSR_BAD_SHAPE;
    DenseArgs a{};
    TSR_TRY(adam_scalars(a.s, t, h->beta1, h->beta2, h->eps));
    a.step = (float)((double)h->lr * (double)h->scale);
    if (!aligned(g_scale, 4) || !std::isfinite(h->lr) || !std::isfinite(h->wd) || !std::isfinite(a.step)) return TSR_INVALID_ARG;
    const bool eps8 = h->eps == 0.0f || (h->eps >= DENSE_EPS8_LEAST && h->eps <= DENSE_EPS8_MOST);
    for (int i = 0; i < count; ++i) {
        TSR_TRY(check_tensor(tensors[i]));
        if (tensors[i].state == TSR_STATE_8BIT && !eps8) return TSR_INVALID_ARG;
        if (!std::isfinite(decay_of(tensors[i], *h))) return TSR_INVALID_ARG;
    }
    TSR_TRY(check_ranges(tensors, count, g_scale));
    a.g_scale = g_scale;
    const unsigned key = mix32(mix32(mix32((unsigned)seed) ^ (unsigned)(seed >> 32)) ^ (unsigned)t);
    unsigned groups = 0;                     // of the launch that is being filled
    auto flush = [&]() -> int {
        if (!a.count) return TSR_OK;
        TSR_HIP(launch_adamw(a, groups, (hipStream_t)stream));
        a.count = 0;
        groups = 0;
        return TSR_OK;
    };
    for (int i = 0; i < count; ++i) {
        const tsr_tensor_desc& d = tensors[i];
        if (!d.count) continue;
        const unsigned need = (unsigned)((d.count + DENSE_CHUNK - 1) / DENSE_CHUNK);
        if (a.count == DENSE_ITEMS || groups + need > MOST_GROUPS) TSR_TRY(flush());
        a.first[a.count] = groups;
        a.item[a.count++] = item_of(d, *h, mix32(key + (unsigned)i * 0x9E3779B1u));
        groups += need;
    }
    return flush();
}

size_t tsr_grad_norm_workspace_bytes(const tsr_tensor_desc* tensors, int count) {
    NormCut c;
    if (!tensors || count <= 0 || cut_norm(tensors, count, c) != TSR_OK) return 0;
    return align_up((size_t)(c.parts > 0 ? c.parts : 1) * sizeof(double));
}

int tsr_grad_norm_batched(const tsr_tensor_desc* tensors, int count, float max_norm, float* norm, float* coef,
                          void* ws, size_t ws_bytes, void* stream) {
    if (!tensors || !norm || !ws) return TSR_INVALID_ARG;
    if (count <= 0) return TSR_BAD_SHAPE;
    if (!(max_norm > 0.0f) || !aligned(norm, 4) || !aligned(coef, 4) || norm == coef) return TSR_INVALID_ARG;
    if ((uintptr_t)ws % ALIGN) return TSR_INVALID_ARG;
    NormCut c;
    TSR_TRY(cut_norm(tensors, count, c));
    if (ws_bytes < (size_t)c.parts * sizeof(double)) return TSR_WORKSPACE_TOO_SMALL;
    const hipStream_t s = (hipStream_t)stream;
    NormArgs a{};
    a.chunk = c.chunk;
    a.max_norm = max_norm; a.norm = norm; a.coef = coef;
    // A few small gradients: one workgroup, unless its 16 waves take longer for their stretches than a second launch does (fp32, in
    // one and in two launches: 1 x 32768 3.75 and 4.9 us, 17 x 512 3.25 and 4.7, 64 x 512 4.6 and 4.75, 120 x 273 8.0 and 5.0).
    long long stretches = 0;
    for (int i = 0; i < count && count <= NORM_ITEMS; ++i) stretches += (tensors[i].count + NORM_STRETCH - 1) / NORM_STRETCH;
    const bool one = c.total <= NORM_ONE && count <= NORM_ITEMS && stretches <= NORM_STRETCHES;
    unsigned groups = 0;
    long long done = 0;
    auto flush = [&]() -> int {
        if (!a.count) return TSR_OK;
        a.partial = (double*)ws + done;
        TSR_HIP(launch_norm_parts(a, groups, s));
        done += groups;
        a.count = 0;
        groups = 0;
        return TSR_OK;
    };
    for (int i = 0; i < count; ++i) {
        const tsr_tensor_desc& d = tensors[i];
        if (!d.count) continue;
        if (a.count == NORM_ITEMS) TSR_TRY(flush());
        const size_t gs = size_of(d.g_dtype);
        a.item[a.count++] = {d.g, d.count, groups, gs == 2 ? DENSE_G16 : 0u};
        const long long each = one ? NORM_STRETCH : c.chunk;
        groups += (unsigned)((d.count + each - 1) / each);
    }
    a.stretches = groups;
    if (one) { TSR_HIP(launch_norm_one(a, s)); return TSR_OK; }
    TSR_TRY(flush());
    TSR_HIP(launch_norm_total((const double*)ws, (int)c.parts, max_norm, norm, coef, s));
    return TSR_OK;
}

}  // extern "C"
