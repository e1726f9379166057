// The element types of the operators in eight bits: vectors of bf16, conversions, tests of alignment.
#pragma once

#include "cdl_internal.h"

namespace cdl {

typedef __bf16 bf16_t;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// A grid holds fewer than 2^32 threads: what has more entries than that goes through in several launches, launch(first, count) for kLaunchThreads at a time.
constexpr int64_t kLaunchThreads = 1ll << 31;
template <class F>
int in_launches(int64_t n, int64_t most, const F &launch)
{
    for (int64_t at = 0; at < n; at += most) {
        launch(at, n - at < most ? n - at : most);
        const int rc = check_launch();
        if (rc != CDL_OK) return rc;
    }
    return CDL_OK;
}

// Eight consecutive entries from 16-byte aligned memory (fp32: two loads), as fp32; past the caches if `stream`.
__device__ __forceinline__ void load8(const float *p, float (&v)[8], bool stream)
{
    const f32x4 *const at = reinterpret_cast<const f32x4 *>(p);
    const f32x4 a = stream ? __builtin_nontemporal_load(at) : at[0], b = stream ? __builtin_nontemporal_load(at + 1) : at[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}
__device__ __forceinline__ void load8(const bf16_t *p, float (&v)[8], bool stream)
{
    const u32x4 *const at = reinterpret_cast<const u32x4 *>(p);
    const u32x4 a = stream ? __builtin_nontemporal_load(at) : *at;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(a[i] << 16);
        v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8], bool stream)
{
    f32x4 *const at = reinterpret_cast<f32x4 *>(p);
    const f32x4 a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
    if (stream) { __builtin_nontemporal_store(a, at); __builtin_nontemporal_store(b, at + 1); }
    else { at[0] = a; at[1] = b; }
}
// (one rounding, to nearest even)
__device__ __forceinline__ void store8(bf16_t *p, const float (&v)[8], bool stream)
{
    union { bf16x8 h; u32x4 u; } a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a.h[i] = (bf16_t)v[i];
    u32x4 *const at = reinterpret_cast<u32x4 *>(p);
    if (stream) __builtin_nontemporal_store(a.u, at);
    else *at = a.u;
}

}  // namespace cdl
