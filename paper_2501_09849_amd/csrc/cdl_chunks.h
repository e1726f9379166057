// Eight consecutive entries of a row as a lane's share: loads kept packed until they are used, rows that start anywhere, rows that end inside the eight.
#pragma once

#include "cdl_types.h"

namespace cdl {

template <class T> struct Raw8;
template <> struct Raw8<bf16_t> { u32x4 a; };
template <> struct Raw8<float> { f32x4 a, b; };

// The first n of eight entries (n may be 0 or less, or more than 8), zeros behind them.  RAGGED: from any address of an entry, any n; else 16-byte aligned, n in
// whole eights.  Past the caches if `stream`.
template <bool RAGGED>
__device__ __forceinline__ Raw8<bf16_t> load_raw(const bf16_t *p, int n, bool stream)
{
    Raw8<bf16_t> r{{0, 0, 0, 0}};
    if (n >= 8) {
        if constexpr (RAGGED) r.a = *reinterpret_cast<const u32x4_any *>(p);
        else r.a = stream ? __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p)) : *reinterpret_cast<const u32x4 *>(p);
    } else if (RAGGED) {
        const uint16_t *const h = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < n) r.a[k >> 1] |= (uint32_t)h[k] << (16 * (k & 1));
    }
    return r;
}
template <bool RAGGED>
__device__ __forceinline__ Raw8<float> load_raw(const float *p, int n, bool stream)
{
    Raw8<float> r{{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
    if (n >= 8) {
        if constexpr (RAGGED) {
            r.a = *reinterpret_cast<const f32x4_any *>(p);
            r.b = *reinterpret_cast<const f32x4_any *>(p + 4);
        } else {
            const f32x4 *const at = reinterpret_cast<const f32x4 *>(p);
            r.a = stream ? __builtin_nontemporal_load(at) : at[0];
            r.b = stream ? __builtin_nontemporal_load(at + 1) : at[1];
        }
    } else if (RAGGED) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (k < n) r.a[k] = p[k];
            if (k + 4 < n) r.b[k] = p[k + 4];
        }
    }
    return r;
}
__device__ __forceinline__ void unpack(const Raw8<bf16_t> &r, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(r.a[i] << 16);
        v[2 * i + 1] = __uint_as_float(r.a[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(const Raw8<float> &r, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = r.a[i]; v[4 + i] = r.b[i]; }
}

// The first n of eight entries to memory, one rounding each.
template <bool RAGGED>
__device__ __forceinline__ void store_first(bf16_t *p, int n, const float (&v)[8], bool stream)
{
    if (n >= 8) {
        if constexpr (RAGGED) {
            union { bf16x8 h; u32x4 u; } a;
#pragma unroll
            for (int i = 0; i < 8; ++i) a.h[i] = (bf16_t)v[i];
            *reinterpret_cast<u32x4_any *>(p) = a.u;
        } else {
            store8(p, v, stream);
        }
    } else if (RAGGED) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < n) p[k] = (bf16_t)v[k];
    }
}
template <bool RAGGED>
__device__ __forceinline__ void store_first(float *p, int n, const float (&v)[8], bool stream)
{
    if (n >= 8) {
        if constexpr (RAGGED) {
            *reinterpret_cast<f32x4_any *>(p) = f32x4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4_any *>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
        } else {
            store8(p, v, stream);
        }
    } else if (RAGGED) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < n) p[k] = v[k];
    }
}

// ... of a vector that starts on 16 bytes, `missing` where there is none
template <bool RAGGED>
__device__ __forceinline__ void load_vector(const float *p, int n, float missing, float (&v)[8])
{
    if (!p) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = missing;
        return;
    }
    unpack(load_raw<RAGGED>(p, n, false), v);
}

}  // namespace cdl
