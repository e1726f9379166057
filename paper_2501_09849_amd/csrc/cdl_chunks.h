// Eight consecutive entries of a row as a lane's share: loads kept packed until they are used, rows that start anywhere, rows that end inside the eight.
#pragma once

#include "cdl_types.h"

namespace cdl {

template <class T> struct Raw8;
template <> struct Raw8<bf16_t> { u32x4 a; };
template <> struct Raw8<float> { f32x4 a, b; };

// Pieces of a row to any address of an entry
template <class V, class T>
__device__ __forceinline__ void store_at(T *p, V v)
{
    typedef V any_t __attribute__((aligned(sizeof(T))));
    *reinterpret_cast<any_t *>(p) = v;
}

// Eight entries at p of a row (or vector) that has n more from there on (n may be 0 or less, or more than 8), zeros beyond its end once they are unpacked.  RAGGED: at any address of an
// entry, any n; else 16-byte aligned, n in whole eights.  Past the caches if `stream`.  Where the row ends inside the eight its last eight entries are loaded and moved down in
// unpack(), so that a load is one access (fp32: two) for all lanes and nothing waits for it here; rows of fewer than eight entries (SHORT) come entry by entry.
// (Entry by entry for the last chunk of every row, 4099 x 1021 in bf16, layer norm backward, took 21.2 us instead of 15.8.)
template <bool RAGGED>
__device__ __forceinline__ Raw8<bf16_t> load_raw(const bf16_t *p, int n, bool stream, bool is_short)
{
    Raw8<bf16_t> r{{0, 0, 0, 0}};
    if (!RAGGED) {
        if (n > 0) r.a = stream ? __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p)) : *reinterpret_cast<const u32x4 *>(p);
    } else if (!is_short) {
        r.a = *reinterpret_cast<const u32x4_any *>(n < 8 ? p + n - 8 : p);
    } else {
        const uint16_t *const h = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < n) r.a[k >> 1] |= (uint32_t)h[k] << (16 * (k & 1));
    }
    return r;
}
template <bool RAGGED>
__device__ __forceinline__ Raw8<float> load_raw(const float *p, int n, bool stream, bool is_short)
{
    Raw8<float> r{{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
    if (!RAGGED) {
        if (n > 0) {
            const f32x4 *const at = reinterpret_cast<const f32x4 *>(p);
            r.a = stream ? __builtin_nontemporal_load(at) : at[0];
            r.b = stream ? __builtin_nontemporal_load(at + 1) : at[1];
        }
    } else if (!is_short) {
        const float *const at = n < 8 ? p + n - 8 : p;
        r.a = *reinterpret_cast<const f32x4_any *>(at);
        r.b = *reinterpret_cast<const f32x4_any *>(at + 4);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (k < n) r.a[k] = p[k];
            if (k + 4 < n) r.b[k] = p[k + 4];
        }
    }
    return r;
}
template <bool RAGGED>
__device__ __forceinline__ void unpack(const Raw8<bf16_t> &r, int n, bool is_short, float (&v)[8])
{
    uint32_t a[4] = {r.a[0], r.a[1], r.a[2], r.a[3]};
    if (RAGGED && !is_short && n < 8) {
        const int by = 8 - n;      // entries down
        if (by & 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = (a[i] >> 16) | (i < 3 ? a[i + 1 < 4 ? i + 1 : 3] << 16 : 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = by & 2 ? (i < 3 ? a[i + 1 < 4 ? i + 1 : 3] : 0) : a[i];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = n <= 0 ? 0 : by & 4 ? (i < 2 ? a[i + 2 < 4 ? i + 2 : 3] : 0) : a[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(a[i] << 16);
        v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
}
template <bool RAGGED>
__device__ __forceinline__ void unpack(const Raw8<float> &r, int n, bool is_short, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = r.a[i]; v[4 + i] = r.b[i]; }
    if (RAGGED && !is_short && n < 8) {
        const int by = 8 - n;
#pragma unroll
        for (int d = 1; d < 8; d *= 2)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = by & d ? (i + d < 8 ? v[i + d < 8 ? i + d : 7] : 0.0f) : v[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = n <= 0 ? 0.0f : v[i];
    }
}

// The first n of eight entries to memory, one rounding each.
template <bool RAGGED>
__device__ __forceinline__ void store_first(bf16_t *p, int n, const float (&v)[8], bool stream)
{
    if (!RAGGED) {
        if (n > 0) store8(p, v, stream);
        return;
    }
    union { bf16x8 h; u32x4 u; } a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a.h[i] = (bf16_t)v[i];
    if (n >= 8) *reinterpret_cast<u32x4_any *>(p) = a.u;
    const int m = n >= 8 ? 0 : max(n, 0);
    const uint32_t two = m & 4 ? a.u[2] : a.u[0], after = m & 4 ? a.u[3] : a.u[1], one = m & 2 ? after : two;
    if (m & 4) store_at(p, u32x2{a.u[0], a.u[1]});
    if (m & 2) store_at(p + (m & 4), two);
    if (m & 1) store_at(p + (m & 6), (uint16_t)one);
}
template <bool RAGGED>
__device__ __forceinline__ void store_first(float *p, int n, const float (&v)[8], bool stream)
{
    if (!RAGGED) {
        if (n > 0) store8(p, v, stream);
        return;
    }
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x4 lo = {v[0], v[1], v[2], v[3]}, hi = {v[4], v[5], v[6], v[7]};
    if (n >= 8) {
        *reinterpret_cast<f32x4_any *>(p) = lo;
        *reinterpret_cast<f32x4_any *>(p + 4) = hi;
    }
    const int m = n >= 8 ? 0 : max(n, 0);
    const f32x4 rest = m & 4 ? hi : lo;
    if (m & 4) store_at(p, lo);
    if (m & 2) store_at(p + (m & 4), f32x2{rest[0], rest[1]});
    if (m & 1) p[m & 6] = m & 2 ? rest[2] : rest[0];
}

// ... of a vector, `missing` where there is none
template <bool RAGGED>
__device__ __forceinline__ void load_vector(const float *p, int n, bool is_short, float missing, float (&v)[8])
{
    if (!p) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = missing;
        return;
    }
    unpack<RAGGED>(load_raw<RAGGED>(p, n, false, is_short), n, is_short, v);
}

}  // namespace cdl
