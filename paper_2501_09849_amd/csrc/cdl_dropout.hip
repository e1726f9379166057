// Dropout with a mask that is computed where it is needed and never stored.
#include "cdl_types.h"

namespace cdl {
namespace {

// Philox 4x32 (J. Salmon, M. Moraes, R. Dror, D. Shaw: Parallel random numbers: as easy as 1, 2, 3; SC 2011): a bijection of
// 128-bit counters keyed by 64 bits, ten rounds of two 32 x 32 -> 64 bit products.
struct Words { uint32_t w[4]; };
__device__ __forceinline__ Words philox(uint64_t counter, uint32_t k0, uint32_t k1)
{
    uint32_t x0 = (uint32_t)counter, x1 = (uint32_t)(counter >> 32), x2 = 0, x3 = 0;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p = (uint64_t)x0 * 0xD2511F53u, q = (uint64_t)x2 * 0xCD9E8D57u;
        x0 = (uint32_t)(q >> 32) ^ x1 ^ k0;
        x1 = (uint32_t)q;
        x2 = (uint32_t)(p >> 32) ^ x3 ^ k1;
        x3 = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{x0, x1, x2, x3}};
}

constexpr int kThreads = 256;

// A thread: eight consecutive entries, one counter.  Sixteen bits an entry, not 32: the generator's products take a quarter of
// the rate of other instructions, and with a word for every entry bf16 tensors would wait for them, not for memory.
// Bound by memory: 50 M entries in bf16 and a residual 53 us, 5.7 TB/s.
template <class T, bool ADD>
__global__ __launch_bounds__(kThreads)
void dropout_kernel(const T *x, const T *add, T *y, int64_t n, uint32_t share, float scale, uint64_t seed, uint64_t counter, bool stream)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x, e = i * 8;
    if (e >= n) return;
    float v[8], a[8];
    const bool whole = e + 8 <= n;
    if (whole) {
        load8(x + e, v, stream);
        if (ADD) load8(add + e, a, stream);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            v[k] = e + k < n ? (float)x[e + k] : 0.0f;
            if (ADD) a[k] = e + k < n ? (float)add[e + k] : 0.0f;
        }
    }
    const Words w = philox(counter + (uint64_t)i, (uint32_t)seed, (uint32_t)(seed >> 32));
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t bits = k & 1 ? w.w[k >> 1] >> 16 : w.w[k >> 1] & 0xffffu;
        const float kept = bits >= share ? v[k] * scale : 0.0f;      // (a choice, not a product with 0: what is dropped may be infinite)
        v[k] = ADD ? kept + a[k] : kept;
    }
    if (whole) {
        store8(y + e, v, stream);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (e + k < n) y[e + k] = (T)v[k];
    }
}

template <class T>
int launch(const void *x, const void *add, int64_t n, uint32_t share, uint64_t seed, uint64_t counter, void *y, hipStream_t stream)
{
    const float scale = share < 65536 ? 65536.0f / (float)(65536 - share) : 0.0f;
    const bool past = n * (int64_t)sizeof(T) >= kStreamFrom * 4;
    const auto kernel = add ? dropout_kernel<T, true> : dropout_kernel<T, false>;
    return in_launches(n, 8 * kLaunchThreads, [&](int64_t at, int64_t count) {
        const int64_t blocks = ((count + 7) / 8 + kThreads - 1) / kThreads;
        CDL_LAUNCH("dropout_kernel", stream, kernel, dim3((unsigned)blocks), dim3(kThreads), 0, (const T *)x + at, add ? (const T *)add + at : nullptr, (T *)y + at, count, share,
                   scale, seed, counter + (uint64_t)at / 8, past);
    });
}

}  // namespace

int launch_dropout(const void *x, const void *add, int32_t type, int64_t n, float p, uint64_t seed, uint64_t counter, void *y, hipStream_t stream)
{
    if (n == 0) return CDL_OK;
    const uint32_t share = (uint32_t)rintf(p * 65536.0f);
    return type == CDL_BF16 ? launch<bf16_t>(x, add, n, share, seed, counter, y, stream) : launch<float>(x, add, n, share, seed, counter, y, stream);
}

}  // namespace cdl
