// The block-scaled product with what stands behind it for a few rows, down to one: the weights go from memory into the fragments of the matrix instructions, once.
#pragma once

#include "cdl_act_ring.h"

namespace cdl {

// A block: 16 rows of the weights (of both matrices, if GATED) and 16 QT rows of a, its eight waves every eighth K-tile each; their sums meet in LDS.  Nothing
// is staged and no wave waits for another before that: a lane loads 32 bytes of its row of a K-tile, 16 of either half, and which bytes of a K-tile go to which place of the
// contraction does not matter as long as both operands agree.
// Bound by latency for small layers (4 x 4096 x 1024 5.3 us a call, 3.7 of them the kernel) and by the way of the weights for large ones (16 x 4096 x 4096 7.6 us for 17 MB).  In
// tiles of 128 x 64 through LDS the first took 7.4 us for the product alone.
typedef float v4f __attribute__((ext_vector_type(4)));
struct ThinJob {
    const uint8_t *a, *b[2], *sa, *sb[2];
    int64_t ld, pitch_a, pitch_b;
    int nk;
    ActTarget to;
};

constexpr int kThinWaves = 8;
// Rows of a that a block takes at most, in sixteens.  Two projections' exact products with 64 rows do not fit the registers: 23 spilled in the loop, 64 x 2048 x 1536 gated took 9.4 us
// (32 rows 5.4), 52 x 2000 x 3000 14.0 (8.4); where the loop is short it was as good or better, 64 x 4096 x 512 5.6 (6.0).
constexpr int thin_most(bool gated, bool exact) { return gated && exact ? 2 : 4; }

template <int FA, int FB, bool EXACT>
__device__ __forceinline__ void thin_product(v4f &acc, const v8i &b, const v8i &a, int sb, int sa)
{
    if constexpr (EXACT) {
        typedef OpF8<FB, FA, true> Op;
#pragma unroll
        for (int g = 0; g < 4; ++g)
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(Op::template widen<FB>(b[2 * g], b[2 * g + 1], __int_as_float(sb << 23)),
                                                          Op::template widen<FA>(a[2 * g], a[2 * g + 1], __int_as_float(sa << 23)), acc, 0, 0, 0);
    } else {
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, acc, FB, FA, 0, sb, 0, sa);
    }
}

template <int FA, int FB, bool GATED, int QT, class T>
__global__ __launch_bounds__(kThinWaves * 64)
void block8_thin_kernel(ThinJob job)
{
    constexpr int S = GATED ? 2 : 1;
    constexpr bool kExact = sizeof(T) == 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, part = lane >> 4;
    const int p0 = (int)blockIdx.x * 16, q0 = (int)blockIdx.y * 16 * QT;
    const int p = min(p0 + row, job.to.N - 1);      // (rows beyond the matrices: their last ones again, whose results nobody stores)
    const uint8_t *from_b[S], *from_a[QT], *scale_b[S], *scale_a[QT];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        from_b[s] = job.b[s] + p * job.ld + part * 16;
        scale_b[s] = job.sb[s] + p;
    }
#pragma unroll
    for (int j = 0; j < QT; ++j) {
        const int q = min(q0 + j * 16 + row, job.to.M - 1);
        from_a[j] = job.a + q * job.ld + part * 16;
        scale_a[j] = job.sa + q;
    }
    v4f acc[S][QT];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int j = 0; j < QT; ++j) acc[s][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    v8i b[2][S], a[2][QT];
    int sb[2][S], sa[2][QT];
    auto load = [&](int kt, auto set_c) {
        constexpr int N = decltype(set_c)::value;
        auto piece = [&](const uint8_t *at) {
            const v4i lo = *reinterpret_cast<const v4i *>(at + (int64_t)kt * kRingRow), hi = *reinterpret_cast<const v4i *>(at + (int64_t)kt * kRingRow + 64);
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };
#pragma unroll
        for (int s = 0; s < S; ++s) {
            b[N][s] = piece(from_b[s]);
            sb[N][s] = scale_b[s][kt * job.pitch_b];
        }
#pragma unroll
        for (int j = 0; j < QT; ++j) {
            a[N][j] = piece(from_a[j]);
            sa[N][j] = scale_a[j][kt * job.pitch_a];
        }
    };
    auto multiply = [&](auto set_c) {
        constexpr int N = decltype(set_c)::value;
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int j = 0; j < QT; ++j) thin_product<FA, FB, kExact>(acc[s][j], b[N][s], a[N][j], sb[N][s], sa[N][j]);
    };
    typedef std::integral_constant<int, 0> Zero;
    typedef std::integral_constant<int, 1> One;
    if (wave < job.nk) load(wave, Zero{});
    for (int kt = wave; kt < job.nk; kt += 2 * kThinWaves) {
        if (kt + kThinWaves < job.nk) load(kt + kThinWaves, One{});
        multiply(Zero{});
        if (kt + kThinWaves >= job.nk) break;
        if (kt + 2 * kThinWaves < job.nk) load(kt + 2 * kThinWaves, Zero{});
        multiply(One{});
    }

    // a lane holds entries p0 + 4 part + r of column q0 + 16 j + row
    __shared__ float sums[kThinWaves][S][QT][16][17];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int j = 0; j < QT; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) sums[wave][s][j][row][4 * part + r] = acc[s][j][r];
    __syncthreads();
    const ActTarget &to = job.to;
    for (int e = threadIdx.x; e < 256 * QT; e += kThinWaves * 64) {
        const int at_p = e & 15, at_q = e >> 4, p = p0 + at_p, q = q0 + at_q;
        if (p >= to.N || q >= to.M) continue;
        float z[S];
#pragma unroll
        for (int s = 0; s < S; ++s) {
            z[s] = 0.0f;
#pragma unroll
            for (int w = 0; w < kThinWaves; ++w) z[s] += sums[w][s][at_q >> 4][at_q & 15][at_p];
            if (to.bias[s]) z[s] += to.bias[s][p];
        }
        const int64_t at = (int64_t)q * to.N + p;
#pragma unroll
        for (int s = 0; s < S; ++s)
            if (to.z[s]) ((T *)to.z[s])[at] = (T)z[s];
        float y = to.act == CDL_ACT_RELU ? act_value<CDL_ACT_RELU>(z[0]) : to.act == CDL_ACT_GELU ? act_value<CDL_ACT_GELU>(z[0]) : to.act == CDL_ACT_SILU ? act_value<CDL_ACT_SILU>(z[0]) : z[0];
        if constexpr (GATED) y *= z[1];
        else if (to.add) y += (float)((const T *)to.add)[at];
        ((T *)to.y)[at] = (T)y;
    }
}

template <int FA, int FB, bool GATED, class T>
int launch_thin(const ThinJob &job, int qt, hipStream_t stream)
{
    const auto kernel = qt == 1 ? block8_thin_kernel<FA, FB, GATED, 1, T> : qt == 2 ? block8_thin_kernel<FA, FB, GATED, 2, T> : block8_thin_kernel<FA, FB, GATED, thin_most(GATED, sizeof(T) == 4), T>;
    const dim3 grid((unsigned)((job.to.N + 15) / 16), (unsigned)((job.to.M + 16 * qt - 1) / (16 * qt)));
    CDL_LAUNCH(GATED ? "block8_gated_thin_kernel" : "block8_act_thin_kernel", stream, kernel, grid, dim3(kThinWaves * 64), 0, job);
    return check_launch();
}
template <bool GATED, class T>
int launch_thin(const ThinJob &job, int qt, int a_format, int b_format, hipStream_t stream)
{
    if (b_format == CDL_E4M3) return a_format == CDL_E4M3 ? launch_thin<0, 0, GATED, T>(job, qt, stream) : launch_thin<1, 0, GATED, T>(job, qt, stream);
    return a_format == CDL_E4M3 ? launch_thin<0, 1, GATED, T>(job, qt, stream) : launch_thin<1, 1, GATED, T>(job, qt, stream);
}
int launch_thin_any(const ThinJob &job, int qt, bool gated, int y_type, int a_format, int b_format, hipStream_t stream);

}  // namespace cdl
