// What the tiles of a block-scaled product become in a layer: bias, activation, residual, the gated product of two projections; straight from the accumulators.
//
// In a GATED form a wave's first half of accumulators along P is of the gate and the second of the same entries of the other projection, so that the product of the two needs no other wave.
// What it costs: a wave of 128 x 128 is alone on its SIMD and issues the end of a tile in 7500 cycles, with silu in 12700, with gelu in 28600, where six K-tiles take 24500; its stores, one
// behind the other with those of every other compute unit, take as long as memory takes (128 KB a tile and compute unit in 4.7 us at the 7.2 TB/s that all stores together reach in the caches), and
// the loads of the next tile come in order behind them.  65536 x 4096 x 768 into bf16: 170 us products and loads alone, 270 with the stores, gelu 392 (in tiles of 128 x 128, where the other block
// multiplies meanwhile, 363), gelu with z kept 452.  65536 x 2048 x 768 gated, all three results kept: 313 us, on other cards 322 to 332; 805 MB written.
#pragma once

#include "cdl_act.h"
#include "cdl_ring.h"

namespace cdl {

struct ActTarget {
    const float *bias[2];
    const void *add;
    void *y, *z[2];
    int M, N, act;
};

// Sixteen results of a lane (entries p + 8 n + 4 (lane / 32) + k of row lane % 32 at 4 n + k) as shares of 16 bytes that lie side by side in memory, without a way through LDS.
// bf16: the halves of the wave swap fours, so that each has eight consecutive entries twice, of 32 rows; then the odd rows of 16 lanes swap with the even ones of the other
// eight.  fp32, where four entries are a share: the second swap alone, of shares 0 and 1, 2 and 3.  Either way an access is 64 bytes of 16 rows: share n of a lane is of row
// lane % 16 + 16 (n % 2).  (As 32 bytes of 32 rows 65536 x 4096 x 768 into bf16 took 278 us in tiles of 256 x 256, so 272.)
__device__ __forceinline__ void swap_halves(uint32_t &a, uint32_t &b)      // a's upper half of the wave with b's lower one
{
    const auto s = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = s[0];
    b = s[1];
}
__device__ __forceinline__ void swap_rows(uint32_t &a, uint32_t &b)      // a's odd rows of 16 lanes with b's even ones
{
    const auto s = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = s[0];
    b = s[1];
}
template <class T> struct Share;
template <> struct Share<float> {
    static constexpr int kCount = 4, kEntries = 4;
    typedef f32x4_any any_t;
    static __device__ __forceinline__ int entry(int n, int lane) { return 16 * (n >> 1) + 8 * (lane >> 4 & 1) + 4 * (lane >> 5); }
    static __device__ __forceinline__ void pack(const float (&v)[16], any_t (&out)[4])
    {
#pragma unroll
        for (int n = 0; n < 4; n += 2)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t a = __float_as_uint(v[4 * n + k]), b = __float_as_uint(v[4 * n + 4 + k]);
                swap_rows(a, b);
                out[n][k] = __uint_as_float(a);
                out[n + 1][k] = __uint_as_float(b);
            }
    }
    static __device__ __forceinline__ void unpack(const any_t (&in)[4], float (&v)[16])
    {
#pragma unroll
        for (int n = 0; n < 4; n += 2)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t a = __float_as_uint(in[n][k]), b = __float_as_uint(in[n + 1][k]);
                swap_rows(a, b);
                v[4 * n + k] = __uint_as_float(a);
                v[4 * n + 4 + k] = __uint_as_float(b);
            }
    }
};
template <> struct Share<bf16_t> {
    static constexpr int kCount = 2, kEntries = 8;
    typedef u32x4_any any_t;
    static __device__ __forceinline__ int entry(int, int lane) { return 16 * (lane >> 4 & 1) + 8 * (lane >> 5); }
    static __device__ __forceinline__ uint32_t two(float a, float b)
    {
        union { bf16x2 h; uint32_t u; } v;
        v.h = bf16x2{(bf16_t)a, (bf16_t)b};
        return v.u;
    }
    static __device__ __forceinline__ void pack(const float (&v)[16], any_t (&out)[2])
    {
        uint32_t w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = two(v[2 * k], v[2 * k + 1]);
#pragma unroll
        for (int n = 0; n < 8; n += 4) {      // eight entries: w[n], w[n + 1], w[n + 2], w[n + 3]
            swap_halves(w[n], w[n + 2]);
            swap_halves(w[n + 1], w[n + 3]);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            swap_rows(w[k], w[4 + k]);
            out[0][k] = w[k];
            out[1][k] = w[4 + k];
        }
    }
    static __device__ __forceinline__ void unpack(const any_t (&in)[2], float (&v)[16])
    {
        uint32_t w[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            w[k] = in[0][k];
            w[4 + k] = in[1][k];
            swap_rows(w[k], w[4 + k]);
        }
#pragma unroll
        for (int n = 0; n < 8; n += 4) {
            swap_halves(w[n], w[n + 2]);
            swap_halves(w[n + 1], w[n + 3]);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            v[2 * k] = __uint_as_float(w[k] << 16);
            v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
        }
    }
};

template <class FORM, class T>
struct ActStore {
    static constexpr bool kGated = FORM::GATED;
    static constexpr int S = kGated ? 2 : 1, TPO = FORM::TP / S, TQ = FORM::TQ, kCount = Share<T>::kCount;
    static constexpr int kStores = TPO * TQ * kCount;
    typedef typename Share<T>::any_t any_t;
    ActTarget to;

    // a tile of 32 x 32 at p, q
    template <bool FULL>
    __device__ __forceinline__ void load_shares(const T *from, int p, int q, int lane, any_t (&out)[kCount]) const
    {
        const int row = q + (lane & 15);
        const T *const base = from + (int64_t)row * to.N + p;
#pragma unroll
        for (int n = 0; n < kCount; ++n) {
            const int e = Share<T>::entry(n, lane);
            const T *const at = base + (n & 1 ? 16 * (int64_t)to.N : 0) + e;
            const int left = FULL || row + 16 * (n & 1) < to.M ? to.N - p - e : 0;      // entries that are there
            union { any_t a; T t[Share<T>::kEntries]; } u;
            if (FULL) {
                u.a = *reinterpret_cast<const any_t *>(at);
            } else {
#pragma unroll
                for (int k = 0; k < Share<T>::kEntries; ++k) u.t[k] = (T)0.0f;
                if (left >= Share<T>::kEntries) u.a = *reinterpret_cast<const any_t *>(at);
                if (to.N % Share<T>::kEntries != 0) {
#pragma unroll
                    for (int k = 0; k < Share<T>::kEntries; ++k)
                        if (left < Share<T>::kEntries && k < left) u.t[k] = at[k];
                }
            }
            out[n] = u.a;
        }
    }
    template <bool FULL>
    __device__ __forceinline__ void store_shares(T *into, int p, int q, int lane, const any_t (&in)[kCount]) const
    {
        const int row = q + (lane & 15);
        T *const base = into + (int64_t)row * to.N + p;
#pragma unroll
        for (int n = 0; n < kCount; ++n) {
            const int e = Share<T>::entry(n, lane);
            T *const at = base + (n & 1 ? 16 * (int64_t)to.N : 0) + e;
            const int left = FULL || row + 16 * (n & 1) < to.M ? to.N - p - e : 0;
            if (FULL || left >= Share<T>::kEntries) *reinterpret_cast<any_t *>(at) = in[n];
            if (!FULL && to.N % Share<T>::kEntries != 0) {
                union { any_t a; T t[Share<T>::kEntries]; } u;
                u.a = in[n];
#pragma unroll
                for (int k = 0; k < Share<T>::kEntries; ++k)
                    if (left < Share<T>::kEntries && k < left) at[k] = u.t[k];
            }
        }
    }

    // kSide tiles of an output one behind the other: the halves of a cache line meet in L2.  (With other outputs' between them 17 % more was written than there is, and 65536 x 2048 x 768
    // gated, all three results kept, took 371 us instead of 313.)
    static constexpr int kSide = sizeof(T) == 2 && TPO % 2 == 0 ? 2 : 1;
    template <bool FULL>
    __device__ __forceinline__ void store_side_by_side(T *into, int p, int q, int lane, const any_t (&in)[kSide][kCount]) const
    {
#pragma unroll
        for (int i = 0; i < kSide; ++i) store_shares<FULL>(into, p + 32 * i, q, lane, in[i]);
    }
    // PLAIN: neither z nor a residual
    template <int ACT, bool FULL, bool PLAIN>
    __device__ __forceinline__ void body(const v16f (&acc)[FORM::TP][FORM::TQ], int p0, int q0, int lane) const
    {
        const int half = lane >> 5, N = to.N;
        const bool with_add = !kGated && !PLAIN && to.add;
        float bias[S][TPO][16];
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int i = 0; i < TPO; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int p = p0 + i * 32 + 8 * r + 4 * half;
                    f32x4 b = {0.0f, 0.0f, 0.0f, 0.0f};
                    if (to.bias[s]) {
                        if (FULL || p + 4 <= N) b = *reinterpret_cast<const f32x4 *>(to.bias[s] + p);
                        else {
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                if (p + k < N) b[k] = to.bias[s][p + k];
                        }
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) bias[s][i][4 * r + k] = b[k];
                }
        // the residual of the next 32 columns is under way while these are finished: its wait would otherwise be one for their stores (in fp32 there are no registers for that)
        constexpr int kAhead = sizeof(T) == 2 ? 2 : 1;
        any_t add[kAhead][TPO][kCount];
        auto fetch = [&](int j) {
#pragma unroll
            for (int i = 0; i < TPO; ++i) load_shares<FULL>((const T *)to.add, p0 + i * 32, q0 + j * 32, lane, add[j % kAhead][i]);
        };
        if (with_add && kAhead == 2) fetch(0);
#pragma unroll
        for (int j = 0; j < TQ; ++j) {
            if (with_add && j + kAhead - 1 < TQ) fetch(j + kAhead - 1);
#pragma unroll
            for (int i0 = 0; i0 < TPO; i0 += kSide) {
                any_t out[kSide][kCount];
                float z[kSide][S][16], y[16];
#pragma unroll
                for (int s = 0; s < S; ++s) {
#pragma unroll
                    for (int i = 0; i < kSide; ++i)
#pragma unroll
                        for (int e = 0; e < 16; ++e) z[i][s][e] = result<FORM>(acc[s * TPO + i0 + i][j], e) + bias[s][i0 + i][e];
                    if (!PLAIN && to.z[s]) {
#pragma unroll
                        for (int i = 0; i < kSide; ++i) Share<T>::pack(z[i][s], out[i]);
                        store_side_by_side<FULL>((T *)to.z[s], p0 + i0 * 32, q0 + j * 32, lane, out);
                    }
                }
#pragma unroll
                for (int i = 0; i < kSide; ++i) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        y[e] = act_value<ACT>(z[i][0][e]);
                        if constexpr (kGated) y[e] *= z[i][1][e];
                    }
                    if (with_add) {
                        float other[16];
                        Share<T>::unpack(add[j % kAhead][i0 + i], other);
#pragma unroll
                        for (int e = 0; e < 16; ++e) y[e] += other[e];
                    }
                    Share<T>::pack(y, out[i]);
                }
                store_side_by_side<FULL>((T *)to.y, p0 + i0 * 32, q0 + j * 32, lane, out);
                __builtin_amdgcn_sched_barrier(0);      // (these results' registers at a time)
            }
        }
    }
    template <int ACT>
    __device__ __forceinline__ void by_outputs(const v16f (&acc)[FORM::TP][FORM::TQ], int p0, int q0, int lane) const
    {
        if (p0 + TPO * 32 <= to.N && q0 + TQ * 32 <= to.M) {
            if (to.add || to.z[0] || to.z[1]) body<ACT, true, false>(acc, p0, q0, lane);
            else body<ACT, true, true>(acc, p0, q0, lane);
        } else {
            body<ACT, false, false>(acc, p0, q0, lane);
            __builtin_amdgcn_s_waitcnt(wait_imm(0));
        }
    }
    __device__ __forceinline__ void operator()(const v16f (&acc)[FORM::TP][FORM::TQ], int p0, int q0, int, uint8_t *, int lane) const
    {
        switch (to.act) {
            case CDL_ACT_RELU: by_outputs<CDL_ACT_RELU>(acc, p0, q0, lane); break;
            case CDL_ACT_GELU: by_outputs<CDL_ACT_GELU>(acc, p0, q0, lane); break;
            case CDL_ACT_SILU: by_outputs<CDL_ACT_SILU>(acc, p0, q0, lane); break;
            default: by_outputs<CDL_ACT_NONE>(acc, p0, q0, lane); break;
        }
    }
};

template <class FORM, int FP, int FQ, bool EXACT, class T>
__global__ __launch_bounds__(FORM::kThreads, FORM::PER_CU)
void block8_act_kernel(RingCall<ActStore<FORM, T>> call)
{
    ring<FORM, OpF8<FP, FQ, EXACT>, false, false, false>(call);
}

// Tiles of 256 x 256, one block on a compute unit; of 128 x 128, two: while one finishes a tile, the other multiplies; of 64 x 64 (gated: 128 x 64, 64 of either matrix), two, with more
// K-tiles under way: for products of so few tiles that their latency counts.  (The staging of the first two is what ring() asks for of rings of two; nothing is written there.)
template <bool GATED> using ActWide = RingForm<2, 2, 4, 4, 2, 2, 1, 4096, true, GATED>;
template <bool GATED> using ActPair = RingForm<2, 2, 2, 2, 2, 2, 2, 2048, true, GATED>;
template <bool GATED> using ActSmall = std::conditional_t<GATED, RingForm<2, 2, 2, 1, 3, 3, 2, 0, true, true>, RingForm<2, 2, 1, 1, 4, 4, 2, 0, true, false>>;
enum class ActForm { kWide, kPair, kSmall };

template <class FORM, bool EXACT, class T>
int launch_act_form(RingJob job, const ActTarget &to, int a_format, int b_format, hipStream_t stream)
{
    const auto kernel = b_format == CDL_E4M3 ? (a_format == CDL_E4M3 ? block8_act_kernel<FORM, 0, 0, EXACT, T> : block8_act_kernel<FORM, 0, 1, EXACT, T>)
                                             : (a_format == CDL_E4M3 ? block8_act_kernel<FORM, 1, 0, EXACT, T> : block8_act_kernel<FORM, 1, 1, EXACT, T>);
    const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, FORM::kLds);
    if (e != hipSuccess) return hip_failed(e);
    job.tiles_p = (to.N + FORM::kAcross - 1) / FORM::kAcross;
    job.tiles_q = (to.M + FORM::kQ - 1) / FORM::kQ;
    const int64_t grid = ring_blocks((int64_t)job.tiles_p * job.tiles_q, FORM::PER_CU);
    CDL_LAUNCH(FORM::GATED ? "block8_gated_kernel" : "block8_act_kernel", stream, kernel, dim3((unsigned)grid), dim3(FORM::kThreads), FORM::kLds,
               (RingCall<ActStore<FORM, T>>{ring_ready(job), {to}}));
    return check_launch();
}

// One file for each type of results and number of projections: they take a minute or two each to compile.
template <bool GATED, class T>
int launch_act_ring(ActForm form, const RingJob &job, const ActTarget &to, int a_format, int b_format, hipStream_t stream)
{
    constexpr bool kExact = sizeof(T) == 4;
    if (form == ActForm::kSmall) return launch_act_form<ActSmall<GATED>, kExact, T>(job, to, a_format, b_format, stream);
    if constexpr (!kExact || GATED) {      // (exact products in wide tiles of one matrix spill: choose() does not take them)
        if (form == ActForm::kWide) return launch_act_form<ActWide<GATED>, kExact, T>(job, to, a_format, b_format, stream);
    }
    return launch_act_form<ActPair<GATED>, kExact, T>(job, to, a_format, b_format, stream);
}
int launch_act_bf16(ActForm form, const RingJob &job, const ActTarget &to, int a_format, int b_format, hipStream_t stream);
int launch_act_f32(ActForm form, const RingJob &job, const ActTarget &to, int a_format, int b_format, hipStream_t stream);
int launch_gated_bf16(ActForm form, const RingJob &job, const ActTarget &to, int a_format, int b_format, hipStream_t stream);
int launch_gated_f32(ActForm form, const RingJob &job, const ActTarget &to, int a_format, int b_format, hipStream_t stream);

}  // namespace cdl
