// The product of two matrices in 8-bit floating point with a scale for every block of 128 entries of the contraction.
//
//   y[m,n] = sum_kb 2^(a_scale[kb,m] + b_scale[kb,n] - 254) * sum_{k in kb} a[m,k] * b[n,k]
//
// Scales are powers of two, so the matrix instructions apply them.  65536 x 3072 x 768 into bf16 185 us, call after call, at the power limit, 221: 146 of them products and loads, 35
// turning results into rows and 42 storing 403 MB, during both of which a compute unit's only block of 256 x 256 multiplies nothing; 3072 x 768 x 65536 into fp32 256 us, the matrix cores busy 62 %.
#include "cdl_ring.h"

namespace cdl {
namespace {

using Wide = RingForm<2, 2, 4, 4, 2, 2, 1, 4096, true>;        // 256 x 256
using Square = RingForm<2, 2, 2, 2, 4, 4, 1, 4096, true>;      // 128 x 128
using Thin = RingForm<4, 1, 1, 2, 3, 3, 2, 0, true>;           // 128 of b, 64 of a

template <class FORM, class T>
struct Store {
    static constexpr int kStores = row_stores<FORM, T>();
    RowTarget<T> to;
    int64_t part;      // entries between the parts of a split contraction
    __device__ __forceinline__ void operator()(const v16f (&acc)[FORM::TP][FORM::TQ], int p0, int q0, int split, uint8_t *staging, int lane) const
    {
        RowTarget<T> at = to;
        at.out += split * part;
        store_rows<FORM, T, false>(acc, at, p0, q0, staging, lane, [](float v, int, int) { return v; });
    }
};

template <class FORM, int FP, int FQ, bool EXACT, class T>
__global__ __launch_bounds__(FORM::kThreads, FORM::PER_CU)
void block8_gemm_kernel(RingCall<Store<FORM, T>> call)
{
    ring<FORM, OpF8<FP, FQ, EXACT>, false, false, false>(call);
}

// The parts of a split contraction added up, in order.
template <class T>
__global__ __launch_bounds__(256)
void block8_sum_kernel(const float *__restrict__ parts, int splits, int64_t n, T *__restrict__ y)
{
    const int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (e >= n) return;
    if (e + 4 <= n && (n & 3) == 0) {
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = 0; s < splits; ++s) sum += *reinterpret_cast<const f32x4 *>(parts + s * n + e);
        typename Four<T>::type out;
#pragma unroll
        for (int k = 0; k < 4; ++k) out[k] = (T)sum[k];
        *reinterpret_cast<typename Four<T>::type *>(y + e) = out;
    } else {
        for (int k = 0; k < 4 && e + k < n; ++k) {
            float sum = 0.0f;
            for (int s = 0; s < splits; ++s) sum += parts[s * n + e + k];
            y[e + k] = (T)sum;
        }
    }
}

template <class T>
__global__ __launch_bounds__(256)
void zero_kernel(T *y, int64_t n)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) y[i] = (T)0.0f;
}

enum Form { kWide, kSquare, kThin };
struct Layout {
    Form form;
    int tiles_p, tiles_q, splits, k_per;
    float cost;
};

// A product in one form, and what it takes, in K-tiles of a block of 128 x 128 alone on its compute unit (0.6 us): rounds of blocks over the chip, 3.3 for a K-tile of
// 256 x 256, 1.1 for two blocks of 128 x 64 on a compute unit, 0.55 where there is one.  The contraction is split where tiles leave compute units idle and it is
// 48 K-tiles long, into parts of 16 at least: adding the parts up takes a launch, 8 us, and their way to memory and back (1000 x 1000 x 2048 in two parts 22.1 us, in one
// 11.7; 4 x 8192 x 8192 in eight parts 24.0, in four 21.5).
Layout layout_of(Form form, int32_t M, int32_t N, int nk)
{
    Layout l;
    l.form = form;
    const int p = form == kWide ? 256 : 128, q = form == kWide ? 256 : form == kSquare ? 128 : 64, per_cu = form == kThin ? 2 : 1;
    l.tiles_p = (N + p - 1) / p;
    l.tiles_q = (M + q - 1) / q;
    const int64_t tiles = (int64_t)l.tiles_p * l.tiles_q, places = 256 * per_cu;
    const int64_t most = nk < 48 ? 1 : nk / 16;
    int64_t splits = tiles >= places ? 1 : places / tiles;
    splits = splits < most ? splits : most;
    const int per = (int)((nk + splits - 1) / splits);
    l.splits = (nk + per - 1) / per;
    l.k_per = per;
    const int64_t units = tiles * l.splits;
    const float each = form == kWide ? 3.3f : form == kSquare ? 1.0f : units <= 256 ? 0.55f : 1.1f;
    l.cost = (float)((units + places - 1) / places) * (float)per * each + (l.splits > 1 ? 13.0f + (float)l.splits * (float)M * (float)N * 1.7e-6f : 0.0f);
    return l;
}

// The form that takes least; for few tokens, of which a wider tile would hold one row of tiles, the thin one.  Results bf16, us, as Wide, Square, Thin:
//   1000 x 1000 x 520     -    9.4   8.0        2048 x 2048 x 2048   30.4  16.7   -          4096 x 4096 x 768    22.3  25.0   -
//   1000 x 1000 x 4096    -   21.6  16.5        2048 x 2048 x 8192   56.6  40.1   -          8192 x 4096 x 2048   64.8  78.3   -
//   1700 x 1700 x 2048    -   20.4  17.7        1024 x 1024 x 16384  43.6  33.4   -          65536 x 1024 x 512   47.1  60.6   -
Layout layout(int32_t M, int32_t N, int32_t K)
{
    const int nk = (int)(block8_pitch(K) / kRingRow);
    Layout best = layout_of(kThin, M, N, nk);
    if (M <= 64) return best;
    for (Form form : {kSquare, kWide}) {
        const Layout l = layout_of(form, M, N, nk);
        if (l.cost < best.cost) best = l;
    }
    return best;
}

template <class FORM, bool EXACT, class T>
int launch_form(const RingJob &job, int a_format, int b_format, const Store<FORM, T> &store, hipStream_t stream)
{
    const auto kernel = b_format == CDL_E4M3 ? (a_format == CDL_E4M3 ? block8_gemm_kernel<FORM, 0, 0, EXACT, T> : block8_gemm_kernel<FORM, 0, 1, EXACT, T>)
                                             : (a_format == CDL_E4M3 ? block8_gemm_kernel<FORM, 1, 0, EXACT, T> : block8_gemm_kernel<FORM, 1, 1, EXACT, T>);
    const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, FORM::kLds);
    if (e != hipSuccess) return hip_failed(e);
    const int64_t grid = ring_blocks((int64_t)job.tiles_p * job.tiles_q * job.splits, FORM::PER_CU);
    CDL_LAUNCH("block8_gemm_kernel", stream, kernel, dim3((unsigned)grid), dim3(FORM::kThreads), FORM::kLds, (RingCall<Store<FORM, T>>{ring_ready(job), store}));
    return check_launch();
}

template <bool EXACT, class T>
int launch_product(const RingJob &job, const Layout &l, int a_format, int b_format, T *y, int32_t M, int32_t N, hipStream_t stream)
{
    const RowTarget<T> to{y, N, N, M, row_width(y, (int64_t)N * (int64_t)sizeof(T))};
    const int64_t part = (int64_t)M * N;
    switch (l.form) {
        case kWide: return launch_form<Wide, EXACT, T>(job, a_format, b_format, Store<Wide, T>{to, part}, stream);
        case kSquare: return launch_form<Square, EXACT, T>(job, a_format, b_format, Store<Square, T>{to, part}, stream);
        default: return launch_form<Thin, EXACT, T>(job, a_format, b_format, Store<Thin, T>{to, part}, stream);
    }
}

}  // namespace

size_t block8_gemm_workspace_bytes(int32_t M, int32_t N, int32_t K)
{
    if (M == 0 || N == 0 || K == 0) return 0;
    const Layout l = layout(M, N, K);
    return l.splits > 1 ? align_up((size_t)l.splits * (size_t)M * (size_t)N * sizeof(float), 256) : 0;
}

int launch_block8_gemm(const uint8_t *a, const uint8_t *a_scale, const uint8_t *b, const uint8_t *b_scale, int32_t M, int32_t N, int32_t K, int32_t a_format,
                       int32_t b_format, void *y, int32_t y_type, void *ws, hipStream_t stream)
{
    const int64_t n = (int64_t)M * N;
    if (n == 0) return CDL_OK;
    if (K == 0) {
        return in_launches(n, kLaunchThreads, [&](int64_t at, int64_t count) {
            const unsigned blocks = (unsigned)((count + 255) / 256);
            if (y_type == CDL_BF16) CDL_LAUNCH("block8_zero_kernel", stream, zero_kernel<bf16_t>, dim3(blocks), dim3(256), 0, (bf16_t *)y + at, count);
            else CDL_LAUNCH("block8_zero_kernel", stream, zero_kernel<float>, dim3(blocks), dim3(256), 0, (float *)y + at, count);
        });
    }
    const Layout l = layout(M, N, K);
    const int64_t ld = block8_pitch(K);
    RingJob job{};
    job.P = b;
    job.Q = a;
    job.ldp = job.ldq = ld;
    job.rowsP = N;
    job.rowsQ = M;
    job.nk = (int)(ld / kRingRow);
    job.tiles_p = l.tiles_p;
    job.tiles_q = l.tiles_q;
    job.splits = l.splits;
    job.k_per = l.k_per;
    job.sp = b_scale;
    job.sq = a_scale;
    job.pitch_sp = block8_pitch(N);
    job.pitch_sq = block8_pitch(M);
    if (l.splits == 1)
        return y_type == CDL_BF16 ? launch_product<false>(job, l, a_format, b_format, (bf16_t *)y, M, N, stream) : launch_product<true>(job, l, a_format, b_format, (float *)y, M, N, stream);
    const int rc = y_type == CDL_BF16 ? launch_product<false>(job, l, a_format, b_format, (float *)ws, M, N, stream)
                                      : launch_product<true>(job, l, a_format, b_format, (float *)ws, M, N, stream);
    if (rc != CDL_OK) return rc;
    const unsigned blocks = (unsigned)((n + 1023) / 1024);
    if (y_type == CDL_BF16) CDL_LAUNCH("block8_sum_kernel", stream, block8_sum_kernel<bf16_t>, dim3(blocks), dim3(256), 0, (const float *)ws, l.splits, n, (bf16_t *)y);
    else CDL_LAUNCH("block8_sum_kernel", stream, block8_sum_kernel<float>, dim3(blocks), dim3(256), 0, (const float *)ws, l.splits, n, (float *)y);
    return check_launch();
}

}  // namespace cdl
