// The block-scaled product with what stands behind it in a layer, and the gated product of two projections:
//
//   z = a b^T + bias,  y = act(z) + add                    y = act(a gate^T + bias) * (a up^T + bias)
#include "cdl_act.h"
#include "cdl_chunks.h"

namespace cdl {
namespace {

// Products that went to memory as fp32 sums of parts of the contraction: added up, in order, and finished.  A thread takes eight consecutive entries of a row.
constexpr int kLanes = 32, kRows = 8, kThreads = kLanes * kRows, kCols = kLanes * 8;

struct Finish {
    const float *parts[2];
    int splits, M, N, col_blocks, row_blocks;
    const float *bias[2];
    const void *add;
    void *y, *z[2];
};

template <class T, int ACT, bool GATED, bool RAGGED>
__global__ __launch_bounds__(kThreads)
void block8_finish_kernel(Finish f)
{
    constexpr int S = GATED ? 2 : 1;
    const int col = (int)(blockIdx.x % (unsigned)f.col_blocks) * kCols + (int)(threadIdx.x % kLanes) * 8, left = f.N - col;
    const int64_t whole = (int64_t)f.M * f.N;
    float bias[S][8];
#pragma unroll
    for (int s = 0; s < S; ++s) load_vector<RAGGED>(f.bias[s] ? f.bias[s] + col : nullptr, left, 0.0f, bias[s]);
    for (int64_t row = (int64_t)(blockIdx.x / (unsigned)f.col_blocks) * kRows + threadIdx.x / kLanes; row < f.M; row += (int64_t)f.row_blocks * kRows) {
        const int64_t at = row * f.N + col;
        float z[S][8], y[8], add[8];
#pragma unroll
        for (int s = 0; s < S; ++s) {
#pragma unroll
            for (int k = 0; k < 8; ++k) z[s][k] = 0.0f;
            for (int i = 0; i < f.splits; ++i) {
                float v[8];
                unpack(load_raw<RAGGED>(f.parts[s] + i * whole + at, left, false), v);
#pragma unroll
                for (int k = 0; k < 8; ++k) z[s][k] += v[k];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) z[s][k] += bias[s][k];
            if (f.z[s]) store_first<RAGGED>((T *)f.z[s] + at, left, z[s], false);
        }
        if (f.add) unpack(load_raw<RAGGED>((const T *)f.add + at, left, false), add);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float v = act_value<ACT>(z[0][k]);
            if constexpr (GATED) y[k] = v * z[1][k];
            else y[k] = f.add ? v + add[k] : v;
        }
        store_first<RAGGED>((T *)f.y + at, left, y, false);
    }
}

template <class T, bool GATED, bool RAGGED>
int launch_finish(const Finish &f, int act, hipStream_t stream)
{
    const auto kernel = act == CDL_ACT_RELU   ? block8_finish_kernel<T, CDL_ACT_RELU, GATED, RAGGED>
                        : act == CDL_ACT_GELU ? block8_finish_kernel<T, CDL_ACT_GELU, GATED, RAGGED>
                        : act == CDL_ACT_SILU ? block8_finish_kernel<T, CDL_ACT_SILU, GATED, RAGGED>
                                              : block8_finish_kernel<T, CDL_ACT_NONE, GATED, RAGGED>;
    CDL_LAUNCH("block8_finish_kernel", stream, kernel, dim3((unsigned)f.col_blocks * (unsigned)f.row_blocks), dim3(kThreads), 0, f);
    return check_launch();
}
template <class T>
int launch_finish(const Finish &f, int act, bool gated, hipStream_t stream)
{
    if (f.N % 8 == 0) return gated ? launch_finish<T, true, false>(f, act, stream) : launch_finish<T, false, false>(f, act, stream);
    return gated ? launch_finish<T, true, true>(f, act, stream) : launch_finish<T, false, true>(f, act, stream);
}

size_t parts_bytes(int32_t M, int32_t N, int32_t K) { return align_up((size_t)block8_parts(M, N, K) * (size_t)M * (size_t)N * sizeof(float), 256); }

}  // namespace

size_t block8_gemm_act_workspace_bytes(int32_t M, int32_t N, int32_t K, bool gated) { return parts_bytes(M, N, K) * (gated ? 2 : 1); }

int launch_block8_gemm_act(const ProductCall &c, bool gated, hipStream_t stream)
{
    if (c.M == 0 || c.N == 0) return CDL_OK;
    Finish f{};
    f.splits = block8_parts(c.M, c.N, c.K);
    f.M = c.M;
    f.N = c.N;
    f.add = c.add;
    f.y = c.y;
    for (int s = 0; s < (gated ? 2 : 1); ++s) {
        float *const parts = (float *)((uint8_t *)c.ws + s * parts_bytes(c.M, c.N, c.K));
        f.parts[s] = parts;
        f.bias[s] = c.bias[s];
        f.z[s] = c.z[s];
        if (f.splits == 0) continue;
        const int rc = launch_block8_parts(c.a, c.a_scale, c.b[s], c.b_scale[s], c.M, c.N, c.K, c.a_format, c.b_format, c.y_type == CDL_F32, parts, stream);
        if (rc != CDL_OK) return rc;
    }
    f.col_blocks = (c.N + kCols - 1) / kCols;
    const int64_t rows = ((int64_t)c.M + kRows - 1) / kRows, most = (1 << 23) / f.col_blocks;
    f.row_blocks = (int)(rows < most ? rows : most);
    if (f.row_blocks < 1) f.row_blocks = 1;
    return c.y_type == CDL_BF16 ? launch_finish<bf16_t>(f, c.act, gated, stream) : launch_finish<float>(f, c.act, gated, stream);
}

}  // namespace cdl
