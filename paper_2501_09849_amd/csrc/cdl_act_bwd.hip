// Backward passes of what stands behind a product: the activation of a layer, and the gated product of two projections, from their values before it (z) as they are or
// as kept in 8-bit floating point, with the sums over the rows that are the biases' gradients.
//
//   d_z = g act'(z),  y = act(z)          d_gate = g z_up act'(z_gate),  d_up = g act(z_gate),  y = act(z_gate) z_up
//
// Bound by memory, 65536 x 2048 in bf16: gelu 162 us (805 MB, 5.0 TB/s; its 32 instructions an entry take about as long beside), the gated silu from eight bits 221 us (1.08 GB, 4.9 TB/s).
// The sums over the rows come in the same pass, from the gradients before their rounding: a pass of their own would read 268 MB again for each.
#include "cdl_act.h"
#include "cdl_block8.h"
#include "cdl_chunks.h"

namespace cdl {
namespace {

// A block: 256 columns, 32 lanes of eight each, eight rows at a time of its stretch of rows; a thread's sums of its columns stay in registers.  TALL: 64 columns, 64 rows at a
// time, for sums of few rows, which one block then has whole: a second launch that adds up parts takes about
// 3.5 us (74 x 75 in fp32 8.5 us with it, 5.0 without; 384 x 576 in bf16 from eight bits 8.9 and 5.3).  From 385 rows on the longer walk costs what the launch did: gelu, 385 x 2048 in bf16, 7.9 us
// in two launches, 384 rows 7.5 in one; 512 rows 7.9 and 9.0.
// Narrow tensors leave lanes idle, 30 of 32 at 16 columns: gelu, 65536 x 16 in bf16, 17 us, 65536 x 128 19.6.
template <bool TALL> constexpr int kLanes = TALL ? 8 : 32;
template <bool TALL> constexpr int kGroups = TALL ? 64 : 8;
template <bool TALL> constexpr int kThreads = kLanes<TALL> * kGroups<TALL>;
template <bool TALL> constexpr int kCols = kLanes<TALL> * 8;
constexpr int kTallRows = 384;

struct ActBwd {
    const void *g, *z[2];                 // z of the gate (or of the layer), and of the other projection
    const uint8_t *q[2], *scale[2];
    int rows, cols, col_blocks, rows_per;
    void *d[2], *y;
    float *parts;                         // [stretch of rows][1 or 2][part_cols], or null
    float *sums[2];                       // of one stretch alone: where its sums go at once
    int64_t pitch_c, pitch_r, part_cols;
    bool stream;
};

template <class T, int ACT, bool GATED, bool RAGGED, int KEPT, bool TALL>      // KEPT: 0 no, 1 E4M3, 2 E5M2
__global__ __launch_bounds__(kThreads<TALL>)
void act_bwd_kernel(ActBwd a)
{
    constexpr int S = GATED ? 2 : 1, kRows = kGroups<TALL>, kAcross = kCols<TALL>;
    const int lane = threadIdx.x % kLanes<TALL>, group = threadIdx.x / kLanes<TALL>;
    const int cb = (int)(blockIdx.x % (unsigned)a.col_blocks), part = (int)(blockIdx.x / (unsigned)a.col_blocks);
    const int col = cb * kAcross + lane * 8, left = a.cols - col;
    const int64_t first = (int64_t)part * a.rows_per, end = min(first + a.rows_per, (int64_t)a.rows);
    Raw8<T> raw_g, raw_z[S];
    u32x2 kept[S];
    uint32_t byte[S];
    auto fetch = [&](int64_t r) {
        const int64_t at = r * a.cols + col;
        raw_g = load_raw<RAGGED>((const T *)a.g + at, left, a.stream, a.cols < 8);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (KEPT) {
                if (left > 0) {
                    kept[s] = *reinterpret_cast<const u32x2 *>(a.q[s] + r * a.pitch_c + col);
                    byte[s] = a.scale[s][(int64_t)(col >> 7) * a.pitch_r + r];
                } else {
                    kept[s] = u32x2{0, 0};
                    byte[s] = 127;
                }
            } else {
                raw_z[s] = load_raw<RAGGED>((const T *)a.z[s] + at, left, a.stream, a.cols < 8);
            }
        }
    };
    float sums[S][8];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int k = 0; k < 8; ++k) sums[s][k] = 0.0f;
    int64_t row = first + group;
    if (row < end) fetch(row);
    for (; row < end; row += kRows) {
        float g[8], z[S][8], d[S][8], y[8];
        unpack<RAGGED>(raw_g, left, a.cols < 8, g);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (KEPT) {
                values8<KEPT == 2>(kept[s], z[s]);
                const float by = scale_of(byte[s]);
#pragma unroll
                for (int k = 0; k < 8; ++k) z[s][k] *= by;
            } else {
                unpack<RAGGED>(raw_z[s], left, a.cols < 8, z[s]);
            }
        }
        if (row + kRows < end) fetch(row + kRows);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const ValueSlope v = act_both<ACT>(z[0][k]);
            if constexpr (GATED) {
                d[0][k] = g[k] * z[1][k] * v.slope;
                d[1][k] = g[k] * v.value;
                y[k] = v.value * z[1][k];
            } else {
                d[0][k] = g[k] * v.slope;
                y[k] = v.value;
            }
#pragma unroll
            for (int s = 0; s < S; ++s) sums[s][k] += d[s][k];
        }
        const int64_t at = row * a.cols + col;
#pragma unroll
        for (int s = 0; s < S; ++s)
            if (a.d[s]) store_first<RAGGED>((T *)a.d[s] + at, left, d[s], a.stream);
        if (a.y) store_first<RAGGED>((T *)a.y + at, left, y, a.stream);
    }
    if (!a.parts && !a.sums[0] && !a.sums[1]) return;
    __shared__ float all[kRows][kAcross];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        if (s > 0) __syncthreads();
        store8(&all[group][lane * 8], sums[s], false);
        __syncthreads();
        float *const out = a.parts ? a.parts + ((int64_t)part * S + s) * a.part_cols : a.sums[s];
        if (out && threadIdx.x < kAcross && cb * kAcross + (int)threadIdx.x < a.cols) {
            float sum = 0.0f;
#pragma unroll 8
            for (int i = 0; i < kRows; ++i) sum += all[i][threadIdx.x];
            out[cb * kAcross + threadIdx.x] = sum;
        }
    }
}

// Sums of the blocks' parts [parts][sets][pitch] over the first index: 16 columns a block, 64 threads each, whose sums are joined in a fixed order.
__global__ __launch_bounds__(1024)
void column_sums_kernel(const float *__restrict__ parts, int64_t n, int sets, int64_t cols, int64_t pitch, float *out0, float *out1)
{
    __shared__ float all[16][16];
    const int lane = threadIdx.x & 15, group = threadIdx.x >> 4;
    const int64_t col = (int64_t)blockIdx.x * 16 + lane;
    float *const out = blockIdx.y ? out1 : out0;
    if (!out) return;
    float sum = 0.0f;
    if (col < cols) {
#pragma unroll 8
        for (int64_t i = group; i < n; i += 64) sum += parts[(i * sets + blockIdx.y) * pitch + col];
    }
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if ((threadIdx.x & 63) < 16) all[threadIdx.x >> 6][lane] = sum;
    __syncthreads();
    if (threadIdx.x < 16 && col < cols) {
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += all[i][lane];
        out[col] = sum;
    }
}

int64_t part_cols(int32_t cols) { return ((int64_t)cols + 7) / 8 * 8; }

// Stretches of rows: blocks that fill the chip, of at least 16 rows; up to 32 rows, and where sums are asked for up to 384, are one, whose sums take no second launch.
struct Split {
    int col_blocks, parts, rows_per;
    bool tall;
};
Split split_of(int32_t rows, int32_t cols, bool sums)
{
    Split s;
    s.tall = sums && rows > 32 && rows <= kTallRows;
    if (s.tall) {
        s.col_blocks = (cols + kCols<true> - 1) / kCols<true>;
        s.parts = 1;
        s.rows_per = rows;
        return s;
    }
    s.col_blocks = (cols + kCols<false> - 1) / kCols<false>;
    int64_t parts = (2048 + s.col_blocks - 1) / s.col_blocks;
    const int64_t most = rows <= 32 ? 1 : ((int64_t)rows + 15) / 16;
    if (parts > most) parts = most;
    s.rows_per = (int)((rows + parts - 1) / parts);
    s.parts = (rows + s.rows_per - 1) / s.rows_per;
    return s;
}

template <class T, int ACT, bool GATED, bool RAGGED, bool TALL>
int launch_act(const ActBwd &a, int kept, int64_t blocks, hipStream_t stream)
{
    const auto kernel = kept == 0   ? act_bwd_kernel<T, ACT, GATED, RAGGED, 0, TALL>
                        : kept == 1 ? act_bwd_kernel<T, ACT, GATED, RAGGED, 1, TALL>
                                    : act_bwd_kernel<T, ACT, GATED, RAGGED, 2, TALL>;
    CDL_LAUNCH(GATED ? "gated_bwd_kernel" : "act_bwd_kernel", stream, kernel, dim3((unsigned)blocks), dim3(kThreads<TALL>), 0, a);
    return check_launch();
}
template <class T, int ACT, bool GATED, bool RAGGED>
int launch_act(const ActBwd &a, int kept, const Split &s, hipStream_t stream)
{
    const int64_t blocks = (int64_t)s.col_blocks * s.parts;
    return s.tall ? launch_act<T, ACT, GATED, RAGGED, true>(a, kept, blocks, stream) : launch_act<T, ACT, GATED, RAGGED, false>(a, kept, blocks, stream);
}
template <class T, bool GATED, bool RAGGED>
int launch_any(const ActBwd &a, int act, int kept, const Split &s, hipStream_t stream)
{
    switch (act) {
        case CDL_ACT_RELU: return launch_act<T, CDL_ACT_RELU, GATED, RAGGED>(a, kept, s, stream);
        case CDL_ACT_GELU: return launch_act<T, CDL_ACT_GELU, GATED, RAGGED>(a, kept, s, stream);
        case CDL_ACT_SILU: return launch_act<T, CDL_ACT_SILU, GATED, RAGGED>(a, kept, s, stream);
        default: return launch_act<T, CDL_ACT_NONE, GATED, RAGGED>(a, kept, s, stream);
    }
}
template <bool GATED>
int launch_all(ActBwd a, int type, int act, int kept, const Split &s, hipStream_t stream)
{
    if (a.cols % 8 == 0)
        return type == CDL_BF16 ? launch_any<bf16_t, GATED, false>(a, act, kept, s, stream) : launch_any<float, GATED, false>(a, act, kept, s, stream);
    return type == CDL_BF16 ? launch_any<bf16_t, GATED, true>(a, act, kept, s, stream) : launch_any<float, GATED, true>(a, act, kept, s, stream);
}

}  // namespace

int launch_column_sums(const float *parts, int64_t n, int32_t cols, int64_t pitch, float *out0, float *out1, hipStream_t stream, int sets)
{
    const dim3 grid((unsigned)((cols + 15) / 16), (unsigned)sets);
    CDL_LAUNCH("column_sums_kernel", stream, column_sums_kernel, grid, dim3(1024), 0, parts, n, sets, (int64_t)cols, pitch, out0, out1);
    return check_launch();
}

size_t act_bwd_workspace_bytes(int32_t rows, int32_t cols, bool gated)
{
    if (rows == 0 || cols == 0 || split_of(rows, cols, true).parts == 1) return 0;
    return align_up((size_t)split_of(rows, cols, true).parts * (gated ? 2 : 1) * (size_t)part_cols(cols) * sizeof(float), 256);
}

int launch_act_bwd(const ActCall &c, bool gated, hipStream_t stream)
{
    if (c.cols == 0) return CDL_OK;
    const bool sums = c.d_bias[0] || c.d_bias[1];
    const int64_t size = c.type == CDL_BF16 ? 2 : 4;
    int64_t parts = 0;
    if (c.rows > 0) {
        const Split s = split_of(c.rows, c.cols, sums);
        parts = s.parts;
        ActBwd a{};
        a.g = c.g;
        for (int i = 0; i < 2; ++i) {
            a.z[i] = c.z[i];
            a.q[i] = c.q[i];
            a.scale[i] = c.scale[i];
            a.d[i] = c.d[i];
        }
        a.rows = c.rows;
        a.cols = c.cols;
        a.col_blocks = s.col_blocks;
        a.rows_per = s.rows_per;
        a.y = c.y;
        a.parts = sums && parts > 1 ? (float *)c.ws : nullptr;
        for (int i = 0; i < 2; ++i) a.sums[i] = parts == 1 ? c.d_bias[i] : nullptr;
        a.pitch_c = block8_pitch(c.cols);
        a.pitch_r = block8_pitch(c.rows);
        a.part_cols = part_cols(c.cols);
        a.stream = (int64_t)c.rows * c.cols * size >= kStreamFrom * 4;
        const int kept = !c.q[0] ? 0 : c.format == CDL_E5M2 ? 2 : 1;
        const int rc = gated ? launch_all<true>(a, c.type, c.act, kept, s, stream) : launch_all<false>(a, c.type, c.act, kept, s, stream);
        if (rc != CDL_OK) return rc;
    }
    return sums && parts != 1 ? launch_column_sums((const float *)c.ws, parts, c.cols, part_cols(c.cols), c.d_bias[0], c.d_bias[1], stream, gated ? 2 : 1) : CDL_OK;
}

}  // namespace cdl
