// Layer norm of the rows of a matrix, its gradients, and the rows' copy in 8-bit floating point from which the backward pass can be formed.
//
//   m = mean of the row, r = 1 / sqrt(mean of (x - m)^2 + eps), c = (x - m) r;     y = c w + b
//   h = g w:   d_x = r (h - mean of h - c mean of (h c)) + add,     d_w = sum over rows of g c,     d_b = sum over rows of g
//
// A row stays in the registers of L lanes, C chunks of eight entries each, so that it is read once: the mean, then the squares about it (a sum of squares less the mean's square would
// lose rows far from zero), then the results.  The mean's own roundings would enter every entry alike, times r (rows of 1000.1 and no spread came out 0.06 off their bias): it is the first
// entry and the mean of the differences from it, which are all zero in such a row, and what it is still off is the mean of the differences from it, summed beside their squares.  Lanes that are not a whole block are a wave or a quarter of one, and their sums never leave the registers.  Weights, and backward the sums over the rows, stay
// in registers too, so a team takes row after row, the next one's loads under way.
// Bound by memory, 65536 x 768 in bf16: forward with the copy in eight bits 53 us (252 MB, 4.7 TB/s where a copy reaches 5.2), without 41; backward from eight bits onto a residual 70 us
// (353 MB, 5.0 TB/s), from bf16 77, and 4 us for adding up the blocks' sums in a launch of their own.  2000 x 16384: forward 28.5 us, backward 76.
#include "cdl_block8.h"
#include "cdl_chunks.h"

namespace cdl {
namespace {

template <int L>
constexpr int kThreadsOf = L > 256 ? L : 256;

// Sums over the L lanes of a row, in all of them.  `slot` alternates between 0 and 1 from one sum to the next: beyond a wave, one barrier each.
template <int L, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], int slot)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
#define CDL_ROR(D) v[i] += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v[i]), 0x120 + D, 0xf, 0xf, false))
        CDL_ROR(8); CDL_ROR(4); CDL_ROR(2); CDL_ROR(1);
#undef CDL_ROR
        if (L >= 64) {
            v[i] += __shfl_xor(v[i], 16, 64);
            v[i] += __shfl_xor(v[i], 32, 64);
        }
    }
    if constexpr (L > 64) {
        __shared__ float sums[2][N][L / 64];
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) sums[slot][i][threadIdx.x >> 6] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.0f;
#pragma unroll
            for (int w = 0; w < L / 64; ++w) v[i] += sums[slot][i][w];
        }
    }
}

struct NormFwd {
    const void *x;
    const float *weight, *bias;
    int rows, cols;
    float eps, by_cols;
    void *y;
    float *mean, *rstd;
    uint8_t *q, *scale;
    int64_t pitch_c, pitch_r, rows_end;      // rows_end: with q, rows up to whole blocks
    bool stream;
};

template <class T, int L, int C, bool RAGGED, int KEEP>      // KEEP: 0 no copy, 1 E4M3, 2 E5M2
__global__ __launch_bounds__(kThreadsOf<L>)
void layer_norm_fwd_kernel(NormFwd a)
{
    constexpr int kTeams = kThreadsOf<L> / L;
    const int lane = threadIdx.x % L, team = threadIdx.x / L;
    float w[C][8], b[C][8];
    int left[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (c * L + lane) * 8;
        left[c] = a.cols - col;
        load_vector<RAGGED>(a.weight ? a.weight + col : nullptr, left[c], a.cols < 8, 1.0f, w[c]);
        load_vector<RAGGED>(a.bias ? a.bias + col : nullptr, left[c], a.cols < 8, 0.0f, b[c]);
    }
    const int64_t step = (int64_t)gridDim.x * kTeams;
    int64_t row = (int64_t)blockIdx.x * kTeams + team;
    Raw8<T> raw[C];
    T raw_first;
    auto fetch = [&](int64_t r) {
        raw_first = ((const T *)a.x)[r * a.cols];
#pragma unroll
        for (int c = 0; c < C; ++c) raw[c] = load_raw<RAGGED>((const T *)a.x + r * a.cols + (c * L + lane) * 8, left[c], a.stream, a.cols < 8);
    };
    // Entries beyond the row add nothing to a sum of differences: these are selected, or, where the selections' masks would take more scalar registers than there are, such entries
    // are set to what is subtracted, in a branch that most waves skip (4915 x 10239 with the copy: 79 us, 83 with selections).
    constexpr bool kSet = RAGGED && C == 4;
    auto inside = [&](int c, int k, float v) { return !RAGGED || kSet || k < left[c] ? v : 0.0f; };
    auto end_with = [](float (&v)[8], int n, float value) {
        if (kSet && n < 8) {
            asm volatile("" : "+v"(n));      // (compared here, not ahead of the loop)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = k < n ? v[k] : value;
        }
    };
    if (row < a.rows) fetch(row);
    for (; row < a.rows_end; row += step) {
        if (row < a.rows) {
            float v[C][8];
#pragma unroll
            for (int c = 0; c < C; ++c) unpack<RAGGED>(raw[c], left[c], a.cols < 8, v[c]);
            const float first = (float)raw_first;
            if (row + step < a.rows) fetch(row + step);
            float sum[1] = {0.0f};
#pragma unroll
            for (int c = 0; c < C; ++c) {
                end_with(v[c], left[c], first);
                float part = 0.0f;
#pragma unroll
                for (int k = 0; k < 8; ++k) part += inside(c, k, v[c][k] - first);
                sum[0] += kSet || left[c] > 0 ? part : 0.0f;
            }
            row_sums<L>(sum, 0);
            const float near = __builtin_fmaf(sum[0], a.by_cols, first);
            if (KEEP) {
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    end_with(v[c], left[c], 0.0f);
                    uint32_t largest = 0;
#pragma unroll
                    for (int k = 0; k < 8; ++k) largest = max(largest, __float_as_uint(v[c][k]) & 0x7fffffffu);
                    const uint32_t byte = scale_byte(row16_max(largest), KEEP == 2 ? 15 : 8);
                    const float by = inverse(byte);
                    const int col = (c * L + lane) * 8;
                    float s[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) s[k] = v[c][k] * by;
                    if (col < a.pitch_c) {
                        *reinterpret_cast<u32x2 *>(a.q + row * a.pitch_c + col) = eight<KEEP == 2>(s);
                        if ((lane & 15) == 0) a.scale[(int64_t)(col >> 7) * a.pitch_r + row] = (uint8_t)byte;
                    }
                }
            }
            float about[2] = {0.0f, 0.0f};
#pragma unroll
            for (int c = 0; c < C; ++c) {
                end_with(v[c], left[c], near);
                float part[2] = {0.0f, 0.0f};
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    v[c][k] = inside(c, k, v[c][k] - near);
                    part[0] += v[c][k];
                    part[1] = __builtin_fmaf(v[c][k], v[c][k], part[1]);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) about[i] += kSet || left[c] > 0 ? part[i] : 0.0f;
            }
            row_sums<L>(about, 1);
            const float off = about[0] * a.by_cols, var = __builtin_fmaf(-off, off, about[1] * a.by_cols), mean = near + off;
            const float rstd = 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + a.eps), back = -off * rstd;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float y[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = __builtin_fmaf(__builtin_fmaf(v[c][k], rstd, back), w[c][k], b[c][k]);
                store_first<RAGGED>((T *)a.y + row * a.cols + (c * L + lane) * 8, left[c], y, a.stream);
            }
            if (lane == 0) {
                if (a.mean) a.mean[row] = mean;
                if (a.rstd) a.rstd[row] = rstd;
            }
        } else if (KEEP) {      // scales of rows beyond the matrix
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * L + lane) * 8;
                if (col < a.pitch_c && (lane & 15) == 0) a.scale[(int64_t)(col >> 7) * a.pitch_r + row] = (uint8_t)kLeast;
            }
        }
    }
}

struct NormBwd {
    const void *g, *x;
    const uint8_t *q, *scale;
    const float *weight, *mean, *rstd;
    const void *add;
    int rows, cols;
    float by_cols;
    void *d_x;
    float *parts;                      // [block][2][part_cols]: d_w, d_b of the block's rows; or null
    float *sums[2];                    // of one block alone: where they go at once
    int64_t pitch_c, pitch_r, part_cols;
    bool stream;
};

// KEPT: 0 from x, 1 from its copy in E4M3, 2 E5M2
template <class T, int L, int C, bool RAGGED, int KEPT>
__global__ __launch_bounds__(kThreadsOf<L>)
void layer_norm_bwd_kernel(NormBwd a)
{
    constexpr int kTeams = kThreadsOf<L> / L;
    const int lane = threadIdx.x % L, team = threadIdx.x / L;
    float w[C][8], dw[C][8], db[C][8];
    int left[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (c * L + lane) * 8;
        left[c] = a.cols - col;
        load_vector<RAGGED>(a.weight ? a.weight + col : nullptr, left[c], a.cols < 8, 1.0f, w[c]);
#pragma unroll
        for (int k = 0; k < 8; ++k) dw[c][k] = db[c][k] = 0.0f;
    }
    const int64_t step = (int64_t)gridDim.x * kTeams;
    constexpr bool kAhead = L <= 256;      // the next row's loads under way while a row is worked on, as far as there are registers
    Raw8<T> raw_g[C], raw_x[C], raw_add[C];
    u32x2 kept[C];
    uint32_t byte[C];
    float mean = 0.0f, rstd = 0.0f;
    auto fetch = [&](int64_t r) {
        mean = a.mean[r];
        rstd = a.rstd[r];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * L + lane) * 8;
            const int64_t at = r * a.cols + col;
            raw_g[c] = load_raw<RAGGED>((const T *)a.g + at, left[c], a.stream, a.cols < 8);
            if (KEPT) {
                if (left[c] > 0) {
                    kept[c] = *reinterpret_cast<const u32x2 *>(a.q + r * a.pitch_c + col);
                    byte[c] = a.scale[(int64_t)(col >> 7) * a.pitch_r + r];
                } else {
                    kept[c] = u32x2{0, 0};
                    byte[c] = 127;
                }
            } else {
                raw_x[c] = load_raw<RAGGED>((const T *)a.x + at, left[c], a.stream, a.cols < 8);
            }
            if (kAhead && a.add && a.d_x) raw_add[c] = load_raw<RAGGED>((const T *)a.add + at, left[c], a.stream, a.cols < 8);
        }
    };
    int64_t row = (int64_t)blockIdx.x * kTeams + team;
    if (kAhead && row < a.rows) fetch(row);
    int slot = 0;
    for (; row < a.rows; row += step) {
        if (!kAhead) fetch(row);
        float n[C][8], h[C][8], add[C][8];
        const float r = rstd;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (KEPT) {
                values8<KEPT == 2>(kept[c], n[c]);
                const float by = scale_of(byte[c]);
#pragma unroll
                for (int k = 0; k < 8; ++k) n[c][k] *= by;
            } else {
                unpack<RAGGED>(raw_x[c], left[c], a.cols < 8, n[c]);
            }
            unpack<RAGGED>(raw_g[c], left[c], a.cols < 8, h[c]);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                n[c][k] = (n[c][k] - mean) * r;
                dw[c][k] = __builtin_fmaf(h[c][k], n[c][k], dw[c][k]);
                db[c][k] += h[c][k];
                h[c][k] *= w[c][k];
            }
            if (kAhead) {
                if (a.add && a.d_x) unpack<RAGGED>(raw_add[c], left[c], a.cols < 8, add[c]);
                else {
#pragma unroll
                    for (int k = 0; k < 8; ++k) add[c][k] = 0.0f;
                }
            }
        }
        if (kAhead && row + step < a.rows) fetch(row + step);
        if (!a.d_x) continue;
        float sums[2] = {0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                sums[0] += h[c][k];
                sums[1] = __builtin_fmaf(h[c][k], n[c][k], sums[1]);
            }
        row_sums<L>(sums, slot);
        slot ^= 1;
        const float one = sums[0] * a.by_cols, two = sums[1] * a.by_cols;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float d[8];
            if (!kAhead) {
#pragma unroll
                for (int k = 0; k < 8; ++k) add[c][k] = 0.0f;
                if (a.add) unpack<RAGGED>(load_raw<RAGGED>((const T *)a.add + row * a.cols + (c * L + lane) * 8, left[c], a.stream, a.cols < 8), left[c], a.cols < 8, add[c]);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) d[k] = __builtin_fmaf(h[c][k] - one - n[c][k] * two, r, add[c][k]);
            store_first<RAGGED>((T *)a.d_x + row * a.cols + (c * L + lane) * 8, left[c], d, a.stream);
        }
    }
    if (!a.parts && !a.sums[0] && !a.sums[1]) return;
    float *const out[2] = {a.parts ? a.parts + (int64_t)blockIdx.x * 2 * a.part_cols : a.sums[0], a.parts ? a.parts + ((int64_t)blockIdx.x * 2 + 1) * a.part_cols : a.sums[1]};
    if constexpr (kTeams > 1) {      // the teams of a block one after the other
        __shared__ float part[2][L * C * 8];
        for (int t = 0; t < kTeams; ++t) {
            if (team == t) {
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int at = (c * L + lane) * 8 + k;
                        part[0][at] = t ? part[0][at] + dw[c][k] : dw[c][k];
                        part[1][at] = t ? part[1][at] + db[c][k] : db[c][k];
                    }
            }
            __syncthreads();
        }
        for (int at = threadIdx.x; at < a.cols; at += kThreadsOf<L>) {
            if (out[0]) out[0][at] = part[0][at];
            if (out[1]) out[1][at] = part[1][at];
        }
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * L + lane) * 8;
            if (out[0]) store_first<RAGGED>(out[0] + col, left[c], dw[c], false);
            if (out[1]) store_first<RAGGED>(out[1] + col, left[c], db[c], false);
        }
    }
}

constexpr int kForms = 8;
// lanes of a row, chunks of a lane: up to 128, 256, 512, 1024, 2048, 4096, 8192 and 16384 entries (in 1024 lanes the longest would spill: 2000 x 16384 backward 520 us so.
// In 512 lanes nothing does where rows are whole; ragged ones keep 4 to 16 registers of a thread in memory, backward: 2000 x 16383 in bf16 91 us where 16384 take 76, in fp32 136 and 123)
constexpr int kLanes[kForms] = {16, 16, 64, 64, 256, 256, 256, 512}, kChunksOf[kForms] = {1, 2, 1, 2, 1, 2, 4, 4};
static_assert(kLanes[kForms - 1] * kChunksOf[kForms - 1] * 8 == kNormMostCols, "the longest row");
int form_of(int32_t cols)
{
    int f = 0;
    while (f < kForms - 1 && cols > kLanes[f] * kChunksOf[f] * 8) ++f;
    return f;
}
int64_t teams_of(int form) { return (kLanes[form] > 256 ? kLanes[form] : 256) / kLanes[form]; }

int64_t fwd_blocks(int form, int64_t rows)
{
    const int64_t blocks = (rows + teams_of(form) - 1) / teams_of(form), most = kLanes[form] > 256 ? 512 : 2048;
    return blocks < most ? blocks : most;
}
// Backward: as many rows for every team, on the blocks that a compute unit holds two of, or one where a block has one row at a time and a thread many registers.  More blocks leave more
// sums to be added up, and rows that do not come out even (65536 x 768 from eight bits: 384 blocks 82.4 us, 512 71.6, 768 73.7, 1024 81.6; 4096 x 8192: 256 blocks 61.2, 512 70.0).
// Sums of few rows are one block's, which has them without a second launch (16 x 768: 6.9 us instead of 8.9); where none are asked for, every team has a row as long as there are blocks.
int64_t bwd_blocks(int form, int64_t rows, bool sums)
{
    if (sums && rows <= 4 * teams_of(form)) return 1;
    const int64_t teams = teams_of(form), most = teams == 1 && kChunksOf[form] > 1 ? 256 : 512, per = (rows + most * teams - 1) / (most * teams);
    return (rows + per * teams - 1) / (per * teams);
}
int64_t part_cols(int32_t cols) { return ((int64_t)cols + 7) / 8 * 8; }

template <class T, bool RAGGED, int KEEP>
int launch_fwd(const NormFwd &a, hipStream_t stream)
{
    const int form = form_of(a.cols);
    typedef void (*kernel_t)(NormFwd);
    static const kernel_t kernels[kForms] = {layer_norm_fwd_kernel<T, 16, 1, RAGGED, KEEP>, layer_norm_fwd_kernel<T, 16, 2, RAGGED, KEEP>, layer_norm_fwd_kernel<T, 64, 1, RAGGED, KEEP>,
                                             layer_norm_fwd_kernel<T, 64, 2, RAGGED, KEEP>, layer_norm_fwd_kernel<T, 256, 1, RAGGED, KEEP>, layer_norm_fwd_kernel<T, 256, 2, RAGGED, KEEP>,
                                             layer_norm_fwd_kernel<T, 256, 4, RAGGED, KEEP>, layer_norm_fwd_kernel<T, 512, 4, RAGGED, KEEP>};
    CDL_LAUNCH("layer_norm_fwd_kernel", stream, kernels[form], dim3((unsigned)fwd_blocks(form, a.rows_end)), dim3(kLanes[form] > 256 ? kLanes[form] : 256), 0, a);
    return check_launch();
}
template <class T>
int launch_fwd(const NormFwd &a, int keep, hipStream_t stream)
{
    if (a.cols % 8 == 0) return keep == 0 ? launch_fwd<T, false, 0>(a, stream) : keep == 1 ? launch_fwd<T, false, 1>(a, stream) : launch_fwd<T, false, 2>(a, stream);
    return keep == 0 ? launch_fwd<T, true, 0>(a, stream) : keep == 1 ? launch_fwd<T, true, 1>(a, stream) : launch_fwd<T, true, 2>(a, stream);
}

template <class T, bool RAGGED, int KEPT>
int launch_bwd(const NormBwd &a, hipStream_t stream)
{
    const int form = form_of(a.cols);
    typedef void (*kernel_t)(NormBwd);
    static const kernel_t kernels[kForms] = {layer_norm_bwd_kernel<T, 16, 1, RAGGED, KEPT>, layer_norm_bwd_kernel<T, 16, 2, RAGGED, KEPT>, layer_norm_bwd_kernel<T, 64, 1, RAGGED, KEPT>,
                                             layer_norm_bwd_kernel<T, 64, 2, RAGGED, KEPT>, layer_norm_bwd_kernel<T, 256, 1, RAGGED, KEPT>, layer_norm_bwd_kernel<T, 256, 2, RAGGED, KEPT>,
                                             layer_norm_bwd_kernel<T, 256, 4, RAGGED, KEPT>, layer_norm_bwd_kernel<T, 512, 4, RAGGED, KEPT>};
    CDL_LAUNCH("layer_norm_bwd_kernel", stream, kernels[form], dim3((unsigned)bwd_blocks(form, a.rows, a.parts || a.sums[0] || a.sums[1])), dim3(kLanes[form] > 256 ? kLanes[form] : 256), 0, a);
    return check_launch();
}
template <class T>
int launch_bwd(const NormBwd &a, int kept, hipStream_t stream)
{
    if (a.cols % 8 == 0) return kept == 0 ? launch_bwd<T, false, 0>(a, stream) : kept == 1 ? launch_bwd<T, false, 1>(a, stream) : launch_bwd<T, false, 2>(a, stream);
    return kept == 0 ? launch_bwd<T, true, 0>(a, stream) : kept == 1 ? launch_bwd<T, true, 1>(a, stream) : launch_bwd<T, true, 2>(a, stream);
}

}  // namespace

int launch_layer_norm_fwd(const void *x, int32_t type, const float *weight, const float *bias, int32_t rows, int32_t cols, float eps, void *y, float *mean, float *rstd,
                          uint8_t *q, uint8_t *scale, int32_t format, hipStream_t stream)
{
    if (rows == 0) return CDL_OK;
    const int64_t size = type == CDL_BF16 ? 2 : 4;
    const NormFwd a{x, weight, bias, rows, cols, eps, 1.0f / (float)cols, y, mean, rstd, q, scale, block8_pitch(cols), block8_pitch(rows), q ? block8_pitch(rows) : rows,
                    (int64_t)rows * cols * size >= kStreamFrom * 4};
    const int keep = !q ? 0 : format == CDL_E5M2 ? 2 : 1;
    return type == CDL_BF16 ? launch_fwd<bf16_t>(a, keep, stream) : launch_fwd<float>(a, keep, stream);
}

size_t layer_norm_bwd_workspace_bytes(int32_t rows, int32_t cols)
{
    if (rows == 0 || bwd_blocks(form_of(cols), rows, true) == 1) return 0;
    return align_up((size_t)bwd_blocks(form_of(cols), rows, true) * 2 * (size_t)part_cols(cols) * sizeof(float), 256);
}

int launch_layer_norm_bwd(const void *g, int32_t type, const void *x, const uint8_t *q, const uint8_t *scale, int32_t format, const float *weight, const float *mean,
                          const float *rstd, const void *add, int32_t rows, int32_t cols, void *d_x, float *d_weight, float *d_bias, void *ws, hipStream_t stream)
{
    const bool sums = d_weight || d_bias;
    const int64_t blocks = rows > 0 ? bwd_blocks(form_of(cols), rows, sums) : 0;
    const bool at_once = blocks == 1;
    float *const parts = sums && !at_once ? (float *)ws : nullptr;
    const int64_t size = type == CDL_BF16 ? 2 : 4;
    if (rows > 0) {
        const NormBwd a{g, x, q, scale, weight, mean, rstd, add, rows, cols, 1.0f / (float)cols, d_x, parts, {at_once ? d_weight : nullptr, at_once ? d_bias : nullptr}, block8_pitch(cols), block8_pitch(rows), part_cols(cols),
                        (int64_t)rows * cols * size >= kStreamFrom * 4};
        const int kept = !q ? 0 : format == CDL_E5M2 ? 2 : 1;
        const int rc = type == CDL_BF16 ? launch_bwd<bf16_t>(a, kept, stream) : launch_bwd<float>(a, kept, stream);
        if (rc != CDL_OK) return rc;
    }
    if (!sums || at_once) return CDL_OK;
    return launch_column_sums(parts, blocks, cols, part_cols(cols), d_weight, d_bias, stream);
}

}  // namespace cdl
