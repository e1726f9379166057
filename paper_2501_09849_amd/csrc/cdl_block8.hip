// A matrix in 8-bit floating point with a power of two as scale for every block of 128 entries, and its transpose, in one pass.
#include "cdl_block8.h"

namespace cdl {
namespace {

// A block of threads takes a tile of 128 x 128 entries, a thread eight rows of eight columns in registers: 16 lanes side by side
// read 128 entries of a row.  Both forms come from the same registers, so the matrix is read once.  The largest magnitude of a row is
// a maximum over 16 lanes, that of a column one over a thread's rows, four lanes and four waves; magnitudes are compared
// as the bits of their floats, in which an infinity beats every number and NaN beats infinity.  The transposed tile
// goes through LDS as words of eight bytes, eight rows of a column, so that its rows leave as 128 whole bytes too.
// Bound by memory: 65536 x 768 in bf16, both forms, 49 us, 4.1 TB/s where a copy reaches 5.1 (38.5 us where the memory-side cache holds all of it).
constexpr int kTile = 128, kThreads = 256;

struct QuantArgs {
    const void *x;
    int rows, cols, col_blocks;
    int64_t pitch_c, pitch_r;      // cols and rows up to whole blocks
    uint8_t *q, *scale, *q_t, *scale_t;
};

// VEC: rows of x start on 16 bytes and hold whole groups of eight columns
template <class T, bool E5M2, bool TILES, bool VEC>
__global__ __launch_bounds__(kThreads)
void block8_quantize_kernel(QuantArgs a, bool stream)
{
    constexpr int kTop = E5M2 ? 15 : 8;
    __shared__ __attribute__((aligned(16))) uint8_t tile[kTile * kTile];
    __shared__ uint32_t col_max[4][kTile];
    const int tid = threadIdx.x, oct = tid & 15, group = tid >> 4, wave = tid >> 6;
    const int cb = (int)(blockIdx.x % (unsigned)a.col_blocks), rb = (int)(blockIdx.x / (unsigned)a.col_blocks);
    const int row0 = rb * kTile + group * 8, col0 = cb * kTile + oct * 8;
    const T *const x = reinterpret_cast<const T *>(a.x);

    float v[8][8];
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        const int r = row0 + p;
        const T *const at = x + (int64_t)r * a.cols + col0;
        if (VEC) {
            if (r < a.rows && col0 < a.cols) {
                load8(at, v[p], stream);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[p][k] = 0.0f;
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[p][k] = r < a.rows && col0 + k < a.cols ? (float)at[k] : 0.0f;
        }
    }

    uint32_t row_byte[8], col_byte[8];
    uint32_t cmax[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) cmax[k] = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t bits = __float_as_uint(v[p][k]) & 0x7fffffffu;
            m = max(m, bits);
            cmax[k] = max(cmax[k], bits);
        }
        row_byte[p] = m;
    }
    if (TILES) {
        uint32_t m = 0;
#pragma unroll
        for (int p = 0; p < 8; ++p) m = max(m, row_byte[p]);
        m = row16_max(m);
        m = max(m, (uint32_t)__shfl_xor((int)m, 16, 64));
        m = max(m, (uint32_t)__shfl_xor((int)m, 32, 64));
        if ((tid & 63) == 0) col_max[wave][0] = m;
        __syncthreads();
        m = max(max(col_max[0][0], col_max[1][0]), max(col_max[2][0], col_max[3][0]));
        const uint32_t byte = scale_byte(m, kTop);
#pragma unroll
        for (int p = 0; p < 8; ++p) row_byte[p] = col_byte[p] = byte;
    } else {
#pragma unroll
        for (int p = 0; p < 8; ++p) row_byte[p] = scale_byte(row16_max(row_byte[p]), kTop);
        if (a.q_t) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                cmax[k] = max(cmax[k], (uint32_t)__shfl_xor((int)cmax[k], 16, 64));
                cmax[k] = max(cmax[k], (uint32_t)__shfl_xor((int)cmax[k], 32, 64));
            }
            if ((tid & 63) < 16) {
#pragma unroll
                for (int k = 0; k < 8; ++k) col_max[wave][oct * 8 + k] = cmax[k];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int c = oct * 8 + k;
                col_byte[k] = scale_byte(max(max(col_max[0][c], col_max[1][c]), max(col_max[2][c], col_max[3][c])), kTop);
            }
        }
    }

    if (a.q) {
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            const float by = inverse(row_byte[p]);
            float s[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) s[k] = v[p][k] * by;
            if (row0 + p < a.rows) *reinterpret_cast<u32x2 *>(a.q + (int64_t)(row0 + p) * a.pitch_c + col0) = eight<E5M2>(s);
        }
        if (oct == 0) {
            u32x2 bytes = {0, 0};
#pragma unroll
            for (int p = 0; p < 8; ++p) bytes[p >> 2] |= row_byte[p] << (8 * (p & 3));
            *reinterpret_cast<u32x2 *>(a.scale + (int64_t)cb * a.pitch_r + row0) = bytes;
        }
    }
    if (a.q_t) {
        // column c of the tile: 16 words of eight rows, word w at w ^ (c / 8): the 16 lanes of a group, whose columns are eight
        // apart, write to different banks
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float by = inverse(col_byte[k]);
            float s[8];
#pragma unroll
            for (int p = 0; p < 8; ++p) s[p] = v[p][k] * by;
            const int c = oct * 8 + k;
            *reinterpret_cast<u32x2 *>(tile + c * kTile + ((group ^ oct) * 8)) = eight<E5M2>(s);
        }
        if (group == 0) {
            u32x2 bytes = {0, 0};
#pragma unroll
            for (int k = 0; k < 8; ++k) bytes[k >> 2] |= col_byte[k] << (8 * (k & 3));
            *reinterpret_cast<u32x2 *>(a.scale_t + (int64_t)rb * a.pitch_c + cb * kTile + oct * 8) = bytes;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = i * 32 + (tid >> 3), w = (tid & 7) * 2, swz = c >> 3;
            const u32x2 lo = *reinterpret_cast<const u32x2 *>(tile + c * kTile + ((w ^ swz) * 8));
            const u32x2 hi = *reinterpret_cast<const u32x2 *>(tile + c * kTile + (((w + 1) ^ swz) * 8));
            const u32x4 out = {lo.x, lo.y, hi.x, hi.y};
            if (cb * kTile + c < a.cols) *reinterpret_cast<u32x4 *>(a.q_t + (int64_t)(cb * kTile + c) * a.pitch_r + rb * kTile + w * 8) = out;
        }
    }
}

template <class T>
int launch(const QuantArgs &a, bool tiles, bool e5m2, int64_t blocks, hipStream_t stream)
{
    const bool vec = a.cols % 8 == 0, past = (int64_t)a.rows * a.cols * (int64_t)sizeof(T) >= kStreamFrom * 4;
#define CDL_PICK(V) (e5m2 ? (tiles ? block8_quantize_kernel<T, true, true, V> : block8_quantize_kernel<T, true, false, V>) \
                          : (tiles ? block8_quantize_kernel<T, false, true, V> : block8_quantize_kernel<T, false, false, V>))
    const auto kernel = vec ? CDL_PICK(true) : CDL_PICK(false);
#undef CDL_PICK
    CDL_LAUNCH("block8_quantize_kernel", stream, kernel, dim3((unsigned)blocks), dim3(kThreads), 0, a, past);
    return check_launch();
}

}  // namespace

int64_t block8_pitch(int32_t n) { return n <= 0 ? 0 : ((int64_t)n + 127) / 128 * 128; }

int launch_block8_quantize(const void *x, int32_t type, int32_t rows, int32_t cols, int32_t tiles, int32_t format, uint8_t *q, uint8_t *scale, uint8_t *q_t,
                           uint8_t *scale_t, hipStream_t stream)
{
    const int64_t pc = block8_pitch(cols), pr = block8_pitch(rows), blocks = (pc / 128) * (pr / 128);
    if (blocks == 0) return CDL_OK;
    if (blocks * kThreads >= 1ll << 32) return CDL_ERR_RANGE;
    const QuantArgs a{x, rows, cols, (int)(pc / 128), pc, pr, q, scale, q_t, scale_t};
    return type == CDL_BF16 ? launch<bf16_t>(a, tiles != 0, format == CDL_E5M2, blocks, stream) : launch<float>(a, tiles != 0, format == CDL_E5M2, blocks, stream);
}

}  // namespace cdl
