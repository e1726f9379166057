// The block-scaled product with what stands behind it in a layer, and the gated product of two projections:
//
//   z = a b^T + bias,  y = act(z) + add                    y = act(a gate^T + bias) * (a up^T + bias)
#include <cmath>

#include "cdl_act_thin.h"
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
    for (int s = 0; s < S; ++s) load_vector<RAGGED>(f.bias[s] ? f.bias[s] + col : nullptr, left, f.N < 8, 0.0f, bias[s]);
    for (int64_t row = (int64_t)(blockIdx.x / (unsigned)f.col_blocks) * kRows + threadIdx.x / kLanes; row < f.M; row += (int64_t)f.row_blocks * kRows) {
        const int64_t at = row * f.N + col;
        float z[S][8], y[8], add[8];
#pragma unroll
        for (int s = 0; s < S; ++s) {
#pragma unroll
            for (int k = 0; k < 8; ++k) z[s][k] = 0.0f;
            for (int i = 0; i < f.splits; ++i) {
                float v[8];
                unpack<RAGGED>(load_raw<RAGGED>(f.parts[s] + i * whole + at, left, false, f.N < 8), left, f.N < 8, v);
#pragma unroll
                for (int k = 0; k < 8; ++k) z[s][k] += v[k];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) z[s][k] += bias[s][k];
            if (f.z[s]) store_first<RAGGED>((T *)f.z[s] + at, left, z[s], false);
        }
        if (f.add) unpack<RAGGED>(load_raw<RAGGED>((const T *)f.add + at, left, false, f.N < 8), left, f.N < 8, add);
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

// How a product is formed: in fp32 through memory, its contraction in parts; in tiles that are finished from the accumulators; or by blocks of 16 rows of the weights.
enum Way { kParts, kWide, kPair, kSmall, kThin };
struct Choice {
    Way way;
    int rows;      // kThin: rows of a, in sixteens
};

// The way that takes least, in us.  Tiles: rounds of blocks over the chip, of a K-tile for every 128 entries of the contraction and the end of a tile, which a compute unit's other block
// works beside.  Thin blocks read their rows from L2 at 9 MB a us (exact products 6), behind the latency of a wave's own K-tiles.  Measured, us, as Parts, Wide, Pair, Small, Thin:
//   4 x 4096 x 1024 gelu             9.5    -   11.1    -    5.3        1 x 2048 x 768 gated             15.1    -    8.4    -    5.8
//   64 x 4096 x 4096 gelu           16.3    -   26.7    -   12.7        64 x 8192 x 2048 gated           21.4    -   15.8  10.6  17.8
//   300 x 400 x 9000 gelu           13.5    -   52.8  21.3  15.4        256 x 4096 x 4096                17.1    -   24.8  12.0  45.1
//   1021 x 1000 x 520 gelu, fp32    13.4    -   15.4   8.5  13.1        512 x 2048 x 768 gated           16.8    -    8.3   7.2  18.0
//   2048 x 2048 x 2048              23.0  31.7  16.4    -     -         8192 x 2048 x 768 gelu             -   28.1  25.6  39.4    -
//   65536 x 4096 x 768               602   270   308    -     -         65536 x 4096 x 768 gelu           609   392   363    -     -
//   65536 x 2048 x 768 gated         603   255   274    -     -         ... with gelu                       -   302   298    -     -
//   ... and both z kept              687   313   374    -     -         32768 x 4096 x 768 gated, fp32    744   384   434    -     -
//   32768 x 4096 x 768, fp32         436  (423)  272    -     -         4096 x 4096 x 4096                 85  57.8  67.8    -     -
struct Cost { int p, q, places; float alone, full, end, gelu, kept; };      // entries of a tile, blocks at a time; us of a K-tile alone on a compute unit and beside another block; the end of a tile, with gelu and with z kept more
float tiles_us(Way way, bool gated, bool exact, int32_t M, int32_t N, int nk, int act, bool kept)
{
    const Cost c = way == kWide   ? Cost{256, 256, 256, exact ? 3.2f : 1.72f, exact ? 3.2f : 1.72f, gated ? 5.3f : 6.3f, gated ? 3.0f : 7.7f, 3.0f}
                   : way == kPair ? Cost{128, 128, 512, exact ? 1.2f : 0.7f, exact ? 1.8f : 1.0f, gated ? 2.5f : 3.5f, gated ? 0.8f : 1.7f, 3.0f}
                   : gated        ? Cost{128, 64, 512, exact ? 0.6f : 0.28f, exact ? 1.6f : 0.62f, 1.7f, 0.3f, 0.7f}
                                  : Cost{64, 64, 512, exact ? 0.5f : 0.23f, exact ? 0.8f : 0.4f, 1.7f, 0.3f, 0.7f};
    const int p = gated ? c.p / 2 : c.p;
    const int64_t tiles = (((int64_t)N + p - 1) / p) * (((int64_t)M + c.q - 1) / c.q), rounds = (tiles + c.places - 1) / c.places;
    return 4.0f + (float)rounds * ((float)nk * (tiles <= 256 ? c.alone : c.full) + c.end + (act == CDL_ACT_GELU ? c.gelu : 0.0f) + (kept ? c.kept : 0.0f));
}
// The order of a product's sums (of parts, of a block's waves, or of K-tiles one after the other, which all forms of tiles have alike) does not go by `kept`: a call that stores z, for a step whose
// forward pass is formed again, gives the y of the call that does not, bit for bit.  Which tiles does go by it.
Choice choose(int32_t M, int32_t N, int32_t K, bool gated, int y_type, int act, bool kept)
{
    if (K == 0) return {kParts, 0};
    const bool exact = y_type == CDL_F32;
    const int nk = (int)(block8_pitch(K) / kRingRow);
    Choice best{kParts, 0}, tiles{kSmall, 0};
    float least = block8_parts_us(M, N, K) * (gated ? 2.0f : 1.0f) * (exact ? 1.5f : 1.0f), least_tiles = INFINITY;
    bool by_tiles = false;
    for (const Way way : {kSmall, kPair, kWide}) {
        if (way == kWide && exact && !gated) continue;      // (it spills)
        const float bare = tiles_us(way, gated, exact, M, N, nk, act, false), us = kept ? tiles_us(way, gated, exact, M, N, nk, act, true) : bare;
        if (us < least_tiles) {
            least_tiles = us;
            tiles.way = way;
        }
        if (bare < least) {
            least = bare;
            by_tiles = true;
        }
    }
    if (by_tiles) best = tiles;
    for (const int rows : {1, 2, 4}) {
        if (rows > thin_most(gated, exact)) continue;
        const int64_t across = ((int64_t)M + 16 * rows - 1) / (16 * rows), blocks = ((int64_t)N + 15) / 16 * across;
        const float read = (float)((gated ? 2 : 1) + rows);      // sixteens of a block
        const float us = 3.5f + (float)blocks * 16.0f * read * (float)block8_pitch(K) / (exact ? 6e6f : 9e6f) + 0.2f * read * (float)((nk + 7) / 8) + (float)(blocks / 512);
        if (us < least && across <= 65535 && blocks < 1 << 22) {      // (a grid's limits)
            least = us;
            best = {kThin, rows};
        }
    }
    return best;
}

size_t parts_bytes(int32_t M, int32_t N, int32_t K) { return align_up((size_t)block8_parts(M, N, K) * (size_t)M * (size_t)N * sizeof(float), 256); }

}  // namespace

size_t block8_gemm_act_workspace_bytes(int32_t M, int32_t N, int32_t K, bool gated)
{
    if (M == 0 || N == 0 || K == 0) return 0;
    // (whatever the results' type and the activation, which the query does not know)
    for (const int type : {CDL_BF16, CDL_F32})
        for (const int act : {CDL_ACT_NONE, CDL_ACT_GELU})
            if (choose(M, N, K, gated, type, act, false).way == kParts) return parts_bytes(M, N, K) * (gated ? 2 : 1);
    return 0;
}

int launch_block8_gemm_act(const ProductCall &c, bool gated, hipStream_t stream)
{
    if (c.M == 0 || c.N == 0) return CDL_OK;
    const ActTarget to{{c.bias[0], c.bias[1]}, c.add, c.y, {c.z[0], c.z[1]}, c.M, c.N, c.act};
    const int64_t ld = block8_pitch(c.K), pitch_a = block8_pitch(c.M), pitch_b = block8_pitch(c.N);
    const int nk = (int)(ld / kRingRow);
    const Choice choice = choose(c.M, c.N, c.K, gated, c.y_type, c.act, c.z[0] || c.z[1]);
    if (choice.way == kThin)
        return launch_thin_any({c.a, {c.b[0], c.b[1]}, c.a_scale, {c.b_scale[0], c.b_scale[1]}, ld, pitch_a, pitch_b, nk, to}, choice.rows, gated, c.y_type, c.a_format, c.b_format,
                               stream);
    if (choice.way != kParts) {
        RingJob job{};
        job.P = c.b[0];
        job.P2 = c.b[1];
        job.Q = c.a;
        job.ldp = job.ldq = ld;
        job.rowsP = c.N;
        job.rowsQ = c.M;
        job.nk = job.k_per = nk;
        job.splits = 1;
        job.sp = c.b_scale[0];
        job.sp2 = c.b_scale[1];
        job.sq = c.a_scale;
        job.pitch_sp = pitch_b;
        job.pitch_sq = pitch_a;
        const auto launch = c.y_type == CDL_BF16 ? (gated ? launch_gated_bf16 : launch_act_bf16) : gated ? launch_gated_f32 : launch_act_f32;
        const ActForm form = choice.way == kWide ? ActForm::kWide : choice.way == kPair ? ActForm::kPair : ActForm::kSmall;
        return launch(form, job, to, c.a_format, c.b_format, stream);
    }
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
