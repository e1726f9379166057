// Softmax cross entropy of a linear last layer over a large vocabulary, its logits never in memory as a whole, and its gradients.
//
// Forward: the logits of a tile become the largest and the sum of exponentials of every token's stretch of the vocabulary (one pass; the joining of stretches is a second launch).
// Backward: they are formed again, a piece of the vocabulary at a time, and become g, which two products contract over the vocabulary and over the tokens.
// Bound by the matrix cores at the chip's power limit: 8192 tokens, 128000 words, width 2048 in bf16 3.3 ms forward (1300 TFLOP/s), 3.6 for g, 6.7 for the products.  50021 words, width 768:
// 0.58, 0.72, 1.4 ms, a third of the passes over the logits in their epilogues.
#include <cmath>

#include "cdl_ring.h"

namespace cdl {
namespace {

constexpr double kLog2eWhole = 1.44269504088896340736;
constexpr float kLog2e = (float)kLog2eWhole, kLog2eRest = (float)(kLog2eWhole - (double)kLog2e);      // log2 e as the sum of two floats
constexpr float kLn2 = 0.69314718055994530942f;

using Wide = RingForm<2, 2, 4, 4, 3, 2, 1>;        // 256 x 256
using Square = RingForm<2, 2, 2, 2, 3, 2, 2>;      // 128 x 128
using Thin = RingForm<4, 1, 1, 2, 3, 3, 2>;        // 128 x 64

// The logit of a token's target, where it lies in the wave's part of a tile (entry `at` of its 32 TP): the one that the sums are made of, so that a sure
// token's loss and gradient vanish but for a rounding of the log-sum.  Few parts hold any: the search is skipped there.  Every lane stores f(logit), those without a target to `spare`: no
// branch that lanes take apart, around which the compiler would have to move registers that hold addresses.
template <class FORM, class F>
__device__ __forceinline__ void find_target(const v16f (&acc)[FORM::TP][FORM::TQ], int j, int64_t at, int half, float *to, float *spare, const F &f)
{
    const bool here = at >= 0 && at < FORM::TP * 32 && ((int)(at >> 2) & 1) == half;
    if (__builtin_amdgcn_ballot_w64(here) == 0) return;
    const int own = (int)at - 4 * half;
    float z = 0.0f;
#pragma unroll
    for (int i = 0; i < FORM::TP; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) z = i * 32 + 8 * (r >> 2) + (r & 3) == own ? result<FORM>(acc[i][j], r) : z;
    *(here ? to : spare) = f(z);
}

// ---- the logits of a tile, reduced to the largest and the sum of exponentials of every token --------------------------

template <class FORM>
struct Reduce {
    static constexpr int kStores = 0;
    float2 *partial;      // [ceil(V / (32 TP))][T]: the largest logit of a stretch of the vocabulary, and the sum of exp(z - largest)
    const int64_t *target;
    float *at_target;     // [T] and one to spare: the logit of the target
    int V, T;
    __device__ __forceinline__ void operator()(const v16f (&acc)[FORM::TP][FORM::TQ], int p0, int q0, int, uint8_t *, int lane) const
    {
        if (p0 + FORM::TP * 32 <= V) columns<true>(acc, p0, q0, lane);
        else if (p0 < V) columns<false>(acc, p0, q0, lane);
    }
    template <bool FULL>
    __device__ __forceinline__ void columns(const v16f (&acc)[FORM::TP][FORM::TQ], int p0, int q0, int lane) const
    {
        constexpr int TP = FORM::TP, TQ = FORM::TQ;
        const int row = lane & 31, half = lane >> 5, left = V - p0 - 4 * half;
        float2 *const out = partial + (int64_t)(p0 / (TP * 32)) * T;
#pragma unroll
        for (int j = 0; j < TQ; ++j) {
            float m = -INFINITY, s = 0.0f;
            int end = left;
            asm volatile("" : "+v"(end));      // (compared anew each time: the masks of all entries would take more scalar registers than there are)
            auto value = [&](int i, int r) { return FULL || i * 32 + 8 * (r >> 2) + (r & 3) < end ? result<FORM>(acc[i][j], r) : -INFINITY; };
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) m = fmaxf(m, value(i, r));
            asm volatile("" : "+v"(end));
            m = fmaxf(m, __shfl_xor(m, 32, 64));
            // (logits from 2^127 on count as infinite: a stretch of none but -infinity adds nothing, one with +infinity makes the sum infinite; less m they would be no numbers)
            const float shift = fabsf(m) < 0x1p127f ? -m * kLog2e : 0.0f;
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) s += __builtin_amdgcn_exp2f(__builtin_fmaf(value(i, r), kLog2e, shift));
            s += __shfl_xor(s, 32, 64);
            const int t = q0 + j * 32 + row;
            if (half == 0 && t < T) out[t] = make_float2(m, s);
            const int64_t to = t < T ? target[t] : -1;
            find_target<FORM>(acc, j, to < V ? to - p0 : -1, half, at_target + t, at_target + T, [](float z) { return z; });
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

template <class FORM, bool PARTS>
__global__ __launch_bounds__(FORM::kThreads, FORM::PER_CU)
void head_reduce_kernel(RingCall<Reduce<FORM>> call)
{
    ring<FORM, OpBf16, PARTS, false, false>(call);
}

// A block: 1 << bits tokens side by side, whose stretches the other threads share, eight at a time so that as many loads are under way.
// 16 tokens a block where that makes enough blocks, 4 for fewer tokens (16 tokens, 1564 stretches: 4 a block 8.1 us, 16 a block 10.7; 8192 tokens, 391 stretches: 29 and 11).
constexpr int kFinishThreads = 1024;
constexpr int finish_bits(int64_t tokens) { return tokens > 1024 ? 4 : 2; }
__device__ __forceinline__ float scaled(float x, float from, float top) { return x * (from == top ? 1.0f : expf(from - top)); }      // (equal ones, also infinite: no difference of infinities)
__global__ __launch_bounds__(kFinishThreads)
void head_finish_kernel(const float2 *__restrict__ partial, int stretches, const float *__restrict__ at_target, const int64_t *__restrict__ target, int tokens, int V,
                        int bits, float *__restrict__ loss, float *__restrict__ lse)
{
    __shared__ float2 part[16][16];
    const int tid = threadIdx.x, own = tid & ((1 << bits) - 1), group = tid >> bits, groups = kFinishThreads >> bits, t = (int)(blockIdx.x << bits) + own;
    float m = -INFINITY, s = 0.0f;
    if (t < tokens)
        for (int i = group; i < stretches; i += 8 * groups) {
            float2 x[8];
            float top = m;
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = i + k * groups < stretches ? partial[(int64_t)(i + k * groups) * tokens + t] : make_float2(-INFINITY, 0.0f);
#pragma unroll
            for (int k = 0; k < 8; ++k) top = fmaxf(top, x[k].x);
            s = scaled(s, m, top);
#pragma unroll
            for (int k = 0; k < 8; ++k) s += scaled(x[k].y, x[k].x, top);
            m = top;
        }
    // the lanes of a wave, then the waves
    for (int step = 1 << bits; step < 64; step <<= 1) {
        const float m2 = __shfl_xor(m, step, 64), s2 = __shfl_xor(s, step, 64), top = fmaxf(m, m2);
        s = scaled(s, m, top) + scaled(s2, m2, top);
        m = top;
    }
    if ((tid & 63) < 1 << bits) part[tid >> 6][own] = make_float2(m, s);
    __syncthreads();
    if (group != 0 || t >= tokens) return;
    float top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int g = 0; g < 16; ++g) top = fmaxf(top, part[g][own].x);
#pragma unroll
    for (int g = 0; g < 16; ++g) sum += scaled(part[g][own].y, part[g][own].x, top);
    const float all = top + logf(sum);
    lse[t] = all;
    if (loss) {
        const int64_t at = target[t];
        loss[t] = at >= 0 && at < V ? all - at_target[t] : 0.0f;
    }
}

// ---- operands -------------------------------------------------------------------------------------------------------

// x[rows, D] as bf16 rows of Dp entries, zeros beyond D; fp32 in three parts [rows][Dp], plane entries apart, whose sum is x: each the rest rounded to bf16, the first one of a finite entry the
// largest finite bf16 where rounding would give infinity (the rest of it would be infinite too, and their products no numbers).
constexpr float kLargest = 0x1.fep127f;
template <class T>
__global__ __launch_bounds__(256)
void head_rows_kernel(const T *__restrict__ x, int64_t rows, int64_t plane, int D, int Dp, bf16_t *__restrict__ out)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;      // eight entries
    const int per = Dp / 8;
    const int64_t r = i / per;
    if (r >= rows) return;
    const int d = (int)(i - r * per) * 8;
    float v[8];
    const T *const at = x + r * D + d;
    if (D % 8 == 0 && d < D) {
        load8(at, v, false);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = d + k < D ? (float)at[k] : 0.0f;
    }
    bf16_t *to = out + r * Dp + d;
    if constexpr (sizeof(T) == 4) {
        float part[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) part[k] = fabsf(v[k]) < INFINITY ? fminf(fmaxf(v[k], -kLargest), kLargest) : v[k];
        store8(to, part, false);
#pragma unroll
        for (int i = 1; i < 3; ++i) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                v[k] -= (float)(bf16_t)part[k];
                part[k] = v[k];
            }
            to += plane;
            store8(to, part, false);
        }
    } else {
        store8(to, v, false);
    }
}

// ---- gradient of the logits ------------------------------------------------------------------------------------------

// Of a token: the factor of its probabilities and of its target, over `unit`, its log-sum, the target.
struct Token { float factor, lse; int target; float at_target; };

__global__ __launch_bounds__(1024)
void head_unit_kernel(const int64_t *__restrict__ target, const float *__restrict__ d_loss, const float *__restrict__ d_lse, int T, int V, float *__restrict__ unit)
{
    __shared__ float part[16];
    float m = 0.0f;
    for (int t0 = threadIdx.x; t0 < T; t0 += 8 * 1024) {      // eight tokens a thread, all loads under way together
        int64_t at[8];
        float a[8], b[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int t = min(t0 + k * 1024, T - 1);
            at[k] = target[t];
            a[k] = d_loss ? d_loss[t] : 1.0f;
            b[k] = d_lse ? d_lse[t] : 0.0f;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) m = fmaxf(m, (at[k] >= 0 && at[k] < V ? fabsf(a[k]) : 0.0f) + fabsf(b[k]));
    }
#pragma unroll
    for (int s = 32; s; s >>= 1) m = fmaxf(m, __shfl_xor(m, s, 64));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 16; ++i) m = fmaxf(m, part[i]);
        *unit = m > 0.0f && m < INFINITY ? m : 1.0f;
    }
}

__global__ __launch_bounds__(256)
void head_tokens_kernel(const int64_t *__restrict__ target, const float *__restrict__ lse, const float *__restrict__ d_loss, const float *__restrict__ d_lse, int tokens,
                        int padded, int V, const float *__restrict__ unit, Token *__restrict__ out)
{
    const int t = blockIdx.x * 256 + threadIdx.x;
    if (t >= padded) return;
    Token k{0.0f, INFINITY, -1, 0.0f};      // (beyond the tokens: probabilities exp(-inf))
    if (t < tokens) {
        const int64_t at = target[t];
        const bool in = at >= 0 && at < V;
        const float by = *unit, dl = in ? (d_loss ? d_loss[t] : 1.0f) : 0.0f;
        k.lse = lse[t];
        k.factor = (dl + (d_lse ? d_lse[t] : 0.0f)) / by;
        k.target = in ? (int)at : -1;
        k.at_target = dl / by;
    }
    out[t] = k;
}

// g of a piece of the vocabulary, as bf16, the products' type (in 32 bits, gradients would be 1.66e-3 off instead of 1.7e-3 to 2.4e-3, by how tokens weigh and how likely targets are, and
// two bf16 parts would double the products), [T][ld], zeros from `cols` up to ld; PARTS: in three parts `plane` entries apart
template <class FORM, bool PARTS>
struct Gradient {
    static constexpr int kStores = row_stores<FORM, bf16_t>();
    RowTarget<bf16_t> to;
    const Token *tokens;      // padded to whole tiles
    float *at_target;         // [T] and one to spare: the probability of the target, where it lies in the piece
    int T, first, cols;       // first: of the piece, in the vocabulary
    int64_t plane;
    __device__ __forceinline__ static float probability(float z, float lse)
    {
        if (!PARTS) return __builtin_amdgcn_exp2f(__builtin_fmaf(z, kLog2e, -lse));      // (lse times log2 e)
        // exp(e) = 2^hi 2^lo, hi the rounded product with log2 e and lo what it leaves: 2^lo = 1 + lo ln 2, as lo is below 2^-16
        const float e = z - lse, hi = e * kLog2e, lo = __builtin_fmaf(e, kLog2e, -hi) + e * kLog2eRest, x = __builtin_amdgcn_exp2f(hi);
        // (exp(-150) is below half of the smallest float; further down hi and lo become infinite.  NaN is not below.)
        return e < -150.0f ? 0.0f : __builtin_fmaf(x, lo * kLn2, x);
    }
    __device__ __forceinline__ void operator()(const v16f (&acc)[FORM::TP][FORM::TQ], int p0, int q0, int, uint8_t *staging, int lane) const
    {
        const int half = lane >> 5, left = cols - p0 - 4 * half;
        float factor[FORM::TQ], lse[FORM::TQ];
#pragma unroll
        for (int j = 0; j < FORM::TQ; ++j) {
            const int t = q0 + j * 32 + (lane & 31);
            const Token k = tokens[t];
            factor[j] = k.factor;
            lse[j] = PARTS ? k.lse : k.lse * kLog2e;
            find_target<FORM>(acc, j, k.target < 0 ? -1 : (int64_t)k.target - first - p0, half, at_target + t, at_target + T,
                              [&](float z) { return probability(z, lse[j]); });
            __builtin_amdgcn_sched_barrier(0);
        }
        auto g = [&](float z, int, int j) { return probability(z, lse[j]) * factor[j]; };
        auto edge = [&](float z, int p, int j) {
            int end = left;
            asm("" : "+v"(end) : "v"(z));      // (compared anew each time: the masks of all entries would take more scalar registers than there are)
            return p < end ? g(z, p, j) : 0.0f;
        };
        store_rows<FORM, bf16_t, false>(acc, to, p0, q0, staging, lane, cols, g, edge);
        if (PARTS) {
            RowTarget<bf16_t> at = to;
            at.out += plane;
            auto second = [](float x) { return x - (float)(bf16_t)x; };
            store_rows<FORM, bf16_t, false>(acc, at, p0, q0, staging, lane, cols, [&](float z, int p, int j) { return second(g(z, p, j)); },
                                            [&](float z, int p, int j) { return second(edge(z, p, j)); });
            at.out += plane;
            store_rows<FORM, bf16_t, false>(acc, at, p0, q0, staging, lane, cols, [&](float z, int p, int j) { return second(second(g(z, p, j))); },
                                            [&](float z, int p, int j) { return second(second(edge(z, p, j))); });
        }
    }
};

template <class FORM, bool PARTS>
__global__ __launch_bounds__(FORM::kThreads, FORM::PER_CU)
void head_gradient_kernel(RingCall<Gradient<FORM, PARTS>> call)
{
    ring<FORM, OpBf16, PARTS, false, false>(call);
}

// the targets: what is left out above
__global__ __launch_bounds__(256)
void head_target_kernel(const Token *__restrict__ tokens, const float *__restrict__ at_target, int T, int v0, int cols, bf16_t *__restrict__ g, int64_t ld, int64_t plane, int parts)
{
    const int t = blockIdx.x * 256 + threadIdx.x;
    if (t >= T) return;
    const Token k = tokens[t];
    const int v = k.target - v0;
    if (k.target < 0 || v < 0 || v >= cols) return;
    float x = k.factor * at_target[t] - k.at_target;
    for (int i = 0; i < parts; ++i) {
        const bf16_t part = (bf16_t)x;
        g[i * plane + (int64_t)t * ld + v] = part;
        x -= (float)part;
    }
}

// ---- products with it -------------------------------------------------------------------------------------------------

// by: results times *by; ADD: onto what is there; parts of a split contraction `part` entries apart
template <class FORM, class T, bool ADD>
struct Store {
    static constexpr int kStores = row_stores<FORM, T>();
    RowTarget<T> to;
    int64_t part;
    const float *by;
    __device__ __forceinline__ void operator()(const v16f (&acc)[FORM::TP][FORM::TQ], int p0, int q0, int split, uint8_t *staging, int lane) const
    {
        RowTarget<T> at = to;
        at.out += split * part;
        const float scale = by ? *by : 1.0f;
        store_rows<FORM, T, ADD>(acc, at, p0, q0, staging, lane, [&](float v, int, int) { return v * scale; });
    }
};

// P the vocabulary or the states, down whose rows the contraction runs, and for the gradient of the vocabulary (DOWN) g too
template <class FORM, bool PARTS, class T, bool ADD, bool DOWN>
__global__ __launch_bounds__(FORM::kThreads, FORM::PER_CU)
void head_product_kernel(RingCall<Store<FORM, T, ADD>> call)
{
    ring<FORM, OpBf16, PARTS, true, DOWN>(call);
}

template <class T>
__global__ __launch_bounds__(256)
void head_sum_kernel(const float *__restrict__ parts, int splits, int64_t part, int64_t n, const float *__restrict__ by, T *__restrict__ y)
{
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= n) return;
    float sum = 0.0f;
    for (int s = 0; s < splits; ++s) sum += parts[s * part + e];
    y[e] = (T)(sum * *by);
}

template <class T>
__global__ __launch_bounds__(256)
void head_zero_kernel(T *y, int64_t n)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) y[i] = (T)0.0f;
}

// ---- layouts ----------------------------------------------------------------------------------------------------------

enum Form { kWide, kSquare, kThin };
constexpr int form_p(Form f) { return f == kWide ? 256 : 128; }
constexpr int form_q(Form f) { return f == kWide ? 256 : f == kSquare ? 128 : 64; }
constexpr int form_per_cu(Form f) { return f == kWide ? 1 : 2; }
constexpr int form_stretch(Form f) { return f == kWide ? 128 : f == kSquare ? 64 : 32; }      // entries of P of a wave

// Thin for few tokens, whose tile would be mostly empty; Wide where it gives half of the compute units a tile (8192 tokens, 128000 words, width 2048, a step: Wide 13.7 ms, Square
// 16.9; 50021 words, width 768: 3.00 and 3.13).
Form choose_form(int64_t rows_p, int64_t rows_q)
{
    if (rows_q <= 64) return kThin;
    return ((rows_p + 255) / 256) * ((rows_q + 255) / 256) >= 128 ? kWide : kSquare;
}

int64_t up(int64_t n, int64_t by) { return (n + by - 1) / by * by; }

// Pitch of rows of n entries (a multiple of 64) in the workspace: an odd number of cache lines, so that the rows of a tile do not start in the same memory channel.
int64_t line_pitch(int64_t n) { return n / 64 % 2 ? n : n + 64; }

struct Split { int splits, k_per; };
Split choose_splits(int64_t tiles, int per_cu, int nk)
{
    int64_t s = 256 * per_cu / tiles;
    s = s < nk / 4 ? s : nk / 4;
    if (s < 1) s = 1;
    const int per = (int)((nk + s - 1) / s);
    return {(nk + per - 1) / per, per};
}

// Entries of g that are in memory at a time: 256 MB of bf16, which the memory-side cache holds (a step over 128000 words 13.8 ms; half of it 14.1, twice as much 13.8).
constexpr int64_t kPieceEntries = 1 << 27;

struct Plan {
    int parts;
    int64_t Dp, Tp;                   // up to multiples of 64
    bool copy;                        // the operands as rows of Dp entries in the workspace
    Form reduce;
    int64_t stretches;
    // training
    int64_t piece, piece_l;           // entries of the vocabulary at a time; pitch of their rows
    Form gradient, form_h, form_w;
    Split split_h;
    int64_t tokens;                   // of the table, whole tiles
    // offsets in the workspace
    size_t rows_h, rows_w, at_target, partial, unit, table, g, sums, bytes;
};

Plan make_plan(int64_t T, int64_t V, int64_t D, int32_t type, bool train)
{
    Plan p{};
    p.parts = type == CDL_F32 ? 3 : 1;
    p.Dp = D == 0 ? 64 : up(D, 64);
    p.Tp = up(T, 64);
    p.copy = type == CDL_F32 || p.Dp != D;
    p.reduce = choose_form(V, T);
    p.stretches = (V + form_stretch(p.reduce) - 1) / form_stretch(p.reduce);
    size_t at = 0;
    auto take = [&](int64_t bytes) { const size_t here = at; at += align_up((size_t)bytes, 256); return here; };
    if (p.copy) {
        p.rows_h = take(p.parts * T * p.Dp * 2);
        p.rows_w = take(p.parts * V * p.Dp * 2);
    }
    p.at_target = take((T + 1) * 4);
    const size_t kept = at;
    p.partial = take(p.stretches * T * 8);
    if (train) {
        const size_t forward = at;
        at = kept;      // the sums of the forward call are not needed any more
        p.unit = take(256);
        p.tokens = up(T, 256);
        p.table = take(p.tokens * (int64_t)sizeof(Token));
        int64_t most = up(kPieceEntries / (T < 1 ? 1 : T) / p.parts, 2048);
        most = most < 2048 ? 2048 : most > 1 << 22 ? 1 << 22 : most;      // (256 rows of g within 32-bit offsets)
        const int64_t pieces = (V + most - 1) / most;
        p.piece = pieces == 1 ? V : up((V + pieces - 1) / pieces, 256);
        p.piece_l = line_pitch(up(p.piece, 64));
        p.gradient = choose_form(p.piece, T);
        p.form_h = choose_form(D, T);
        p.form_w = choose_form(D, p.piece);
        const int64_t tiles = ((D + form_p(p.form_h) - 1) / form_p(p.form_h)) * ((T + form_q(p.form_h) - 1) / form_q(p.form_h));
        p.split_h = choose_splits(tiles < 1 ? 1 : tiles, form_per_cu(p.form_h), (int)(up(p.piece, 64) / 64 * (p.parts == 3 ? 6 : 1)));
        p.g = take(p.parts * p.Tp * p.piece_l * 2);
        p.sums = take((int64_t)p.split_h.splits * T * D * 4);
        if (at < forward) at = forward;
    }
    p.bytes = at;
    return p;
}

unsigned blocks_of(int64_t n, int64_t per) { return (unsigned)((n + per - 1) / per); }

template <class KERNEL, class EPILOGUE>
int launch_ring(const char *name, KERNEL kernel, int lds, int threads, int per_cu, const RingJob &job, const EPILOGUE &e, hipStream_t stream)
{
    const hipError_t err = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (err != hipSuccess) return hip_failed(err);
    const int64_t grid = ring_blocks((int64_t)job.tiles_p * job.tiles_q * job.splits, per_cu);
    CDL_LAUNCH(name, stream, kernel, dim3((unsigned)grid), dim3((unsigned)threads), lds, (RingCall<EPILOGUE>{ring_ready(job), e}));
    return check_launch();
}
#define CDL_RING(NAME, FORM, KERNEL, JOB, E, STREAM) launch_ring(NAME, KERNEL, FORM::kLds, FORM::kThreads, FORM::PER_CU, JOB, E, STREAM)

RingJob ring_job(Form form, const void *P, int64_t ldp, int64_t rows_p, const void *Q, int64_t ldq, int64_t rows_q, int64_t entries, int parts, int64_t plane_p, int64_t plane_q)
{
    RingJob job{};
    job.P = (const uint8_t *)P;
    job.Q = (const uint8_t *)Q;
    job.ldp = ldp * 2;
    job.ldq = ldq * 2;
    job.rowsP = (int)rows_p;
    job.rowsQ = (int)rows_q;
    job.plane_nk = (int)(entries / 64);
    job.nk = job.plane_nk * (parts == 3 ? 6 : 1);
    job.plane_p = plane_p * 2;
    job.plane_q = plane_q * 2;
    job.tiles_p = (int)((rows_p + form_p(form) - 1) / form_p(form));
    job.tiles_q = (int)((rows_q + form_q(form) - 1) / form_q(form));
    job.splits = 1;
    job.k_per = job.nk;
    return job;
}

template <bool PARTS>
int run_reduce(const Plan &p, const RingJob &job, float2 *partial, const int64_t *target, float *at_target, int V, int T, hipStream_t stream)
{
    switch (p.reduce) {
        case kWide: return CDL_RING("head_reduce_kernel", Wide, (head_reduce_kernel<Wide, PARTS>), job, (Reduce<Wide>{partial, target, at_target, V, T}), stream);
        case kSquare: return CDL_RING("head_reduce_kernel", Square, (head_reduce_kernel<Square, PARTS>), job, (Reduce<Square>{partial, target, at_target, V, T}), stream);
        default: return CDL_RING("head_reduce_kernel", Thin, (head_reduce_kernel<Thin, PARTS>), job, (Reduce<Thin>{partial, target, at_target, V, T}), stream);
    }
}

template <bool PARTS>
int run_gradient(const Plan &p, const RingJob &job, const RowTarget<bf16_t> &to, const Token *tokens, float *at_target, int T, int first, int cols, int64_t plane, hipStream_t stream)
{
    switch (p.gradient) {
        case kWide: return CDL_RING("head_gradient_kernel", Wide, (head_gradient_kernel<Wide, PARTS>), job, (Gradient<Wide, PARTS>{to, tokens, at_target, T, first, cols, plane}), stream);
        case kSquare: return CDL_RING("head_gradient_kernel", Square, (head_gradient_kernel<Square, PARTS>), job, (Gradient<Square, PARTS>{to, tokens, at_target, T, first, cols, plane}), stream);
        default: return CDL_RING("head_gradient_kernel", Thin, (head_gradient_kernel<Thin, PARTS>), job, (Gradient<Thin, PARTS>{to, tokens, at_target, T, first, cols, plane}), stream);
    }
}

template <bool PARTS, class T, bool ADD, bool DOWN>
int run_product(Form form, const RingJob &job, const RowTarget<T> &to, int64_t part, const float *by, hipStream_t stream)
{
    switch (form) {
        case kWide: return CDL_RING("head_product_kernel", Wide, (head_product_kernel<Wide, PARTS, T, ADD, DOWN>), job, (Store<Wide, T, ADD>{to, part, by}), stream);
        case kSquare: return CDL_RING("head_product_kernel", Square, (head_product_kernel<Square, PARTS, T, ADD, DOWN>), job, (Store<Square, T, ADD>{to, part, by}), stream);
        default: return CDL_RING("head_product_kernel", Thin, (head_product_kernel<Thin, PARTS, T, ADD, DOWN>), job, (Store<Thin, T, ADD>{to, part, by}), stream);
    }
}

#define CDL_TRY(X) do { const int cdl_rc_ = (X); if (cdl_rc_ != CDL_OK) return cdl_rc_; } while (0)

template <class T>
int to_rows(const T *x, int64_t rows, int64_t D, int64_t Dp, bf16_t *out, hipStream_t stream)
{
    return in_launches(rows, kLaunchThreads / (Dp / 8), [&](int64_t at, int64_t count) {
        CDL_LAUNCH("head_rows_kernel", stream, head_rows_kernel<T>, dim3(blocks_of(count * (Dp / 8), 256)), dim3(256), 0, x + at * D, count, rows * Dp, (int)D, (int)Dp, out + at * Dp);
    });
}

template <class T>
int forward(const T *h, const T *w, int32_t type, const int64_t *target, int32_t tokens, int32_t V, int32_t D, float *loss, float *lse, char *ws, hipStream_t stream)
{
    const Plan p = make_plan(tokens, V, D, type, false);
    const bf16_t *ph = (const bf16_t *)h, *pw = (const bf16_t *)w;
    if (p.copy) {
        CDL_TRY(to_rows(h, tokens, D, p.Dp, (bf16_t *)(ws + p.rows_h), stream));
        CDL_TRY(to_rows(w, V, D, p.Dp, (bf16_t *)(ws + p.rows_w), stream));
        ph = (const bf16_t *)(ws + p.rows_h);
        pw = (const bf16_t *)(ws + p.rows_w);
    }
    float2 *const partial = (float2 *)(ws + p.partial);
    const RingJob job = ring_job(p.reduce, pw, p.Dp, V, ph, p.Dp, tokens, p.Dp, p.parts, V * p.Dp, tokens * p.Dp);
    float *const at_target = (float *)(ws + p.at_target);
    CDL_TRY(run_reduce<sizeof(T) == 4>(p, job, partial, target, at_target, V, tokens, stream));
    CDL_LAUNCH("head_finish_kernel", stream, head_finish_kernel, dim3(blocks_of(tokens, 1 << finish_bits(tokens))), dim3(kFinishThreads), 0, (const float2 *)partial,
               (int)p.stretches, (const float *)at_target, target, tokens, V, finish_bits(tokens), loss, lse);
    return check_launch();
}

template <class T>
int backward(const T *h, const T *w, int32_t type, const int64_t *target, const float *lse, const float *d_loss, const float *d_lse, int32_t tokens, int32_t V,
             int32_t D, T *d_h, T *d_w, char *ws, hipStream_t stream)
{
    constexpr bool PARTS = sizeof(T) == 4;
    const Plan p = make_plan(tokens, V, D, type, true);
    const bf16_t *ph = (const bf16_t *)h, *pw = (const bf16_t *)w;
    if (p.copy) {
        CDL_TRY(to_rows(h, tokens, D, p.Dp, (bf16_t *)(ws + p.rows_h), stream));
        CDL_TRY(to_rows(w, V, D, p.Dp, (bf16_t *)(ws + p.rows_w), stream));
        ph = (const bf16_t *)(ws + p.rows_h);
        pw = (const bf16_t *)(ws + p.rows_w);
    }
    float *const unit = (float *)(ws + p.unit), *const at_target = (float *)(ws + p.at_target), *const sums = (float *)(ws + p.sums);
    Token *const table = (Token *)(ws + p.table);
    CDL_LAUNCH("head_unit_kernel", stream, head_unit_kernel, dim3(1), dim3(1024), 0, target, d_loss, d_lse, tokens, V, unit);
    CDL_LAUNCH("head_tokens_kernel", stream, head_tokens_kernel, dim3(blocks_of(p.tokens, 256)), dim3(256), 0, target, lse, d_loss, d_lse, tokens, (int)p.tokens, V,
               (const float *)unit, table);
    CDL_TRY(check_launch());
    bf16_t *const g = (bf16_t *)(ws + p.g);
    const int64_t plane_g = p.Tp * p.piece_l;
    for (int64_t v0 = 0; v0 < V; v0 += p.piece) {
        const int64_t cols = v0 + p.piece <= V ? p.piece : V - v0, padded = up(cols, 64);
        const bf16_t *const piece = pw + v0 * p.Dp;
        {
            const RingJob job = ring_job(p.gradient, piece, p.Dp, cols, ph, p.Dp, tokens, p.Dp, p.parts, V * p.Dp, tokens * p.Dp);
            CDL_TRY(run_gradient<PARTS>(p, job, RowTarget<bf16_t>{g, p.piece_l, (int)padded, (int)p.Tp, 16}, table, at_target, tokens, (int)v0, (int)cols, plane_g, stream));
            CDL_LAUNCH("head_target_kernel", stream, head_target_kernel, dim3(blocks_of(tokens, 256)), dim3(256), 0, (const Token *)table, (const float *)at_target, tokens, (int)v0, (int)cols, g, p.piece_l,
                       plane_g, p.parts);
            CDL_TRY(check_launch());
        }
        if (d_h) {
            RingJob job = ring_job(p.form_h, piece, p.Dp, D, g, p.piece_l, tokens, padded, p.parts, V * p.Dp, plane_g);
            job.downP = (int)cols;
            job.k_per = p.split_h.k_per;
            job.splits = (job.nk + job.k_per - 1) / job.k_per;      // (a last, shorter piece: fewer parts)
            const RowTarget<float> to{sums, D, D, tokens, row_width(sums, (int64_t)D * 4)};
            const int64_t part = (int64_t)tokens * D;
            CDL_TRY(v0 == 0 ? (run_product<PARTS, float, false, false>(p.form_h, job, to, part, nullptr, stream)) : (run_product<PARTS, float, true, false>(p.form_h, job, to, part, nullptr, stream)));
        }
        if (d_w) {
            RingJob job = ring_job(p.form_w, ph, p.Dp, D, g, p.piece_l, cols, p.Tp, p.parts, tokens * p.Dp, plane_g);
            job.downP = tokens;
            job.downQ = (int)p.Tp;
            T *const out = d_w + v0 * D;
            CDL_TRY((run_product<PARTS, T, false, true>(p.form_w, job, RowTarget<T>{out, D, D, (int)cols, row_width(out, (int64_t)D * (int64_t)sizeof(T))}, 0, unit, stream)));
        }
    }
    if (d_h) {
        const int64_t n = (int64_t)tokens * D;
        CDL_TRY(in_launches(n, kLaunchThreads, [&](int64_t at, int64_t count) {
            CDL_LAUNCH("head_sum_kernel", stream, head_sum_kernel<T>, dim3(blocks_of(count, 256)), dim3(256), 0, (const float *)sums + at, p.split_h.splits, n, count,
                       (const float *)unit, d_h + at);
        }));
    }
    return check_launch();
}

template <class T>
int zero(T *y, int64_t n, hipStream_t stream)
{
    if (!y || n == 0) return CDL_OK;
    return in_launches(n, kLaunchThreads, [&](int64_t at, int64_t count) {
        CDL_LAUNCH("head_zero_kernel", stream, head_zero_kernel<T>, dim3(blocks_of(count, 256)), dim3(256), 0, y + at, count);
    });
}

}  // namespace

size_t head_loss_workspace_bytes(int32_t T, int32_t V, int32_t D, int32_t type, bool train)
{
    return T == 0 || V == 0 ? 0 : make_plan(T, V, D, type, train).bytes;
}

int launch_head_loss_fwd(const void *h, const void *w, int32_t type, const int64_t *target, int32_t T, int32_t V, int32_t D, float *loss, float *lse, void *ws,
                         hipStream_t stream)
{
    if (T == 0) return CDL_OK;
    return type == CDL_BF16 ? forward((const bf16_t *)h, (const bf16_t *)w, type, target, T, V, D, loss, lse, (char *)ws, stream)
                            : forward((const float *)h, (const float *)w, type, target, T, V, D, loss, lse, (char *)ws, stream);
}

int launch_head_loss_bwd(const void *h, const void *w, int32_t type, const int64_t *target, const float *lse, const float *d_loss, const float *d_lse,
                         int32_t T, int32_t V, int32_t D, void *d_h, void *d_w, void *ws, hipStream_t stream)
{
    const int64_t n_w = (int64_t)V * D;
    if (D == 0) return CDL_OK;
    if (T == 0) return type == CDL_BF16 ? zero((bf16_t *)d_w, n_w, stream) : zero((float *)d_w, n_w, stream);
    return type == CDL_BF16 ? backward((const bf16_t *)h, (const bf16_t *)w, type, target, lse, d_loss, d_lse, T, V, D, (bf16_t *)d_h, (bf16_t *)d_w, (char *)ws, stream)
                            : backward((const float *)h, (const float *)w, type, target, lse, d_loss, d_lse, T, V, D, (float *)d_h, (float *)d_w, (char *)ws, stream);
}

}  // namespace cdl
