// Products of two matrices over their contiguous dimension on the matrix cores, bf16 or 8-bit floating point: the loop over
// K-tiles that the block-scaled product and the loss of the last layer share.
//
//   D[p,q] = sum_k P[p,k] * Q[q,k]
//
// A block of threads owns kP x kQ entries of D, its waves TP x TQ accumulators of 32 x 32 each.  K-tiles are 64 bytes of every row of both
// operands.  They come by direct global->LDS loads through a ring of RING stages, RING - 1 of them under way, across the ends of tiles: a block
// takes tile after tile as one sequence of K-tiles.  What bounds it is the LDS and the loads, not the matrix cores, wherever a wave's
// tile is small: a wave reads (32 TP + 32 TQ) * 64 bytes for TP * TQ * 64 cycles of its matrix core, so the widest form has four
// waves of 128 x 128, whose 256 accumulators leave one wave to a SIMD.  The fragments of a step are therefore read behind
// the products of the step before, and the products of one step cover the loads of the next.
//
// In the accumulators of a 32 x 32 product a lane holds one column (q) and four consecutive rows (p) at a time, so D goes to memory as [q][p]:
// P is the operand whose rows are contiguous in the result.
#pragma once

#include <type_traits>

#include "cdl_limbs.h"
#include "cdl_types.h"

namespace cdl {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v8i __attribute__((ext_vector_type(8)));

constexpr int kRingRow = 64;      // bytes of a row in a K-tile
// s_waitcnt of loads (and stores) still under way, and of all LDS reads
constexpr int wait_imm(int vm) { return (vm & 15) | ((vm >> 4) << 14) | 0x0070; }

// WP x WQ waves of TP x TQ accumulators; STAGING: LDS bytes in which a wave turns its results into rows; SCALES: a byte for every row comes with a K-tile
template <int WP_, int WQ_, int TP_, int TQ_, int RING_, int PER_CU_, int STAGING_, bool SCALES_ = false>
struct RingForm {
    static constexpr int WP = WP_, WQ = WQ_, TP = TP_, TQ = TQ_, RING = RING_, PER_CU = PER_CU_, STAGING = STAGING_;
    static constexpr bool SCALES = SCALES_;
    static constexpr int kWaves = WP * WQ, kThreads = 64 * kWaves, kP = WP * TP * 32, kQ = WQ * TQ * 32;
    static constexpr int kOperands = (kP + kQ) * kRingRow, kScaleBytes = 256, kStage = kOperands + (SCALES ? 2 * kScaleBytes : 0);
    static constexpr int kLds = RING * kStage + kWaves * STAGING;
    static constexpr int kLoadsP = kP / 16 / kWaves, kLoadsQ = kQ / 16 / kWaves, kLoads = kLoadsP + kLoadsQ + (SCALES ? 1 : 0);      // of a wave and K-tile
    static_assert(kLoadsP * 16 * kWaves == kP && kLoadsQ * 16 * kWaves == kQ && RING >= 3, "whole loads of 1 KB; a stage free while the next is read");
    static_assert(PER_CU * kLds <= 160 << 10 && kP <= 256 && kQ <= 256 && kWaves % 2 == 0, "LDS; scales of an operand in one load");
};

struct RingJob {
    const uint8_t *P, *Q;          // 16-byte aligned, rows ldp, ldq bytes apart (multiples of 16, 256 of them within 4 GiB)
    int64_t ldp, ldq;
    int rowsP, rowsQ;
    int nk;                        // K-tiles in all, even
    int tiles_p, tiles_q;
    int splits, k_per;             // the contraction in `splits` parts of k_per K-tiles (even; the last may be shorter, none is empty)
    // an operand in three parts: their products one after the other, plane_nk K-tiles each, parts plane_p and plane_q bytes apart
    int plane_nk;
    int64_t plane_p, plane_q;
    const uint8_t *sp, *sq;        // scales: [128 bytes of K][pitch], pitches multiples of 128
    int64_t pitch_sp, pitch_sq;
};

// Tile of a unit of work: groups of four rows of tiles, column by column, so that tiles worked on together share rows and columns.
struct RingUnit { int p0, q0, split; };
template <class FORM>
__device__ __forceinline__ RingUnit ring_unit(const RingJob &job, int unit)
{
    const int tiles = job.tiles_p * job.tiles_q, split = unit / tiles, t = unit - split * tiles;
    const int group = t / (4 * job.tiles_p), in = t - group * 4 * job.tiles_p, high = min(4, job.tiles_q - 4 * group);
    const int p = in / high, q = 4 * group + in - p * high;
    return {p * FORM::kP, q * FORM::kQ, split};
}

struct OpBf16 {
    static constexpr int KS = 2;      // steps of a K-tile
    typedef bf16x8 Frag;
    static __device__ __forceinline__ Frag read(const uint8_t *row, const int *chunk, int ks)
    {
        return *reinterpret_cast<const bf16x8 *>(row + chunk[ks]);
    }
    template <bool FIRST, int TP, int TQ>
    static __device__ __forceinline__ void products(v16f (&acc)[TP][TQ], const Frag (&p)[TP], const Frag (&q)[TQ], const int (&)[TP], const int (&)[TQ])
    {
        const v16f zero = {};
#pragma unroll
        for (int i = 0; i < TP; ++i)
#pragma unroll
            for (int j = 0; j < TQ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(p[i], q[j], FIRST ? zero : acc[i][j], 0, 0, 0);
    }
};

// Operands in 8-bit floating point of the formats FP and FQ (CDL_E4M3 = 0, CDL_E5M2 = 1, which is how the instruction numbers them too), a scale's byte for
// every row of a fragment.
//
// The instructions for 8-bit operands add up groups of 8 or 16 products before they reach the accumulator, and keep of each only what lies above
// 2^-14 of the group's largest (32x32x64, 16x16x128, 32x32x16 and 16x16x32 alike, seen from sums of two powers of two; the accumulator itself is
// fp32).  Over random operands that is 1.5e-5 of the result: a hundredth of a rounding to bf16, but a hundred roundings to fp32.
// Results in bf16 therefore come from these instructions, results in fp32 from EXACT: the bytes become bf16, which holds them and their scales whole, and go to
// the bf16 instruction, whose products and sums are those of fp32, at half the rate.
template <int FP, int FQ, bool EXACT>
struct OpF8 {
    static constexpr int KS = 1;
    typedef v8i Frag;
    static __device__ __forceinline__ Frag read(const uint8_t *row, const int *chunk, int)
    {
        const v4i a = *reinterpret_cast<const v4i *>(row + chunk[0]), b = *reinterpret_cast<const v4i *>(row + chunk[1]);
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    template <int F>
    static __device__ __forceinline__ bf16x8 widen(int lo, int hi, float scale)
    {
        union { bf16x2 h[4]; bf16x8 all; } v;
#define CDL_WIDEN(W, S) (F == CDL_E4M3 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)(W), scale, S) : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((uint32_t)(W), scale, S))
        v.h[0] = CDL_WIDEN(lo, false);
        v.h[1] = CDL_WIDEN(lo, true);
        v.h[2] = CDL_WIDEN(hi, false);
        v.h[3] = CDL_WIDEN(hi, true);
#undef CDL_WIDEN
        return v.all;
    }
    template <bool FIRST, int TP, int TQ>
    static __device__ __forceinline__ void products(v16f (&acc)[TP][TQ], const Frag (&p)[TP], const Frag (&q)[TQ], const int (&sp)[TP], const int (&sq)[TQ])
    {
        const v16f zero = {};
        if constexpr (EXACT) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                bf16x8 wp[TP], wq[TQ];
#pragma unroll
                for (int i = 0; i < TP; ++i) wp[i] = widen<FP>(p[i][2 * g], p[i][2 * g + 1], __int_as_float(sp[i] << 23));
#pragma unroll
                for (int j = 0; j < TQ; ++j) wq[j] = widen<FQ>(q[j][2 * g], q[j][2 * g + 1], __int_as_float(sq[j] << 23));
#pragma unroll
                for (int i = 0; i < TP; ++i)
#pragma unroll
                    for (int j = 0; j < TQ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wp[i], wq[j], FIRST && g == 0 ? zero : acc[i][j], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int j = 0; j < TQ; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(p[i], q[j], FIRST ? zero : acc[i][j], FP, FQ, 0, sp[i], 0, sq[j]);
        }
    }
};

// Where a wave's loads come from.
template <class FORM, bool PLANES>
struct RingSource {
    const RingJob &job;
    int unit, last, each, kt, end, in_plane, product;
    const uint8_t *src_p, *src_q, *src_s;
    uint32_t off_p[FORM::kLoadsP], off_q[FORM::kLoadsQ], off_s;
    int64_t step_s;

    // parts multiplied, of P and of Q: (0,0) (0,1) (1,0) (1,1) (0,2) (2,0)
    static __device__ __forceinline__ int part_p(int product) { return (0x850 >> (2 * product)) & 3; }
    static __device__ __forceinline__ int part_q(int product) { return (0x244 >> (2 * product)) & 3; }

    __device__ __forceinline__ void start(int wave, int lane)
    {
        const RingUnit u = ring_unit<FORM>(job, unit);
        kt = u.split * job.k_per;
        end = min(kt + job.k_per, job.nk);
        product = PLANES ? kt / job.plane_nk : 0;
        in_plane = PLANES ? kt - product * job.plane_nk : kt;
        src_p = job.P + (int64_t)u.p0 * job.ldp + (int64_t)in_plane * kRingRow + (PLANES ? part_p(product) * job.plane_p : 0);
        src_q = job.Q + (int64_t)u.q0 * job.ldq + (int64_t)in_plane * kRingRow + (PLANES ? part_q(product) * job.plane_q : 0);
        const uint32_t chunk = (uint32_t)(((lane & 3) ^ ((lane >> 4) & 3)) * 16);
#pragma unroll
        for (int i = 0; i < FORM::kLoadsP; ++i)      // (rows beyond the matrix: its last one again, whose results nobody stores)
            off_p[i] = (uint32_t)min((wave * FORM::kLoadsP + i) * 16 + (lane >> 2), job.rowsP - 1 - u.p0) * (uint32_t)job.ldp + chunk;
#pragma unroll
        for (int i = 0; i < FORM::kLoadsQ; ++i)
            off_q[i] = (uint32_t)min((wave * FORM::kLoadsQ + i) * 16 + (lane >> 2), job.rowsQ - 1 - u.q0) * (uint32_t)job.ldq + chunk;
        if (FORM::SCALES) {      // four bytes a lane; half of the waves load those of P, the others those of Q
            const bool q = wave & 1;
            const int64_t pitch = q ? job.pitch_sq : job.pitch_sp;
            const int at = q ? u.q0 : u.p0;
            src_s = (q ? job.sq : job.sp) + at + (int64_t)(kt >> 1) * pitch;
            off_s = (uint32_t)min((int64_t)lane * 4, pitch - 4 - at);
            step_s = pitch;
        }
    }
    __device__ __forceinline__ void issue(uint8_t *stage, int wave, int lane)
    {
        uint8_t *const to_p = stage + wave * FORM::kLoadsP * 1024, *const to_q = stage + FORM::kP * kRingRow + wave * FORM::kLoadsQ * 1024;
#pragma unroll
        for (int i = 0; i < FORM::kLoadsP; ++i) __builtin_amdgcn_global_load_lds((gptr_t)(src_p + off_p[i]), (lptr_t)(to_p + i * 1024), 16, 0, 0);
#pragma unroll
        for (int i = 0; i < FORM::kLoadsQ; ++i) __builtin_amdgcn_global_load_lds((gptr_t)(src_q + off_q[i]), (lptr_t)(to_q + i * 1024), 16, 0, 0);
        if (FORM::SCALES) {
            __builtin_amdgcn_global_load_lds((gptr_t)(src_s + off_s), (lptr_t)(stage + FORM::kOperands + (wave & 1) * FORM::kScaleBytes), 4, 0, 0);
            if (kt & 1) src_s += step_s;      // (one scale for 128 bytes of a row: two K-tiles)
        }
        src_p += kRingRow;
        src_q += kRingRow;
        ++kt;
        if (PLANES && ++in_plane == job.plane_nk) {
            in_plane = 0;
            ++product;
            if (kt < end) {
                src_p += (part_p(product) - part_p(product - 1)) * job.plane_p - (int64_t)job.plane_nk * kRingRow;
                src_q += (part_q(product) - part_q(product - 1)) * job.plane_q - (int64_t)job.plane_nk * kRingRow;
            }
        }
        if (kt == end) {
            unit = min(unit + each, last);      // (past the last unit: the last one again, which nobody reads)
            start(wave, lane);
        }
    }
};

// epilogue(acc, p0, q0, split): first entries of the wave's part of a tile; stores at least EPILOGUE::kStores times for a wave or waits for its stores.
template <class FORM, class OP, bool PLANES, class EPILOGUE>
__device__ __forceinline__ void ring(const RingJob &job, EPILOGUE &epilogue)
{
    constexpr int TP = FORM::TP, TQ = FORM::TQ, AHEAD = FORM::RING - 1, KS = OP::KS;
    extern __shared__ __attribute__((aligned(16))) uint8_t ring_lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wp = wave / FORM::WQ, wq = wave % FORM::WQ;

    // Workgroups go to the eight XCDs round-robin; XCD x takes the x-th eighth of the units, its blocks side by side through them.
    const int total = job.tiles_p * job.tiles_q * job.splits, share = (total + 7) >> 3, xcd = (int)blockIdx.x & 7, each = (int)gridDim.x >> 3;
    const int first = xcd * share + ((int)blockIdx.x >> 3), end = min(total, (xcd + 1) * share);
    if (first >= end) return;

    RingSource<FORM, PLANES> source{job};
    source.unit = first;
    source.each = each;
    source.last = total - 1;
    source.start(wave, lane);

    const int row = lane & 31, half = lane >> 5, swz = (row >> 2) & 3;
    const int chunk[2] = {row * kRingRow + (half ^ swz) * 16, row * kRingRow + ((2 + half) ^ swz) * 16};
    const int at_p = wp * TP * 32 * kRingRow, at_q = (FORM::kP + wq * TQ * 32) * kRingRow;

    v16f acc[TP][TQ];
    typename OP::Frag fp[2][TP], fq[2][TQ];
    int sp[2][TP], sq[2][TQ];
    auto read = [&](int stage, int ks, auto set_c) {
        constexpr int S = decltype(set_c)::value;
        const uint8_t *const base = ring_lds + stage * FORM::kStage;
#pragma unroll
        for (int i = 0; i < TP; ++i) fp[S][i] = OP::read(base + at_p + i * 32 * kRingRow, chunk, ks);
#pragma unroll
        for (int j = 0; j < TQ; ++j) fq[S][j] = OP::read(base + at_q + j * 32 * kRingRow, chunk, ks);
        if (FORM::SCALES) {
#pragma unroll
            for (int i = 0; i < TP; ++i) sp[S][i] = base[FORM::kOperands + (wp * TP + i) * 32 + row];
#pragma unroll
            for (int j = 0; j < TQ; ++j) sq[S][j] = base[FORM::kOperands + FORM::kScaleBytes + (wq * TQ + j) * 32 + row];
        }
    };
    auto multiply = [&](auto set_c, auto first_c) {
        constexpr int S = decltype(set_c)::value;
        OP::template products<decltype(first_c)::value>(acc, fp[S], fq[S], sp[S], sq[S]);
    };
    typedef std::integral_constant<int, 0> Zero;
    typedef std::integral_constant<int, 1> One;

    int stage = 0, since = 1 << 20;      // K-tiles since a tile's stores
    // The loads of the next K-tile have landed - younger are those of RING - 3 K-tiles, and, where they were asked for before the stores of the last tile, at least
    // those: loads and stores are counted together, up to 63, in order -, this wave has its fragments, and every wave has left the stage before.
    auto turn = [&]() {
        constexpr int kLoads = (FORM::RING - 3) * FORM::kLoads, kBoth = kLoads + EPILOGUE::kStores < 63 ? kLoads + EPILOGUE::kStores : 63;
        if (since < FORM::RING - 2) __builtin_amdgcn_s_waitcnt(wait_imm(kBoth));
        else __builtin_amdgcn_s_waitcnt(wait_imm(kLoads));
        ++since;
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        source.issue(ring_lds + (stage == 0 ? FORM::RING - 1 : stage - 1) * FORM::kStage, wave, lane);
        stage = stage + 1 == FORM::RING ? 0 : stage + 1;
    };
    auto pair = [&](auto first_c) {      // two K-tiles
        typedef decltype(first_c) First;
        if constexpr (KS == 2) {
            read(stage, 1, One{});
            multiply(Zero{}, First{});
            turn();
            read(stage, 0, Zero{});
            multiply(One{}, std::false_type{});
            read(stage, 1, One{});
            multiply(Zero{}, std::false_type{});
            turn();
            read(stage, 0, Zero{});
            multiply(One{}, std::false_type{});
        } else {
            turn();
            read(stage, 0, One{});
            multiply(Zero{}, First{});
            turn();
            read(stage, 0, Zero{});
            multiply(One{}, std::false_type{});
        }
    };

    for (int s = 0; s < AHEAD; ++s) source.issue(ring_lds + s * FORM::kStage, wave, lane);
    __builtin_amdgcn_s_waitcnt(wait_imm((AHEAD - 1) * FORM::kLoads));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    read(0, 0, Zero{});
    for (int unit = first; unit < end; unit += each) {
        const RingUnit u = ring_unit<FORM>(job, unit);
        const int pairs = (min(job.k_per, job.nk - u.split * job.k_per)) >> 1;
        pair(std::true_type{});
        for (int k = 1; k < pairs; ++k) pair(std::false_type{});
        int own = lane;
        asm volatile("" : "+v"(own));      // (what the results' places are made of is formed here, not held through the loop)
        epilogue(acc, u.p0 + wp * TP * 32, u.q0 + wq * TQ * 32, u.split, ring_lds + FORM::RING * FORM::kStage + wave * FORM::STAGING, own);
        since = 0;
    }
    __builtin_amdgcn_s_waitcnt(wait_imm(0));      // the loads behind the last step write LDS: done before this wave ends
}

// ---- a wave's results as rows [q][p] -------------------------------------------------------------------------------

// Where results go: rows ld entries apart, rows q < rows_q, entries p < rows_p.  width: what every row starts a multiple of, in bytes: 16, 4 or 2.
template <class T>
struct RowTarget {
    T *out;
    int64_t ld;
    int rows_p, rows_q, width;
};

template <class T> struct Four;
template <> struct Four<float> { typedef f32x4 type; };
template <> struct Four<bf16_t> { typedef bf16x4 type; };

// The results of TP x TQ accumulators, by f(value, p, j), as T: entry p + 4 (lane / 32) of the wave's, column tile j.  32 rows of staging at a time: the four
// consecutive entries that a lane holds go in, 16 bytes a lane come out, side by side along rows, so that whole lines reach memory.  16-byte chunks
// at chunk ^ (row), as far as a row has chunks: neither writes nor reads meet in a bank.  ADD: added to what is there (fp32).  FULL: nothing of it
// beyond the result, rows on 16 bytes.
template <class FORM, class T, bool ADD, bool FULL, class F>
__device__ __forceinline__ void store_strips(const v16f (&acc)[FORM::TP][FORM::TQ], const RowTarget<T> &to, int p0, int q0, uint8_t *staging, int lane, const F &f)
{
    typedef typename Four<T>::type four_t;
    constexpr int TP = FORM::TP, TQ = FORM::TQ, S = (int)sizeof(T);
    constexpr int kRow = FORM::STAGING / 32 < TP * 32 * S ? FORM::STAGING / 32 : TP * 32 * S;      // bytes of a staged row
    constexpr int kChunks = kRow / 16, kTiles = kRow / S / 32, kTurn = 16 / kChunks, kReads = kChunks / 2, kStep = 64 / kChunks;
    static_assert(kRow >= 32 * S && TP % kTiles == 0 && kChunks <= 16 && (!ADD || S == 4), "whole tiles; sixteen chunks");
    const int row = lane & 31, half = lane >> 5, swz = row / kTurn & (kChunks - 1);
    const int rr0 = lane / kChunks, c = lane % kChunks;      // of the first read; kStep rows further with each
    T *base = to.out + (int64_t)(q0 + rr0) * to.ld + p0 + c * (16 / S);
#pragma unroll
    for (int j = 0; j < TQ; ++j)
#pragma unroll
        for (int i0 = 0; i0 < TP; i0 += kTiles) {
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    four_t v;
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = (T)f(acc[i0 + i][j][4 * r + k], (i0 + i) * 32 + 8 * r + k, j);
                    const int byte = (i * 32 + 8 * r) * S + 4 * half * S;
                    *reinterpret_cast<four_t *>(staging + row * kRow + (((byte >> 4) ^ swz) << 4) + (byte & 15)) = v;
                }
            asm volatile("" ::: "memory");
            const int p_at = p0 + i0 * 32, q_at = q0 + j * 32;
            if (FULL || to.width == 16) {
                T *at[kReads];
                u32x4 v[kReads];
                bool inside[kReads];
#pragma unroll
                for (int n = 0; n < kReads; ++n) {
                    const int rr = rr0 + n * kStep;
                    inside[n] = FULL || (p_at + c * (16 / S) < to.rows_p && q_at + rr < to.rows_q);
                    at[n] = base + (int64_t)(j * 32 + n * kStep) * to.ld + i0 * 32;
                    v[n] = *reinterpret_cast<const u32x4 *>(staging + rr * kRow + ((c ^ (rr / kTurn & (kChunks - 1))) << 4));
                }
                if (ADD) {
                    f32x4 old[kReads];
#pragma unroll
                    for (int n = 0; n < kReads; ++n)
                        if (inside[n]) old[n] = *reinterpret_cast<const f32x4 *>(at[n]);
#pragma unroll
                    for (int n = 0; n < kReads; ++n) {
                        union { u32x4 u; f32x4 x; } sum{v[n]};
                        sum.x += old[n];
                        v[n] = sum.u;
                    }
                }
#pragma unroll
                for (int n = 0; n < kReads; ++n)
                    if (inside[n]) *reinterpret_cast<u32x4 *>(at[n]) = v[n];
            } else {
                // rows that start anywhere: words, or halves, side by side
                auto pieces = [&](auto *piece) {
                    typedef std::remove_pointer_t<decltype(piece)> piece_t;
                    constexpr int kPer = kRow / (int)sizeof(piece_t);
                    for (int n = lane; n < 32 * kPer; n += 64) {
                        const int rr = n / kPer, byte = n % kPer * (int)sizeof(piece_t), p = p_at + byte / S, q = q_at + rr;
                        if (p >= to.rows_p || q >= to.rows_q) continue;
                        const piece_t x = *reinterpret_cast<const piece_t *>(staging + rr * kRow + (((byte >> 4) ^ (rr / kTurn & (kChunks - 1))) << 4) + (byte & 15));
                        piece_t *const at = reinterpret_cast<piece_t *>(to.out + (int64_t)q * to.ld + p);
                        if constexpr (ADD) *at += x;
                        else *at = x;
                    }
                };
                if constexpr (S == 4) pieces((float *)nullptr);
                else if (to.width == 4) pieces((uint32_t *)nullptr);
                else pieces((uint16_t *)nullptr);
            }
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);      // (one strip's registers at a time)
        }
}
template <class FORM, class T, bool ADD, class F>
__device__ __forceinline__ void store_rows(const v16f (&acc)[FORM::TP][FORM::TQ], const RowTarget<T> &to, int p0, int q0, uint8_t *staging, int lane, const F &f)
{
    if (p0 + FORM::TP * 32 <= to.rows_p && q0 + FORM::TQ * 32 <= to.rows_q && to.width == 16) {
        store_strips<FORM, T, ADD, true>(acc, to, p0, q0, staging, lane, f);
    } else {
        store_strips<FORM, T, ADD, false>(acc, to, p0, q0, staging, lane, f);
        __builtin_amdgcn_s_waitcnt(wait_imm(0));
    }
}
// stores of a wave where its part is whole
template <class FORM, class T>
constexpr int row_stores() { return FORM::TP * FORM::TQ * 32 * 32 * (int)sizeof(T) / 1024; }

inline int row_width(const void *out, int64_t row_bytes)
{
    const uint64_t both = (uint64_t)(uintptr_t)out | (uint64_t)row_bytes;
    return both % 16 == 0 ? 16 : both % 4 == 0 ? 4 : 2;
}

// Blocks of a launch: as many as the chip holds at a time, whole rounds over the XCDs.
inline int64_t ring_blocks(int64_t units, int per_cu)
{
    int dev = 0, n_cu = 0;
    if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n_cu <= 0) n_cu = 256;
    const int64_t places = (int64_t)per_cu * n_cu;
    return units < places ? (units + 7) / 8 * 8 : places / 8 * 8;
}

}  // namespace cdl
