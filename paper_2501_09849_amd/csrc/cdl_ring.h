// Products of two matrices over their contiguous dimension on the matrix cores, bf16 or 8-bit floating point: the loop over
// K-tiles that the block-scaled product, its forms for layers and the loss of the last layer share.
//
//   D[p,q] = sum_k P[p,k] * Q[q,k]
//
// A block of threads owns kP x kQ entries of D, its waves TP x TQ accumulators of 32 x 32 each.  K-tiles are 128 bytes of every row of both
// operands, which come by direct global->LDS loads, across the ends of tiles: a block takes tile after tile as one sequence of K-tiles.
// In LDS each operand has a ring of its own, NP and NQ K-tiles long.  The widest form, four waves of 128 x 128, has room for 3 + 2 and nothing else; its results
// turn into rows in the slot of P that waits for its loads.
// What bounds it: the matrix cores run at the chip's power limit (1.8 GHz of 2.4), and beside them the loads.  Rows in pieces of 64 bytes, half a
// cache line, come at 10 TB/s over the chip and no more: 64-byte K-tiles in a ring of four took 0.82 us a K-tile of the widest form, the same
// bytes as whole lines 0.70, no loads at all 0.63.  A wave of 128 x 128 leaves one wave to a SIMD, so its fragments are read
// behind the products of the step before.
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

constexpr int kRingRow = 128;      // bytes of a row in a K-tile
// s_waitcnt of loads (and stores) still under way, and of all LDS reads
constexpr int wait_imm(int vm) { return (vm & 15) | ((vm >> 4) << 14) | 0x0070; }

// WP x WQ waves of TP x TQ accumulators; NP, NQ: K-tiles of each operand in LDS; STAGING: LDS bytes in which a wave turns its results into rows, 0: in the slot of P
// that is free then; SCALES: a byte for every row comes with a K-tile.
// GATED: P is two matrices of the same shape, and a tile holds half as many entries of either, side by side for each wave: of a wave's accumulators along P the first half
// are of the first matrix, the others of the same entries of the second.
// After a K-tile its slots are free.  The loads of Q into its slot go out with the last products of the K-tile, those of P with the first ones of the next K-tile
// (behind a tile's results), or with those of Q where P has no third slot.
template <int WP_, int WQ_, int TP_, int TQ_, int NP_, int NQ_, int PER_CU_, int STAGING_ = 0, bool SCALES_ = false, bool GATED_ = false>
struct RingForm {
    static constexpr int WP = WP_, WQ = WQ_, TP = TP_, TQ = TQ_, NP = NP_, NQ = NQ_, PER_CU = PER_CU_;
    static constexpr bool SCALES = SCALES_, GATED = GATED_, kTogether = NP == 2;
    static constexpr int kWaves = WP * WQ, kThreads = 64 * kWaves, kP = WP * TP * 32, kQ = WQ * TQ * 32;
    static constexpr int kAcross = GATED ? kP / 2 : kP, kWaveAcross = kAcross / WP;      // entries of the result along P of a tile, of a wave
    static constexpr int kSlotP = kP * kRingRow, kSlotQ = kQ * kRingRow, kScaleBytes = 256, kSlotS = SCALES ? 2 * kScaleBytes : 0;
    static constexpr int kAtQ = NP * kSlotP, kAtS = kAtQ + NQ * kSlotQ, kAtStaging = kAtS + NQ * kSlotS, kLds = kAtStaging + kWaves * STAGING_;
    static constexpr int kLoadsP = kP / 8 / kWaves, kLoadsQ = kQ / 8 / kWaves, kMoreQ = kLoadsQ + (SCALES ? 1 : 0);      // of a wave and K-tile, 1 KB each; and the scales
    static constexpr int STAGING = STAGING_ ? STAGING_ : kLoadsP * 1024;
    static_assert(kLoadsP * 8 * kWaves == kP && kLoadsQ * 8 * kWaves == kQ && (NP == NQ || NP == NQ + 1) && NQ >= 2, "whole loads; the order of the loads");
    static_assert(!GATED || (WQ == 2 && TP % 2 == 0), "a wave's loads are of one matrix");
    static_assert(!kTogether || STAGING_ > 0, "a free slot of P between tiles");
    static_assert(PER_CU * kLds <= 160 << 10 && kP <= 256 && kQ <= 256 && kWaves % 2 == 0, "LDS; scales of an operand in one load");
};

struct RingJob {
    const uint8_t *P, *Q;          // 16-byte aligned, rows ldp, ldq bytes apart (multiples of 16, 256 of them within 4 GiB - 8 KiB)
    int64_t ldp, ldq;
    int rowsP, rowsQ;
    int nk;                        // K-tiles in all
    int tiles_p, tiles_q;
    int splits, k_per;             // the contraction in `splits` parts of k_per K-tiles (the last may be shorter, none is empty)
    // an operand in three parts: their products one after the other, plane_nk K-tiles each, parts plane_p and plane_q bytes apart
    int plane_nk;
    int64_t plane_p, plane_q;
    const uint8_t *sp, *sq;        // scales: [K-tile][pitch], pitches multiples of 128
    int64_t pitch_sp, pitch_sq;
    int downP, downQ;              // rows in memory of an operand whose contraction runs down its rows
    const uint8_t *P2, *sp2;       // GATED: the second matrix, its scales
    uint64_t by_tiles, by_group;   // 1 / (tiles_p tiles_q) and 1 / (4 tiles_p), of a launch: ring_ready()
};

// n / d for n < 2^31 as a product: 2^63 / d rounded up, off by less than 1, makes the quotient too large by less than n / 2^63 < 1 / d.  (The compiler's division by a number
// that is not known takes some 30 instructions one behind the other; a tile needed twelve of them, 1 us.)
inline uint64_t reciprocal(uint64_t d) { return ((1ull << 63) + d - 1) / d; }
__device__ __forceinline__ int divide(int n, uint64_t by) { return (int)__umul64hi((uint64_t)(uint32_t)n << 1, by); }

// What a kernel of this loop is launched with, its only argument.  Between the tiles it is read again from where the launch put it (start(), the epilogue): scalar
// registers do not hold it all through the loop beside what the loop needs, and what the compiler spilled came back from memory in every K-tile.
template <class EPILOGUE>
struct RingCall {
    RingJob job;
    EPILOGUE epilogue;
};
template <class CALL>
__device__ __forceinline__ const CALL &again(const CALL &)
{
    uint64_t at = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    return *(const CALL *)(const __attribute__((address_space(4))) CALL *)at;
}

inline RingJob ring_ready(RingJob job)
{
    job.by_tiles = reciprocal((uint64_t)job.tiles_p * (uint64_t)job.tiles_q);
    job.by_group = reciprocal(4 * (uint64_t)job.tiles_p);
    return job;
}

// Tile of a unit of work: groups of four rows of tiles, column by column, so that tiles worked on together share rows and columns.
struct RingUnit { int p0, q0, split; };
template <class FORM>
__device__ __forceinline__ RingUnit ring_unit(const RingJob &job, int unit)
{
    const int split = divide(unit, job.by_tiles), t = unit - split * job.tiles_p * job.tiles_q;
    const int group = divide(t, job.by_group), in = t - group * 4 * job.tiles_p, high = min(4, job.tiles_q - 4 * group);
    const int p = high == 4 ? in >> 2 : high == 3 ? (int)((uint32_t)in / 3u) : in >> (high - 1), q = 4 * group + in - p * high;
    return {p * FORM::kAcross, q * FORM::kQ, split};
}

struct OpBf16 {
    static constexpr bool kPin = false;
    static constexpr int KS = 4, kReads = 1, kPerPair = 1, kConversions = 0;      // steps of a K-tile; reads of a fragment, instructions of a product, conversions beside each
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
    static constexpr bool kPin = true;
    static constexpr int KS = 2, kReads = 2, kPerPair = EXACT ? 4 : 1, kConversions = EXACT ? 2 : 0;
    typedef v8i Frag;
    static __device__ __forceinline__ Frag read(const uint8_t *row, const int *chunk, int ks)
    {
        const v4i a = *reinterpret_cast<const v4i *>(row + chunk[2 * ks]), b = *reinterpret_cast<const v4i *>(row + chunk[2 * ks + 1]);
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

// Where the loads of an operand come from: K-tile after K-tile, `left` of them before change() has to be called, which goes on to the next unit of work (or to
// the next product of parts).  Four loads share a base in LDS: the instruction's offset counts on both sides, so a lane's offset into memory
// takes it back.
//
// DOWN: the contraction runs down the rows of the operand (bf16), which is [k][p]: a K-tile is 64 rows of it, of each the tile's entries side by side, in LDS too.
// What lies beyond the matrix in memory is read as its last 16 bytes; rows beyond the contraction meet zeros of the other operand.
template <class FORM, bool PLANES, bool IS_P, bool DOWN>
struct RingStream {
    static constexpr int kLoads = IS_P ? FORM::kLoadsP : FORM::kLoadsQ, kBack = 4096;      // (offsets stay positive)
    static constexpr bool kGated = FORM::GATED && IS_P;
    static constexpr int kEntries = IS_P ? FORM::kP : FORM::kQ, kChunks = kEntries / 8, kRows = 64 / kChunks;      // DOWN: 16-byte chunks of a row, rows of a load
    int unit, left, end, product, rows_in;
    const uint8_t *src, *src_s;
    uint32_t off[kLoads], off_s, limit;
    int64_t step, rest, step_s;      // DOWN: bytes from a K-tile to the next, from its first byte to the last chunk of the matrix

    // 16-byte chunk c of row k at chunk c ^ turned(k), so that four rows of 64 bytes read together lie in different banks
    static __device__ __forceinline__ int turned(int k) { return kChunks >= 16 ? (k & 3) << 2 : (k >> 1 & 1) << 2; }

    // parts multiplied, of P and of Q: (0,0) (0,1) (1,0) (1,1) (0,2) (2,0)
    static __device__ __forceinline__ int part(int product) { return ((IS_P ? 0x850 : 0x244) >> (2 * product)) & 3; }

    struct Place {
        const uint8_t *src;
        int left, product;
        int64_t rest;
    };
    __device__ __forceinline__ void start(const RingJob &job, int wave, int lane) { go(of_unit(job, wave, lane)); }
    __device__ __forceinline__ void go(const Place &to)
    {
        src = to.src;
        left = to.left;
        product = to.product;
        rest = to.rest;
        bound();
    }
    __device__ __forceinline__ void bound()
    {
        if (DOWN) limit = (uint32_t)min(rest, (int64_t)0x7fffffff) + kBack;
    }
    __device__ __forceinline__ void advance()
    {
        src += DOWN ? step : (int64_t)kRingRow;
        if (DOWN) rest -= step;
        bound();
    }
    __device__ __forceinline__ Place of_unit(const RingJob &job, int wave, int lane)
    {
        const RingUnit u = ring_unit<FORM>(job, unit);
        const int kt = u.split * job.k_per, row0 = IS_P ? u.p0 : u.q0, rows = IS_P ? job.rowsP : job.rowsQ;
        const int64_t ld = IS_P ? job.ldp : job.ldq;
        end = min(kt + job.k_per, job.nk);
        const int product = PLANES ? kt / job.plane_nk : 0, in_plane = PLANES ? kt - product * job.plane_nk : kt;
        const int left = PLANES ? min(job.plane_nk - in_plane, end - kt) : end - kt;
        step = 64 * ld;
        const int64_t at = DOWN ? (int64_t)row0 * 2 + in_plane * step : (int64_t)row0 * ld + (int64_t)in_plane * kRingRow;
        const int64_t rest = DOWN ? (IS_P ? job.downP : job.downQ) * ld - 16 - at : 0;
        const uint8_t *const src = (kGated && (wave & 1) ? job.P2 : IS_P ? job.P : job.Q) + at + (PLANES ? part(product) * (IS_P ? job.plane_p : job.plane_q) : 0) - kBack;
        const int most = DOWN ? 0 : min(rows - 1 - row0, kEntries - 1), from = kGated ? wave >> 1 : wave;      // GATED: even waves load the first matrix, odd ones the same rows of the second
        if (most != rows_in) {
            rows_in = most;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {      // load i fills LDS rows 8 n ... 8 n + 7, chunk c of a row at c ^ (row / 2); rows beyond the matrix: its last one again, whose results nobody stores
                const int n = wave * kLoads + i, k = n * kRows + lane / kChunks;
                if (DOWN) off[i] = (uint32_t)k * (uint32_t)ld + (uint32_t)(lane % kChunks ^ turned(k)) * 16 + kBack - (i & 3) * 1024;
                else off[i] = (uint32_t)min((from * kLoads + i) * 8 + (lane >> 3), most) * (uint32_t)ld + (uint32_t)((lane & 7) ^ ((4 * n + (lane >> 4)) & 7)) * 16 + kBack - (i & 3) * 1024;
            }
        }
        if (FORM::SCALES && !IS_P) {      // four bytes a lane; half of the waves load those of Q, the others those of P
            const bool q = wave & 1;
            const int64_t pitch = q ? job.pitch_sq : job.pitch_sp;
            const int at = q ? u.q0 : u.p0;
            src_s = (q ? job.sq : job.sp) + at + (int64_t)kt * pitch;
            off_s = (uint32_t)min((int64_t)lane * 4, pitch - 4 - at);
            if (FORM::GATED && !q) {      // a lane's four rows are of one matrix
                constexpr int kRows = FORM::kP / FORM::kWaves;
                const int part = lane * 4 / kRows;
                off_s = (uint32_t)min((int64_t)(part >> 1) * kRows + lane * 4 % kRows, pitch - 4 - at);
                if (part & 1) src_s += job.sp2 - job.sp;
            }
            step_s = pitch;
        }
        return {src, left, product, rest};
    }
    __device__ __forceinline__ Place of_next(const RingJob &job, int each, int last, int wave, int lane)
    {
        if (PLANES) {
            const int next = (product + 1) * job.plane_nk;
            if (next < end) {
                const int64_t parts = part(product + 1) - part(product);
                const int64_t back = job.plane_nk * (DOWN ? step : (int64_t)kRingRow);
                return {src + parts * (IS_P ? job.plane_p : job.plane_q) - back, min(job.plane_nk, end - next), product + 1, rest + back};
            }
        }
        unit = min(unit + each, last);      // (past the last unit: the last one again, which nobody reads)
        return of_unit(job, wave, lane);
    }
    // (one set of stores for both ways: the compiler would join stores to different members, and keep the members in memory)
    __device__ __forceinline__ void change(const RingJob &job, int each, int last, int wave, int lane) { go(of_next(job, each, last, wave, lane)); }
    // loads FROM .. TO - 1 of a K-tile
    template <int FROM, int TO>
    __device__ __forceinline__ void issue(uint8_t *slot, int wave) const
    {
        if constexpr (FROM < TO) {
            const uint32_t at = DOWN ? min(off[FROM], limit - (FROM & 3) * 1024) : off[FROM];
            __builtin_amdgcn_global_load_lds((gptr_t)(src + at), (lptr_t)(slot + wave * kLoads * 1024 + (FROM & ~3) * 1024), 16, (FROM & 3) * 1024, 0);
            issue<FROM + 1, TO>(slot, wave);
        }
    }
    __device__ __forceinline__ void issue_scales(uint8_t *slot, int wave)
    {
        __builtin_amdgcn_global_load_lds((gptr_t)(src_s + off_s), (lptr_t)(slot + (wave & 1) * FORM::kScaleBytes), 4, 0, 0);
        src_s += step_s;
    }
};

// The order of instructions that the loop asks for: reads behind the first products, so that they have come by the next step, loads evenly.
template <int I, int PRODUCTS, int READS, int LOADS, int CONVERSIONS>
__device__ __forceinline__ void mix_slots()
{
    if constexpr (I < PRODUCTS) {
        constexpr int kHalf = PRODUCTS / 2 > 0 ? PRODUCTS / 2 : 1, kReads = I < kHalf ? (I + 1) * READS / kHalf - I * READS / kHalf : 0;
        constexpr int kLoads = (I + 1) * LOADS / PRODUCTS - I * LOADS / PRODUCTS;
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if constexpr (CONVERSIONS > 0) __builtin_amdgcn_sched_group_barrier(0x002, CONVERSIONS, 0);
        if constexpr (kReads > 0) __builtin_amdgcn_sched_group_barrier(0x100, kReads, 0);
        if constexpr (kLoads > 0) __builtin_amdgcn_sched_group_barrier(0x010, kLoads, 0);
        mix_slots<I + 1, PRODUCTS, READS, LOADS, CONVERSIONS>();
    }
}

// The accumulators of the widest form fill the half of the registers that only the matrix cores and moves reach.  The results are moved out one at a time, where they are
// used: left to itself the compiler moves whole accumulators, spills what there was, and every reload waits for the stores before it (an epilogue of
// 128 x 128 results a wave took 20 to 50 us).
template <class FORM>
__device__ __forceinline__ float result(const v16f &acc, int r)
{
    if constexpr (FORM::TP * FORM::TQ >= 16) {
        float x;
        asm("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(acc[r]));
        return x;
    } else {
        return acc[r];
    }
}
// ... behind the last products: the compiler does not know that the moves read what the matrix cores have yet to write (at most 19 cycles later)
template <class FORM>
__device__ __forceinline__ void results_ready(v16f (&acc)[FORM::TP][FORM::TQ])
{
    if constexpr (FORM::TP == 4 && FORM::TQ == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) asm volatile("s_nop 15\n\ts_nop 15" : "+a"(acc[i][0]), "+a"(acc[i][1]), "+a"(acc[i][2]), "+a"(acc[i][3]));
    }
}

// A fragment of 32 entries and 16 k of an operand [k][entries]: eight k of one entry for a lane.  A group of 16 lanes reads four k of 16 entries, and each lane gets one entry's.
// (__restrict__ is what tells the compiler that these reads are not of what the loads on their way write; without it every one waited for all of them, and a product took half as long again.)
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef s16x4 __attribute__((address_space(3))) *down_t;
template <int ENTRIES>
__device__ __forceinline__ bf16x8 read_down(const uint8_t *__restrict__ at, int ks)
{
    union { s16x4 h[2]; bf16x8 all; } v;
    v.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((down_t)(at + ks * 16 * ENTRIES * 2));
    v.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((down_t)(at + (ks * 16 + 4) * ENTRIES * 2));
    return v.all;
}

// epilogue(acc, p0, q0, split, staging, lane): first entries of the wave's part of a tile; stores at least EPILOGUE::kStores times for a wave or waits for its stores.
template <class FORM, class OP, bool PLANES, bool DOWN_P, bool DOWN_Q, class EPILOGUE>
__device__ __forceinline__ void ring(const RingCall<EPILOGUE> &call)
{
    const RingJob &job = call.job;
    constexpr int TP = FORM::TP, TQ = FORM::TQ, KS = OP::KS;
    extern __shared__ __attribute__((aligned(16))) uint8_t ring_lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wp = wave / FORM::WQ, wq = wave % FORM::WQ;

    // Workgroups go to the eight XCDs round-robin; XCD x takes the x-th eighth of the units, its blocks side by side through them.
    const int total = job.tiles_p * job.tiles_q * job.splits, share = (total + 7) >> 3, xcd = (int)blockIdx.x & 7, each = (int)gridDim.x >> 3;
    const int first = xcd * share + ((int)blockIdx.x >> 3), end = min(total, (xcd + 1) * share);
    if (first >= end) return;

    typedef RingStream<FORM, PLANES, true, DOWN_P> FromP;
    typedef RingStream<FORM, PLANES, false, DOWN_Q> FromQ;
    FromP from_p;
    FromQ from_q;
    from_p.unit = from_q.unit = first;
    from_p.rows_in = from_q.rows_in = -1;
    from_p.start(job, wave, lane);
    from_q.start(job, wave, lane);

    const int row = lane & 31, half = lane >> 5;
    int chunk[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) chunk[c] = row * kRingRow + (((2 * c + half) ^ (row >> 1)) & 7) * 16;

    // DOWN: where a lane of a 16 x 16 transposing read starts in the first step's rows of a fragment
    int down_p[TP], down_q[TQ];
    const int down_k = half * 8 + ((lane & 15) >> 2), in_tile = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
#pragma unroll
    for (int i = 0; i < TP; ++i) down_p[i] = down_k * FORM::kP * 2 + ((((wp * TP + i) * 4 + in_tile) ^ FromP::turned(down_k)) << 4) + (lane & 1) * 8;
#pragma unroll
    for (int j = 0; j < TQ; ++j) down_q[j] = down_k * FORM::kQ * 2 + ((((wq * TQ + j) * 4 + in_tile) ^ FromQ::turned(down_k)) << 4) + (lane & 1) * 8;

    v16f acc[TP][TQ];
    typename OP::Frag fp[2][TP], fq[2][TQ];
    int sp[2][TP], sq[2][TQ];
    int at_p = 0, at_q = 0, at_s = 0;      // of the K-tile being multiplied: its slots
    auto read = [&](int ks, auto set_c) {
        constexpr int S = decltype(set_c)::value;
        const uint8_t *const p = ring_lds + at_p + wp * TP * 32 * kRingRow, *const q = ring_lds + FORM::kAtQ + at_q + wq * TQ * 32 * kRingRow;
#pragma unroll
        for (int i = 0; i < TP; ++i) {
            if constexpr (DOWN_P) fp[S][i] = read_down<FORM::kP>(ring_lds + at_p + down_p[i], ks);
            else fp[S][i] = OP::read(p + i * 32 * kRingRow, chunk, ks);
        }
#pragma unroll
        for (int j = 0; j < TQ; ++j) {
            if constexpr (DOWN_Q) fq[S][j] = read_down<FORM::kQ>(ring_lds + FORM::kAtQ + at_q + down_q[j], ks);
            else fq[S][j] = OP::read(q + j * 32 * kRingRow, chunk, ks);
        }
        if (FORM::SCALES) {
            const uint8_t *const scales = ring_lds + FORM::kAtS + at_s;
#pragma unroll
            for (int i = 0; i < TP; ++i) sp[S][i] = scales[(wp * TP + i) * 32 + row];
#pragma unroll
            for (int j = 0; j < TQ; ++j) sq[S][j] = scales[FORM::kScaleBytes + (wq * TQ + j) * 32 + row];
        }
    };
    auto multiply = [&](auto set_c, auto first_c) {
        constexpr int S = decltype(set_c)::value;
        OP::template products<decltype(first_c)::value>(acc, fp[S], fq[S], sp[S], sq[S]);
    };
    typedef std::integral_constant<int, 0> Zero;
    typedef std::integral_constant<int, 1> One;
    typedef std::true_type Yes;
    typedef std::false_type No;

    int free_p = 0, free_q = 0, free_s = 0;      // the slots that the next loads fill
    auto loaded_p = [&]() {
        free_p = free_p == (FORM::NP - 1) * FORM::kSlotP ? 0 : free_p + FORM::kSlotP;
        from_p.advance();
        __builtin_amdgcn_sched_barrier(0);
        if (--from_p.left == 0) from_p.change(again(call).job, each, total - 1, wave, lane);
    };
    auto issue_q = [&]() {
        from_q.template issue<0, FORM::kLoadsQ>(ring_lds + FORM::kAtQ + free_q, wave);
        if (FORM::SCALES) from_q.issue_scales(ring_lds + FORM::kAtS + free_s, wave);
    };
    auto loaded_q = [&]() {
        free_q = free_q == (FORM::NQ - 1) * FORM::kSlotQ ? 0 : free_q + FORM::kSlotQ;
        if (FORM::SCALES) free_s = free_s == (FORM::NQ - 1) * FORM::kSlotS ? 0 : free_s + FORM::kSlotS;
        from_q.advance();
        __builtin_amdgcn_sched_barrier(0);
        if (--from_q.left == 0) from_q.change(again(call).job, each, total - 1, wave, lane);
    };
    auto barrier = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // The loads of the next K-tile have landed - younger are those of NQ - 2 whole K-tiles and of one more of P where it has a slot more, and for the first K-tile of a
    // tile the stores of the tile before, at least: loads and stores are counted together, up to 63, in order -, this wave has its fragments, and every
    // wave has read what it needs of the K-tile.
    bool stored = false;
    auto turn = [&](auto early_c) {
        constexpr int kYounger = (FORM::NQ - 2) * (FORM::kLoadsP + FORM::kMoreQ) + (FORM::NP > FORM::NQ ? FORM::kLoadsP : 0);
        constexpr int kBoth = kYounger + EPILOGUE::kStores < 63 ? kYounger + EPILOGUE::kStores : 63;
        static_assert(kYounger < 64, "loads that the counter holds");
        __builtin_amdgcn_sched_barrier(0);
        if (decltype(early_c)::value && stored) __builtin_amdgcn_s_waitcnt(wait_imm(kBoth));
        else __builtin_amdgcn_s_waitcnt(wait_imm(kYounger));
        barrier();
    };
    // Nothing else fills a SIMD's matrix cores while its only wave reads or loads, so reads and loads go between the products, and the products of a step stay on their side
    // of the barrier (left to itself the compiler gathers the reads before the wait and the products behind it).
    constexpr int kFragments = TP * (DOWN_P ? 2 : OP::kReads) + TQ * (DOWN_Q ? 2 : OP::kReads) + (FORM::SCALES ? TP + TQ : 0), kProducts = TP * TQ * OP::kPerPair;
    auto step = [&](auto first_c) {      // a K-tile, the first one of a tile or a later one
        typedef decltype(first_c) First;
        auto inner = [&](auto r_c) {
            constexpr int R = decltype(r_c)::value, kFrom = FORM::kTogether ? 0 : FORM::kLoadsP * R / (KS - 1), kTo = FORM::kTogether ? 0 : FORM::kLoadsP * (R + 1) / (KS - 1);
            read(R + 1, std::integral_constant<int, (R + 1) & 1>{});
            from_p.template issue<kFrom, kTo>(ring_lds + free_p, wave);
            multiply(std::integral_constant<int, R & 1>{}, std::integral_constant<bool, First::value && R == 0>{});
            mix_slots<0, kProducts, kFragments, kTo - kFrom, OP::kConversions>();
            __builtin_amdgcn_sched_barrier(0);
        };
        inner(Zero{});
        if constexpr (KS == 4) {
            inner(One{});
            inner(std::integral_constant<int, 2>{});
        }
        if constexpr (!FORM::kTogether) loaded_p();
        turn(First{});
        at_p = at_p == (FORM::NP - 1) * FORM::kSlotP ? 0 : at_p + FORM::kSlotP;
        at_q = at_q == (FORM::NQ - 1) * FORM::kSlotQ ? 0 : at_q + FORM::kSlotQ;
        if (FORM::SCALES) at_s = at_s == (FORM::NQ - 1) * FORM::kSlotS ? 0 : at_s + FORM::kSlotS;
        read(0, Zero{});
        issue_q();
        if constexpr (FORM::kTogether) from_p.template issue<0, FORM::kLoadsP>(ring_lds + free_p, wave);
        multiply(One{}, No{});
        mix_slots<0, kProducts, kFragments, FORM::kMoreQ + (FORM::kTogether ? FORM::kLoadsP : 0), OP::kConversions>();
        if constexpr (OP::kPin) {      // (a use of the products on this side of the branch below: the compiler would move them behind it, away from the reads and loads)
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int j = 0; j < TQ; ++j) asm volatile("" ::"a"(acc[i][j]));
        }
        loaded_q();
        if constexpr (FORM::kTogether) loaded_p();
    };

    // the order that the loop keeps: Q of a K-tile, then P of that K-tile, or of the next one where P has a slot more; the last one of P comes with the first step
#pragma unroll
    for (int k = FORM::NQ - FORM::NP; k < FORM::NQ; ++k) {
        if (k >= 0) {
            issue_q();
            loaded_q();
        }
        if (k < FORM::NQ - 1 || FORM::kTogether) {
            from_p.template issue<0, FORM::kLoadsP>(ring_lds + free_p, wave);
            loaded_p();
        }
    }
    __builtin_amdgcn_s_waitcnt(wait_imm((FORM::NP - (FORM::kTogether ? 1 : 2)) * FORM::kLoadsP + (FORM::NQ - 1) * FORM::kMoreQ));
    barrier();
    read(0, Zero{});
    for (int unit = first; unit < end; unit += each) {
        const RingCall<EPILOGUE> &now = again(call);
        const int from = ring_unit<FORM>(now.job, unit).split * now.job.k_per, count = min(now.job.k_per, now.job.nk - from);
        step(Yes{});
        for (int k = 1; k < count; ++k) step(No{});
        results_ready<FORM>(acc);
        int own = lane;
        asm volatile("" : "+v"(own));      // (what the results' places are made of is formed here, not held through the loop)
        // the wave's own part of the free slot of P, which its own next loads fill; every wave has left that K-tile
        uint8_t *const staging = ring_lds + (FORM::kTogether || FORM::kLds > FORM::kAtStaging ? FORM::kAtStaging + wave * FORM::STAGING : free_p + wave * FORM::kLoadsP * 1024);
        const RingCall<EPILOGUE> &then = again(call);
        const RingUnit u = ring_unit<FORM>(then.job, unit);
        then.epilogue(acc, u.p0 + wp * FORM::kWaveAcross, u.q0 + wq * TQ * 32, u.split, staging, own);
        stored = true;
        read(0, Zero{});      // (again: the fragments would take registers that the results need)
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
    constexpr int kAcross = TP / kTiles, kStrips = TQ * kAcross;
    four_t mine[kTiles][4];      // of the strip at hand: taken from the accumulators while the strip before it comes back from LDS
    auto take = [&](int strip) {
        const int j = strip / kAcross, i0 = strip % kAcross * kTiles;
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int k = 0; k < 4; ++k) mine[i][r][k] = (T)f(result<FORM>(acc[i0 + i][j], 4 * r + k), (i0 + i) * 32 + 8 * r + k, j);
    };
    take(0);
#pragma unroll
    for (int strip = 0; strip < kStrips; ++strip) {
        const int j = strip / kAcross, i0 = strip % kAcross * kTiles;
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int byte = (i * 32 + 8 * r) * S + 4 * half * S;
                *reinterpret_cast<four_t *>(staging + row * kRow + (((byte >> 4) ^ swz) << 4) + (byte & 15)) = mine[i][r];
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
            f32x4 old[kReads];
            if (ADD) {
#pragma unroll
                for (int n = 0; n < kReads; ++n)
                    if (inside[n]) old[n] = *reinterpret_cast<const f32x4 *>(at[n]);
            }
            if (FULL) {
                __builtin_amdgcn_sched_barrier(0);
                if (strip + 1 < kStrips) take(strip + 1);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (ADD) {
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
        if (!FULL && strip + 1 < kStrips) take(strip + 1);
    }
}
// edge: f where the wave's part may reach beyond the entry `end`
template <class FORM, class T, bool ADD, class F, class G>
__device__ __forceinline__ void store_rows(const v16f (&acc)[FORM::TP][FORM::TQ], const RowTarget<T> &to, int p0, int q0, uint8_t *staging, int lane, int end, const F &f,
                                           const G &edge)
{
    if (p0 + FORM::TP * 32 <= end && q0 + FORM::TQ * 32 <= to.rows_q && to.width == 16) {
        store_strips<FORM, T, ADD, true>(acc, to, p0, q0, staging, lane, f);
    } else {
        store_strips<FORM, T, ADD, false>(acc, to, p0, q0, staging, lane, edge);
        __builtin_amdgcn_s_waitcnt(wait_imm(0));
    }
}
template <class FORM, class T, bool ADD, class F>
__device__ __forceinline__ void store_rows(const v16f (&acc)[FORM::TP][FORM::TQ], const RowTarget<T> &to, int p0, int q0, uint8_t *staging, int lane, const F &f)
{
    store_rows<FORM, T, ADD>(acc, to, p0, q0, staging, lane, to.rows_p, f, f);
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
