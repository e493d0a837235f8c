// Products on the matrix cores for the kernels of the operators: tiles of two
// operands in LDS, and the loop that multiplies them.  What becomes of a tile
// is its user's (Early, Finish).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "ops_internal.h"

namespace ckpt {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u16x4 u16x4_any __attribute__((aligned(2)));
typedef u16x8 u16x8_any __attribute__((aligned(2)));

__device__ inline uint16_t bf16_of(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// ---- tiles of an operand in LDS ----
//
// A tile is B rows by BK values of k, in 16-byte chunks that the loads write
// straight to LDS, one wave 64 consecutive chunks at a time; which chunk of
// global memory goes to a slot is chosen so that the reads below meet every
// bank once.
template <int B, int BK, bool ACROSS>
struct Tile {
    static constexpr int kElems = B * BK, kChunks = kElems / 8;

    // k contiguous: rows of BK; a chunk moves by its row, which spreads the 16 rows that a quarter of a wave reads.
    static __device__ inline uint32_t turn(uint32_t row)
    {
        constexpr uint32_t slots = BK / 8;
        return (row / (16 / slots)) & (slots - 1);
    }
    // k across rows: BK rows of B; pairs of chunks (16 values) move by k, which spreads the 4 rows and 2 pairs
    // that half a wave reads.
    static __device__ inline uint32_t turn_pair(uint32_t k)
    {
        return B >= 128 ? (k & 3) << 1 : B == 64 ? (k & 2) : 0;
    }

    // Load instructions of a wave.
    template <int THREADS>
    static constexpr int loads()
    {
        return (kChunks + THREADS - 1) / THREADS;
    }
    // What a lane keeps for its loads: byte offsets from the tile's first row (below 2^31: 256 rows of 2^22 values), or
    // for k across rows the column's, which all its loads share.
    template <int THREADS>
    struct Lane {
        uint32_t off[ACROSS ? 1 : loads<THREADS>()];
        __device__ inline Lane(const Operand& o, uint32_t row0)
        {
            if constexpr (!ACROSS) {
#pragma unroll
                for (int i = 0; i < loads<THREADS>(); ++i) {
                    const uint32_t s = i * THREADS + threadIdx.x, r = s / (BK / 8), c = (s % (BK / 8)) ^ turn(r);
                    off[i] = (min(row0 + r, o.rows - 1) - row0) * (uint32_t)o.ld * 2 + c * 16;
                }
            } else {
                static_assert(THREADS / (B / 8) % 4 == 0, "a lane's loads are of rows with the same turn");
                const uint32_t k = threadIdx.x / (B / 8), at = threadIdx.x % (B / 8);
                off[0] = min(row0 + (((at >> 1) ^ turn_pair(k)) << 1 | (at & 1)) * 8, o.cols - 8) * 2;
            }
        }
    };
    // The wave's load `i`.  Nothing is fetched unless `any`: a buffer of no bytes.
    template <int THREADS>
    static __device__ inline void load(const Operand& o, const uint16_t* base, const Lane<THREADS>& lane, uint32_t row0,
                                       uint32_t k0, bool any, int i, uint16_t* lds)
    {
        static_assert(kChunks % THREADS == 0, "every wave has the same loads");
        const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        // The last values of k may lie past the operand altogether (k runs to a multiple of 64, BK may be less).
        if constexpr (ACROSS) k0 = min(k0, o.rows - 1);
        const uint16_t* from = base + (ACROSS ? (uint64_t)k0 * o.ld : (uint64_t)row0 * o.ld + k0);
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
            (void*)from, 0, __builtin_amdgcn_readfirstlane(any ? -1 : 0), 0x00020000);
        uint32_t off = lane.off[ACROSS ? 0 : i];
        if constexpr (ACROSS)
            off += min((uint32_t)((i * THREADS + threadIdx.x) / (B / 8)), o.rows - 1 - k0) * (uint32_t)o.ld * 2;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            r, (__attribute__((address_space(3))) void*)(lds + (i * THREADS + wave * 64) * 8), 16, off, 0, 0, 0);
    }

    // The lane's 8 values of rows [r0, r0 + 32), k [16 step, 16 step + 16): row lane % 32, k 8 (lane / 32) + 0..7.
    static __device__ inline bf16x8 read(const uint16_t* lds, uint32_t r0, uint32_t step)
    {
        const uint32_t lane = threadIdx.x & 63;
        if constexpr (!ACROSS) {
            const uint32_t r = r0 + (lane & 31), c = step * 2 + (lane >> 5);
            return *(const bf16x8*)(lds + (r * (BK / 8) + (c ^ turn(r))) * 8);
        } else {
            // Transposing reads: 16 lanes name 4 rows of 16 values and each receives a column of them.
            typedef __attribute__((address_space(3))) i16x4* Ptr;
            i16x4 h[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t k = step * 16 + 8 * (lane >> 5) + 4 * u + ((lane >> 2) & 3);
                const uint32_t pair = (r0 >> 4) + ((lane >> 4) & 1), half = (lane >> 1) & 1;
                h[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (Ptr)(lds + (k * (B / 8) + ((pair ^ turn_pair(k)) << 1 | half)) * 8 + (lane & 1) * 4));
            }
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// What a lane reads for its epilogue ahead of the products.
template <class End, int TQ>
struct Early {
    __device__ inline Early(const End&, uint32_t) {}
};
// What becomes of a tile: run(end, early, acc, p0, q0, slice, lds) for a wave's accumulators; `lds` is the product's first
// buffer, free once all waves of the workgroup have met.  acc[tp][tq] holds out[q][p] of
// 32 x 32 tiles: q = q0 + 32 tq + lane % 32 and, for register i, p = p0 + 32 tp + 8 (i / 4) + 4 (lane / 32) + i % 4: every
// lane has runs of 4 consecutive p of one q.
template <class End, int TP, int TQ>
struct Finish;

// Two runs of 4 values in 16 bits, p + 4 half.. and p + 8 + 4 half.., of the lanes of both halves: as 8 consecutive ones,
// p + 8 half.., for one store of 16 bytes.
__device__ inline u16x8 pair_of(uint2 a, uint2 b)
{
    const auto x = __builtin_amdgcn_permlane32_swap(a.x, b.x, false, false);
    const auto y = __builtin_amdgcn_permlane32_swap(a.y, b.y, false, false);
    const uint4 r = {x[0], y[0], x[1], y[1]};
    return __builtin_bit_cast(u16x8, r);
}

// Which tile a workgroup takes.  Workgroups go round the 8 XCDs, each with an L2 of its own: an XCD gets a run of
// consecutive tiles, and runs go through bands of kBand tiles of q, so that the tiles which an XCD works on at a time
// share their operands' rows.
constexpr uint32_t kXcds = 8, kBand = 4;
__device__ inline uint2 tile_of(uint32_t block, uint32_t np, uint32_t nq)
{
    const uint32_t n = np * nq, each = n / kXcds, more = n % kXcds;
    const uint32_t xcd = block % kXcds, at = block / kXcds;
    const uint32_t t = xcd * each + min(xcd, more) + at;
    const uint32_t band = t / (kBand * np), in = t % (kBand * np), width = min(kBand, nq - band * kBand);
    return make_uint2(in / width, band * kBand + in % width);
}

// ---- the product ----
//
// A workgroup of NWP x NWQ waves makes a BP x BQ tile of out[q][p] = sum_k P(p, k) Q(q, k), each wave a part of it in
// registers.  Two buffers in LDS: while one is multiplied the loads of the next BK values of k write the other one.
// ZP and ZQ planes an operand.  3 and 3: fp32 operands as 3 bf16 planes; of the 9 products of planes the 6 whose sum of
// indexes is at most 2 are made, smallest first.  The others are at most 2 * 2^-8 * 2^-17 + 2^-34 of the value, 2^-24, of
// either sign (2^-23 within 2^-8 of fp32's largest value).
//
// 2 and 2 (HALF): planes of fp16, hi = x and lo = x - hi rounded to nearest, 22 bits together; hi hi, hi lo and lo hi are
// made, and lo lo, 2^-22 of the value, is left out unless ALL.
//
// PARTS: the sums of every `chunk` values of k are added up in registers of their own.  A sum that grows is rounded by more
// and more (of squares, 8192 values of k: 9.5e-7 of it in one go), with two planes 3 times for every 16 values.
template <int ZP_, int ZQ_, bool PA_, bool QA_, int BP_, int BQ_, int NWP_, int NWQ_, int BK_, int BUFS_, bool HALF_ = false,
          bool PARTS_ = false, bool ALL_ = false>
struct Shape {
    static constexpr int ZP = ZP_, ZQ = ZQ_, BP = BP_, BQ = BQ_, NWP = NWP_, NWQ = NWQ_, BK = BK_, BUFS = BUFS_;
    static constexpr bool PA = PA_, QA = QA_, HALF = HALF_, PARTS = PARTS_;
    // Products of planes whose indexes sum to more than this are left out.
    static constexpr int kMostSum = ZP == 3 && ZQ == 3 ? 2 : HALF && !ALL_ && ZP == 2 && ZQ == 2 ? 1 : ZP + ZQ - 2;
    static constexpr int kThreads = NWP * NWQ * 64;
    static constexpr int kBuffer = (ZP * BP + ZQ * BQ) * BK; // elements
    static_assert(BUFS >= 2 && BUFS <= 4, "");
};

// LDS of a kernel that makes products of shapes A and B.  Arrays of their own, so that the compiler sees that a read of
// one waits for no load into another.
#define CKPT_BUFFERS(A, B)                                                                                          \
    constexpr int kBuf01 = std::max(A::kBuffer, B::kBuffer);                                                        \
    constexpr int kBuf2 = std::max(A::BUFS > 2 ? A::kBuffer : 1, B::BUFS > 2 ? B::kBuffer : 1);                     \
    constexpr int kBuf3 = std::max(A::BUFS > 3 ? A::kBuffer : 1, B::BUFS > 3 ? B::kBuffer : 1);                     \
    __shared__ __attribute__((aligned(16))) uint16_t s0[kBuf01], s1[kBuf01], s2[kBuf2], s3[kBuf3]

// Tile `tile` (of p and q) by the `block`-th of the tiles' workgroups, for run `slice` of k.
template <class S, class End>
__device__ inline void product(const Operand& P, const Operand& Q, const ProductShape& shape, const End& end,
                               uint2 tile, uint32_t block, uint32_t slice, uint16_t* s0, uint16_t* s1, uint16_t* s2, uint16_t* s3,
                               uint32_t chunk = 0)
{
    constexpr int ZP = S::ZP, ZQ = S::ZQ, BK = S::BK, BUFS = S::BUFS, kThreads = S::kThreads;
    constexpr int TP = S::BP / S::NWP / 32, TQ = S::BQ / S::NWQ / 32;
    using TileP = Tile<S::BP, BK, S::PA>;
    using TileQ = Tile<S::BQ, BK, S::QA>;
    constexpr int kAtQ = ZP * TileP::kElems;

    const uint32_t p0 = __builtin_amdgcn_readfirstlane(tile.x * S::BP), q0 = __builtin_amdgcn_readfirstlane(tile.y * S::BQ);
    const uint32_t steps = shape.k / BK;
    const uint32_t first = __builtin_amdgcn_readfirstlane((uint64_t)steps * slice / shape.slices);
    const uint32_t last = __builtin_amdgcn_readfirstlane((uint64_t)steps * (slice + 1) / shape.slices);
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wp = (wave % S::NWP) * 32 * TP, wq = (wave / S::NWP) * 32 * TQ;

    f32x16 acc[TP][TQ];
#pragma unroll
    for (int a = 0; a < TP; ++a)
#pragma unroll
        for (int b = 0; b < TQ; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[a][b][i] = 0;

    const typename TileP::template Lane<kThreads> lane_p(P, p0);
    const typename TileQ::template Lane<kThreads> lane_q(Q, q0);
    // The wave's load `i` of a step's kLoads into buffer s; none past the last step.
    constexpr int kLoadsP = TileP::template loads<kThreads>(), kLoadsQ = TileQ::template loads<kThreads>();
    constexpr int kLoads = ZP * kLoadsP + ZQ * kLoadsQ;
    // shape.around: each workgroup goes round its steps from another one.
    const uint32_t round = last - first;
    const uint32_t ahead = shape.around && round ? __builtin_amdgcn_readfirstlane(block % round) : 0;
    auto load = [&](uint16_t* s, uint32_t step, int i) {
        const bool any = step < last;
        const uint32_t at = step + ahead, k0 = any ? (at < last ? at : at - round) * BK : 0;
        if (i < ZP * kLoadsP) {
            const int z = i % ZP, j = i / ZP;
            TileP::template load<kThreads>(P, P.base + z * P.plane, lane_p, p0, k0, any, j, s + z * TileP::kElems);
        } else {
            const int z = (i - ZP * kLoadsP) % ZQ, j = (i - ZP * kLoadsP) / ZQ;
            TileQ::template load<kThreads>(Q, Q.base + z * Q.plane, lane_q, q0, k0, any, j, s + kAtQ + z * TileQ::kElems);
        }
    };
    struct Part { // a wave's operands of 16 values of k
        bf16x8 a[ZP][TP], b[ZQ][TQ];
    };
    auto read = [&](Part& f, const uint16_t* s, int k) {
#pragma unroll
        for (int z = 0; z < ZP; ++z)
#pragma unroll
            for (int t = 0; t < TP; ++t) f.a[z][t] = TileP::read(s + z * TileP::kElems, wp + 32 * t, k);
#pragma unroll
        for (int z = 0; z < ZQ; ++z)
#pragma unroll
            for (int t = 0; t < TQ; ++t) f.b[z][t] = TileQ::read(s + kAtQ + z * TileQ::kElems, wq + 32 * t, k);
    };
    // Nothing moves past: a part's reads stay ahead of the products that hide them, and loads between products.
    auto hold = [] { __builtin_amdgcn_sched_barrier(0); };
    // The products of a part, with the first `loads` loads of `step` into s spread among them: issued at once by all
    // waves they fill the queue to the caches, and no wave gets past it to its products (8192 x 4096 x 32000: 1.97 ms,
    // spread 1.65 ms).
    auto multiply = [&](const Part& f, uint16_t* s, uint32_t step, int loads) {
        constexpr int kPairs = S::kMostSum < ZP + ZQ - 2 ? (ZP == 3 ? 6 : 3) : ZP * ZQ, kProducts = TP * TQ * kPairs;
        int n = 0;
#pragma unroll
        for (int sum = S::kMostSum; sum >= 0; --sum)
#pragma unroll
            for (int z = 0; z <= sum; ++z) {
                if (z >= ZP || sum - z >= ZQ) continue;
#pragma unroll
                for (int t = 0; t < TP; ++t)
#pragma unroll
                    for (int u = 0; u < TQ; ++u) {
                        if constexpr (S::HALF)
                            acc[t][u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
                                __builtin_bit_cast(f16x8, f.a[z][t]), __builtin_bit_cast(f16x8, f.b[sum - z][u]),
                                acc[t][u], 0, 0, 0);
                        else
                            acc[t][u] =
                                __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.a[z][t], f.b[sum - z][u], acc[t][u], 0, 0, 0);
                        ++n;
                        for (int i = loads * (n - 1) / kProducts; i < loads * n / kProducts; ++i) {
                            hold();
                            load(s, step, i);
                            hold();
                        }
                    }
            }
    };
    // Once this wave's reads are done and its loads but those of the last BUFS - 2 steps have landed: when that is so
    // for all.
    auto meet = [] {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((BUFS - 2) * kLoads) : "memory");
    };
    // One step on buffer s: each part is read while the one before is multiplied.  All of s is in registers before the
    // last part is multiplied, so the waves meet there: behind that part's products s is filled again and the next
    // buffer's first part is read.  There is no branch around the loads and reads past the last step: a branch would
    // make the compiler wait for what its other path has not loaded, and what they fetch is not used.
    Part even, odd;
    auto one_step = [&](uint16_t* s, uint16_t* next, uint32_t step) {
        constexpr int kParts = BK / 16;
        static_assert(kParts % 2 == 0, "a step ends with its parts where it began");
#pragma unroll
        for (int k = 0; k < kParts; k += 2) {
            const bool end_part = k + 2 == kParts;
            read(odd, s, k + 1);
            hold();
            multiply(even, s, step, 0);
            hold();
            if (end_part) meet();
            read(even, end_part ? next : s, end_part ? 0 : k + 2);
            hold();
            multiply(odd, s, step + BUFS, end_part ? kLoads : 0);
            hold();
        }
    };
#pragma unroll
    for (int i = 0; i < BUFS * kLoads; ++i)
        load(i / kLoads == 0 ? s0 : i / kLoads == 1 ? s1 : i / kLoads == 2 ? s2 : s3, first + i / kLoads, i % kLoads);
    const Early<End, TQ> early(end, q0 + wq); // waits for all that was loaded before it
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((BUFS - 1) * kLoads) : "memory");
    read(even, s0, 0);
    uint32_t step = first;
    // PARTS: `chunk` is a multiple of 64, or 0 for one sum of all.
    f32x16 sum[S::PARTS ? TP : 1][S::PARTS ? TQ : 1];
    uint32_t part_end = chunk ? first + chunk / BK : 0xffffffffu;
    if constexpr (S::PARTS) {
#pragma unroll
        for (int a = 0; a < TP; ++a)
#pragma unroll
            for (int b = 0; b < TQ; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[a][b][i] = 0;
    }
    auto begin = [&](uint32_t at) { // a step
        if constexpr (S::PARTS) {
            if (at != part_end) return;
            part_end += chunk / BK;
#pragma unroll
            for (int a = 0; a < TP; ++a)
#pragma unroll
                for (int b = 0; b < TQ; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) sum[a][b][i] += acc[a][b][i], acc[a][b][i] = 0;
        }
    };
    for (; step + BUFS <= last; step += BUFS) {
        begin(step);
        one_step(s0, s1, step);
        begin(step + 1);
        one_step(s1, BUFS > 2 ? s2 : s0, step + 1);
        if constexpr (BUFS > 2) {
            begin(step + 2);
            one_step(s2, BUFS > 3 ? s3 : s0, step + 2);
        }
        if constexpr (BUFS > 3) {
            begin(step + 3);
            one_step(s3, s0, step + 3);
        }
    }
    begin(step);
    if (step < last) one_step(s0, s1, step);
    begin(step + 1);
    if (BUFS > 2 && step + 1 < last) one_step(s1, s2, step + 1);
    begin(step + 2);
    if (BUFS > 3 && step + 2 < last) one_step(s2, s3, step + 2);
    if constexpr (S::PARTS) {
#pragma unroll
        for (int a = 0; a < TP; ++a)
#pragma unroll
            for (int b = 0; b < TQ; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[a][b][i] += sum[a][b][i];
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // no load is left that would write the LDS of another workgroup
    Finish<End, TP, TQ>::run(end, early, acc, p0 + wp, q0 + wq, slice, s0);
}

} // namespace
} // namespace ckpt
