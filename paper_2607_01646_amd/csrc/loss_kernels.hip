// loss_kernels.hip -- gfx950 kernels of the vocabulary head's losses.
//
// Three products on the matrix cores, with what comes before and after them:
//   logits    l = hidden weight^T           statistics of each row, the logits of a piece
//   d_hidden  = d_logits weight             contraction over the words
//   d_weight  = d_logits^T hidden           contraction over the tokens
// each 2 tokens * vocab * dim operations, and the row kernel that turns a
// piece's logits into their gradient.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "ops_internal.h"

namespace ckpt {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u16x4 u16x4_any __attribute__((aligned(2)));
typedef u16x8 u16x8_any __attribute__((aligned(2)));

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kInf = __builtin_inff();

__device__ inline float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
__device__ inline uint16_t bf16_of(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// An fp32 value as the sum of 3 bf16: each rounds what the ones before it leave, which is exact: 24 bits, less 8 and a
// sign each time.  Rounded and not cut off, so that the second is at most 2^-8 and the third 2^-17 of the leading power of
// two, of either sign: that is what the products below leave out.  A value whose rounding would be infinite is cut off
// instead.  An infinity is its third plane alone: that one meets only the other operand's first, so the product is infinity
// times the value; as a first plane it would meet all three, and a 0 among them gives NaN.  (Where both operands are infinite
// it is NaN; all logits of such a token are infinite or NaN, and its loss is no number either way.)  A NaN is its first plane
// (one whose bits would all be cut off keeps one).
__device__ inline void split3(float x, uint16_t (&p)[3])
{
    const uint32_t u = __float_as_uint(x);
    if ((u & 0x7F800000u) == 0x7F800000u) {
        const bool nan = (u & 0x007FFFFFu) != 0;
        p[0] = nan ? (uint16_t)(u >> 16 | 0x40) : 0;
        p[1] = 0;
        p[2] = nan ? 0 : (uint16_t)(u >> 16);
        return;
    }
    p[0] = (u & 0x7FFFFFFFu) >= 0x7F7F8000u ? (uint16_t)(u >> 16) : bf16_of(x);
    const float r = x - __uint_as_float((uint32_t)p[0] << 16);
    p[1] = bf16_of(r);
    p[2] = bf16_of(r - __uint_as_float((uint32_t)p[1] << 16));
}

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

// ---- epilogues ----
//
// acc[tp][tq] holds out[q][p] of 32 x 32 tiles: q = q0 + 32 tq + lane % 32 and, for register i,
// p = p0 + 32 tp + 8 (i / 4) + 4 (lane / 32) + i % 4: every lane has runs of 4 consecutive p of one q.  They are what a
// workgroup does while no product is made, so they are kept short: tiles that lie inside the output check no bounds.

// Two runs of 4 values in 16 bits, p + 4 half.. and p + 8 + 4 half.., of the lanes of both halves: as 8 consecutive ones,
// p + 8 half.., for one store of 16 bytes.
__device__ inline u16x8 pair_of(uint2 a, uint2 b)
{
    const auto x = __builtin_amdgcn_permlane32_swap(a.x, b.x, false, false);
    const auto y = __builtin_amdgcn_permlane32_swap(a.y, b.y, false, false);
    const uint4 r = {x[0], y[0], x[1], y[1]};
    return __builtin_bit_cast(u16x8, r);
}
__device__ inline uint2 bf16_run(f32x4 x)
{
    return __builtin_bit_cast(uint2, u16x4{bf16_of(x[0]), bf16_of(x[1]), bf16_of(x[2]), bf16_of(x[3])});
}

// Two values of [0, 1] in 16 bits each: the 7 exponent bits that fp32 has for them and 9 of the significand, to nearest.
// The whole range of exp is kept, and the rounding is a quarter of bf16's.  (A NaN does not fit: it is known from the
// sums.)
__device__ inline uint32_t pack_e16(float a, float b)
{
    const uint32_t half = 1u << 13;
    return (__float_as_uint(a) + half) >> 14 | ((__float_as_uint(b) + half) << 2 & 0xFFFF0000u);
}
__device__ inline float unpack_e16(uint16_t x) { return __uint_as_float((uint32_t)x << 14); }

// What a lane reads for its epilogue ahead of the products.
template <class End, int TQ>
struct Early {
    __device__ inline Early(const End&, uint32_t) {}
};
template <int TQ>
struct Early<LogitsOut, TQ> {
    int32_t target[TQ];
    __device__ inline Early(const LogitsOut& o, uint32_t q0)
    {
#pragma unroll
        for (int t = 0; t < TQ; ++t) {
            const uint32_t q = q0 + 32 * t + (threadIdx.x & 31);
            const int64_t y = o.target && q < o.tokens ? o.target[q] : -1;
            target[t] = y >= 0 && y < o.vocab ? (int32_t)y : -1;
        }
    }
};

template <int TP, int TQ>
__device__ inline void finish(const LogitsOut& o, const Early<LogitsOut, TQ>& early, f32x16 (&acc)[TP][TQ],
                              uint32_t wave_p0, uint32_t q0, uint32_t)
{
    constexpr int kTiles = kPartWords / 32, kMine = kTiles * 16; // of a part; a lane's words of it
    static_assert(TP % kTiles == 0, "a wave's words are whole parts");
    const uint32_t lane = threadIdx.x & 63, half = lane >> 5;
#pragma unroll
    for (int part = 0; part < TP / kTiles; ++part) {
        const uint32_t p0 = wave_p0 + part * kPartWords;
        if (p0 >= o.vocab) break;
        const bool whole = p0 + kPartWords <= o.vocab;
#pragma unroll
        for (int tq = 0; tq < TQ; ++tq) {
            const uint32_t q = q0 + 32 * tq + (lane & 31);
            const bool here = q < o.tokens;
            float x[kMine]; // of words p0 + 32 (j / 16) + 8 (j / 4 % 4) + 4 half + j % 4
#pragma unroll
            for (int j = 0; j < kMine; ++j) x[j] = acc[part * kTiles + j / 16][tq][j % 16];
            if (!whole) {
#pragma unroll
                for (int j = 0; j < kMine; ++j)
                    if (p0 + 32 * (j / 16) + 8 * (j / 4 % 4) + 4 * half + j % 4 >= o.vocab) x[j] = -kInf;
            }
            const uint32_t t = (uint32_t)early.target[tq] - p0;
            if (t < kPartWords && (t >> 2 & 1) == half) {
                const uint32_t mine = (t >> 5) * 16 + (t >> 3 & 3) * 4 + (t & 3);
                float l = 0;
#pragma unroll
                for (int j = 0; j < kMine; ++j) l = mine == j ? x[j] : l;
                o.target_logit[q] = l;
            }
            if (o.logits && here) {
                float* row = o.logits + (uint64_t)q * o.ld + p0 + 4 * half; // ld covers whole parts
#pragma unroll
                for (int j = 0; j < kMine; j += 4)
                    *(f32x4*)(row + 32 * (j / 16) + 8 * (j / 4 % 4)) = {x[j], x[j + 1], x[j + 2], x[j + 3]};
            }
            float top = -kInf; // fmaxf passes a NaN by; the sum below does not
#pragma unroll
            for (int j = 0; j < kMine; ++j) top = fmaxf(top, x[j]);
            top = fmaxf(top, __shfl_xor(top, 32));
            const float low = top == -kInf ? 0.0f : top;
            float sum = 0, sum_t = 0;
            if (o.part_t) {
#pragma unroll
                for (int j = 0; j < kMine; ++j) sum_t += exp_of((x[j] - low) * o.inv_t);
                sum_t += __shfl_xor(sum_t, 32);
            }
#pragma unroll
            for (int j = 0; j < kMine; ++j) {
                x[j] = exp_of(x[j] - low);
                sum += x[j];
            }
            sum += __shfl_xor(sum, 32);
            if (here && half == 0) {
                const uint64_t at = (uint64_t)q * o.parts + p0 / kPartWords;
                o.part[at] = make_float2(top, sum);
                if (o.part_t) o.part_t[at] = sum_t;
            }
            if (o.e16) {
                uint16_t* row = o.e16 + (uint64_t)q * o.ld + p0 + 8 * half;
#pragma unroll
                for (int j = 0; j < kMine; j += 8) {
                    const u16x8 v = pair_of(make_uint2(pack_e16(x[j], x[j + 1]), pack_e16(x[j + 2], x[j + 3])),
                                            make_uint2(pack_e16(x[j + 4], x[j + 5]), pack_e16(x[j + 6], x[j + 7])));
                    if (here) *(u16x8*)(row + 32 * (j / 16) + 8 * (j / 4 % 4)) = v;
                }
            }
        }
    }
}

struct GradEnd {
    GradOut o;
    uint32_t p, q;
};

// The factor that all rows share, and the loss: one wave's sums, in an order of their own (of few tokens, where a
// launch for them alone takes longer).
__device__ inline float few_sums(const LossSums& s, bool total)
{
    double weight = 0, loss = 0;
    for (uint32_t n = threadIdx.x & 63; n < s.tokens; n += 64) {
        const float w = s.row_weight[n];
        weight += w;
        if (total && w != 0) loss += (double)w * s.token_loss[n];
    }
    for (int o = 32; o; o >>= 1) {
        weight += __shfl_xor(weight, o);
        loss += __shfl_xor(loss, o);
    }
    const double over = s.mean ? (weight != 0 ? 1 / weight : 0.0) : 1.0;
    if (total && threadIdx.x == 0) *s.loss = (float)(loss * over);
    return (float)(over * (s.grad_scale ? *s.grad_scale : 1.0f));
}

template <int TQ>
struct Early<GradEnd, TQ> {
    float scale;
    __device__ inline Early(const GradEnd& e, uint32_t)
    {
        scale = e.o.sums.tokens ? few_sums(e.o.sums, e.o.total && blockIdx.x + 1 == gridDim.x)
                                : (e.o.scale ? *e.o.scale : 1.0f);
    }
};

template <int TP, int TQ>
__device__ inline void finish(const GradEnd& e, const Early<GradEnd, TQ>& early, f32x16 (&acc)[TP][TQ], uint32_t p0,
                              uint32_t q0, uint32_t slice)
{
    const GradOut& o = e.o;
    const uint32_t lane = threadIdx.x & 63, half = lane >> 5;
    const bool whole = p0 + 32 * TP <= e.p;
#pragma unroll
    for (int tq = 0; tq < TQ; ++tq) {
        const uint32_t q = q0 + 32 * tq + (lane & 31);
        const bool here = q < e.q;
        const uint64_t row = (uint64_t)slice * o.slice + (uint64_t)q * o.ld;
#pragma unroll
        for (int tp = 0; tp < TP; ++tp)
#pragma unroll
            for (int i = 0; i < 16; i += 8) {
                f32x4 x[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int r = i + 4 * u;
                    const uint32_t p = p0 + 32 * tp + 2 * r + 4 * half;
                    x[u] = {acc[tp][tq][r], acc[tp][tq][r + 1], acc[tp][tq][r + 2], acc[tp][tq][r + 3]};
                    if (o.add && here) {
                        const float* add = o.add + (uint64_t)q * o.add_ld + p;
                        for (uint32_t j = 0; j < 4; ++j)
                            if (p + j < e.p) x[u][j] += add[j];
                    }
                    x[u] *= early.scale;
                    if (o.f32 && here) {
                        float* out = (float*)o.out + row + p;
                        if (whole)
                            *(f32x4_any*)out = x[u];
                        else
                            for (uint32_t j = 0; j < 4; ++j)
                                if (p + j < e.p) out[j] = x[u][j];
                    }
                }
                if (o.f32) continue;
                const u16x8 v = pair_of(bf16_run(x[0]), bf16_run(x[1]));
                const uint32_t p = p0 + 32 * tp + 2 * i + 8 * half;
                uint16_t* out = (uint16_t*)o.out + row + p;
                if (!here) continue;
                if (whole)
                    *(u16x8_any*)out = v;
                else
                    for (uint32_t j = 0; j < 8; ++j)
                        if (p + j < e.p) out[j] = v[j];
            }
    }
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
template <int ZP_, int ZQ_, bool PA_, bool QA_, int BP_, int BQ_, int NWP_, int NWQ_, int BK_, int BUFS_>
struct Shape {
    static constexpr int ZP = ZP_, ZQ = ZQ_, BP = BP_, BQ = BQ_, NWP = NWP_, NWQ = NWQ_, BK = BK_, BUFS = BUFS_;
    static constexpr bool PA = PA_, QA = QA_;
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

// `block` of the tiles' workgroups, for run `slice` of k.
template <class S, class End>
__device__ inline void product(const Operand& P, const Operand& Q, const ProductShape& shape, const End& end,
                               uint32_t block, uint32_t slice, uint16_t* s0, uint16_t* s1, uint16_t* s2, uint16_t* s3)
{
    constexpr int ZP = S::ZP, ZQ = S::ZQ, BK = S::BK, BUFS = S::BUFS, kThreads = S::kThreads;
    constexpr int TP = S::BP / S::NWP / 32, TQ = S::BQ / S::NWQ / 32;
    using TileP = Tile<S::BP, BK, S::PA>;
    using TileQ = Tile<S::BQ, BK, S::QA>;
    constexpr int kAtQ = ZP * TileP::kElems;

    const uint32_t np = (shape.p + S::BP - 1) / S::BP, nq = (shape.q + S::BQ - 1) / S::BQ;
    const uint2 tile = tile_of(block, np, nq);
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
        constexpr int kPairs = ZP == 3 && ZQ == 3 ? 6 : ZP * ZQ, kProducts = TP * TQ * kPairs;
        int n = 0;
#pragma unroll
        for (int sum = kPairs == 6 ? 2 : ZP + ZQ - 2; sum >= 0; --sum)
#pragma unroll
            for (int z = 0; z <= sum; ++z) {
                if (z >= ZP || sum - z >= ZQ) continue;
#pragma unroll
                for (int t = 0; t < TP; ++t)
#pragma unroll
                    for (int u = 0; u < TQ; ++u) {
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
    for (; step + BUFS <= last; step += BUFS) {
        one_step(s0, s1, step);
        one_step(s1, BUFS > 2 ? s2 : s0, step + 1);
        if constexpr (BUFS > 2) one_step(s2, BUFS > 3 ? s3 : s0, step + 2);
        if constexpr (BUFS > 3) one_step(s3, s0, step + 3);
    }
    if (step < last) one_step(s0, s1, step);
    if (BUFS > 2 && step + 1 < last) one_step(s1, s2, step + 1);
    if (BUFS > 3 && step + 2 < last) one_step(s2, s3, step + 2);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // no load is left that would write the LDS of another workgroup
    finish<TP, TQ>(end, early, acc, p0 + wp, q0 + wq, slice);
}

template <class S, class End>
__global__ __launch_bounds__(S::kThreads, S::kThreads >= 512 ? 2 : 1) void product_kernel(
    const Operand P, const Operand Q, const ProductShape shape, const End end)
{
    CKPT_BUFFERS(S, S);
    product<S>(P, Q, shape, end, blockIdx.x, blockIdx.y, s0, s1, s2, s3);
}

// Two products that do not wait for each other in one launch: d_hidden's workgroups, then d_weight's.
struct Both {
    Operand hp, hq, wp, wq;
    ProductShape hs, ws;
    uint32_t h_tiles; // workgroups of one run of k
    uint32_t h_all;
};
template <class H, class W>
__global__ __launch_bounds__(H::kThreads, 1) void both_kernel(const Both b, const GradEnd h_end, const GradEnd w_end)
{
    static_assert(H::kThreads == W::kThreads, "");
    CKPT_BUFFERS(H, W);
    if (blockIdx.x < b.h_all)
        product<H>(b.hp, b.hq, b.hs, h_end, blockIdx.x % b.h_tiles, blockIdx.x / b.h_tiles, s0, s1, s2, s3);
    else
        product<W>(b.wp, b.wq, b.ws, w_end, blockIdx.x - b.h_all, 0, s0, s1, s2, s3);
}

template <class S>
uint64_t tiles_of(const ProductShape& s)
{
    return (uint64_t)((s.p + S::BP - 1) / S::BP) * ((s.q + S::BQ - 1) / S::BQ);
}

template <class S, class End>
hipError_t launch_product(const Operand& P, const Operand& Q, const ProductShape& s, const End& end, hipStream_t stream)
{
    const uint64_t tiles = tiles_of<S>(s);
    if (tiles == 0 || tiles * S::kThreads > 0xffffffffu || s.slices == 0 || s.slices > 65535 || s.k % S::BK)
        return hipErrorInvalidValue;
    product_kernel<S, End><<<dim3((uint32_t)tiles, s.slices), S::kThreads, 0, stream>>>(P, Q, s, end);
    return hipGetLastError();
}

template <class H, class W>
hipError_t launch_both(Both b, const GradEnd& h_end, const GradEnd& w_end, hipStream_t stream)
{
    const uint64_t h_tiles = tiles_of<H>(b.hs), all = h_tiles * b.hs.slices + tiles_of<W>(b.ws);
    if (h_tiles == 0 || all * H::kThreads > 0xffffffffu || b.hs.k % H::BK || b.ws.k % W::BK) return hipErrorInvalidValue;
    b.h_tiles = (uint32_t)h_tiles;
    b.h_all = (uint32_t)(h_tiles * b.hs.slices);
    both_kernel<H, W><<<(uint32_t)all, H::kThreads, 0, stream>>>(b, h_end, w_end);
    return hipGetLastError();
}

// ---- rows ----

__device__ inline float load1(const void* p, uint64_t at, bool f32)
{
    return f32 ? ((const float*)p)[at] : __uint_as_float((uint32_t)((const uint16_t*)p)[at] << 16);
}

constexpr int kRowThreads = 256;

__device__ inline float wave_max(float x)
{
    for (int o = 32; o; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
    return x;
}
__device__ inline float wave_sum(float x)
{
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
    return x;
}
// Over the workgroup: the maxima of the first MAX values and the sums of the others, the waves' in their order.  s holds
// a value of each for every wave and is used once (one barrier).
template <int WAVES, int MAX, int N>
__device__ inline void block_reduce(float (&x)[N], float* s)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = i < MAX ? wave_max(x[i]) : wave_sum(x[i]);
        if ((threadIdx.x & 63) == 0) s[i * WAVES + (threadIdx.x >> 6)] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = s[i * WAVES];
        for (int w = 1; w < WAVES; ++w) x[i] = i < MAX ? fmaxf(x[i], s[i * WAVES + w]) : x[i] + s[i * WAVES + w];
    }
}

// A teacher entry that is there: a word, and any logit but -inf.
__device__ inline bool entry(const LossRows& r, uint64_t n, uint32_t k, int64_t* word, float* logit)
{
    *word = r.t_index[n * r.t_index_ld + k];
    *logit = load1(r.t_logits, n * r.t_logits_ld + k, r.t_f32);
    return *word >= 0 && *logit != -kInf;
}

// 8 values as PLANES planes of bf16, `plane` apart: rounded, 2 bf16 whose sum has 16 bits, or the 3 of an fp32 value.
template <int PLANES>
__device__ inline void put8(uint16_t* to, uint64_t plane, const float (&g)[8])
{
    u16x8 x[PLANES];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if constexpr (PLANES == 3) {
            uint16_t y[3];
            split3(g[j], y);
            for (int z = 0; z < 3; ++z) x[z][j] = y[z];
        } else {
            x[0][j] = bf16_of(g[j]);
            if constexpr (PLANES == 2) x[1][j] = bf16_of(g[j] - __uint_as_float((uint32_t)x[0][j] << 16));
        }
    }
#pragma unroll
    for (int z = 0; z < PLANES; ++z) *(u16x8*)(to + z * plane) = x[z];
}
// One wave a row.
__global__ __launch_bounds__(kRowThreads) void prepare_kernel(const LossRows r, bool weigh, uint32_t row0, uint32_t rows,
                                                              const RowCopy c)
{
    const uint32_t lane = threadIdx.x & 63, row = blockIdx.x * (kRowThreads / 64) + (threadIdx.x >> 6);
    bool counts = row < rows;
    if (weigh && counts) {
        const uint64_t n = row0 + row;
        const float w = r.token_weight ? r.token_weight[n] : 1.0f;
        counts = r.target && r.alpha < 1 && r.target[n] != r.ignore_index;
        for (uint32_t k = lane; k < r.topk && r.alpha > 0; k += 64) {
            int64_t word;
            float logit;
            counts |= entry(r, n, k, &word, &logit);
        }
        counts = __ballot(counts) != 0 && w != 0;
        if (lane == 0) r.row_weight[n] = counts ? w : 0.0f;
    }
    if (!c.src || row >= c.dst_rows) return;
    const uint64_t src = (uint64_t)(row0 + row) * c.src_ld;
    uint16_t* dst = c.dst + (uint64_t)row * c.dst_cols;
    for (uint32_t at = 8 * lane; at < c.dst_cols; at += 512) { // dst_cols: a multiple of 64
        if (c.f32) {
            const float* from = (const float*)c.src + src + at;
            float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (counts && at + 8 <= c.cols) {
                const f32x4 a = *(const f32x4_any*)from, b = *(const f32x4_any*)(from + 4);
                for (int j = 0; j < 4; ++j) x[j] = a[j], x[4 + j] = b[j];
            } else if (counts) {
                for (int j = 0; j < 7; ++j)
                    if (at + j < c.cols) x[j] = from[j];
            }
            put8<3>(dst + at, c.plane, x);
        } else {
            u16x8 x = {0, 0, 0, 0, 0, 0, 0, 0};
            const uint16_t* from = (const uint16_t*)c.src + src + at;
            if (counts && at + 8 <= c.cols)
                x = *(const u16x8_any*)from;
            else if (counts)
                for (int j = 0; j < 7; ++j)
                    if (at + j < c.cols) x[j] = from[j];
            *(u16x8*)(dst + at) = x;
        }
    }
}

__device__ inline void put1(const LossPiece& p, uint16_t* dl, uint32_t v, float g)
{
    if (p.planes == 3) {
        uint16_t x[3];
        split3(g, x);
        for (int z = 0; z < 3; ++z) dl[z * p.dl_plane + v] = x[z];
        return;
    }
    dl[v] = bf16_of(g);
    if (p.planes == 2) dl[p.dl_plane + v] = bf16_of(g - __uint_as_float((uint32_t)dl[v] << 16));
}

// The row of hidden states as d_weight reads it: zeros where the row does not count.
template <int THREADS>
__device__ inline void copy_row(const RowCopy& c, uint32_t row, uint64_t n, bool counts)
{
    if (!c.src) return;
    const uint16_t* from = (const uint16_t*)c.src + n * c.src_ld;
    uint16_t* to = c.dst + (uint64_t)row * c.dst_cols;
    for (uint32_t at = 8 * threadIdx.x; at < c.dst_cols; at += 8 * THREADS)
        *(u16x8*)(to + at) = counts ? *(const u16x8*)(from + at) : u16x8{0, 0, 0, 0, 0, 0, 0, 0};
}

template <int THREADS>
__device__ inline void zero_row(const LossPiece& p, uint16_t* dl)
{
    if (!dl) return;
    for (uint32_t z = 0; z < p.planes; ++z)
        for (uint64_t v = 8 * threadIdx.x; v < p.dl_ld; v += 8 * THREADS) // dl_ld: a multiple of 64
            *(u16x8*)(dl + z * p.dl_plane + v) = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
}

// The row's target where the cross entropy has a share in it, else -1; *word: whether it is one of the vocabulary.
__device__ inline bool labelled(const LossRows& r, uint64_t n, int64_t* label, bool* word)
{
    *label = -1;
    *word = false;
    if (!r.target || r.alpha >= 1 || r.target[n] == r.ignore_index) return false;
    *label = r.target[n];
    *word = *label >= 0 && *label < r.vocab;
    return true;
}

// The loss of one token alone.
__device__ inline void only_row(const LossRows& r, float weight, float loss)
{
    if (r.tokens != 1) return;
    const double over = r.mean ? (weight != 0 ? 1.0 / weight : 0.0) : 1.0;
    *r.loss = weight != 0 ? (float)((double)weight * loss * over) : 0.0f;
    *r.scale = (float)(over * (r.grad_scale ? *r.grad_scale : 1.0f));
}

// One workgroup a row: its log-sum-exp and loss and, with d_logits, its row of
//   w (alpha T (p^T - q) + (1 - alpha) (p - 1_y)).
// The factor that all rows share (grad_scale and the mean's) is left to the products' fp32 sums: here the label's term
// is near -1 for most tokens of a new model, which bf16 holds exactly, and -1/tokens would be rounded the same way in
// all of them.  Rounding d_logits to bf16 is what feeds the matrix cores; its errors are independent from word to word
// and of the size of the gradients' own rounding.
//
// E16: the logits are held as exponentials in 16 bits (cross entropy in bf16), in the place where d_logits goes, and
// the factors of the parts in LDS: 4 bytes of traffic a word, not 6.  Bound by HBM.
template <int WAVES, bool E16>
__global__ __launch_bounds__(WAVES * 64) void rows_kernel(const LossRows r, const LossPiece p, const RowCopy copy)
{
    extern __shared__ float s_more[]; // E16: a factor for each part; else the teacher's entries
    __shared__ float s_first[3 * WAVES], s_second[3 * WAVES], s_third[WAVES];
    constexpr uint32_t kThreads = WAVES * 64;
    const uint32_t row = blockIdx.x, tid = threadIdx.x;
    const uint64_t n = p.row0 + (uint64_t)row;
    uint16_t* dl = p.d_logits ? p.d_logits + (uint64_t)row * p.dl_ld : nullptr;
    if (row >= p.rows) {
        copy_row<kThreads>(copy, row, n, false);
        zero_row<kThreads>(p, dl);
        return;
    }
    const float given = r.token_weight ? r.token_weight[n] : 1.0f;
    int64_t label;
    bool word;
    const bool has_label = labelled(r, n, &label, &word);
    const bool teach = !E16 && r.alpha > 0;
    const float inv_t = 1 / r.temperature;
    constexpr float kBad = 4096; // for an entry that is no word of the vocabulary: above the entries a row can have
    // The teacher's entries: logit, then q; word, -1 where there is none; the student's logit.
    float* s_q = s_more;
    float* s_own = s_more + r.topk;
    int* s_word = (int*)(s_more + 2 * r.topk);
    const float* logits = E16 ? nullptr : p.logits + (uint64_t)row * p.ld;
    const float2* part = p.part + (uint64_t)row * p.parts;
    const float* part_t = p.part_t ? p.part_t + (uint64_t)row * p.parts : nullptr;
    float first[3] = {-kInf, -kInf, 0}; // the largest logit, the teacher's largest, the count of entries
    // What does not wait for anything is asked for first: two parts a lane (the others of a larger vocabulary are read
    // twice), the label's logit.
    constexpr int kAhead = 2;
    float2 ahead[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
        const uint32_t k = tid + u * kThreads;
        ahead[u] = k < p.parts ? part[k] : make_float2(-kInf, 0);
    }
    const float target_logit = word ? r.target_logit[n] : 0.0f;
    for (uint32_t k = tid + kAhead * kThreads; k < p.parts; k += kThreads) first[0] = fmaxf(first[0], part[k].x);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) first[0] = fmaxf(first[0], ahead[u].x);
    if (teach) {
        for (uint32_t k = tid; k < r.topk; k += kThreads) {
            int64_t at;
            float t;
            const bool there = entry(r, n, k, &at, &t), known = there && at < r.vocab;
            s_q[k] = there ? t : -kInf;
            s_word[k] = known ? (int)at : -1;
            s_own[k] = known ? logits[at] : 0.0f;
            if (there) {
                first[1] = fmaxf(first[1], t);
                first[2] += known ? 1 : kBad;
            }
        }
    }
    block_reduce<WAVES, 2>(first, s_first);
    const float low = first[0] == -kInf ? 0.0f : first[0], t_top = first[1], t_count = first[2];
    const bool counts = (has_label || t_count > 0) && given != 0;
    const float weight = counts ? given : 0.0f;
    if (tid == 0) r.row_weight[n] = weight;
    copy_row<kThreads>(copy, row, n, counts);
    if (!counts) {
        if (tid == 0) {
            r.token_loss[n] = r.lse[n] = 0;
            only_row(r, 0, 0);
        }
        zero_row<kThreads>(p, dl);
        return;
    }

    float second[3] = {0, 0, 0}; // the sums of exponentials: the words', at the temperature, the teacher's
    auto add_part = [&](uint32_t k, float2 x) {
        // A maximum of -inf: all words at -inf and sums of 0, or NaN among them, which a maximum passes by and the sums show.
        const bool none = x.x == -kInf;
        const float f = none ? x.y : exp_of(x.x - low);
        second[0] += x.y * f;
        if (E16) s_more[k] = f;
        if (part_t) second[1] += part_t[k] * (none ? x.y : exp_of((x.x - low) * inv_t));
    };
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
        if (tid + u * kThreads < p.parts) add_part(tid + u * kThreads, ahead[u]);
    for (uint32_t k = tid + kAhead * kThreads; k < p.parts; k += kThreads) add_part(k, part[k]);
    if (teach)
        for (uint32_t k = tid; k < r.topk; k += kThreads) second[2] += exp_of((s_q[k] - t_top) * inv_t);
    block_reduce<WAVES, 0>(second, s_second);
    const float sum = second[0], lse = low + __builtin_amdgcn_logf(sum) * kLn2;
    const float lse_t = part_t ? low * inv_t + __builtin_amdgcn_logf(second[1]) * kLn2 : lse;

    const uint32_t target = word ? (uint32_t)label : ~0u; // no word is as large
    float loss = 0, hard = 0;
    if (has_label) {
        hard = word ? 1 - r.alpha : __builtin_nanf(""); // the loss and the gradient show a label that is no word
        loss = word ? hard * (lse - target_logit) : hard;
    }
    if constexpr (E16) {
        if (tid == 0) {
            r.token_loss[n] = loss;
            r.lse[n] = lse;
            only_row(r, weight, loss);
        }
        const float scale = weight * hard / sum;
        for (uint32_t v = 8 * tid; v < p.dl_ld; v += 8 * kThreads) {
            const u16x8 e = *(const u16x8*)(dl + v);
            const float f = v < r.vocab ? scale * s_more[v / kPartWords] : 0.0f;
            float g[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = f * unpack_e16(e[j]);
            if (target - v < 8) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (target - v == j) g[j] -= weight * hard;
            }
            if (v + 8 > r.vocab) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (v + j >= r.vocab) g[j] = 0;
            }
            put8<1>(dl + v, 0, g);
        }
        return;
    }

    float soft = 0;
    if (teach) {
        const float log_sum = __builtin_amdgcn_logf(second[2]) * kLn2;
        float kd[1] = {0};
        for (uint32_t k = tid; k < r.topk; k += kThreads) {
            const float log_q = (s_q[k] - t_top) * inv_t - log_sum, q = t_count > 0 ? exp_of(log_q) : 0.0f;
            s_q[k] = q;
            if (s_word[k] >= 0 && q != 0) kd[0] += q * (log_q - (s_own[k] * inv_t - lse_t));
        }
        block_reduce<WAVES, 0>(kd, s_third);
        if (t_count > 0) {
            soft = t_count >= kBad ? __builtin_nanf("") : r.alpha * r.temperature;
            loss += soft * r.temperature * kd[0];
        }
    }
    if (tid == 0) {
        r.token_loss[n] = loss;
        r.lse[n] = teach ? lse_t : lse;
        only_row(r, weight, loss);
    }
    if (!dl) return;

    const float soft_w = weight * soft, hard_w = weight * hard;
    auto gradient = [&](float l) {
        float g = 0;
        if (hard != 0) g = hard_w * exp_of(l - lse);
        if (soft != 0) g += soft_w * exp_of(l * inv_t - lse_t);
        return g;
    };
    auto store = [&](auto planes) {
        for (uint32_t v = 8 * tid; v < p.dl_ld; v += 8 * kThreads) {
            const f32x4 a = *(const f32x4*)(logits + v), b = *(const f32x4*)(logits + v + 4);
            float g[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) g[j] = gradient(a[j]), g[4 + j] = gradient(b[j]);
            if (target - v < 8) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (target - v == j) g[j] -= hard_w;
            }
            if (v + 8 > r.vocab) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (v + j >= r.vocab) g[j] = 0;
            }
            put8<planes>(dl + v, p.dl_plane, g);
        }
    };
    if (p.planes == 1)
        store(std::integral_constant<int, 1>());
    else if (p.planes == 2)
        store(std::integral_constant<int, 2>());
    else
        store(std::integral_constant<int, 3>());
    if (soft == 0) return;
    // The teacher's words once more, each by the first of its entries, when the stores above have been made.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    for (uint32_t k = tid; k < r.topk; k += kThreads) {
        const int at = s_word[k];
        if (at < 0) continue;
        float q = 0;
        bool first = true;
        for (uint32_t j = 0; j < r.topk; ++j) {
            if (s_word[j] != at) continue;
            first &= j >= k;
            q += s_q[j];
        }
        if (first) put1(p, dl, at, gradient(s_own[k]) - soft_w * q - ((uint32_t)at == target ? hard_w : 0.0f));
    }
}

__global__ __launch_bounds__(1024) void finish_kernel(const LossRows r, bool total)
{
    __shared__ double s[2][16];
    double weight = 0, loss = 0;
    for (uint32_t n0 = 4 * threadIdx.x; n0 < r.tokens; n0 += 4096) {
        f32x4 w = {0, 0, 0, 0}, x = {0, 0, 0, 0};
        if (n0 + 4 <= r.tokens) {
            w = *(const f32x4_any*)(r.row_weight + n0);
            if (total) x = *(const f32x4_any*)(r.token_loss + n0);
        } else {
            for (int j = 0; j < 3; ++j)
                if (n0 + j < r.tokens) {
                    w[j] = r.row_weight[n0 + j];
                    if (total) x[j] = r.token_loss[n0 + j];
                }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            weight += w[j];
            if (w[j] != 0) loss += (double)w[j] * x[j];
        }
    }
    for (int o = 32; o; o >>= 1) {
        weight += __shfl_xor(weight, o);
        loss += __shfl_xor(loss, o);
    }
    if ((threadIdx.x & 63) == 0) {
        s[0][threadIdx.x >> 6] = weight;
        s[1][threadIdx.x >> 6] = loss;
    }
    __syncthreads();
    if (threadIdx.x) return;
    weight = loss = 0;
    for (int w = 0; w < 16; ++w) {
        weight += s[0][w];
        loss += s[1][w];
    }
    const double over = r.mean ? (weight != 0 ? 1 / weight : 0.0) : 1.0;
    *r.scale = (float)(over * (r.grad_scale ? *r.grad_scale : 1.0f));
    if (total) *r.loss = (float)(loss * over);
}

// ---- logits of a few tokens ----
//
// For up to 4 tokens (fp32: some more, 8 at a time) the head's rows are all that is read, and the matrix cores would wait
// for them: a workgroup takes the 64 words of a part, each wave 8, and multiplies a run of 1 KiB of each row with the
// tokens' own on the vector units, the next runs on their way.  No operand is copied or split first: any stride and
// alignment, and fp32 as it is.  Bound by HBM: one token against 32000 x 4096 in bf16 44 us, 5.9 TB/s.
constexpr int kDotWords = 8, kDotWaves = kPartWords / kDotWords;

template <bool F32>
struct Run { // a lane's values of one row
    static constexpr int kValues = F32 ? 4 : 8;
    uint4 raw;
    __device__ inline float at(int j) const
    {
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
        if (F32) return __uint_as_float(w[j]);
        return __uint_as_float(j & 1 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
    }
    // Values k.. of a row of dim, zeros past its end.
    __device__ inline void load(const void* base, uint64_t row, uint64_t k, uint64_t dim)
    {
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
        typedef u32x4 any __attribute__((aligned(2)));
        if (k + kValues <= dim) {
            const u32x4 x = __builtin_nontemporal_load((const any*)((const uint8_t*)base + (row + k) * (F32 ? 4 : 2)));
            raw = {x[0], x[1], x[2], x[3]};
            return;
        }
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < kValues - 1; ++j) {
            if (k + j >= dim) continue;
            if (F32)
                w[j] = ((const uint32_t*)base)[row + k + j];
            else
                w[j / 2] |= (uint32_t)((const uint16_t*)base)[row + k + j] << (j & 1 ? 16 : 0);
        }
        raw = {w[0], w[1], w[2], w[3]};
    }
};

template <int N, bool F32>
__global__ __launch_bounds__(kDotWaves * 64, 2) void dots_kernel(const DotOperand W, const DotOperand H, uint32_t dim, const LogitsOut o)
{
    constexpr uint32_t kRun = 64 * Run<F32>::kValues;
    __shared__ float s_logit[N][kPartWords];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t p0 = blockIdx.x * kPartWords, mine = p0 + wave * kDotWords;
    float acc[N][kDotWords];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < kDotWords; ++i) acc[n][i] = 0;
    Run<F32> now[kDotWords], next[kDotWords], h[N], h_next[N];
    auto load = [&](Run<F32>* w, Run<F32>* t, uint32_t k0) {
#pragma unroll
        for (int i = 0; i < kDotWords; ++i)
            w[i].load(W.base, (uint64_t)min(mine + i, o.vocab - 1) * W.ld, k0 + Run<F32>::kValues * lane, dim);
#pragma unroll
        for (int n = 0; n < N; ++n)
            t[n].load(H.base, (uint64_t)min((uint32_t)n, o.tokens - 1) * H.ld, k0 + Run<F32>::kValues * lane, dim);
    };
    // Each wave begins at another run of its rows: rows lie a power of two apart for most heads, and waves at the same
    // place in them would all wait for the same memory channels.
    const uint32_t runs = (dim + kRun - 1) / kRun;
    uint32_t at = (blockIdx.x * kDotWaves + wave) % runs;
    load(now, h, at * kRun);
    for (uint32_t c = 0; c < runs; ++c) {
        at = at + 1 == runs ? 0 : at + 1;
        if (c + 1 < runs) load(next, h_next, at * kRun);
#pragma unroll
        for (int i = 0; i < kDotWords; ++i)
#pragma unroll
            for (int j = 0; j < Run<F32>::kValues; ++j)
#pragma unroll
                for (int n = 0; n < N; ++n) acc[n][i] = __builtin_fmaf(now[i].at(j), h[n].at(j), acc[n][i]);
#pragma unroll
        for (int i = 0; i < kDotWords; ++i) now[i] = next[i];
#pragma unroll
        for (int n = 0; n < N; ++n) h[n] = h_next[n];
    }
    // The lanes' sums: each exchange halves the words that a lane answers for.
#pragma unroll
    for (int n = 0; n < N; ++n) {
        int left = kDotWords;
#pragma unroll
        for (int step = 32; step > 4; step /= 2) {
            left /= 2;
            const bool high = lane & step;
#pragma unroll
            for (int i = 0; i < left; ++i) {
                const float keep = high ? acc[n][i + left] : acc[n][i], give = high ? acc[n][i] : acc[n][i + left];
                acc[n][i] = keep + __shfl_xor(give, step);
            }
        }
        float x = acc[n][0];
        for (int step = 4; step; step /= 2) x += __shfl_xor(x, step);
        const uint32_t word = (lane >> 5 & 1) * 4 + (lane >> 4 & 1) * 2 + (lane >> 3 & 1);
        if ((lane & 7) == 0) s_logit[n][wave * kDotWords + word] = x;
    }
    __syncthreads();
    if (wave >= N || wave >= o.tokens) return;
    const uint32_t q = wave, p = p0 + lane;
    const float x = p < o.vocab ? s_logit[q < N ? q : 0][lane] : -kInf;
    if (o.logits) o.logits[(uint64_t)q * o.ld + p] = x; // ld covers whole parts
    if (o.target && o.target[q] == (int64_t)p && p < o.vocab) o.target_logit[q] = x;
    const float top = wave_max(x), low = top == -kInf ? 0.0f : top;
    const float sum = wave_sum(exp_of(x - low)), sum_t = o.part_t ? wave_sum(exp_of((x - low) * o.inv_t)) : 0.0f;
    if (lane == 0) {
        const uint64_t at = (uint64_t)q * o.parts + blockIdx.x;
        o.part[at] = make_float2(top, sum);
        if (o.part_t) o.part_t[at] = sum_t;
    }
}

template <bool F32>
hipError_t dots_of(const DotOperand& w, const DotOperand& h, uint32_t dim, const LogitsOut& o, hipStream_t stream)
{
    constexpr uint32_t kThreads = kDotWaves * 64;
    if (o.tokens == 1)
        dots_kernel<1, F32><<<o.parts, kThreads, 0, stream>>>(w, h, dim, o);
    else if (o.tokens == 2)
        dots_kernel<2, F32><<<o.parts, kThreads, 0, stream>>>(w, h, dim, o);
    else if (o.tokens <= 4)
        dots_kernel<4, F32><<<o.parts, kThreads, 0, stream>>>(w, h, dim, o);
    else
        dots_kernel<8, F32><<<o.parts, kThreads, 0, stream>>>(w, h, dim, o);
    return hipGetLastError();
}

__global__ __launch_bounds__(256) void zero_kernel(void* out, uint32_t rows, uint32_t cols, uint64_t ld, bool f32)
{
    for (uint64_t row = blockIdx.x; row < rows; row += gridDim.x)
        for (uint32_t c = threadIdx.x; c < cols; c += 256)
            if (f32)
                ((float*)out)[row * ld + c] = 0;
            else
                ((uint16_t*)out)[row * ld + c] = 0;
}

// One row of q a y, 4 values a lane: p is a multiple of 4 in `slices` (rows of ld_s).
__global__ __launch_bounds__(256) void join_kernel(const float* slices, uint64_t slice, uint32_t ld_s, uint32_t n, uint32_t p,
                                                   const GradOut o)
{
    const uint32_t at = 4 * (blockIdx.x * 256 + threadIdx.x), q = blockIdx.y;
    const float scale = o.sums.tokens ? few_sums(o.sums, false) : (o.scale ? *o.scale : 1.0f);
    if (at >= p) return;
    const float* from = slices + (uint64_t)q * ld_s + at;
    f32x4 x = {0, 0, 0, 0};
    for (uint32_t k = 0; k < n; ++k) x += *(const f32x4*)(from + k * slice);
    x *= scale;
    const uint64_t to = (uint64_t)q * o.ld + at;
    for (int j = 0; j < 4; ++j) {
        if (at + j >= p) break;
        if (o.f32)
            ((float*)o.out)[to + j] = x[j];
        else
            ((uint16_t*)o.out)[to + j] = bf16_of(x[j]);
    }
}

} // namespace

namespace {

// Workgroup tiles, and what a step of 64 values of k takes one of them (us) where the compute units have one, and
// where all have two; each round of tiles takes 3 us more.
//   bf16:     256 x 256 (8 waves of 64 x 128): bound by the matrix cores, 1.2-1.3 PFLOP/s with all units busy
//             128 x 128 (4 waves of 64 x 64): 1.0-1.07 PFLOP/s; alone on a unit its steps wait for their loads
//             64 x 64 (2 waves of 64 x 32): 4 buffers hide that; for few tokens, where loads are all of the time
//             (64 x 2048 x 8192: 9.8 us, 128 x 128 23.6 us)
//   2 planes of d_logits: the smaller two (they are used for few tokens)
//   3 planes: 256 x 128 (8 waves of 64 x 64; LDS has no room for more), 128 x 128 and 64 x 64
enum Size { kSmall, kMiddle, kLarge };
struct Tiling {
    Size size;
    uint32_t slices;
};

// The tile and the number of runs of k that finish first.
Tiling tiling(const ProductShape& s, uint32_t zp, uint32_t zq, uint32_t most)
{
    Tiling best = {kMiddle, 1};
    double least = 1e30;
    for (int size = kSmall; size <= kLarge; ++size) {
        if (size == kLarge && zp != zq) continue;
        const uint32_t bp = size == kSmall ? 64 : size == kMiddle ? 128 : 256;
        const uint32_t bq = size == kLarge && zp == 3 ? 128 : bp;
        const double alone = zp == 3 ? (size == kSmall ? 0.95 : size == kMiddle ? 3.0 : 4.6)
                                     : (size == kSmall ? 0.25 : size == kMiddle ? 0.65 : 1.7) * zq;
        const double both = size == kLarge || zp == 3 ? 2 * alone : (size == kSmall ? 0.38 : 1.02) * zq;
        const uint64_t tiles = (uint64_t)((s.p + bp - 1) / bp) * ((s.q + bq - 1) / bq);
        for (uint32_t n = 1; n <= std::min({most, 64u, std::max(1u, s.k / 256)}); ++n) {
            const uint64_t all = tiles * n, pairs = all / 512, left = all % 512;
            const double steps = (double)((s.k / 64 + n - 1) / n);
            const double t = pairs * (steps * both + 3) +
                             (left == 0 ? 0 : left <= 256 ? steps * alone + 3 : steps * both + 3) +
                             (n > 1 ? 3 + 0.8 * n + 8.0 * s.p * s.q * n / 6e6 : 0);
            if (t < least) least = t, best = {(Size)size, n};
        }
    }
    return best;
}

// The shapes.  The smaller two of gradients have 4 waves each, for one launch of both, and together no more LDS than
// lets two workgroups share a unit (fp32: no such shapes).
template <int ZP, int ZQ, bool PA, bool QA>
using Large = std::conditional_t<
    ZP == 3, Shape<ZP, ZQ, PA, QA, 256, 128, 4, 2, 32, 2>,
    std::conditional_t<PA, Shape<ZP, ZQ, PA, QA, 256, 256, 4, 2, 32, 4>, Shape<ZP, ZQ, PA, QA, 256, 256, 2, 4, 64, 2>>>;
template <int ZP, int ZQ, bool PA, bool QA>
using Middle = Shape<ZP, ZQ, PA, QA, 128, 128, 2, 2, ZP == 3 || ZQ == 2 ? 32 : 64, 2>;
template <int ZP, int ZQ, bool PA, bool QA>
using Small = Shape<ZP, ZQ, PA, QA, 64, 64, PA ? 2 : 1, 2, ZP == 3 ? 32 : 64, PA || ZP == 3 ? 3 : 4>;

template <int Z>
hipError_t logits_of(const Operand& w, const Operand& h, const ProductShape& s, const LogitsOut& o, hipStream_t stream)
{
    const Size size = tiling(s, Z, Z, 1).size;
    return size == kLarge    ? launch_product<Large<Z, Z, false, false>>(w, h, s, o, stream)
           : size == kMiddle ? launch_product<Middle<Z, Z, false, false>>(w, h, s, o, stream)
                             : launch_product<Small<Z, Z, false, false>>(w, h, s, o, stream);
}

template <int ZP, int ZQ>
hipError_t gradients_of(const Both& b, const GradEnd& he, const GradEnd& we, hipStream_t stream)
{
    const Size h = tiling(b.hs, ZP, ZQ, b.hs.slices).size, w = tiling(b.ws, ZP, ZQ, 1).size;
    using HM = Middle<ZP, ZQ, true, false>;
    using HS = Small<ZP, ZQ, true, false>;
    using WM = Middle<ZP, ZQ, true, true>;
    using WS = Small<ZP, ZQ, true, true>;
    if (h != kLarge && w != kLarge)
        return h == kMiddle ? (w == kMiddle ? launch_both<HM, WM>(b, he, we, stream) : launch_both<HM, WS>(b, he, we, stream))
                            : (w == kMiddle ? launch_both<HS, WM>(b, he, we, stream) : launch_both<HS, WS>(b, he, we, stream));
    if constexpr (ZP == ZQ) { // (1, 2) has no large shape
        using HL = Large<ZP, ZQ, true, false>;
        using WL = Large<ZP, ZQ, true, true>;
        const hipError_t e = h == kLarge    ? launch_product<HL>(b.hp, b.hq, b.hs, he, stream)
                             : h == kMiddle ? launch_product<HM>(b.hp, b.hq, b.hs, he, stream)
                                            : launch_product<HS>(b.hp, b.hq, b.hs, he, stream);
        if (e != hipSuccess) return e;
        return w == kLarge    ? launch_product<WL>(b.wp, b.wq, b.ws, we, stream)
               : w == kMiddle ? launch_product<WM>(b.wp, b.wq, b.ws, we, stream)
                              : launch_product<WS>(b.wp, b.wq, b.ws, we, stream);
    }
    return hipErrorInvalidValue;
}

} // namespace

hipError_t launch_logits(const Operand& w, const Operand& h, const ProductShape& s, uint32_t planes,
                         const LogitsOut& o, hipStream_t stream)
{
    return planes == 3 ? logits_of<3>(w, h, s, o, stream) : logits_of<1>(w, h, s, o, stream);
}

hipError_t launch_dots(const DotOperand& w, const DotOperand& h, uint32_t dim, bool f32, const LogitsOut& o,
                       hipStream_t stream)
{
    if (o.e16) return hipErrorInvalidValue;
    for (uint32_t n = 0; n < o.tokens; n += 8) { // the tokens of a launch
        LogitsOut part = o;
        part.tokens = std::min(8u, o.tokens - n);
        part.target = o.target ? o.target + n : nullptr;
        part.target_logit = o.target_logit + n;
        part.part = o.part + (uint64_t)n * o.parts;
        part.part_t = o.part_t ? o.part_t + (uint64_t)n * o.parts : nullptr;
        part.logits = o.logits ? o.logits + (uint64_t)n * o.ld : nullptr;
        const DotOperand rows = {(const uint8_t*)h.base + (uint64_t)n * h.ld * (f32 ? 4 : 2), h.ld};
        const hipError_t e = f32 ? dots_of<true>(w, rows, dim, part, stream) : dots_of<false>(w, rows, dim, part, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_gradients(const Operand& w, const Operand& h, uint32_t zp, const Operand& dl, uint32_t zq,
                            const ProductShape& dh, const GradOut& dho, const ProductShape& dw, const GradOut& dwo,
                            hipStream_t stream)
{
    const Both b = {w, dl, h, dl, dh, dw, 0, 0};
    const GradEnd he = {dho, dh.p, dh.q}, we = {dwo, dw.p, dw.q};
    return zp == 3   ? gradients_of<3, 3>(b, he, we, stream)
           : zq == 2 ? gradients_of<1, 2>(b, he, we, stream)
                     : gradients_of<1, 1>(b, he, we, stream);
}

uint32_t d_hidden_slices(uint32_t p, uint32_t q, uint32_t k, uint32_t zp, uint32_t zq, uint32_t most)
{
    return tiling({p, q, k, 1, false}, zp, zq, std::max(1u, most)).slices;
}

hipError_t launch_join(const float* slices, uint64_t slice, uint32_t ld_s, uint32_t n, uint32_t p, uint32_t q,
                       const GradOut& o, hipStream_t stream)
{
    for (uint32_t q0 = 0; q0 < q; q0 += 65535) { // rows of a launch
        GradOut part = o;
        part.out = (uint8_t*)o.out + (uint64_t)q0 * o.ld * (o.f32 ? 4 : 2);
        join_kernel<<<dim3((p + 1023) / 1024, std::min(q - q0, 65535u)), 256, 0, stream>>>(
            slices + (uint64_t)q0 * ld_s, slice, ld_s, n, p, part);
    }
    return hipGetLastError();
}

hipError_t launch_zero(void* out, uint32_t rows, uint32_t cols, uint64_t ld, bool f32, hipStream_t stream)
{
    zero_kernel<<<std::min(rows, 16384u), 256, 0, stream>>>(out, rows, cols, ld, f32);
    return hipGetLastError();
}

hipError_t launch_prepare(const LossRows* r, uint32_t row0, uint32_t rows, const RowCopy& c, hipStream_t stream)
{
    const uint32_t all = c.src ? std::max(rows, c.dst_rows) : rows;
    constexpr uint32_t kRows = 1u << 24; // of a launch, a wave each: 2^30 lanes
    if (c.src && all > kRows) return hipErrorInvalidValue;
    for (uint32_t at = 0; at < all; at += kRows) {
        const uint32_t n = std::min(kRows, all - at);
        prepare_kernel<<<(n + 3) / 4, kRowThreads, 0, stream>>>(r ? *r : LossRows(), r != nullptr, row0 + at,
                                                               std::min(n, rows - std::min(rows, at)), c);
    }
    return hipGetLastError();
}

hipError_t launch_rows(const LossRows& r, const LossPiece& p, const RowCopy& copy, hipStream_t stream)
{
    const uint32_t all = std::max({p.rows, p.d_logits ? p.dl_rows : 0, copy.src ? copy.dst_rows : 0});
    if (all == 0) return hipSuccess;
    if (p.e16)
        rows_kernel<4, true><<<all, 256, p.parts * 4, stream>>>(r, p, copy);
    else
        rows_kernel<4, false><<<all, 256, r.topk * 12, stream>>>(r, p, copy);
    return hipGetLastError();
}

hipError_t launch_finish(const LossRows& r, bool total, hipStream_t stream)
{
    finish_kernel<<<1, 1024, 0, stream>>>(r, total);
    return hipGetLastError();
}

} // namespace ckpt
