// muon_kernels.hip -- gfx950 kernels of the orthogonalised optimizer step.
//
// A matrix's update is divided by its norm and goes `steps` times through
//   A = X X^T,  B = ca I + cb A + cc A A,  X <- B X
// with X laid out so that its rows are the shorter side.  All of it is bound
// by the matrix cores.  The operands are two planes of fp16, 22 bits, and three
// products of planes are made for each product: what is left out is 2^-22 of
// it.  One plane would take a third of the time and leave the result 1.3e-3
// off for gradients without structure, 6e-3 for those of few directions (one
// of bf16 1e-2 and 5e-2): the small singular values of X go through 3.4^steps,
// and what is rounded off beside the large ones goes with them.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "product.h"

namespace ckpt {
namespace {

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

// fp16 holds 4096 times every value of X, A and B: they are at most some 4, and those of a large matrix 2^-13 in X, 2^-18 in
// A, which are normal numbers so.
constexpr float kUp = 4096.0f, kDown = 1.0f / 4096.0f;

__device__ inline f32x4 load4(const float* p) { return *(const f32x4_any*)p; }
__device__ inline f32x4 load4(const uint16_t* p)
{
    const u16x4 u = *(const u16x4_any*)p;
    f32x4 r;
    for (int j = 0; j < 4; ++j) r[j] = __uint_as_float((uint32_t)u[j] << 16);
    return r;
}
__device__ inline float load1(const float* p) { return *p; }
__device__ inline float load1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }

// Values c .. c + 3 of a row of `cols`, zeros past its end.
template <class T>
__device__ inline f32x4 load_row(const T* row, uint32_t c, uint32_t cols)
{
    if (c + 4 <= cols) return load4(row + c);
    f32x4 r = {0, 0, 0, 0};
#pragma unroll
    for (uint32_t j = 0; j < 3; ++j)
        if (c + j < cols) r[j] = load1(row + c + j);
    return r;
}

// x as hi + lo, each to nearest.
__device__ inline void split2(f32x4 x, uint2& hi, uint2& lo)
{
    f16x4 h, l;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        h[j] = (_Float16)x[j];
        l[j] = (_Float16)(x[j] - (float)h[j]);
    }
    hi = __builtin_bit_cast(uint2, h);
    lo = __builtin_bit_cast(uint2, l);
}

__device__ inline uint32_t up64(uint32_t x) { return (x + 63) & ~63u; }

// The matrix of tile t: the last whose first tile is not beyond it.
__device__ inline uint32_t matrix_of(const MuonArgs& a, uint32_t t)
{
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t before = __ballot(lane < a.count && a.m[lane < kMuonMats ? lane : 0].first <= t);
    return __builtin_amdgcn_readfirstlane(63 - __builtin_clzll(before));
}

__device__ inline double wave_sum(double x)
{
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
    return x;
}
// The workgroup's sum in every lane, the waves' in their order.
__device__ inline double block_sum(double x, double* s_wave)
{
    x = wave_sum(x);
    if ((threadIdx.x & 63) == 0) s_wave[threadIdx.x >> 6] = x;
    __syncthreads();
    x = s_wave[0];
    for (int w = 1; w < kThreads / 64; ++w) x += s_wave[w];
    return x;
}

__device__ inline float update(const MuonArgs& a, float m, float cg)
{
    return a.nesterov ? a.beta * m + a.one_beta * cg : m;
}

// ---- the update and its norm ----
//
// Bound by HBM: gradient and momentum are read, the momentum written.  The squares' sums are in 64 bits, a tile's each,
// and added up in their order by every workgroup that needs the norm (at most 2^13 of them for a matrix of 2^25 elements,
// 64 KiB from the L2; a launch of its own would take longer).
template <class G>
__global__ __launch_bounds__(kThreads) void first_kernel(const MuonArgs a)
{
    __shared__ double s_wave[kThreads / 64];
    const uint32_t f = matrix_of(a, blockIdx.x), t = blockIdx.x - a.m[f].first;
    const uint32_t rows = a.m[f].rows, cols = a.m[f].cols, nc = (cols + kMuonCols - 1) / kMuonCols;
    const uint32_t r0 = t / nc * kMuonRows + (threadIdx.x >> 6) * 4, c = t % nc * kMuonCols + (threadIdx.x & 63) * 4;
    const uint64_t ld = a.m[f].in_ld;
    const G* in = (const G*)a.m[f].in;
    float* momentum = (float*)a.m[f].momentum;
    const float cs = a.grad_scale ? *a.grad_scale : 1.0f;
    f32x4 g[4], m[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const uint64_t row = min(r0 + i, rows - 1);
        g[i] = load_row(in + row * ld, c, cols);
        if (momentum) m[i] = load_row(momentum + row * cols, c, cols);
    }
    double sum = 0;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        if (r0 + i >= rows) continue;
        if (momentum) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float cg = cs * g[i][j];
                m[i][j] = a.beta * m[i][j] + a.one_beta * cg;
                g[i][j] = update(a, m[i][j], cg);
            }
            float* to = momentum + (uint64_t)(r0 + i) * cols + c;
            if (c + 4 <= cols)
                *(f32x4_any*)to = m[i];
            else
#pragma unroll
                for (uint32_t j = 0; j < 3; ++j)
                    if (c + j < cols) to[j] = m[i][j];
        }
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
            if (c + j < cols) sum += (double)g[i][j] * (double)g[i][j]; // (zero gradients past the end need not be zero updates)
    }
    sum = block_sum(sum, s_wave);
    if (threadIdx.x == 0) ((double*)a.m[f].part)[t] = sum;
}

template <class G>
__global__ __launch_bounds__(kThreads) void pack_kernel(const MuonArgs a)
{
    __shared__ double s_wave[kThreads / 64];
    __shared__ float s_turn[kMuonTurn][kMuonTurn + 1];
    const uint32_t f = matrix_of(a, blockIdx.x), t = blockIdx.x - a.m[f].first;
    const uint32_t rows = a.m[f].rows, cols = a.m[f].cols;
    const uint32_t s = min(rows, cols), ldx = up64(max(rows, cols));
    const uint64_t plane = (uint64_t)s * ldx, ld = a.m[f].in_ld;
    const G* in = (const G*)a.m[f].in;
    const float* momentum = (const float*)a.m[f].momentum;
    const float cs = a.grad_scale ? *a.grad_scale : 1.0f;
    uint16_t* x = (uint16_t*)a.m[f].x;
    double sum = 0;
    for (uint32_t k = threadIdx.x; k < a.m[f].part_n; k += kThreads) sum += ((const double*)a.m[f].part)[k];
    sum = block_sum(sum, s_wave);
    const float over = (float)((double)kUp / (sqrt(sum) + a.eps));
    // Four values of U over its norm.
    auto values = [&](uint32_t row, uint32_t c) {
        const bool any = row < rows && c < cols;
        const uint64_t r = any ? row : 0;
        f32x4 v = {0, 0, 0, 0};
        if (!any) return v;
        if (!momentum || a.nesterov) v = load_row(in + r * ld, c, cols);
        if (momentum) {
            const f32x4 m = load_row(momentum + r * cols, c, cols);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = update(a, m[j], cs * v[j]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = c + j < cols ? v[j] * over : 0.0f;
        return v;
    };
    auto store = [&](uint64_t at, f32x4 v) {
        uint2 hi, lo;
        split2(v, hi, lo);
        *(uint2*)(x + at) = hi;
        *(uint2*)(x + plane + at) = lo;
    };
    if (rows <= cols) {
        const uint32_t nc = (ldx + kMuonCols - 1) / kMuonCols;
        const uint32_t r0 = t / nc * kMuonRows + (threadIdx.x >> 6) * 4, c = t % nc * kMuonCols + (threadIdx.x & 63) * 4;
        if (c >= ldx) return;
        f32x4 v[4];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) v[i] = values(r0 + i, c);
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (r0 + i < rows) store((uint64_t)(r0 + i) * ldx + c, v[i]);
        return;
    }
    // Tall: X is the transpose, tiles of it through LDS.
    const uint32_t nc = (cols + kMuonTurn - 1) / kMuonTurn;
    const uint32_t r0 = t / nc * kMuonTurn, c0 = t % nc * kMuonTurn;
    const uint32_t at = (threadIdx.x & 15) * 4, line = threadIdx.x >> 4;
    f32x4 v[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) v[i] = values(r0 + line + 16 * i, c0 + at);
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s_turn[line + 16 * i][at + j] = v[i][j];
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const uint32_t c = line + 16 * i;
        if (c0 + c >= cols) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i][j] = s_turn[at + j][c];
        store((uint64_t)(c0 + c) * ldx + r0 + at, v[i]); // ldx covers whole tiles of rows
    }
}

// ---- the products ----

// A tile of A or B, and its mirror image: only the tiles on and below the diagonal are made, and of those only values on and
// below it are used.  So both are symmetric to the last bit, and a value does not depend on the size of the tiles: the
// matrices of a call do not change each other's results.
struct GramEnd {
    uint16_t* out;
    const uint16_t* in; // A, for B
    uint64_t plane;
    uint32_t s, ld;
    float ca, cb, cc;
    bool poly;
};

// Another mapping of a 32 x 32 tile's values: row p of q.  One wave's, through its own LDS.
constexpr uint32_t kTurnLd = 40;
constexpr uint32_t kTurnWave = 32 * kTurnLd;

// What the lanes of this wave have written to LDS is there for its others.
__device__ inline void same_wave()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <int TP, int TQ>
struct Finish<GramEnd, TP, TQ> {
    static __device__ inline void run(const GramEnd& e, const Early<GramEnd, TQ>&, f32x16 (&acc)[TP][TQ], uint32_t p0,
                                      uint32_t q0, uint32_t, uint16_t* lds)
    {
        const uint32_t lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        uint16_t* turn = lds + wave * kTurnWave;
        __syncthreads(); // the buffers are free
#pragma unroll
        for (int tq = 0; tq < TQ; ++tq)
#pragma unroll
            for (int tp = 0; tp < TP; ++tp) {
                const uint32_t ps = p0 + 32 * tp, qs = q0 + 32 * tq, q = qs + (lane & 31);
                if (ps > qs || qs >= e.ld) continue; // ld covers whole tiles of 32
                uint2 hi[4], lo[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint32_t p = ps + 8 * r + 4 * half;
                    f32x4 v;
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = acc[tp][tq][4 * r + j] * kDown;
                    if (e.poly) {
                        f16x4 ah = {0, 0, 0, 0}, al = ah;
                        if (q < e.s) {
                            ah = *(const f16x4*)(e.in + (uint64_t)q * e.ld + p);
                            al = *(const f16x4*)(e.in + e.plane + (uint64_t)q * e.ld + p);
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            v[j] = e.cc * v[j] + e.cb * ((float)ah[j] + (float)al[j]) + (p + j == q ? e.ca * kUp : 0.0f);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = p + j < e.s && q < e.s ? v[j] : 0.0f;
                    split2(v, hi[r], lo[r]);
                }
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const uint2* w = z ? lo : hi;
                    uint16_t* out = e.out + z * e.plane;
                    const u16x8 a = pair_of(w[0], w[1]), b = pair_of(w[2], w[3]);
                    if (ps < qs && q < e.s) {
                        uint16_t* row = out + (uint64_t)q * e.ld + ps + 8 * half;
                        *(u16x8*)row = a;
                        *(u16x8*)(row + 16) = b;
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const u16x4 u = __builtin_bit_cast(u16x4, w[r]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t p = 8 * r + 4 * half + j;
                            if (ps < qs || p <= (lane & 31)) turn[p * kTurnLd + (lane & 31)] = u[j];
                            if (ps == qs && p <= (lane & 31)) turn[(lane & 31) * kTurnLd + p] = u[j];
                        }
                    }
                    same_wave();
                    const uint16_t* from = turn + (lane >> 1) * kTurnLd + (lane & 1) * 16;
                    const u16x8 c = *(const u16x8*)from, d = *(const u16x8*)(from + 8);
                    uint16_t* row = out + (uint64_t)(ps + (lane >> 1)) * e.ld + qs + (lane & 1) * 16;
                    if (ps + (lane >> 1) < e.s) {
                        *(u16x8*)row = c;
                        *(u16x8*)(row + 8) = d;
                    }
                    same_wave();
                }
            }
    }
};

// The next X.
struct NextEnd {
    uint16_t* out;
    uint64_t plane;
    uint32_t s, ld;
};
template <int TP, int TQ>
struct Finish<NextEnd, TP, TQ> {
    static __device__ inline void run(const NextEnd& e, const Early<NextEnd, TQ>&, f32x16 (&acc)[TP][TQ], uint32_t p0,
                                      uint32_t q0, uint32_t, uint16_t*)
    {
        const uint32_t lane = threadIdx.x & 63, half = lane >> 5;
#pragma unroll
        for (int tq = 0; tq < TQ; ++tq)
#pragma unroll
            for (int tp = 0; tp < TP; ++tp) {
                const uint32_t ps = p0 + 32 * tp, q = q0 + 32 * tq + (lane & 31);
                if (ps >= e.ld) continue;
                uint2 hi[4], lo[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    f32x4 v;
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = acc[tp][tq][4 * r + j] * kDown;
                    split2(v, hi[r], lo[r]);
                }
                uint16_t* row = e.out + (uint64_t)q * e.ld + ps + 8 * half;
                const u16x8 h0 = pair_of(hi[0], hi[1]), h1 = pair_of(hi[2], hi[3]);
                const u16x8 l0 = pair_of(lo[0], lo[1]), l1 = pair_of(lo[2], lo[3]);
                if (q >= e.s) continue;
                *(u16x8*)row = h0;
                *(u16x8*)(row + 16) = h1;
                *(u16x8*)(row + e.plane) = l0;
                *(u16x8*)(row + e.plane + 16) = l1;
            }
    }
};

// The last X, [q][p] as the matrix itself lies: into the master copy and the parameter, or as the result.
struct LastEnd {
    float* master; // or nullptr
    void* out;
    uint64_t out_ld;
    uint32_t p, q;
    float keep, lr;
    bool f32;
};
template <int TP, int TQ>
struct Finish<LastEnd, TP, TQ> {
    static __device__ inline void run(const LastEnd& e, const Early<LastEnd, TQ>&, f32x16 (&acc)[TP][TQ], uint32_t p0,
                                      uint32_t q0, uint32_t, uint16_t*)
    {
        const uint32_t lane = threadIdx.x & 63, half = lane >> 5;
#pragma unroll
        for (int tq = 0; tq < TQ; ++tq)
#pragma unroll
            for (int tp = 0; tp < TP; ++tp) {
                const uint32_t q = q0 + 32 * tq + (lane & 31);
                if (q >= e.q) continue;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint32_t p = p0 + 32 * tp + 8 * r + 4 * half;
                    f32x4 v;
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = acc[tp][tq][4 * r + j] * (kDown * kDown);
                    if (p + 4 <= e.p) {
                        if (e.master) {
                            float* w = e.master + (uint64_t)q * e.p + p;
                            v = load4(w) * e.keep - v * e.lr;
                            *(f32x4_any*)w = v;
                        }
                        if (e.f32)
                            *(f32x4_any*)((float*)e.out + (uint64_t)q * e.out_ld + p) = v;
                        else
                            *(u16x4_any*)((uint16_t*)e.out + (uint64_t)q * e.out_ld + p) =
                                u16x4{bf16_of(v[0]), bf16_of(v[1]), bf16_of(v[2]), bf16_of(v[3])};
                    } else {
#pragma unroll
                        for (uint32_t j = 0; j < 3; ++j) {
                            if (p + j >= e.p) continue;
                            float y = v[j];
                            if (e.master) {
                                float* w = e.master + (uint64_t)q * e.p + p + j;
                                y = *w * e.keep - y * e.lr;
                                *w = y;
                            }
                            if (e.f32)
                                ((float*)e.out)[(uint64_t)q * e.out_ld + p + j] = y;
                            else
                                ((uint16_t*)e.out)[(uint64_t)q * e.out_ld + p + j] = bf16_of(y);
                        }
                    }
                }
            }
    }
};

// An XCD gets a run of consecutive tiles.
__device__ inline uint32_t run_of(uint32_t block, uint32_t n)
{
    const uint32_t each = n / kXcds, more = n % kXcds, xcd = block % kXcds;
    return xcd * each + min(xcd, more) + block / kXcds;
}

template <class S>
__global__ __launch_bounds__(S::kThreads, S::kThreads >= 512 ? 2 : 1) void gram_kernel(const MuonArgs a, bool poly)
{
    CKPT_BUFFERS(S, S);
    static_assert(S::BP == S::BQ && S::kThreads / 64 * kTurnWave <= S::kBuffer, "");
    const uint32_t t0 = run_of(blockIdx.x, gridDim.x), f = matrix_of(a, t0), t = t0 - a.m[f].first;
    const uint32_t rows = a.m[f].rows, cols = a.m[f].cols, s = min(rows, cols);
    const uint32_t ldx = up64(max(rows, cols)), lda = up64(s), ld = poly ? lda : ldx;
    // Row i of the triangle begins at tile i (i + 1) / 2.
    uint32_t i = (uint32_t)((__builtin_sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
    while (i * (i + 1) / 2 > t) --i;
    while ((i + 1) * (i + 2) / 2 <= t) ++i;
    const uint32_t j = t - i * (i + 1) / 2;
    const Operand X = {(const uint16_t*)(poly ? a.m[f].a : a.m[f].x), (uint64_t)s * ld, ld, s, ld};
    const GramEnd end = {(uint16_t*)(poly ? a.m[f].b : a.m[f].a), (const uint16_t*)a.m[f].a, (uint64_t)s * lda, s, lda,
                         a.ca, a.cb, a.cc, poly};
    product<S>(X, X, {s, s, ld, 1, false}, end, make_uint2(__builtin_amdgcn_readfirstlane(j), __builtin_amdgcn_readfirstlane(i)),
               t, 0, s0, s1, s2, s3);
}

// WIDE: [q][p] is [short][long]; else [long][short], where the last product of a tall matrix leaves it as it lies.
template <class End>
__device__ inline End apply_end(const MuonArgs& a, uint32_t f)
{
    const MuonMatrix& m = a.m[f];
    const uint32_t s = min(m.rows, m.cols), ldx = up64(max(m.rows, m.cols));
    if constexpr (std::is_same_v<End, NextEnd>)
        return {(uint16_t*)m.y, (uint64_t)s * ldx, s, ldx};
    else
        return {(float*)m.master, (void*)m.out, m.out_ld, m.cols, m.rows, a.keep, m.scale, a.out_f32};
}
template <class S, class End>
__global__ __launch_bounds__(S::kThreads, S::kThreads >= 512 ? 2 : 1) void apply_kernel(const MuonArgs a)
{
    CKPT_BUFFERS(S, S);
    constexpr bool WIDE = S::PA;
    const uint32_t t0 = run_of(blockIdx.x, gridDim.x), f = matrix_of(a, t0), t = t0 - a.m[f].first;
    const uint32_t rows = a.m[f].rows, cols = a.m[f].cols, s = min(rows, cols), l = max(rows, cols);
    const uint32_t ldx = up64(l), lda = up64(s);
    const Operand X = {(const uint16_t*)a.m[f].x, (uint64_t)s * ldx, ldx, s, ldx};
    const Operand B = {(const uint16_t*)a.m[f].b, (uint64_t)s * lda, lda, s, lda};
    const uint32_t p = WIDE ? l : s, q = WIDE ? s : l, np = (p + S::BP - 1) / S::BP, nq = (q + S::BQ - 1) / S::BQ;
    const uint32_t band = t / (kBand * np), in = t % (kBand * np), width = min(kBand, nq - band * kBand);
    const uint2 tile = make_uint2(in / width, band * kBand + in % width);
    product<S>(WIDE ? X : B, WIDE ? B : X, {p, q, lda, 1, false}, apply_end<End>(a, f), tile, t, 0, s0, s1, s2, s3);
}

// ---- shapes ----

enum Size { kSmall, kMiddle, kLarge };
constexpr uint32_t kSide[] = {64, 128, 256};

template <bool PA, bool QA>
using Large = Shape<2, 2, PA, QA, 256, 256, 4, 2, 32, 2, true>;
template <bool PA, bool QA>
using Middle = Shape<2, 2, PA, QA, 128, 128, 2, 2, 32, 2, true>;
template <bool PA, bool QA>
using Small = Shape<2, 2, PA, QA, 64, 64, 2, 1, 32, 3, true>;

uint32_t blocks(uint64_t x, uint32_t side) { return (uint32_t)((x + side - 1) / side); }
uint64_t triangle(uint64_t n) { return n * (n + 1) / 2; }

// Numbers the tiles of each matrix that `tiles` gives it, and returns all.
template <class F>
uint64_t number(MuonArgs& a, F tiles)
{
    uint64_t all = 0;
    for (uint32_t i = 0; i < a.count; ++i) {
        a.m[i].first = (uint32_t)std::min<uint64_t>(all, 0xffffffffu);
        all += tiles(a.m[i]);
    }
    a.tiles = (uint32_t)std::min<uint64_t>(all, 0xffffffffu);
    return all;
}

// The largest tiles that still give each compute unit one.
template <class F>
Size size_of(MuonArgs& a, F tiles)
{
    for (int s = kLarge; s > kSmall; --s) {
        uint64_t all = 0;
        for (uint32_t i = 0; i < a.count; ++i) all += tiles(a.m[i], kSide[s]);
        if (all >= 256) return (Size)s;
    }
    return kSmall;
}

template <class S>
hipError_t gram(const MuonArgs& a, bool poly, hipStream_t stream)
{
    if ((uint64_t)a.tiles * S::kThreads > 0xffffffffu) return hipErrorInvalidValue;
    gram_kernel<S><<<a.tiles, S::kThreads, 0, stream>>>(a, poly);
    return hipGetLastError();
}
template <class S, class End>
hipError_t apply(const MuonArgs& a, hipStream_t stream)
{
    if ((uint64_t)a.tiles * S::kThreads > 0xffffffffu) return hipErrorInvalidValue;
    apply_kernel<S, End><<<a.tiles, S::kThreads, 0, stream>>>(a);
    return hipGetLastError();
}
template <bool WIDE, class End>
hipError_t apply_sized(MuonArgs& a, hipStream_t stream)
{
    const auto tiles = [](const MuonMatrix& m, uint32_t side) {
        return (uint64_t)blocks(std::min(m.rows, m.cols), side) * blocks(std::max(m.rows, m.cols), side);
    };
    const Size size = size_of(a, tiles);
    number(a, [&](const MuonMatrix& m) { return tiles(m, kSide[size]); });
    return size == kLarge    ? apply<Large<WIDE, !WIDE>, End>(a, stream)
           : size == kMiddle ? apply<Middle<WIDE, !WIDE>, End>(a, stream)
                             : apply<Small<WIDE, !WIDE>, End>(a, stream);
}

} // namespace

hipError_t launch_muon_first(MuonArgs& a, hipStream_t stream)
{
    number(a, [](const MuonMatrix& m) { return (uint64_t)m.part_n; });
    if (a.tiles == 0 || (uint64_t)a.tiles * kThreads > 0xffffffffu) return hipErrorInvalidValue;
    if (a.in_f32)
        first_kernel<float><<<a.tiles, kThreads, 0, stream>>>(a);
    else
        first_kernel<uint16_t><<<a.tiles, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_muon_pack(MuonArgs& a, hipStream_t stream)
{
    number(a, [](const MuonMatrix& m) {
        return m.rows <= m.cols ? (uint64_t)blocks(m.rows, kMuonRows) * blocks(((uint64_t)m.cols + 63) / 64 * 64, kMuonCols)
                                : (uint64_t)blocks(m.rows, kMuonTurn) * blocks(m.cols, kMuonTurn);
    });
    if (a.tiles == 0 || (uint64_t)a.tiles * kThreads > 0xffffffffu) return hipErrorInvalidValue;
    if (a.in_f32)
        pack_kernel<float><<<a.tiles, kThreads, 0, stream>>>(a);
    else
        pack_kernel<uint16_t><<<a.tiles, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_muon_gram(MuonArgs& a, bool poly, hipStream_t stream)
{
    const auto tiles = [](const MuonMatrix& m, uint32_t side) { return triangle(blocks(std::min(m.rows, m.cols), side)); };
    const Size size = size_of(a, tiles);
    number(a, [&](const MuonMatrix& m) { return tiles(m, kSide[size]); });
    return size == kLarge    ? gram<Large<false, false>>(a, poly, stream)
           : size == kMiddle ? gram<Middle<false, false>>(a, poly, stream)
                             : gram<Small<false, false>>(a, poly, stream);
}

hipError_t launch_muon_apply(MuonArgs& a, bool last, hipStream_t stream)
{
    if (!last) return apply_sized<true, NextEnd>(a, stream);
    // Wide and tall matrices end with products of their own.
    MuonArgs some = a;
    for (const bool wide : {true, false}) {
        some.count = 0;
        for (uint32_t i = 0; i < a.count; ++i)
            if ((a.m[i].rows <= a.m[i].cols) == wide) some.m[some.count++] = a.m[i];
        if (some.count == 0) continue;
        const hipError_t e = wide ? apply_sized<true, LastEnd>(some, stream) : apply_sized<false, LastEnd>(some, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

} // namespace ckpt
