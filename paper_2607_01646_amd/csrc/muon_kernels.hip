// muon_kernels.hip -- gfx950 kernels of the orthogonalised optimizer step.
//
// A matrix's update is divided by its norm and goes `steps` times through
//   A = X X^T,  B = ca I + cb A + cc A A,  X <- B X
// with X laid out so that its rows are the shorter side; two steps are made
// from one A where that is worth it (ckpt_muon.cpp).  Large matrices are bound
// by the matrix cores (7 of 4096 x 4096 to 11008: 36 ms, 1.1 PFLOP/s on the
// planes over all launches), small ones by the launches' latencies.
//
// The operands are two planes of fp16, 22 bits, and three products of planes
// are made for each product: what is left out is 2^-22 of it (four for short
// sides up to kMuonAll, which leave nothing out).  The result is
// as far from 64 bits as with products in fp32 (1e-6 to 5e-6).  One plane
// would take a third of the time and leave it 1.3e-3 off for gradients without
// structure, 6e-3 for those of few directions (one of bf16 1e-2 and 5e-2): the
// small singular values of X grow 3.4 times a step, and what is rounded off
// beside the large ones grows with them.
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

// Values c[i] .. c[i] + 3 of rows of `cols`, zeros past their ends.  The loads are in no branch of their own, which each
// would wait for what it loads: those that would go past the end begin before it.
template <int N, class T>
__device__ inline void load_rows(const T* const (&row)[N], const uint32_t (&c)[N], uint32_t cols, f32x4 (&v)[N])
{
    if (cols < 4) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) v[i][j] = load1(row[i] + min(c[i] + j, cols - 1));
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) v[i][j] = c[i] + j < cols ? v[i][j] : 0.0f;
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = load4(row[i] + min(c[i], cols - 4));
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t by = c[i] - min(c[i], cols - 4);
        if (by & 1) v[i] = {v[i][1], v[i][2], v[i][3], 0};
        if (by & 2) v[i] = {v[i][2], v[i][3], 0, 0};
        if (by >= 4) v[i] = {0, 0, 0, 0};
    }
}

__device__ inline void store4(float* p, f32x4 x) { *(f32x4_any*)p = x; }
__device__ inline void store4(uint16_t* p, f32x4 x)
{
    *(u16x4_any*)p = u16x4{bf16_of(x[0]), bf16_of(x[1]), bf16_of(x[2]), bf16_of(x[3])};
}
__device__ inline void store1(float* p, float x) { *p = x; }
__device__ inline void store1(uint16_t* p, float x) { *p = bf16_of(x); }
template <class T>
__device__ inline void store_row(T* row, uint32_t c, uint32_t cols, f32x4 x)
{
    if (c + 4 <= cols) return store4(row + c, x);
#pragma unroll
    for (uint32_t j = 0; j < 3; ++j)
        if (c + j < cols) store1(row + c + j, x[j]);
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
template <int THREADS = kThreads>
__device__ inline double block_sum(double x, double* s_wave)
{
    x = wave_sum(x);
    if ((threadIdx.x & 63) == 0) s_wave[threadIdx.x >> 6] = x;
    __syncthreads();
    x = s_wave[0];
    for (int w = 1; w < THREADS / 64; ++w) x += s_wave[w];
    return x;
}

__device__ inline float update(const MuonArgs& a, float m, float cg)
{
    return a.nesterov ? a.beta * m + a.one_beta * cg : m;
}

// ---- the update and its norm ----
//
// Bound by HBM: gradient and momentum are read, the momentum written.  The squares' sums are in 64 bits, a tile's each.
// Few are added up by every workgroup that needs the norm; more than kMuonParts by one, in a launch of its own (11008 x
// 4096: each of 11008 workgroups would read 88 KiB).  A matrix's own number of tiles decides that.
template <class G>
__global__ __launch_bounds__(kThreads) void first_kernel(const MuonArgs a)
{
    __shared__ double s_wave[kThreads / 64];
    const uint32_t f = matrix_of(a, blockIdx.x), t = blockIdx.x - a.m[f].first;
    const uint32_t rows = a.m[f].rows, cols = a.m[f].cols, nc = (cols + kMuonCols - 1) / kMuonCols;
    const uint32_t r0 = t / nc * kMuonRows + (threadIdx.x >> 6) * 4, c = t % nc * kMuonCols + (threadIdx.x & 63) * 4;
    const uint64_t ld = a.m[f].in_ld;
    const G* in = (const G*)a.m[f].in;
    float* momentum = a.m[f].momentum;
    const float cs = a.grad_scale ? *a.grad_scale : 1.0f;
    f32x4 g[4], m[4];
    const G* from[4];
    const float* old[4];
    const uint32_t cs4[4] = {c, c, c, c};
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const uint64_t row = min(r0 + i, rows - 1);
        from[i] = in + row * ld;
        old[i] = momentum + row * cols;
    }
    if (momentum) load_rows(old, cs4, cols, m);
    load_rows(from, cs4, cols, g);
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
            store_row(momentum + (uint64_t)(r0 + i) * cols, c, cols, m[i]);
        }
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
            if (c + j < cols) sum += (double)g[i][j] * (double)g[i][j]; // (zero gradients past the end need not be zero updates)
    }
    sum = block_sum(sum, s_wave);
    if (threadIdx.x == 0) a.m[f].part[t] = sum;
}

__global__ __launch_bounds__(1024) void norm_kernel(const MuonArgs a)
{
    __shared__ double s_wave[16];
    const MuonMatrix& m = a.m[blockIdx.x];
    if (m.part_n <= kMuonParts) return;
    double sum = 0;
    for (uint32_t k = threadIdx.x; k < m.part_n; k += 1024) sum += m.part[k];
    sum = block_sum<1024>(sum, s_wave);
    if (threadIdx.x == 0) m.part[0] = sum; // every part was read before the workgroup met
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
    const float* momentum = a.m[f].momentum;
    const float cs = a.grad_scale ? *a.grad_scale : 1.0f;
    uint16_t* x = a.m[f].x;
    double sum = 0;
    const uint32_t parts = a.m[f].part_n <= kMuonParts ? a.m[f].part_n : 1;
    for (uint32_t k = threadIdx.x; k < parts; k += kThreads) sum += a.m[f].part[k];
    sum = block_sum(sum, s_wave);
    const float over = (float)((double)kUp / (sqrt(sum) + a.eps));
    // Runs of four values of U over its norm, of the rows r0, r0 + by, ..; zeros outside the matrix.
    auto values = [&](uint32_t r0, uint32_t by, uint32_t c, f32x4 (&v)[4]) {
        const G* from[4];
        const float* old[4];
        const uint32_t cs4[4] = {c, c, c, c};
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint64_t row = min(r0 + i * by, rows - 1);
            from[i] = in + row * ld;
            old[i] = momentum + row * cols;
        }
        f32x4 m[4];
        if (momentum) load_rows(old, cs4, cols, m);
        if (!momentum || a.nesterov) load_rows(from, cs4, cols, v);
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            if (momentum) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i][j] = update(a, m[i][j], cs * v[i][j]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] = r0 + i * by < rows && c + j < cols ? v[i][j] * over : 0.0f;
        }
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
        values(r0, 1, c, v);
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
    values(r0 + line, 16, c0 + at, v);
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

// Two planes of a run of 4 values of a row.
struct Planes {
    uint2 hi, lo;
    __device__ inline void load(const uint16_t* p, uint64_t plane)
    {
        hi = *(const uint2*)p;
        lo = *(const uint2*)(p + plane);
    }
    __device__ inline float at(int j) const
    {
        return (float)__builtin_bit_cast(f16x4, hi)[j] + (float)__builtin_bit_cast(f16x4, lo)[j];
    }
};

// What the lanes of this wave have written to LDS is there for its others.
__device__ inline void same_wave()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A tile of a symmetric product, out = ca I + cb C + cc P Q, and its mirror image: only the tiles on and below the diagonal
// are made, and of those only values on and below it are used.  So the result is symmetric to the last bit, and a value
// does not depend on the size of the tiles: the matrices of a call do not change each other's results.
struct TriEnd {
    uint16_t* out;
    const uint16_t* c; // or nullptr
    uint64_t plane;
    uint32_t s, ld;
    float ca, cb, cc;
};

// Where a wave turns a 32 x 32 tile: rows of p, q across.
constexpr uint32_t kTurnLd = 40, kTurnWave = 32 * kTurnLd;

template <int TP, int TQ>
struct Finish<TriEnd, TP, TQ> {
    static __device__ inline void run(const TriEnd& e, const Early<TriEnd, TQ>&, f32x16 (&acc)[TP][TQ], uint32_t p0,
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
                {
                    Planes c[4];
                    if (e.c) {
                        const uint16_t* row = e.c + (uint64_t)min(q, e.s - 1) * e.ld + ps + 4 * half;
#pragma unroll
                        for (int r = 0; r < 4; ++r) c[r].load(row + 8 * r, e.plane);
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const uint32_t p = ps + 8 * r + 4 * half;
                        f32x4 v;
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[j] = e.cc * (acc[tp][tq][4 * r + j] * kDown);
                        if (e.c) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) v[j] += e.cb * c[r].at(j) + (p + j == q ? e.ca * kUp : 0.0f);
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[j] = p + j < e.s && q < e.s ? v[j] : 0.0f;
                        split2(v, hi[r], lo[r]);
                    }
                }
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const uint2* w = z ? lo : hi;
                    uint16_t* out = e.out + z * e.plane;
                    if (ps < qs) {
                        const u16x8 a = pair_of(w[0], w[1]), b = pair_of(w[2], w[3]);
                        if (q < e.s) {
                            uint16_t* row = out + (uint64_t)q * e.ld + ps + 8 * half;
                            *(u16x8*)row = a;
                            *(u16x8*)(row + 16) = b;
                        }
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const u16x4 u = __builtin_bit_cast(u16x4, w[r]);
#pragma unroll
                            for (int j = 0; j < 4; ++j) turn[(8 * r + 4 * half + j) * kTurnLd + (lane & 31)] = u[j];
                        }
                    } else { // on the diagonal: below it, and its image
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const u16x4 u = __builtin_bit_cast(u16x4, w[r]);
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const uint32_t p = 8 * r + 4 * half + j;
                                if (p <= (lane & 31)) turn[p * kTurnLd + (lane & 31)] = turn[(lane & 31) * kTurnLd + p] = u[j];
                            }
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
                const uint32_t ps = p0 + 32 * tp, q = q0 + 32 * tq + (lane & 31), p = ps + 4 * half;
                f32x4 v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[r][j] = acc[tp][tq][4 * r + j] * (kDown * kDown);
                if (q >= e.q || ps >= e.p) continue;
                float* w = e.master ? e.master + (uint64_t)q * e.p + p : nullptr;
                const uint64_t to = (uint64_t)q * e.out_ld + p;
                if (ps + 32 <= e.p) {
                    if (w) {
                        f32x4 old[4];
#pragma unroll
                        for (int r = 0; r < 4; ++r) old[r] = load4(w + 8 * r);
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            v[r] = old[r] * e.keep - v[r] * e.lr;
                            store4(w + 8 * r, v[r]);
                        }
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (e.f32)
                            store4((float*)e.out + to + 8 * r, v[r]);
                        else
                            store4((uint16_t*)e.out + to + 8 * r, v[r]);
                    continue;
                }
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j) {
                        if (p + 8 * r + j >= e.p) continue;
                        float y = v[r][j];
                        if (w) {
                            y = w[8 * r + j] * e.keep - y * e.lr;
                            w[8 * r + j] = y;
                        }
                        if (e.f32)
                            ((float*)e.out)[to + 8 * r + j] = y;
                        else
                            ((uint16_t*)e.out)[to + 8 * r + j] = bf16_of(y);
                    }
            }
    }
};

// Workgroups go round the XCDs, each with an L2 of its own.  Where all tiles take the same time an XCD gets a run of them,
// so that it reads few matrices (A of 7 of 1024 x 8192, tiles of 128: 187 us,
// with shares 331); else it gets a share of each
// matrix, a run too, and the longest first: a run of all would leave it only long ones or only short ones.
// shares: the workgroups of a matrix are a multiple of 8 and begin at one.
__device__ inline uint32_t run_begin(uint32_t n, uint32_t xcd) { return xcd * (n / kXcds) + min(xcd, n % kXcds); }
__device__ inline uint32_t nth_tile(bool shares, uint32_t n) // of n in all
{
    return shares ? blockIdx.x : run_begin(n, blockIdx.x % kXcds) + blockIdx.x / kXcds;
}
__device__ inline bool tile_in(bool shares, uint32_t at, uint32_t n, uint32_t& tile) // at-th of a matrix's n
{
    tile = at;
    if (!shares) return true;
    const uint32_t xcd = at % kXcds;
    tile = run_begin(n, xcd) + at / kXcds;
    return tile < run_begin(n, xcd + 1);
}

template <class S>
__global__ __launch_bounds__(S::kThreads, S::kThreads >= 512 ? 2 : 1) void tri_kernel(const TriArgs a)
{
    CKPT_BUFFERS(S, S);
    static_assert(S::BQ % S::BP == 0 && S::kThreads / 64 * kTurnWave <= S::kBuffer, "");
    const uint32_t lane = threadIdx.x & 63;
    const uint32_t at = nth_tile(a.shares, gridDim.x);
    const uint64_t before = __ballot(lane < a.count && a.m[lane < kMuonMats ? lane : 0].first <= at);
    const TriMatrix m = a.m[__builtin_amdgcn_readfirstlane(63 - __builtin_clzll(before))];
    // Row i of the triangle, of BQ values of q, has kWide tiles more than the one before it.
    constexpr uint32_t kWide = S::BQ / S::BP;
    const uint32_t n = (m.s + S::BQ - 1) / S::BQ;
    uint32_t t;
    if (!tile_in(a.shares, at - m.first, kWide * (n * (n + 1) / 2), t)) return;
    uint32_t i = (uint32_t)((__builtin_sqrtf(8.0f * (t / kWide) + 1.0f) - 1.0f) * 0.5f);
    while (kWide * (i * (i + 1) / 2) > t) --i;
    while (kWide * ((i + 1) * (i + 2) / 2) <= t) ++i;
    const uint32_t j = t - kWide * (i * (i + 1) / 2);
    if (j * S::BP >= m.s) return; // past the matrix: its last row of tiles may be less than half full
    const Operand P = {m.p, (uint64_t)m.s * m.k, m.k, m.s, m.k};
    const Operand Q = {m.q, (uint64_t)m.s * m.k, m.k, m.s, m.k};
    const uint32_t ld = up64(m.s);
    const TriEnd end = {m.out, m.c, (uint64_t)m.s * ld, m.s, ld, a.ca, a.cb, a.cc};
    product<S>(P, Q, {m.s, m.s, m.k, 1, false}, end, make_uint2(__builtin_amdgcn_readfirstlane(j), __builtin_amdgcn_readfirstlane(i)),
               t, 0, s0, s1, s2, s3, m.chunk);
}

// Few rows that are long have few tiles, and a tile's workgroup goes through all of k (X X^T of 64 x 8192: 60 us).  Here each
// chunk of k has a workgroup, and join_kernel adds up what they leave in the order of tri_kernel's own sums: the bits are the
// same, whichever way a call goes.  All five steps of 64 x 8192 356 -> 120 us, of 448 x 8192 439 -> 251, of 17 x 100000 3310 ->
// 238; launch_muon_tri estimates both ways.
struct PartEnd {
    float* out;
    uint32_t s, ld;
};
template <int TP, int TQ>
struct Finish<PartEnd, TP, TQ> {
    static __device__ inline void run(const PartEnd& e, const Early<PartEnd, TQ>&, f32x16 (&acc)[TP][TQ], uint32_t p0,
                                      uint32_t q0, uint32_t, uint16_t*)
    {
        const uint32_t lane = threadIdx.x & 63, half = lane >> 5;
#pragma unroll
        for (int tq = 0; tq < TQ; ++tq)
#pragma unroll
            for (int tp = 0; tp < TP; ++tp)
#pragma unroll
                for (uint32_t r = 0; r < 4; ++r) {
                    const uint32_t p = p0 + 32 * tp + 8 * r + 4 * half, q = q0 + 32 * tq + (lane & 31);
                    if (p > q || q >= e.s) continue;
                    f32x4 v;
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = acc[tp][tq][4 * r + j];
                    *(f32x4*)(e.out + (uint64_t)q * e.ld + p) = v;
                }
    }
};

template <class S>
__global__ __launch_bounds__(S::kThreads) void slices_kernel(const TriArgs a)
{
    CKPT_BUFFERS(S, S);
    static_assert(S::BQ == S::BP, "");
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t before = __ballot(lane < a.count && a.m[lane < kMuonMats ? lane : 0].first <= blockIdx.x);
    const TriMatrix m = a.m[__builtin_amdgcn_readfirstlane(63 - __builtin_clzll(before))];
    const uint32_t at = blockIdx.x - m.first, slice = at % m.slices, t = at / m.slices;
    uint32_t i = (uint32_t)((__builtin_sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
    while (i * (i + 1) / 2 > t) --i;
    while ((i + 1) * (i + 2) / 2 <= t) ++i;
    const uint32_t j = t - i * (i + 1) / 2, k0 = slice * m.chunk, k = m.slices > 1 ? min(m.chunk, m.k - k0) : m.k;
    const Operand X = {m.p + k0, (uint64_t)m.s * m.k, m.k, m.s, k};
    const uint32_t ld = (m.s + 3) / 4 * 4;
    const PartEnd end = {m.part + (uint64_t)slice * m.s * ld, m.s, ld};
    product<S>(X, X, {m.s, m.s, k, 1, false}, end, make_uint2(__builtin_amdgcn_readfirstlane(j), __builtin_amdgcn_readfirstlane(i)),
               t, 0, s0, s1, s2, s3, m.chunk);
}

__global__ __launch_bounds__(kThreads) void join_kernel(const TriArgs a)
{
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t before = __ballot(lane < a.count && a.m[lane < kMuonMats ? lane : 0].first <= blockIdx.x);
    const TriMatrix m = a.m[__builtin_amdgcn_readfirstlane(63 - __builtin_clzll(before))];
    const uint32_t s = m.s, ld = up64(s), part_ld = (s + 3) / 4 * 4, at = (blockIdx.x - m.first) * kThreads + threadIdx.x;
    const uint32_t q = at / (ld / 4), p = at % (ld / 4) * 4; // 4 values of p, up to the diagonal
    if (q >= s || (p > q && p + 4 <= s)) return;
    f32x4 v = {0, 0, 0, 0};
    if (p <= q) {
        const float* part = m.part + (uint64_t)q * part_ld + p;
#pragma unroll 8
        for (uint32_t k = 0; k < m.slices; ++k) v += *(const f32x4*)(part + (uint64_t)k * s * part_ld);
    }
    v = a.cc * (v * kDown);
    uint2 hi, lo;
    split2(v, hi, lo);
    const uint64_t plane = (uint64_t)s * ld;
#pragma unroll
    for (int z = 0; z < 2; ++z) {
        const u16x4 u = __builtin_bit_cast(u16x4, z ? lo : hi);
        uint16_t* out = m.out + z * plane;
        if (p + 3 <= q || p >= s) *(u16x4*)(out + (uint64_t)q * ld + p) = u;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            if (p + j <= q) out[(uint64_t)q * ld + p + j] = out[(uint64_t)(p + j) * ld + q] = u[j];
            else if (p + j >= s) out[(uint64_t)q * ld + p + j] = 0;
        }
    }
}

// [q][p] is [short][long]; for the last X of a tall matrix [long][short], as it lies.  W: the shape of the one, T: of the other.
template <class W, class T, class End>
__global__ __launch_bounds__(W::kThreads, W::kThreads >= 512 ? 2 : 1) void apply_kernel(const MuonArgs a)
{
    CKPT_BUFFERS(W, T);
    const uint32_t at = nth_tile(a.shares, gridDim.x);
    const MuonMatrix& m = a.m[matrix_of(a, at)];
    const uint32_t s = min(m.rows, m.cols), l = max(m.rows, m.cols), ldx = up64(l), lda = up64(s);
    const bool wide = std::is_same_v<End, NextEnd> || m.rows <= m.cols;
    static_assert(W::BP == T::BP && W::BQ == T::BQ, "");
    const uint32_t p = wide ? l : s, q = wide ? s : l, np = (p + W::BP - 1) / W::BP, nq = (q + W::BQ - 1) / W::BQ;
    uint32_t t;
    if (!tile_in(a.shares, at - m.first, np * nq, t)) return;
    const uint32_t chunk = muon_chunk(lda, false);
    const uint32_t band = t / (kBand * np), in = t % (kBand * np), width = min(kBand, nq - band * kBand);
    const uint2 tile = make_uint2(in / width, band * kBand + in % width);
    const Operand X = {m.x, (uint64_t)s * ldx, ldx, s, ldx};
    const Operand B = {m.f, (uint64_t)s * lda, lda, s, lda};
    if constexpr (std::is_same_v<End, NextEnd>) {
        const NextEnd end = {m.y, (uint64_t)s * ldx, s, ldx};
        product<W>(X, B, {p, q, lda, 1, false}, end, tile, t, 0, s0, s1, s2, s3, chunk);
    } else {
        const LastEnd end = {m.master, m.out, m.out_ld, p, q, a.keep, m.scale, a.out_f32};
        if (wide)
            product<W>(X, B, {p, q, lda, 1, false}, end, tile, t, 0, s0, s1, s2, s3, chunk);
        else
            product<T>(B, X, {p, q, lda, 1, false}, end, tile, t, 0, s0, s1, s2, s3, chunk);
    }
}

// ---- thin matrices ----
//
// Short sides up to 16: all steps are polynomials of one Gram matrix, G = U U^T, which is so small that it is kept in 64
// bits: a launch makes it, one goes through the steps (A <- B A B, F <- B F) and the last makes X = F U.  Few terms do not
// average the roundings of 22 bits (2 x 1033: 1.6e-6 off with planes, 5e-7 with products in fp32), and five steps from one
// Gram matrix, which in fewer bits are not stable, are so in 64 (fits_thin in ckpt_muon.cpp).  Bound by the launches'
// latencies (2 x 1033: 14 us, by planes 114), of long rows by the sums from LDS (16 x 1048576: 136 us for 192 MB read and
// written; its transpose, whose lanes read rows of their own, 213).
constexpr uint32_t kThinLd = kThreads + 4; // of LDS rows: 16 bytes further apart than a power of two

// The update's s values at `at` of the long side; KEEP: the momentum's new ones are stored, else they are.
template <class G, bool KEEP>
__device__ inline void thin_values(const MuonArgs& a, const MuonMatrix& m, bool wide, uint32_t s, uint32_t at, float (&u)[kThin])
{
    const float cs = a.grad_scale ? *a.grad_scale : 1.0f;
    float old[kThin];
    const uint64_t in_step = wide ? m.in_ld : 1, step = wide ? m.cols : 1;
    const G* in = (const G*)m.in + (wide ? at : at * m.in_ld);
    float* momentum = m.momentum + (wide ? at : (uint64_t)at * m.cols);
#pragma unroll
    for (uint32_t i = 0; i < kThin; ++i) u[i] = load1(in + min(i, s - 1) * in_step);
    if (m.momentum) {
#pragma unroll
        for (uint32_t i = 0; i < kThin; ++i) old[i] = momentum[min(i, s - 1) * step];
#pragma unroll
        for (uint32_t i = 0; i < kThin; ++i) {
            const float cg = cs * u[i];
            if (KEEP) {
                old[i] = a.beta * old[i] + a.one_beta * cg;
                if (i < s) momentum[i * step] = old[i];
            }
            u[i] = update(a, old[i], cg);
        }
    }
#pragma unroll
    for (uint32_t i = 0; i < kThin; ++i) u[i] = i < s ? u[i] : 0.0f;
}

// Momentum, and a workgroup's share of G: part_n shares of runs of 256 places of the long side.  A thread sums one element of
// G over as many of a run's places as G's side, to a power of two, has elements.
template <class G>
__global__ __launch_bounds__(kThreads) void thin_gram_kernel(const MuonArgs a)
{
    __shared__ __attribute__((aligned(16))) float s_u[kThin][kThinLd];
    const uint32_t f = matrix_of(a, blockIdx.x), t = blockIdx.x - a.m[f].first;
    const MuonMatrix& m = a.m[f];
    const bool wide = m.rows <= m.cols;
    const uint32_t s = min(m.rows, m.cols), l = max(m.rows, m.cols), runs = (l + kThreads - 1) / kThreads;
    const uint32_t log2 = s > 1 ? 32 - __clz(s - 1) : 0, pair = threadIdx.x & ((1u << 2 * log2) - 1);
    const uint32_t i = pair >> log2, j = pair & ((1u << log2) - 1), k0 = threadIdx.x - pair, span = 1u << 2 * log2;
    double sum = 0;
    for (uint32_t run = t; run < runs; run += m.part_n) {
        const uint32_t at = run * kThreads + threadIdx.x;
        float u[kThin];
        if (at < l) thin_values<G, true>(a, m, wide, s, at, u);
#pragma unroll
        for (uint32_t k = 0; k < kThin; ++k) s_u[k][threadIdx.x] = at < l ? u[k] : 0.0f;
        __syncthreads();
        if (s == 1) {
            sum += (double)s_u[0][threadIdx.x] * (double)s_u[0][threadIdx.x];
        } else if (i < s && j <= i) {
            for (uint32_t k = k0; k < k0 + span; k += 4) {
                const f32x4 x = *(const f32x4*)&s_u[i][k], y = *(const f32x4*)&s_u[j][k];
#pragma unroll
                for (int v = 0; v < 4; ++v) sum += (double)x[v] * (double)y[v];
            }
        }
        __syncthreads();
    }
    double* s_sum = (double*)s_u;
    s_sum[threadIdx.x] = sum;
    __syncthreads();
    for (uint32_t n = kThreads / 2; n >= span; n /= 2) {
        if (threadIdx.x < n) s_sum[threadIdx.x] += s_sum[threadIdx.x + n];
        __syncthreads();
    }
    // Elements behind the s-th, and above the diagonal, are not read (thin_steps_kernel).
    if (threadIdx.x < span && i < s) m.part[(uint64_t)t * kThreads + i * kThin + j] = s_sum[threadIdx.x];
}

// All steps of a matrix by one workgroup, an element a thread: F over the norm, where X would be.
__global__ __launch_bounds__(kThreads) void thin_steps_kernel(const MuonArgs a, const MuonPolynomial n)
{
    __shared__ double s_a[kThin][kThin + 1], s_b[kThin][kThin + 1], s_f[kThin][kThin + 1], s_t[kThin][kThin + 1];
    const MuonMatrix& m = a.m[blockIdx.x];
    const uint32_t s = min(m.rows, m.cols);
    const uint32_t i = threadIdx.x / kThin, j = threadIdx.x % kThin;
    double g = 0;
    if (max(i, j) < s) {
#pragma unroll 8
        for (uint32_t t = 0; t < m.part_n; ++t) g += m.part[(uint64_t)t * kThreads + max(i, j) * kThin + min(i, j)];
    }
    s_a[i][j] = g;
    __syncthreads();
    double squares = 0;
    for (uint32_t k = 0; k < s; ++k) squares += s_a[k][k];
    __syncthreads();
    const double norm = sqrt(squares) + a.eps;
    double x = s_a[i][j] = g / norm / norm, f = i == j ? 1 / norm : 0;
    s_f[i][j] = f;
    __syncthreads();
    const auto product = [&](const double (&p)[kThin][kThin + 1], const double (&q)[kThin][kThin + 1]) {
        double sum = 0;
        for (uint32_t k = 0; k < s; ++k) sum += p[i][k] * q[k][j];
        return sum;
    };
    for (uint32_t step = 0; step < n.steps; ++step) {
        s_b[i][j] = (i == j ? n.ca : 0.0) + n.cb * x + n.cc * product(s_a, s_a);
        __syncthreads();
        f = product(s_b, s_f);
        s_t[i][j] = product(s_b, s_a);
        __syncthreads();
        s_f[i][j] = f;
        x = s_a[i][j] = product(s_t, s_b);
        __syncthreads();
    }
    ((double*)m.x)[threadIdx.x] = f;
}

template <class G>
__global__ __launch_bounds__(kThreads) void thin_apply_kernel(const MuonArgs a)
{
    __shared__ double s_f[kThin][kThin];
    const uint32_t index = matrix_of(a, blockIdx.x), t = blockIdx.x - a.m[index].first;
    const MuonMatrix& m = a.m[index];
    const bool wide = m.rows <= m.cols;
    const uint32_t s = min(m.rows, m.cols), l = max(m.rows, m.cols), at = t * kThreads + threadIdx.x;
    s_f[threadIdx.x / kThin][threadIdx.x % kThin] = ((const double*)m.x)[threadIdx.x];
    __syncthreads();
    if (at >= l) return;
    float u[kThin];
    thin_values<G, false>(a, m, wide, s, at, u);
    for (uint32_t i = 0; i < s; ++i) {
        double sum = 0;
#pragma unroll
        for (uint32_t k = 0; k < kThin; ++k) sum += s_f[i][k] * (double)u[k];
        const uint64_t row = wide ? i : at, col = wide ? at : i;
        float y = (float)sum;
        if (m.master) {
            float* w = m.master + row * m.cols + col;
            y = *w * a.keep - y * m.scale;
            *w = y;
        }
        if (a.out_f32)
            ((float*)m.out)[row * m.out_ld + col] = y;
        else
            ((uint16_t*)m.out)[row * m.out_ld + col] = bf16_of(y);
    }
}

// ---- small matrices ----
//
// Up to 64 x 256: a workgroup makes all of a matrix's step, X, A and B in LDS, in the time that the launches' latencies
// would take many times over (4 matrices of 64 x 64 to 256: 36 us, 112 by the kernels above).  The same sums of the same
// operands, but step by step.  X is padded with zeros to 64 rows and 256 columns; rows lie 16 bytes further
// apart than they are long, which spreads the 16 rows that a quarter of a wave reads over the banks.
constexpr int kTinyThreads = 512, kTinyX = kTinyLong + 8, kTinyA = kTinyShort + 8;

// Products of 16 x 16 x 32: there are tiles enough for each wave to have several sums on their way.
// The lane's 8 values of rows [r0, r0 + 16), k [k0, k0 + 32): row lane % 16, k 8 (lane / 16) + 0..7.
__device__ inline f16x8 row_part(const uint16_t* m, uint32_t ld, uint32_t r0, uint32_t k0)
{
    const uint32_t lane = threadIdx.x & 63;
    return *(const f16x8*)(m + (r0 + (lane & 15)) * ld + k0 + 8 * (lane >> 4));
}
// The same of columns [c0, c0 + 16), k down the rows: 16 lanes name 4 rows of 16 values and each receives a column of them.
__device__ inline f16x8 column_part(const uint16_t* m, uint32_t ld, uint32_t c0, uint32_t k0)
{
    typedef __attribute__((address_space(3))) i16x4* Ptr;
    const uint32_t lane = threadIdx.x & 63;
    i16x4 h[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const uint32_t k = k0 + 8 * (lane >> 4) + 4 * u + ((lane >> 2) & 3);
        h[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(m + k * ld + c0 + 4 * (lane & 3)));
    }
    return __builtin_bit_cast(f16x8, __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
}
// out[q][p]: q = lane % 16, p = 4 (lane / 16) + 0..3.
__device__ inline void multiply2(f32x4& acc, const f16x8 (&p)[2], const f16x8 (&q)[2])
{
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[1], q[1], acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[0], q[1], acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[1], q[0], acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[0], q[0], acc, 0, 0, 0);
}

template <class G>
__global__ __launch_bounds__(kTinyThreads) void tiny_kernel(const MuonArgs a, const MuonPolynomial n)
{
    constexpr uint32_t kXPlane = kTinyShort * kTinyX, kAPlane = kTinyShort * kTinyA;
    __shared__ __attribute__((aligned(16))) uint16_t s_x[2 * kXPlane], s_a[2 * kAPlane], s_b[2 * kAPlane];
    __shared__ double s_wave[kTinyThreads / 64];
    const MuonMatrix& m = a.m[blockIdx.x];
    const uint32_t rows = m.rows, cols = m.cols, l64 = up64(max(rows, cols));
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool wide = rows <= cols;

    // The update, in registers until its norm is known.
    constexpr uint32_t kMost = kTinyShort * kTinyLong / 4 / kTinyThreads;
    const uint32_t in_row = (cols + 3) / 4, all = rows * in_row;
    const G* in = (const G*)m.in;
    float* momentum = m.momentum;
    const float cs = a.grad_scale ? *a.grad_scale : 1.0f;
    f32x4 g[kMost], u[kMost];
    uint32_t row[kMost], col[kMost];
    {
        const G* from[kMost];
        const float* old[kMost];
#pragma unroll
        for (uint32_t i = 0; i < kMost; ++i) {
            const uint32_t at = min(i * kTinyThreads + threadIdx.x, all - 1);
            row[i] = at / in_row;
            col[i] = at % in_row * 4;
            from[i] = in + row[i] * m.in_ld;
            old[i] = momentum + row[i] * cols;
        }
        if (momentum) load_rows(old, col, cols, u);
        load_rows(from, col, cols, g);
    }
    for (uint32_t k = threadIdx.x; k < 2 * kXPlane / 8; k += kTinyThreads) ((uint4*)s_x)[k] = make_uint4(0, 0, 0, 0);
    double sum = 0;
#pragma unroll
    for (uint32_t i = 0; i < kMost; ++i) {
        if (i * kTinyThreads + threadIdx.x >= all) continue;
        const uint32_t c = col[i];
        if (momentum) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float cg = cs * g[i][j];
                u[i][j] = a.beta * u[i][j] + a.one_beta * cg;
                g[i][j] = update(a, u[i][j], cg);
            }
            store_row(momentum + row[i] * cols, c, cols, u[i]);
        }
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            if (c + j >= cols) g[i][j] = 0;
            sum += (double)g[i][j] * (double)g[i][j];
        }
    }
    sum = block_sum<kTinyThreads>(sum, s_wave); // and the zeros are there
    const float over = (float)((double)kUp / (sqrt(sum) + a.eps));
#pragma unroll
    for (uint32_t i = 0; i < kMost; ++i) {
        if (i * kTinyThreads + threadIdx.x >= all) continue;
        const uint32_t c = col[i];
        uint2 hi, lo;
        split2(g[i] * over, hi, lo);
        if (wide) {
            *(uint2*)(s_x + row[i] * kTinyX + c) = hi;
            *(uint2*)(s_x + kXPlane + row[i] * kTinyX + c) = lo;
        } else {
            const u16x4 h = __builtin_bit_cast(u16x4, hi), l = __builtin_bit_cast(u16x4, lo);
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                if (c + j >= cols) continue;
                s_x[(c + j) * kTinyX + row[i]] = h[j];
                s_x[kXPlane + (c + j) * kTinyX + row[i]] = l[j];
            }
        }
    }
    __syncthreads();

    const float ca = (float)n.ca, cb = (float)n.cb, cc = (float)n.cc;
    // P P^T: two tiles a wave, of the same q.
    auto square = [&](const uint16_t* p, uint32_t ld, uint32_t plane, uint32_t k, const uint16_t* c, uint16_t* out) {
        const uint32_t q0 = 16 * (wave >> 1), p0 = 32 * (wave & 1), q = q0 + (lane & 15), p1 = p0 + 4 * (lane >> 4);
        f32x4 acc[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
        for (uint32_t k0 = 0; k0 < k; k0 += 64) {
            f16x8 y[2][2], x[2][2][2];
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h)
#pragma unroll
                for (uint32_t z = 0; z < 2; ++z) {
                    y[h][z] = row_part(p + z * plane, ld, q0, k0 + 32 * h);
                    x[h][0][z] = row_part(p + z * plane, ld, p0, k0 + 32 * h);
                    x[h][1][z] = row_part(p + z * plane, ld, p0 + 16, k0 + 32 * h);
                }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                multiply2(acc[0], x[h][0], y[h]);
                multiply2(acc[1], x[h][1], y[h]);
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint32_t at = q * kTinyA + p1 + 16 * t;
            f32x4 v = acc[t] * kDown;
            if (c) {
                Planes old;
                old.load(c + at, kAPlane);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = cc * v[j] + cb * old.at(j) + (p1 + 16 * t + j == q ? ca * kUp : 0.0f);
            }
            uint2 hi, lo;
            split2(v, hi, lo);
            *(uint2*)(out + at) = hi;
            *(uint2*)(out + kAPlane + at) = lo;
        }
        __syncthreads();
    };
    // B X: a wave has 32 columns of X (those past the matrix are zeros), which it reads once: two strips of 16, 4 tiles each.
    constexpr int kTiles = 8;
    static_assert(kTinyShort == 64 && kTinyLong == 32 * (kTinyThreads / 64), "");
    f32x4 acc[kTiles];
    auto i0 = [](int t) { return 16u * (t & 3); };
    auto j0 = [&](int t) { return 32 * wave + 16 * (t >> 2); };
    auto apply = [&](auto turned) { // turned: [q][p] is [long][short]
#pragma unroll
        for (int t = 0; t < kTiles; ++t) acc[t] = {0, 0, 0, 0};
#pragma unroll
        for (uint32_t k0 = 0; k0 < kTinyShort; k0 += 32) {
            f16x8 x[2][2], b[4][2];
#pragma unroll
            for (int z = 0; z < 2; ++z) {
#pragma unroll
                for (int t = 0; t < 2; ++t) x[t][z] = column_part(s_x + z * kXPlane, kTinyX, j0(4 * t), k0);
#pragma unroll
                for (int t = 0; t < 4; ++t) b[t][z] = row_part(s_b + z * kAPlane, kTinyA, i0(t), k0);
            }
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                if constexpr (turned)
                    multiply2(acc[t], b[t & 3], x[t >> 2]);
                else
                    multiply2(acc[t], x[t >> 2], b[t & 3]);
            }
        }
    };
    const bool mine = 32 * wave < l64; // the wave's columns are not all zeros
    for (uint32_t step = 0;; ++step) {
        square(s_x, kTinyX, kXPlane, l64, nullptr, s_a);
        square(s_a, kTinyA, kAPlane, kTinyShort, s_a, s_b);
        if (step + 1 == n.steps) break;
        if (mine) apply(std::false_type());
        __syncthreads();
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            if (!mine) break;
            uint2 hi, lo;
            split2(acc[t] * kDown, hi, lo);
            uint16_t* to = s_x + (i0(t) + (lane & 15)) * kTinyX + j0(t) + 4 * (lane >> 4);
            *(uint2*)to = hi;
            *(uint2*)(to + kXPlane) = lo;
        }
        __syncthreads();
    }
    if (!mine) return;
    // The last as the matrix lies, in runs of 4 values of its rows.
    uint32_t r[kTiles], c[kTiles];
    const float* w[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        r[t] = (wide ? i0(t) : j0(t)) + (lane & 15);
        c[t] = (wide ? j0(t) : i0(t)) + 4 * (lane >> 4);
        w[t] = m.master + min(r[t], rows - 1) * cols;
    }
    f32x4 old[kTiles];
    if (m.master) load_rows(w, c, cols, old);
    if (wide)
        apply(std::false_type());
    else
        apply(std::true_type());
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        if (r[t] >= rows || c[t] >= cols) continue;
        f32x4 v = acc[t] * (kDown * kDown);
        if (m.master) {
            v = old[t] * a.keep - v * m.scale;
            store_row(m.master + r[t] * cols, c[t], cols, v);
        }
        if (a.out_f32)
            store_row((float*)m.out + r[t] * m.out_ld, c[t], cols, v);
        else
            store_row((uint16_t*)m.out + r[t] * m.out_ld, c[t], cols, v);
    }
}

// ---- shapes ----

// Workgroup tiles, and what a step of 64 values of k takes one of them (us) where each compute unit has one; for its first
// loads and its end each takes some us more.  One workgroup a unit.
//   256 x 256, 8 waves of 64 x 128: 1.33 PFLOP/s on the planes while all units are busy; no registers for sums in parts
//   128 x 256, 8 waves of 64 x 64: 1.17
//   128 x 128, 8 waves of 64 x 32: 1.0; the quickest where there are no more tiles than units (A of 2048 x 8192: 126 us;
//              by 4 waves, two workgroups a unit, 173)
//   64 x 64,   4 waves of 32 x 32, for few tiles and short k; three buffers, as its loads come from other XCDs' writes (a
//              matrix of 777 x 1003: 202 us, with two 239)
enum Size { kSmall, kMiddle, kWide, kLarge };
constexpr struct {
    uint32_t p, q;
    double few, many, end; // us a step with up to 128 tiles, and with 256 and more; us a tile
} kTile[] = {{64, 64, 0.48, 0.56, 4}, {128, 128, 1.05, 1.75, 6}, {128, 256, 1.9, 2.75, 8}, {256, 256, 3.4, 4.9, 10}};

constexpr double kJoin = 6; // us of join_kernel

template <bool PA, bool QA>
using Large = Shape<2, 2, PA, QA, 256, 256, 4, 2, 32, 2, true>;
template <bool PA, bool QA>
using Wide = Shape<2, 2, PA, QA, 128, 256, 2, 4, 32, 3, true, true>;
template <bool PA, bool QA, bool ALL>
using Middle = Shape<2, 2, PA, QA, 128, 128, 2, 4, 64, 2, true, true, ALL>;
template <bool PA, bool QA, bool ALL>
using Small = Shape<2, 2, PA, QA, 64, 64, 2, 2, 64, 3, true, true, ALL>;

uint64_t blocks(uint64_t x, uint32_t side) { return (x + side - 1) / side; }

// Numbers the tiles of each matrix that `tiles` gives it, `round` of them at a time, and returns all.
template <class A, class F>
uint64_t number(A& a, uint32_t round, F tiles)
{
    uint64_t all = 0;
    for (uint32_t i = 0; i < a.count; ++i) {
        a.m[i].first = (uint32_t)std::min<uint64_t>(all, 0xffffffffu);
        all += (tiles(a.m[i]) + round - 1) / round * round;
    }
    return all;
}

// The size of tiles that is done first, of products that have `tiles(m, size)` with `steps(m)` of 64 values of k each, the
// longest first; `parts`: some have sums in parts.
template <class A, class T, class K>
Size size_of(const A& a, bool parts, T tiles, K steps, double* time = nullptr)
{
    Size best = kSmall;
    double least = 1e30;
    for (int z = kSmall; z <= kLarge; ++z) {
        if ((z == kLarge && parts) || (z > kMiddle && a.all)) continue;
        const auto& c = kTile[z];
        uint64_t all = 0, work = 0;
        for (uint32_t i = 0; i < a.count; ++i) {
            const uint64_t n = tiles(a.m[i], (Size)z);
            all += n;
            work += n * steps(a.m[i]);
        }
        const double most = (double)steps(a.m[0]), mean = (double)work / (double)all;
        const uint64_t rounds = all / 256, left = all % 256;
        const auto step = [&](uint64_t n) { return n <= 128 ? c.few : c.few + (c.many - c.few) * (double)(std::min<uint64_t>(n, 256) - 128) / 128; };
        double t = (double)rounds * (mean * c.many + c.end);
        if (left) t += mean * step(rounds ? left : all) + c.end;
        t = std::max(t, most * step(all) + c.end);
        if (t < least) least = t, best = (Size)z;
    }
    if (time) *time = least;
    return best;
}

template <class K>
hipError_t launch_tiles(K kernel, const void* args, uint64_t tiles, uint32_t threads, hipStream_t stream)
{
    if (tiles == 0 || tiles * threads > 0xffffffffu) return hipErrorInvalidValue;
    void* list[] = {const_cast<void*>(args)};
    return hipLaunchKernel((const void*)kernel, dim3((uint32_t)tiles), dim3(threads), list, 0, stream);
}

template <class End>
hipError_t apply(MuonArgs& a, hipStream_t stream)
{
    constexpr bool kNext = std::is_same_v<End, NextEnd>;
    const auto tiles = [](const MuonMatrix& m, Size z) {
        const bool wide = kNext || m.rows <= m.cols;
        const uint32_t s = std::min(m.rows, m.cols), l = std::max(m.rows, m.cols);
        return blocks(wide ? l : s, kTile[z].p) * blocks(wide ? s : l, kTile[z].q);
    };
    const auto steps = [](const MuonMatrix& m) { return blocks(std::min(m.rows, m.cols), 64); };
    std::stable_sort(a.m, a.m + a.count, [&](const MuonMatrix& x, const MuonMatrix& y) { return steps(x) > steps(y); });
    bool parts = false;
    for (uint32_t i = 0; i < a.count; ++i) parts |= muon_chunk((uint32_t)steps(a.m[i]) * 64, false) != 0;
    const Size size = size_of(a, parts, tiles, steps);
    a.shares = steps(a.m[0]) != steps(a.m[a.count - 1]);
    const uint64_t all = number(a, a.shares ? kXcds : 1, [&](const MuonMatrix& m) { return tiles(m, size); });
    const auto launch = [&](auto wide, auto turned) { // the shape of wide matrices, and of tall ones' last X
        using W = decltype(wide);
        using T = std::conditional_t<kNext, W, decltype(turned)>;
        return launch_tiles(apply_kernel<W, T, End>, &a, all, W::kThreads, stream);
    };
    return size == kLarge    ? launch(Large<true, false>(), Large<false, true>())
           : size == kWide   ? launch(Wide<true, false>(), Wide<false, true>())
           : size == kMiddle ? (a.all ? launch(Middle<true, false, true>(), Middle<false, true, true>())
                                      : launch(Middle<true, false, false>(), Middle<false, true, false>()))
           : a.all           ? launch(Small<true, false, true>(), Small<false, true, true>())
                             : launch(Small<true, false, false>(), Small<false, true, false>());
}

} // namespace

hipError_t launch_muon_first(MuonArgs& a, hipStream_t stream)
{
    const uint64_t tiles = number(a, 1, [](const MuonMatrix& m) { return (uint64_t)m.part_n; });
    return a.in_f32 ? launch_tiles(first_kernel<float>, &a, tiles, kThreads, stream)
                    : launch_tiles(first_kernel<uint16_t>, &a, tiles, kThreads, stream);
}

hipError_t launch_muon_tiny(const MuonArgs& a, const MuonPolynomial& n, hipStream_t stream)
{
    if (a.count == 0 || a.count > kMuonMats) return hipErrorInvalidValue;
    if (a.in_f32)
        tiny_kernel<float><<<a.count, kTinyThreads, 0, stream>>>(a, n);
    else
        tiny_kernel<uint16_t><<<a.count, kTinyThreads, 0, stream>>>(a, n);
    return hipGetLastError();
}

static hipError_t launch_norms(const MuonArgs& a, hipStream_t stream)
{
    bool many = false;
    for (uint32_t i = 0; i < a.count; ++i) many |= a.m[i].part_n > kMuonParts;
    if (!many) return hipSuccess;
    norm_kernel<<<a.count, 1024, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_muon_thin(MuonArgs& a, const MuonPolynomial& n, hipStream_t stream)
{
    const uint64_t parts = number(a, 1, [](const MuonMatrix& m) { return (uint64_t)m.part_n; });
    hipError_t e = a.in_f32 ? launch_tiles(thin_gram_kernel<float>, &a, parts, kThreads, stream)
                            : launch_tiles(thin_gram_kernel<uint16_t>, &a, parts, kThreads, stream);
    if (e != hipSuccess) return e;
    thin_steps_kernel<<<a.count, kThreads, 0, stream>>>(a, n);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const uint64_t runs = number(a, 1, [](const MuonMatrix& m) { return blocks(std::max(m.rows, m.cols), kThreads); });
    return a.in_f32 ? launch_tiles(thin_apply_kernel<float>, &a, runs, kThreads, stream)
                    : launch_tiles(thin_apply_kernel<uint16_t>, &a, runs, kThreads, stream);
}

hipError_t launch_muon_pack(MuonArgs& a, hipStream_t stream)
{
    if (const hipError_t e = launch_norms(a, stream)) return e;
    const uint64_t tiles = number(a, 1, [](const MuonMatrix& m) {
        return m.rows <= m.cols ? blocks(m.rows, kMuonRows) * blocks(((uint64_t)m.cols + 63) / 64 * 64, kMuonCols)
                                : blocks(m.rows, kMuonTurn) * blocks(m.cols, kMuonTurn);
    });
    return a.in_f32 ? launch_tiles(pack_kernel<float>, &a, tiles, kThreads, stream)
                    : launch_tiles(pack_kernel<uint16_t>, &a, tiles, kThreads, stream);
}

hipError_t launch_muon_tri(TriArgs& a, hipStream_t stream)
{
    const auto tiles = [](const TriMatrix& m, Size z) {
        const uint64_t n = blocks(m.s, kTile[z].q);
        return n * (n + 1) / 2 * (kTile[z].q / kTile[z].p);
    };
    const auto steps = [](const TriMatrix& m) { return (uint64_t)m.k / 64; };
    std::stable_sort(a.m, a.m + a.count, [&](const TriMatrix& x, const TriMatrix& y) { return x.k > y.k; });
    bool parts = false;
    for (uint32_t i = 0; i < a.count; ++i) parts |= a.m[i].chunk != 0;
    double whole;
    const Size size = size_of(a, parts, tiles, steps, &whole);
    if (a.m[0].part) {
        uint64_t most = 0, work = 0;
        for (uint32_t i = 0; i < a.count; ++i) {
            const uint64_t each = a.m[i].slices > 1 ? a.m[i].chunk / 64 : steps(a.m[i]);
            most = std::max(most, each);
            work += tiles(a.m[i], kSmall) * a.m[i].slices * each;
        }
        const uint64_t runs = number(a, 1, [&](const TriMatrix& m) { return tiles(m, kSmall) * m.slices; });
        const auto& c = kTile[kSmall];
        const double mean = (double)work / (double)runs, rounds = (double)blocks(runs, 256);
        if (std::max(rounds * (mean * c.many + c.end), (double)most * c.few + c.end) + kJoin < whole) {
            const hipError_t e = a.all ? launch_tiles(slices_kernel<Small<false, false, true>>, &a, runs, kThreads, stream)
                                       : launch_tiles(slices_kernel<Small<false, false, false>>, &a, runs, kThreads, stream);
            if (e != hipSuccess) return e;
            const uint64_t joins = number(a, 1, [](const TriMatrix& m) { return blocks((uint64_t)m.s * (blocks(m.s, 64) * 16), kThreads); });
            return launch_tiles(join_kernel, &a, joins, kThreads, stream);
        }
    }
    a.shares = steps(a.m[0]) != steps(a.m[a.count - 1]);
    const uint64_t all = number(a, a.shares ? kXcds : 1, [&](const TriMatrix& m) { return tiles(m, size); });
    const auto launch = [&](auto shape) {
        using S = decltype(shape);
        return launch_tiles(tri_kernel<S>, &a, all, S::kThreads, stream);
    };
    return size == kLarge    ? launch(Large<false, false>())
           : size == kWide   ? launch(Wide<false, false>())
           : size == kMiddle ? (a.all ? launch(Middle<false, false, true>()) : launch(Middle<false, false, false>()))
           : a.all           ? launch(Small<false, false, true>())
                             : launch(Small<false, false, false>());
}

hipError_t launch_muon_apply(MuonArgs& a, bool last, hipStream_t stream)
{
    return last ? apply<LastEnd>(a, stream) : apply<NextEnd>(a, stream);
}

} // namespace ckpt
