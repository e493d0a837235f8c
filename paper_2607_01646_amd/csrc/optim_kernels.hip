// optim_kernels.hip -- gfx950 kernels of the optimizer step: the gradients'
// norm and AdamW over a rank's fragments.
//
// Both are bound by HBM: AdamW moves 28 bytes a parameter (bf16 parameter and
// gradient; 32 in full precision) for some 60 instructions, the norm 2 or 4.
// A launch takes the fragments of up to 64 (the norm: 160) parameters as
// kernel arguments, so nothing is allocated or copied for a table; a workgroup
// finds the fragment of its tile with one load per lane and a ballot.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ops_internal.h"

namespace ckpt {
namespace {

// Vectors of four elements at any element's alignment (global memory is read
// and written unaligned by the hardware).
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u16x4 u16x4_any __attribute__((aligned(2)));

__device__ inline f32x4 load4(const float* p) { return __builtin_nontemporal_load((const f32x4_any*)p); }
__device__ inline f32x4 load4(const uint16_t* p)
{
    const u16x4 u = __builtin_nontemporal_load((const u16x4_any*)p);
    f32x4 r;
    for (int j = 0; j < 4; ++j) r[j] = __uint_as_float((uint32_t)u[j] << 16);
    return r;
}
__device__ inline float load1(const float* p) { return *p; }
__device__ inline float load1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }

__device__ inline uint16_t bf16_of(float x)
{
    return __builtin_bit_cast(uint16_t, (__bf16)x); // to nearest even, NaN stays NaN
}
__device__ inline void store4(float* p, f32x4 x) { __builtin_nontemporal_store(x, (f32x4_any*)p); }
__device__ inline void store4(uint16_t* p, f32x4 x)
{
    u16x4 u;
    for (int j = 0; j < 4; ++j) u[j] = bf16_of(x[j]);
    __builtin_nontemporal_store(u, (u16x4_any*)p);
}
__device__ inline void store1(float* p, float x) { *p = x; }
__device__ inline void store1(uint16_t* p, float x) { *p = bf16_of(x); }

struct Moments {
    float master, m, v;
};

__device__ inline Moments adamw(const AdamArgs& a, float c, float g, float master, float m, float v)
{
    g *= c;
    m = a.beta1 * m + a.one_beta1 * g;
    v = a.beta2 * v + a.one_beta2 * g * g;
    master = master * a.keep - a.lr * ((m * a.inv_bc1) / (sqrtf(v * a.inv_bc2) + a.eps));
    return {master, m, v};
}

constexpr int kThreads = 256;

template <class P, class G>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const AdamArgs a)
{
    // The tile's fragment: the last whose first tile is not beyond it.
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t before = __ballot(lane < a.count && a.first[lane] <= blockIdx.x);
    const uint32_t f = __builtin_amdgcn_readfirstlane(63 - __builtin_clzll(before));
    const uint64_t n = a.f[f].numel, begin = (uint64_t)(blockIdx.x - a.first[f]) * kAdamTile;
    P* param = (P*)a.f[f].param + begin;
    float* master = (float*)a.f[f].master + begin;
    float* em = (float*)a.f[f].m + begin;
    float* ev = (float*)a.f[f].v + begin;
    const G* grad = (const G*)a.f[f].grad + begin;
    const float c = a.scale ? *a.scale : 1.0f;
    constexpr int kVecs = kAdamTile / (4 * kThreads);
    const uint64_t left = n - begin;
    if (left >= kAdamTile) {
        f32x4 g[kVecs], w[kVecs], m[kVecs], v[kVecs];
#pragma unroll
        for (int u = 0; u < kVecs; ++u) {
            const uint32_t at = 4 * (u * kThreads + threadIdx.x);
            g[u] = load4(grad + at);
            w[u] = load4(master + at);
            m[u] = load4(em + at);
            v[u] = load4(ev + at);
        }
#pragma unroll
        for (int u = 0; u < kVecs; ++u) {
            const uint32_t at = 4 * (u * kThreads + threadIdx.x);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const Moments r = adamw(a, c, g[u][j], w[u][j], m[u][j], v[u][j]);
                w[u][j] = r.master;
                m[u][j] = r.m;
                v[u][j] = r.v;
            }
            store4(master + at, w[u]);
            store4(em + at, m[u]);
            store4(ev + at, v[u]);
            store4(param + at, w[u]);
        }
        return;
    }
    for (uint32_t at = threadIdx.x; at < left; at += kThreads) {
        const Moments r = adamw(a, c, load1(grad + at), master[at], em[at], ev[at]);
        master[at] = r.master;
        em[at] = r.m;
        ev[at] = r.v;
        store1(param + at, r.master);
    }
}

__device__ inline double wave_sum(double x)
{
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

// The workgroup's sum in lane 0, the waves' in their order.
__device__ inline double block_sum(double x, double* s_wave)
{
    x = wave_sum(x);
    if ((threadIdx.x & 63) == 0) s_wave[threadIdx.x >> 6] = x;
    __syncthreads();
    if (threadIdx.x == 0)
        for (uint32_t w = 1; w < blockDim.x / 64; ++w) x += s_wave[w];
    return x;
}

// The squares of tiles first, first + stride, ...: `lane` is one of LANES that share a tile of TILE elements.  Squares and
// sums are in 64 bits: the sum is exact to its last places for any number of elements, no square overflows, and the
// kernel is bound by its loads all the same.
template <class G, int LANES, uint32_t TILE>
__device__ inline double tile_squares(const NormArgs& a, uint32_t lane, uint32_t first, uint32_t stride)
{
    double sum = 0;
    for (uint32_t t = first; t < a.tiles; t += stride) {
        uint32_t f = 0;
        for (uint32_t base = 0; base < a.count; base += 64) {
            const uint32_t k = base + (threadIdx.x & 63);
            const uint64_t before = __ballot(k < a.count && a.first[k < kNormFrags ? k : 0] <= t);
            if (before) f = base + 63 - __builtin_clzll(before);
        }
        f = __builtin_amdgcn_readfirstlane(f);
        const uint64_t n = a.f[f].numel, begin = (uint64_t)(t - a.first[f]) * TILE;
        const G* g = (const G*)a.f[f].ptr + begin;
        const uint64_t left = n - begin;
        if (left >= TILE) {
            constexpr int kVecs = TILE / (4 * LANES);
            f32x4 x[kVecs];
#pragma unroll
            for (int u = 0; u < kVecs; ++u) x[u] = load4(g + 4 * (u * LANES + lane));
#pragma unroll
            for (int u = 0; u < kVecs; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum += (double)x[u][j] * (double)x[u][j];
        } else {
            for (uint32_t at = 4 * lane; at < left; at += 4 * LANES) {
                if (at + 4 <= left) {
                    const f32x4 x = load4(g + at);
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum += (double)x[j] * (double)x[j];
                } else {
                    for (uint32_t j = at; j < left; ++j) {
                        const double x = load1(g + j);
                        sum += x * x;
                    }
                }
            }
        }
    }
    return sum;
}

__device__ inline void write_norm(double sum, double max_norm, float* out)
{
    const double norm = sqrt(sum);
    const double c = max_norm / (norm + 1e-6);
    out[0] = (float)norm;
    out[1] = max_norm <= 0 || c >= 1 ? 1.0f : (float)c; // a NaN norm gives NaN
}

template <class G>
__global__ __launch_bounds__(kThreads) void norm_kernel(const NormArgs a, double* part, bool fresh)
{
    __shared__ double s_wave[kThreads / 64];
    const double sum = block_sum(tile_squares<G, kThreads, kNormTile>(a, threadIdx.x, blockIdx.x, gridDim.x), s_wave);
    if (threadIdx.x == 0) part[blockIdx.x] = fresh ? sum : part[blockIdx.x] + sum;
    if (fresh && blockIdx.x == 0) // workgroups that this launch does without
        for (uint32_t k = gridDim.x + threadIdx.x; k < kNormBlocks; k += kThreads) part[k] = 0;
}

template <class G>
__global__ __launch_bounds__(1024) void norm_few_kernel(const NormArgs a, double max_norm, float* out)
{
    __shared__ double s_wave[16];
    const double sum = block_sum(
        tile_squares<G, 64, kNormFewTile>(a, threadIdx.x & 63, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), 16), s_wave);
    if (threadIdx.x == 0) write_norm(sum, max_norm, out);
}

__global__ __launch_bounds__(kThreads) void norm_finish_kernel(const double* part, double max_norm, float* out)
{
    __shared__ double s_wave[kThreads / 64];
    double sum = 0;
    for (uint32_t k = threadIdx.x; k < kNormBlocks; k += kThreads) sum += part[k];
    sum = block_sum(sum, s_wave);
    if (threadIdx.x == 0) write_norm(sum, max_norm, out);
}

} // namespace

hipError_t launch_adamw(const AdamArgs& a, bool param_f32, bool grad_f32, hipStream_t s)
{
    if (a.count == 0 || a.count > kAdamFrags) return hipErrorInvalidValue;
    if (a.tiles == 0) return hipSuccess;
    if (param_f32 && grad_f32)
        adamw_kernel<float, float><<<a.tiles, kThreads, 0, s>>>(a);
    else if (param_f32)
        adamw_kernel<float, uint16_t><<<a.tiles, kThreads, 0, s>>>(a);
    else if (grad_f32)
        adamw_kernel<uint16_t, float><<<a.tiles, kThreads, 0, s>>>(a);
    else
        adamw_kernel<uint16_t, uint16_t><<<a.tiles, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_norm(const NormArgs& a, bool f32, bool fresh, double* part, hipStream_t s)
{
    if (a.count > kNormFrags) return hipErrorInvalidValue;
    const uint32_t grid = a.tiles < kNormBlocks ? (a.tiles ? a.tiles : 1) : kNormBlocks;
    if (f32)
        norm_kernel<float><<<grid, kThreads, 0, s>>>(a, part, fresh);
    else
        norm_kernel<uint16_t><<<grid, kThreads, 0, s>>>(a, part, fresh);
    return hipGetLastError();
}

hipError_t launch_norm_few(const NormArgs& a, bool f32, double max_norm, float* out, hipStream_t s)
{
    if (a.count > kNormFrags) return hipErrorInvalidValue;
    if (f32)
        norm_few_kernel<float><<<1, 1024, 0, s>>>(a, max_norm, out);
    else
        norm_few_kernel<uint16_t><<<1, 1024, 0, s>>>(a, max_norm, out);
    return hipGetLastError();
}

hipError_t launch_norm_finish(const double* part, double max_norm, float* out, hipStream_t s)
{
    norm_finish_kernel<<<1, kThreads, 0, s>>>(part, max_norm, out);
    return hipGetLastError();
}

} // namespace ckpt
