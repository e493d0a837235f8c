// embed_kernels.hip -- gfx950 kernels of the vocabulary table: the lookup, and
// its gradient by sorted tokens.
//
// Both are bound by HBM.  The gradient sorts the tokens by word (the order of
// a word's tokens stays), and waves then take runs of the sorted tokens and a
// run of columns each: a word's rows are added up in registers, in fp32, and
// its row of the table is written once.  A word's tokens may lie in several
// runs; their sums go through memory and a launch behind joins them, in order.
// No atomics touch what is summed: the same call gives the same bits.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "ops_internal.h"

namespace ckpt {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));

constexpr int kThreads = 256;
constexpr uint32_t kNoWord = 0xffffffffu;

__device__ inline uint16_t bf16_of(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ inline float float_of(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ inline float float_of(float x) { return x; }

// A lane's 16 bytes of a row: 8 bf16 or 4 fp32, from column c on; any alignment of the elements.
template <class T>
struct Piece {
    static constexpr uint32_t kValues = 16 / sizeof(T);
    u32x4 raw;
    __device__ inline float at(int j) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(raw[j]);
        return __uint_as_float(j & 1 ? raw[j / 2] & 0xFFFF0000u : raw[j / 2] << 16);
    }
    __device__ inline void load(const T* row, uint32_t c, uint32_t dim)
    {
        if (c + kValues <= dim) {
            raw = *(const u32x4_any*)(row + c);
            return;
        }
        raw = {0, 0, 0, 0};
#pragma unroll
        for (uint32_t j = 0; j < kValues - 1; ++j) {
            if (c + j >= dim) continue;
            if constexpr (sizeof(T) == 4)
                raw[j] = __float_as_uint(row[c + j]);
            else
                raw[j / 2] |= (uint32_t)row[c + j] << (j & 1 ? 16 : 0);
        }
    }
};

// N values from column c on, rounded to the row's type.
template <int N, class O>
__device__ inline void store(O* row, uint32_t c, uint32_t dim, const float (&x)[N])
{
    constexpr int kEach = 16 / sizeof(O);
    if (c + N <= dim) {
#pragma unroll
        for (int k = 0; k < N; k += kEach) {
            u32x4 raw = {0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < kEach && k + j < N; ++j) {
                if constexpr (sizeof(O) == 4)
                    raw[j] = __float_as_uint(x[k + j]);
                else
                    raw[j / 2] |= (uint32_t)bf16_of(x[k + j]) << (j & 1 ? 16 : 0);
            }
            if constexpr (kEach <= N)
                *(u32x4_any*)(row + c + k) = raw;
            else { // 4 bf16
                typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
                typedef u32x2 u32x2_any __attribute__((aligned(2)));
                *(u32x2_any*)(row + c + k) = u32x2{raw[0], raw[1]};
            }
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < N - 1; ++j) {
        if (c + j >= dim) continue;
        if constexpr (sizeof(O) == 4)
            row[c + j] = x[j];
        else
            row[c + j] = bf16_of(x[j]);
    }
}

// ---- the lookup ----
//
// A wave takes `UNROLL` KiB of a token's row, all of its loads ahead of its stores.
template <class T, int UNROLL>
__global__ __launch_bounds__(kThreads) void lookup_kernel(const EmbedArgs a, uint32_t runs)
{
    constexpr uint32_t kValues = Piece<T>::kValues, kRun = 64 * kValues;
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t job = __builtin_amdgcn_readfirstlane(blockIdx.x) * 4ull + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t t = (uint32_t)(job / runs), run = (uint32_t)(job % runs);
    if (t >= a.tokens) return;
    const int64_t id = a.ids[t];
    const bool there = id >= 0 && id < (int64_t)a.vocab && id != a.ignore_index;
    const T* from = (const T*)a.table + (there ? (uint64_t)id : 0) * a.table_ld;
    T* to = (T*)a.rows + (uint64_t)t * a.rows_ld;
    const uint32_t c0 = run * UNROLL * kRun + lane * kValues;
    const float instead = id == a.ignore_index ? 0.0f : __builtin_nanf("");
    Piece<T> p[UNROLL];
    if (there) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
            if (c0 + u * kRun < a.dim) p[u].load(from, c0 + u * kRun, a.dim);
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        if (c0 + u * kRun >= a.dim) continue;
        float x[kValues];
#pragma unroll
        for (int j = 0; j < (int)kValues; ++j) x[j] = there ? p[u].at(j) * a.scale : instead;
        store(to, c0 + u * kRun, a.dim, x);
    }
}

// ---- the tokens by word ----
//
// A workgroup has `range` words.  It goes over all ids twice (they stay in the L2): the first time each wave counts its
// own sixteenth of the tokens for each of the words, and those below all of them, which is where the workgroup's tokens
// begin; the second time each wave puts its tokens in their places.  A wave's places of a word follow those of the waves
// before it, a lane's those of the lanes before it: the order is the tokens' own.
__global__ __launch_bounds__(kSortWaves * 64) void sort_kernel(const EmbedArgs a)
{
    extern __shared__ uint32_t s_place[]; // [kSortWaves][range]
    __shared__ uint32_t s_below[kSortWaves], s_sum[kSortWaves];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t first = blockIdx.x * a.range, words = min(a.range, a.vocab - first);
    for (uint32_t k = threadIdx.x; k < kSortWaves * a.range; k += kSortWaves * 64) s_place[k] = 0;
    __syncthreads();
    uint32_t* mine = s_place + wave * a.range;
    const uint32_t each = (uint32_t)((((uint64_t)a.tokens + kSortWaves - 1) / kSortWaves + 63) / 64 * 64);
    const uint64_t begin = (uint64_t)wave * each, end = min(begin + each, (uint64_t)a.tokens);
    constexpr int kAhead = 4;
    // The words of a wave's next tokens: kNoWord for those that do not count.
    auto load = [&](uint64_t t0, uint32_t (&w)[kAhead]) {
        int64_t id[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint64_t t = t0 + 64 * u + lane;
            id[u] = t < end ? a.ids[t] : -1;
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            w[u] = id[u] >= 0 && id[u] < (int64_t)a.vocab && id[u] != a.ignore_index ? (uint32_t)id[u] : kNoWord;
    };
    uint32_t below = 0;
    for (uint64_t t = begin; t < end; t += 64 * kAhead) {
        uint32_t w[kAhead];
        load(t, w);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            below += __builtin_popcountll(__ballot(w[u] < first));
            if (w[u] - first < words) atomicAdd(mine + (w[u] - first), 1u);
        }
    }
    if (lane == 0) s_below[wave] = below;
    __syncthreads();
    // Word r's tokens of all waves, and of all words before it.
    const uint32_t r = threadIdx.x;
    uint32_t count = 0;
    if (r < words)
        for (uint32_t w = 0; w < kSortWaves; ++w) count += s_place[w * a.range + r];
    uint32_t upto = count;
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t x = __shfl_up(upto, o);
        if (lane >= (uint32_t)o) upto += x;
    }
    if (lane == 63) s_sum[wave] = upto;
    __syncthreads();
    uint32_t at = upto - count;
    for (uint32_t w = 0; w < kSortWaves; ++w) at += s_below[w] + (w < wave ? s_sum[w] : 0);
    if (r < words) {
        a.start[first + r] = at;
        if (first + r + 1 == a.vocab) a.start[a.vocab] = at + count;
        for (uint32_t w = 0; w < kSortWaves; ++w) {
            uint32_t& place = s_place[w * a.range + r];
            const uint32_t here = place;
            place = at;
            at += here;
        }
    }
    __syncthreads();
    const uint32_t bits = 32 - __builtin_clz(words);
    for (uint64_t t = begin; t < end; t += 64 * kAhead) {
        uint32_t w[kAhead];
        load(t, w);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const bool in = w[u] - first < words;
            uint64_t same = __ballot(in);
            if (same == 0) continue;
            const uint32_t d = in ? w[u] - first : 0;
            for (uint32_t b = 0; b < bits; ++b) { // the lanes with this lane's word
                const uint64_t has = __ballot(d >> b & 1);
                same &= d >> b & 1 ? has : ~has;
            }
            if (in) {
                const uint32_t place = mine[d] + __builtin_popcountll(same & ((1ull << lane) - 1));
                a.order[place] = (uint32_t)(t + 64 * u + lane);
                a.word[place] = w[u];
            }
            // Every lane has read its word's place before the last of them moves it on.
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (in && (same >> lane) == 1) mine[d] += __builtin_popcountll(same);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
}

// ---- the sums ----

// A word's sum into its row of the table.
template <class O, int N>
__device__ inline void write_row(const EmbedArgs& a, uint32_t word, uint32_t c, float (&x)[N])
{
    O* row = (O*)a.table + (uint64_t)word * a.table_ld;
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] *= a.scale;
    if (a.add) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (c + j < a.dim) x[j] += float_of(row[c + j]);
    }
    store(row, c, a.dim, x);
}

// Workgroups up to `chunk_blocks`: each wave a chunk of sorted tokens and a run of columns.  The others: rows that no token
// has, 16 a workgroup.
template <class T, class O>
__global__ __launch_bounds__(kThreads) void sums_kernel(const EmbedArgs a, uint32_t chunks, uint32_t runs, uint32_t chunk_blocks)
{
    constexpr int kValues = Piece<T>::kValues, kAhead = 8;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (blockIdx.x >= chunk_blocks) {
        const uint32_t v0 = (blockIdx.x - chunk_blocks) * 16 + wave * 4;
        for (uint32_t v = v0; v < min(v0 + 4, a.vocab); ++v) {
            if (a.start[v] != a.start[v + 1]) continue;
            O* row = (O*)a.table + (uint64_t)v * a.table_ld;
            constexpr int kEach = 16 / sizeof(O);
            const float zero[kEach] = {};
            for (uint32_t c = lane * kEach; c < a.dim; c += 64 * kEach) store(row, c, a.dim, zero);
        }
        return;
    }
    const uint64_t job = blockIdx.x * 4ull + wave;
    const uint32_t chunk = __builtin_amdgcn_readfirstlane((uint32_t)(job / runs)), run = __builtin_amdgcn_readfirstlane((uint32_t)(job % runs));
    const uint32_t all = a.start[a.vocab]; // tokens that count
    const uint64_t lo = (uint64_t)chunk * a.chunk;
    if (chunk >= chunks || lo >= all) return;
    const uint32_t hi = (uint32_t)min(lo + a.chunk, (uint64_t)all);
    const uint32_t c = (run * 64 + lane) * kValues;
    float sum[kValues];
#pragma unroll
    for (int j = 0; j < kValues; ++j) sum[j] = 0;
    uint32_t now = kNoWord, begin = 0; // the word that is summed, and its first token here
    auto flush = [&](uint32_t end) {
        if (c < a.dim) {
            const bool head = begin == lo && a.start[now] < lo, tail = end == hi && a.start[now + 1] > hi;
            if (!head && !tail)
                write_row<O>(a, now, c, sum);
            else
                store(a.part + ((head ? 0 : chunks) + (uint64_t)chunk) * a.part_ld, c, (uint32_t)a.part_ld, sum); // part_ld covers whole pieces
        }
#pragma unroll
        for (int j = 0; j < kValues; ++j) sum[j] = 0;
    };
    for (uint32_t base = (uint32_t)lo; base < hi; base += 64) {
        const uint32_t n = min(64u, hi - base), at = base + min(lane, n - 1);
        const uint32_t tokens = a.order[at], words = a.word[at];
        for (uint32_t i = 0; i < n; i += kAhead) {
            Piece<T> p[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const uint32_t t = __builtin_amdgcn_readlane(tokens, min(i + u, n - 1));
                if (c < a.dim && i + u < n) p[u].load((const T*)a.rows + (uint64_t)t * a.rows_ld, c, a.dim);
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (i + u >= n) break;
                const uint32_t w = __builtin_amdgcn_readlane(words, i + u);
                if (w != now) {
                    if (now != kNoWord) flush(base + i + u);
                    now = w;
                    begin = base + i + u;
                }
                if (c < a.dim) {
#pragma unroll
                    for (int j = 0; j < kValues; ++j) sum[j] += p[u].at(j);
                }
            }
        }
    }
    flush(hi);
}

// Words that begin in a chunk and go on behind it.
template <class O>
__global__ __launch_bounds__(kThreads) void join_sums_kernel(const EmbedArgs a, uint32_t chunks, uint32_t runs)
{
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint64_t job = blockIdx.x * 4ull + wave;
    const uint32_t chunk = __builtin_amdgcn_readfirstlane((uint32_t)(job / runs)), run = __builtin_amdgcn_readfirstlane((uint32_t)(job % runs));
    const uint32_t all = a.start[a.vocab];
    const uint64_t lo = (uint64_t)chunk * a.chunk, hi = lo + a.chunk;
    if (chunk >= chunks || hi >= all) return;
    const uint32_t word = a.word[hi - 1];
    const uint32_t begin = a.start[word], end = a.start[word + 1];
    const uint32_t c = (run * 64 + lane) * 4;
    if (begin < lo || end <= hi || c >= a.dim) return;
    const uint32_t last = (end - 1) / a.chunk;
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    f32x4 sum = *(const f32x4*)(a.part + ((uint64_t)chunks + chunk) * a.part_ld + c);
#pragma unroll 8
    for (uint32_t k = chunk + 1; k <= last; ++k) sum += *(const f32x4*)(a.part + k * a.part_ld + c);
    float x[4] = {sum[0], sum[1], sum[2], sum[3]};
    write_row<O>(a, word, c, x);
}

uint64_t cut(uint64_t x, uint64_t by) { return (x + by - 1) / by; }

template <class T>
hipError_t lookup_of(const EmbedArgs& a, hipStream_t stream)
{
    // A wave's KiB of a row: 4 where there are rows enough for the GPU.
    constexpr uint32_t kRun = 1024 / sizeof(T);
    const bool many = a.tokens * cut(a.dim, 4 * kRun) >= 4096;
    const uint64_t runs = cut(a.dim, (many ? 4 : 1) * kRun), blocks = cut(a.tokens * runs, 4);
    if (runs > 0xffffffffu || blocks * kThreads > 0xffffffffu) return hipErrorInvalidValue;
    if (many)
        lookup_kernel<T, 4><<<(uint32_t)blocks, kThreads, 0, stream>>>(a, (uint32_t)runs);
    else
        lookup_kernel<T, 1><<<(uint32_t)blocks, kThreads, 0, stream>>>(a, (uint32_t)runs);
    return hipGetLastError();
}

template <class T, class O>
hipError_t sums_of(const EmbedArgs& a, hipStream_t stream)
{
    const uint64_t chunks = cut(a.tokens, a.chunk), runs = cut(a.dim, 64 * Piece<T>::kValues);
    const uint64_t chunk_blocks = cut(chunks * runs, 4), zero_blocks = a.add ? 0 : cut(a.vocab, 16);
    if ((chunk_blocks + zero_blocks) * kThreads > 0xffffffffu) return hipErrorInvalidValue;
    if (chunk_blocks + zero_blocks)
        sums_kernel<T, O><<<(uint32_t)(chunk_blocks + zero_blocks), kThreads, 0, stream>>>(a, (uint32_t)chunks, (uint32_t)runs, (uint32_t)chunk_blocks);
    const uint64_t join_runs = cut(a.dim, 256), join_blocks = cut((chunks ? chunks - 1 : 0) * join_runs, 4);
    if (join_blocks * kThreads > 0xffffffffu) return hipErrorInvalidValue;
    if (join_blocks) join_sums_kernel<O><<<(uint32_t)join_blocks, kThreads, 0, stream>>>(a, (uint32_t)chunks, (uint32_t)join_runs);
    return hipGetLastError();
}

} // namespace

hipError_t launch_lookup(const EmbedArgs& a, hipStream_t stream)
{
    if (a.tokens == 0) return hipSuccess;
    return a.rows_f32 ? lookup_of<float>(a, stream) : lookup_of<uint16_t>(a, stream);
}

hipError_t launch_sort(const EmbedArgs& a, hipStream_t stream)
{
    if (a.range == 0 || a.range > kSortRange) return hipErrorInvalidValue;
    const uint32_t blocks = (uint32_t)cut(a.vocab, a.range);
    sort_kernel<<<blocks, kSortWaves * 64, kSortWaves * a.range * 4, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_table_sums(const EmbedArgs& a, hipStream_t stream)
{
    if (a.rows_f32)
        return a.table_f32 ? sums_of<float, float>(a, stream) : sums_of<float, uint16_t>(a, stream);
    return a.table_f32 ? sums_of<uint16_t, float>(a, stream) : sums_of<uint16_t, uint16_t>(a, stream);
}

} // namespace ckpt
