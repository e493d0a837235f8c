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

// A lane's 16 bytes of a row: 8 bf16 or 4 fp32, at any alignment of the elements.  The loads of a wave's rows are in no
// branch: a lane whose columns go past the end has the row's last ones (those of a row of fewer: some of them twice), from
// first() on, and settle() puts its sums in their places.
template <class T>
struct Piece {
    static constexpr uint32_t kValues = 16 / sizeof(T);
    u32x4 raw;
    static __device__ inline uint32_t first(uint32_t c, uint32_t dim) { return dim < kValues ? 0 : min(c, dim - kValues); }
    __device__ inline float at(int j) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(raw[j]);
        return __uint_as_float(j & 1 ? raw[j / 2] & 0xFFFF0000u : raw[j / 2] << 16);
    }
    __device__ inline void load(const T* row, uint32_t from, bool narrow, uint32_t dim)
    {
        if (!narrow) {
            raw = *(const u32x4_any*)(row + from);
            return;
        }
        raw = {0, 0, 0, 0};
#pragma unroll
        for (uint32_t j = 0; j < kValues; ++j) {
            const T x = row[min(j, dim - 1)];
            if constexpr (sizeof(T) == 4)
                raw[j] = __float_as_uint(x);
            else
                raw[j / 2] |= (uint32_t)x << (j & 1 ? 16 : 0);
        }
    }
    // Values that begin at column first(c) to such that begin at c.
    static __device__ inline void settle(float (&x)[kValues], uint32_t c, uint32_t dim)
    {
        const uint32_t by = c - first(c, dim);
#pragma unroll
        for (uint32_t b = 1; b < kValues; b *= 2) {
            const bool move = by & b;
#pragma unroll
            for (uint32_t j = 0; j < kValues; ++j) x[j] = move ? (j + b < kValues ? x[j + b] : 0.0f) : x[j];
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

// A wave's share of a row of zeros, the `run`-th of `runs` of N elements each: cut at addresses that are multiples of 128
// bytes, wherever the row begins, so that a line is written at once (7 tokens of 43667 x 7381 fp32: 396 -> 251 us).  PAST the
// caches where rows are read meanwhile (a table of 32000 x 4096 takes 71 us with its gradient, 75 through them); few tokens
// have none to keep (100 of 32000 x 4096 bf16, which the last cache holds: 47 us past it, 39 through it).
template <uint32_t N, bool PAST, class O>
__device__ inline void clear(O* row, uint32_t dim, uint32_t run, uint32_t runs)
{
    constexpr int kEach = 16 / sizeof(O);
    const int skip = (int)((uintptr_t)row % 128 / sizeof(O)), lane = threadIdx.x & 63;
    const int end = run + 1 < runs ? (int)((run + 1) * N) - skip : (int)dim;
    for (int c = (int)(run * N) - skip + lane * kEach; c < end; c += 64 * kEach) {
        if (c >= 0 && c + kEach <= (int)dim) {
            if constexpr (PAST)
                __builtin_nontemporal_store(u32x4{0, 0, 0, 0}, (u32x4*)(row + c));
            else
                *(u32x4*)(row + c) = u32x4{0, 0, 0, 0};
        } else {
#pragma unroll
            for (int j = 0; j < kEach; ++j)
                if (c + j >= 0 && c + j < (int)dim) row[c + j] = 0;
        }
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
    const bool narrow = a.dim < kValues;
    Piece<T> p[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) p[u].load(from, Piece<T>::first(c0 + u * kRun, a.dim), narrow, a.dim);
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        if (c0 + u * kRun >= a.dim) continue;
        float x[kValues];
#pragma unroll
        for (int j = 0; j < (int)kValues; ++j) x[j] = there ? p[u].at(j) * a.scale : instead;
        if (c0 + u * kRun + kValues > a.dim) Piece<T>::settle(x, c0 + u * kRun, a.dim);
        store(to, c0 + u * kRun, a.dim, x);
    }
}

// ---- the tokens by word ----
//
// A workgroup has `range` words and goes over all ids (they stay in the L2), each wave over its own sixteenth: it counts its
// tokens for each of the words, and those below all of them, which is where the workgroup's tokens begin, and lists the
// ones that are the workgroup's in LDS.  Then each wave puts its tokens in their places.  A wave's places of a word follow
// those of the waves before it, a lane's those of the lanes before it: the order is the tokens' own.  A wave whose tokens
// its list does not hold goes over the ids again and puts 64 in their places at a time (56265 tokens of 64, 3890 of them one
// word: 77 us with lists of 256 and at most the tokens among 64 ids at a time, so 50).  Bound by the instructions of the first pass.
constexpr uint32_t kList = 768;
__global__ __launch_bounds__(kSortWaves * 64) void sort_kernel(const EmbedArgs a)
{
    extern __shared__ uint32_t s_place[]; // [kSortWaves][range]
    __shared__ uint32_t s_list[kSortWaves][kList];
    __shared__ uint32_t s_below[kSortWaves], s_sum[kSortWaves];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t first = blockIdx.x * a.range, words = min(a.range, a.vocab - first);
    for (uint32_t k = threadIdx.x; k < kSortWaves * a.range; k += kSortWaves * 64) s_place[k] = 0;
    __syncthreads();
    uint32_t* mine = s_place + wave * a.range;
    const uint32_t each = (uint32_t)((((uint64_t)a.tokens + kSortWaves - 1) / kSortWaves + 63) / 64 * 64);
    const uint64_t begin = (uint64_t)wave * each, end = min(begin + each, (uint64_t)a.tokens);
    constexpr int kAhead = 8;
    // The words of a wave's next tokens: kNoWord for those that do not count.  An ignored id that is a word's number is one
    // in 2^32 bits; no other has its upper half 0 and its lower below vocab.
    const uint32_t ignored = a.ignore_index >= 0 && a.ignore_index < (int64_t)a.vocab ? (uint32_t)a.ignore_index : kNoWord;
    auto load = [&](uint64_t t0, uint32_t (&w)[kAhead]) {
        uint2 id[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) id[u] = ((const uint2*)a.ids)[min(t0 + 64 * u + lane, end - 1)];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            w[u] = id[u].y == 0 && id[u].x < a.vocab && id[u].x != ignored && t0 + 64 * u + lane < end ? id[u].x : kNoWord;
    };
    uint32_t below = 0, listed = 0;
    for (uint64_t t = begin; t < end; t += 64 * kAhead) {
        uint32_t w[kAhead];
        load(t, w);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            below += __builtin_popcountll(__ballot(w[u] < first));
            const bool in = w[u] - first < words;
            const uint64_t which = __ballot(in);
            if (which == 0) continue;
            const uint32_t place = listed + __builtin_popcountll(which & ((1ull << lane) - 1));
            if (in) {
                atomicAdd(mine + (w[u] - first), 1u);
                if (place < kList) s_list[wave][place] = (uint32_t)(t + 64 * u + lane);
            }
            listed += __builtin_popcountll(which);
        }
    }
    if (lane == 0) s_below[wave] = below;
    __syncthreads();
    // Word r's tokens of all waves, and of all words before it.
    const uint32_t r = threadIdx.x;
    uint32_t of[kSortWaves], count = 0;
#pragma unroll
    for (uint32_t w = 0; w < kSortWaves; ++w) {
        of[w] = s_place[w * a.range + min(r, words - 1)];
        count += r < words ? of[w] : 0;
    }
    uint32_t upto = count;
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t x = __shfl_up(upto, o);
        if (lane >= (uint32_t)o) upto += x;
    }
    if (lane == 63) s_sum[wave] = upto;
    __syncthreads();
    uint32_t at = upto - count;
#pragma unroll
    for (uint32_t w = 0; w < kSortWaves; ++w) at += s_below[w] + (w < wave ? s_sum[w] : 0);
    if (r < words) {
        a.start[first + r] = at;
        if (first + r + 1 == a.vocab) a.start[a.vocab] = at + count;
#pragma unroll
        for (uint32_t w = 0; w < kSortWaves; ++w) {
            s_place[w * a.range + r] = at;
            at += of[w];
        }
    }
    __syncthreads();
    const uint32_t bits = 32 - __builtin_clz(words);
    // The places of up to 64 tokens of this wave, in their lanes' order.
    auto put = [&](bool in, uint32_t token, uint32_t word) {
        uint64_t same = __ballot(in);
        const uint32_t d = in ? word - first : 0;
        for (uint32_t b = 0; b < bits; ++b) { // the lanes with this lane's word
            const uint64_t has = __ballot(d >> b & 1);
            same &= d >> b & 1 ? has : ~has;
        }
        if (in) {
            const uint32_t place = mine[d] + __builtin_popcountll(same & ((1ull << lane) - 1));
            a.order[place] = token;
            a.word[place] = word;
        }
        // Every lane has read its word's place before the last of them moves it on.
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (in && (same >> lane) == 1) mine[d] += __builtin_popcountll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    if (listed <= kList) {
        for (uint32_t k = 0; k < listed; k += 64) {
            const uint32_t token = s_list[wave][min(k + lane, listed - 1)];
            put(k + lane < listed, token, ((const uint2*)a.ids)[token].x);
        }
        return;
    }
    uint32_t* list = s_list[wave];
    uint32_t have = 0;
    auto put_listed = [&] { // the first 64
        const uint32_t token = list[min(lane, have - 1)];
        put(lane < have, token, ((const uint2*)a.ids)[token].x);
    };
    for (uint64_t t = begin; t < end; t += 64 * kAhead) {
        uint32_t w[kAhead];
        load(t, w);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const bool in = w[u] - first < words;
            const uint64_t which = __ballot(in);
            if (in) list[have + __builtin_popcountll(which & ((1ull << lane) - 1))] = (uint32_t)(t + 64 * u + lane);
            have += __builtin_popcountll(which);
            if (have < 64) continue;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            put_listed();
            const uint32_t rest = list[64 + lane];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            have -= 64;
            if (lane < have) list[lane] = rest;
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (have) put_listed();
}

// ---- the sums ----

// N values of a row of the table that a sum is added to, from column `from` on.
template <class O, int N>
struct Old {
    O x[N];
    __device__ inline void load(const O* row, uint32_t from, bool narrow, uint32_t dim)
    {
        typedef O any __attribute__((ext_vector_type(N), aligned(sizeof(O))));
        if (!narrow) {
            const any v = *(const any*)(row + from);
#pragma unroll
            for (int j = 0; j < N; ++j) x[j] = v[j];
        } else {
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) x[j] = row[min(j, dim - 1)];
        }
    }
};

constexpr uint32_t kZeroRows = 32;

// Workgroups up to `chunk_blocks`: each wave a chunk of sorted tokens and a run of columns.  The others: rows that no token
// has, of kZeroRows words a workgroup.
template <class T, class O>
__global__ __launch_bounds__(kThreads) void sums_kernel(const EmbedArgs a, uint32_t chunks, uint32_t runs, uint32_t chunk_blocks)
{
    constexpr int kValues = Piece<T>::kValues, kAhead = 8;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (blockIdx.x >= chunk_blocks) {
        const uint32_t v0 = (blockIdx.x - chunk_blocks) * kZeroRows + wave * (kZeroRows / 4);
        const uint32_t mine = min(v0 + lane, a.vocab - 1);
        const bool none = lane < kZeroRows / 4 && v0 + lane < a.vocab && a.start[mine] == a.start[mine + 1];
        for (uint64_t left = __ballot(none); left; left &= left - 1) {
            O* row = (O*)a.table + (uint64_t)(v0 + __builtin_ctzll(left)) * a.table_ld;
            clear<64 * 16 / sizeof(O), true>(row, a.dim, 0, 1);
        }
        return;
    }
    const uint64_t job = blockIdx.x * 4ull + wave;
    const uint32_t chunk = __builtin_amdgcn_readfirstlane((uint32_t)(job / runs)), run = __builtin_amdgcn_readfirstlane((uint32_t)(job % runs));
    if (chunk >= chunks) return;
    const uint64_t lo = (uint64_t)chunk * a.chunk;
    const uint32_t all = a.start[a.vocab]; // tokens that count
    const uint32_t c = (run * 64 + lane) * kValues, from = Piece<T>::first(c, a.dim);
    const bool narrow = a.dim < (uint32_t)kValues;
    float sum[kValues];
#pragma unroll
    for (int j = 0; j < kValues; ++j) sum[j] = 0;
    uint2 goes_on = make_uint2(kNoWord, 0);
    for (uint64_t base = lo; base < lo + a.chunk; base += 64) {
        // 64 tokens at a time: their words, and where those begin and end (what lies past the last token is not used).
        const uint64_t at = min(base + lane, (uint64_t)a.tokens - 1);
        const uint32_t tokens = a.order[at], words = min(a.word[at], a.vocab - 1);
        const uint32_t begins = a.start[words], ends = a.start[words + 1];
        const uint32_t hi = (uint32_t)min(lo + a.chunk, (uint64_t)all);
        if (base >= hi) break;
        const uint32_t n = min(64u, hi - (uint32_t)base);
        for (uint32_t i = 0; i < n; i += kAhead) {
            Piece<T> p[kAhead];
            Old<O, kValues> old[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const uint32_t k = min(i + u, n - 1), end = __builtin_amdgcn_readlane(ends, k);
                p[u].load((const T*)a.rows + (uint64_t)__builtin_amdgcn_readlane(tokens, k) * a.rows_ld, from, narrow, a.dim);
                if (a.add && end == base + k + 1) // its last token: what the word's sum is added to
                    old[u].load((const O*)a.table + (uint64_t)__builtin_amdgcn_readlane(words, k) * a.table_ld, from, narrow, a.dim);
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (i + u >= n) break;
                const uint32_t here = (uint32_t)base + i + u;
                const uint32_t end = __builtin_amdgcn_readlane(ends, i + u);
#pragma unroll
                for (int j = 0; j < kValues; ++j) sum[j] += p[u].at(j);
                if (here + 1 != end && here + 1 != hi) continue;
                // The word's last token, or the chunk's: its row, or a sum that is joined with others.
                const bool head = __builtin_amdgcn_readlane(begins, i + u) < lo, tail = end > hi;
                if (head || tail) {
                    if (!head) goes_on = make_uint2(__builtin_amdgcn_readlane(words, i + u), (end - 1) / a.chunk);
                    if (c + kValues > a.dim) Piece<T>::settle(sum, c, a.dim);
                    if (c < a.dim) // part_ld covers whole pieces
                        store(a.part + ((head ? 0 : chunks) + (uint64_t)chunk) * a.part_ld, c, (uint32_t)a.part_ld, sum);
                } else {
#pragma unroll
                    for (int j = 0; j < kValues; ++j) sum[j] = sum[j] * a.scale + (a.add ? float_of(old[u].x[j]) : 0.0f);
                    if (c + kValues > a.dim) Piece<T>::settle(sum, c, a.dim);
                    if (c < a.dim) store((O*)a.table + (uint64_t)__builtin_amdgcn_readlane(words, i + u) * a.table_ld, c, a.dim, sum);
                }
#pragma unroll
                for (int j = 0; j < kValues; ++j) sum[j] = 0;
            }
        }
    }
    if (run == 0 && lane == 0) a.join[chunk] = goes_on;
}

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

// Words that begin in a chunk and go on behind it: a workgroup a chunk.
template <class O>
__global__ __launch_bounds__(kThreads) void join_sums_kernel(const EmbedArgs a, uint32_t chunks)
{
    const uint32_t chunk = blockIdx.x;
    const uint2 it = a.join[chunk];
    const uint32_t word = it.x, last = it.y;
    if (word == kNoWord) return;
    constexpr uint32_t kAhead = 16;
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    for (uint32_t c = (blockIdx.y * kThreads + threadIdx.x) * 4; c < a.dim; c += gridDim.y * kThreads * 4) {
        f32x4 sum = *(const f32x4*)(a.part + ((uint64_t)chunks + chunk) * a.part_ld + c);
        for (uint32_t k = chunk + 1; k <= last; k += kAhead) {
            f32x4 part[kAhead];
#pragma unroll
            for (uint32_t u = 0; u < kAhead; ++u) part[u] = *(const f32x4*)(a.part + min(k + u, last) * a.part_ld + c);
#pragma unroll
            for (uint32_t u = 0; u < kAhead; ++u)
                if (k + u <= last) sum += part[u];
        }
        float x[4] = {sum[0], sum[1], sum[2], sum[3]};
        write_row<O>(a, word, c, x);
    }
}

// ---- few tokens ----
//
// Up to 128: every wave has all ids in its registers, finds the tokens of 4 words by ballots and writes those rows' run of
// columns.  One launch and no workspace: sorting so few takes longer than their sums (64 tokens of 64: 4.8 us, sorted 11.5).
template <class T, class O>
__global__ __launch_bounds__(kThreads) void few_kernel(const EmbedArgs a)
{
    constexpr int kValues = Piece<T>::kValues, kIds = kFewRows / 64, kAhead = 4;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t v0 = (blockIdx.x * 4 + wave) * 4;
    const uint32_t c = (blockIdx.y * 64 + lane) * kValues, from = Piece<T>::first(c, a.dim);
    const bool narrow = a.dim < (uint32_t)kValues;
    int64_t id[kIds];
#pragma unroll
    for (int k = 0; k < kIds; ++k) id[k] = a.ids[min(64 * k + lane, a.tokens - 1)];
    uint32_t word[kIds];
#pragma unroll
    for (int k = 0; k < kIds; ++k)
        word[k] = 64 * k + lane < a.tokens && id[k] >= 0 && id[k] < (int64_t)a.vocab && id[k] != a.ignore_index ? (uint32_t)id[k] : kNoWord;
    for (uint32_t v = v0; v < min(v0 + 4, a.vocab); ++v) {
        float sum[kValues];
#pragma unroll
        for (int j = 0; j < kValues; ++j) sum[j] = 0;
        bool any = false;
#pragma unroll
        for (int k = 0; k < kIds; ++k) {
            uint64_t left = __ballot(word[k] == v);
            any |= left != 0;
            while (left) {
                Piece<T> p[kAhead];
                bool there[kAhead];
                uint32_t t = 64 * k;
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    there[u] = left != 0;
                    t = there[u] ? 64 * k + __builtin_ctzll(left | 1ull << 63) : t;
                    left &= left - 1;
                    p[u].load((const T*)a.rows + (uint64_t)t * a.rows_ld, from, narrow, a.dim);
                }
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
#pragma unroll
                    for (int j = 0; j < kValues; ++j) sum[j] += there[u] ? p[u].at(j) : 0.0f;
            }
        }
        if (!any) {
            if (!a.add) clear<64 * kValues, false>((O*)a.table + (uint64_t)v * a.table_ld, a.dim, blockIdx.y, gridDim.y);
            continue;
        }
        if (c >= a.dim) continue;
        if (c + kValues > a.dim) Piece<T>::settle(sum, c, a.dim);
        write_row<O>(a, v, c, sum);
    }
}

uint64_t cut(uint64_t x, uint64_t by) { return (x + by - 1) / by; }

template <class T>
hipError_t lookup_of(const EmbedArgs& a, hipStream_t stream)
{
    // A wave's KiB of a row: 4 where there are rows enough for the GPU.
    constexpr uint32_t kRun = 1024 / sizeof(T);
    const bool many = a.tokens * cut(a.dim, 4 * kRun) >= 4096;
    const uint32_t runs = (uint32_t)cut(a.dim, (many ? 4 : 1) * kRun);
    const uint64_t most = std::max(1u, (1u << 25) / runs); // tokens of a launch: 2^31 lanes
    for (uint64_t t = 0; t < a.tokens; t += most) {
        EmbedArgs part = a;
        part.ids += t;
        part.rows = (T*)a.rows + t * a.rows_ld;
        part.tokens = (uint32_t)std::min<uint64_t>(most, a.tokens - t);
        const uint32_t blocks = (uint32_t)cut((uint64_t)part.tokens * runs, 4);
        if (many)
            lookup_kernel<T, 4><<<blocks, kThreads, 0, stream>>>(part, runs);
        else
            lookup_kernel<T, 1><<<blocks, kThreads, 0, stream>>>(part, runs);
    }
    return hipGetLastError();
}

template <class T, class O>
hipError_t sums_of(const EmbedArgs& a, hipStream_t stream)
{
    const uint64_t chunks = cut(a.tokens, a.chunk), runs = cut(a.dim, 64 * Piece<T>::kValues);
    const uint64_t chunk_blocks = cut(chunks * runs, 4), zero_blocks = a.add ? 0 : cut(a.vocab, kZeroRows);
    if ((chunk_blocks + zero_blocks) * kThreads > 0xffffffffu) return hipErrorInvalidValue;
    if (chunk_blocks + zero_blocks)
        sums_kernel<T, O><<<(uint32_t)(chunk_blocks + zero_blocks), kThreads, 0, stream>>>(a, (uint32_t)chunks, (uint32_t)runs, (uint32_t)chunk_blocks);
    // A chunk's columns by as many workgroups as leave each SIMD some waves where words may be long.
    if (chunks > 1)
        join_sums_kernel<O><<<dim3((uint32_t)chunks - 1, (uint32_t)std::min<uint64_t>(cut(a.dim, 4 * kThreads), 4)), kThreads, 0, stream>>>(a, (uint32_t)chunks);
    return hipGetLastError();
}

template <class T, class O>
hipError_t few_of(const EmbedArgs& a, hipStream_t stream)
{
    const uint64_t blocks = cut(a.vocab, 16), runs = cut(a.dim, 64 * Piece<T>::kValues);
    if (blocks * runs * kThreads > 0xffffffffu || runs > 65535) return hipErrorInvalidValue;
    few_kernel<T, O><<<dim3((uint32_t)blocks, (uint32_t)runs), kThreads, 0, stream>>>(a);
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

hipError_t launch_few_sums(const EmbedArgs& a, hipStream_t stream)
{
    if (a.tokens == 0 || a.tokens > kFewRows) return hipErrorInvalidValue;
    if (a.rows_f32)
        return a.table_f32 ? few_of<float, float>(a, stream) : few_of<float, uint16_t>(a, stream);
    return a.table_f32 ? few_of<uint16_t, float>(a, stream) : few_of<uint16_t, uint16_t>(a, stream);
}

hipError_t launch_table_sums(const EmbedArgs& a, hipStream_t stream)
{
    if (a.rows_f32)
        return a.table_f32 ? sums_of<float, float>(a, stream) : sums_of<float, uint16_t>(a, stream);
    return a.table_f32 ? sums_of<uint16_t, float>(a, stream) : sums_of<uint16_t, uint16_t>(a, stream);
}

} // namespace ckpt
