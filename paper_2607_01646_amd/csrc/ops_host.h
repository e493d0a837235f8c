// What the operators' entry points share: the checks of a call's pointers and
// sizes.
#pragma once

#include "../../include/ckpt_ops.h"
#include "ckpt_host.h"

namespace ckpt {

constexpr uint64_t kMost = 0x7fffffffull;   // tokens
constexpr uint64_t kMostWidth = 1ull << 22; // dim, vocab: a tile's rows of an operand stay within 31 bits of bytes

inline uint64_t up(uint64_t x, uint64_t a) { return (x + a - 1) / a * a; }

// The bytes of a [rows, cols] operand with rows `ld` elements apart; false where 64 bits do not count them.
inline bool extent(uint64_t rows, uint64_t cols, uint64_t ld, uint64_t elem, uint64_t* bytes)
{
    *bytes = 0;
    uint64_t last;
    return rows == 0 || (!__builtin_mul_overflow(rows - 1, ld, &last) && !__builtin_add_overflow(last, cols, &last) &&
                         !__builtin_mul_overflow(last, elem, bytes));
}

inline bool type_bytes(uint32_t type, uint64_t* e)
{
    *e = type == CKPT_TYPE_F32 ? 4 : 2;
    return type == CKPT_TYPE_F32 || type == CKPT_TYPE_BF16;
}

// Allocations that this call has met: most of its pointers share a few (a
// flat buffer's fragments, a caching allocator's segments), and asking the
// runtime about one takes a microsecond.
struct Known {
    static constexpr int kMost = 8;
    uint64_t lo[kMost], hi[kMost];
    int n = 0, at = 0;

    bool holds(uint64_t p, uint64_t bytes) const
    {
        for (int k = 0; k < n; ++k)
            if (p >= lo[k] && p <= hi[k] && bytes <= hi[k] - p) return true;
        return false;
    }
    void add(uint64_t base, uint64_t size)
    {
        lo[at] = base;
        hi[at] = base + size;
        at = (at + 1) % kMost;
        n = n < kMost ? n + 1 : n;
    }
};

struct Given {
    const void* p;
    uint64_t rows, cols, ld, elem;
    const char* what;
};

inline ckpt_status check_given(const Given& g, int device, Known& known)
{
    if (g.rows == 0 || g.cols == 0) return CKPT_OK;
    if (!g.p) return fail_free(CKPT_EINVAL, "%s: null pointer", g.what);
    if ((uintptr_t)g.p % g.elem) return fail_free(CKPT_EINVAL, "%s: not aligned to its elements", g.what);
    if (g.rows > 1 && g.ld < g.cols)
        return fail_free(CKPT_EINVAL, "%s: rows of %llu elements are %llu apart", g.what, (unsigned long long)g.cols,
                         (unsigned long long)g.ld);
    if (g.ld > (1ull << 40)) return fail_free(CKPT_EINVAL, "%s: a stride of %llu", g.what, (unsigned long long)g.ld);
    const uint64_t p = (uint64_t)(uintptr_t)g.p;
    uint64_t bytes;
    if (!extent(g.rows, g.cols, g.ld, g.elem, &bytes)) return fail_free(CKPT_EINVAL, "%s: too large", g.what);
    if (known.holds(p, bytes)) return CKPT_OK;
    if (ckpt_status st = check_range(g.p, bytes, device, g.what)) return st;
    hipDeviceptr_t base = nullptr;
    size_t size = 0;
    if (hipMemGetAddressRange(&base, &size, (hipDeviceptr_t)g.p) == hipSuccess)
        known.add((uint64_t)(uintptr_t)base, size);
    else
        (void)hipGetLastError();
    return CKPT_OK;
}

} // namespace ckpt
