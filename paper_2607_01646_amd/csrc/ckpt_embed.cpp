// ckpt_embed.cpp -- entry points of the vocabulary table
// (include/ckpt_embed.h): argument checks, the layout of the gradient's
// workspace, the order of launches.  Nothing is allocated and nothing outlives
// a call.
#include <algorithm>
#include <cmath>

#include "../../include/ckpt_embed.h"
#include "ops_host.h"
#include "ops_internal.h"

namespace ckpt {
namespace {

ckpt_status check_embed(const ckpt_embed_args* a, bool grad)
{
    if (!a) return fail_free(CKPT_EINVAL, "null argument");
    uint64_t e;
    if (!type_bytes(a->dtype, &e) || !type_bytes(a->table_dtype, &e))
        return fail_free(CKPT_EINVAL, "rows and table are bf16 or fp32, not types %u and %u", a->dtype, a->table_dtype);
    if (!grad && a->dtype != a->table_dtype) return fail_free(CKPT_EINVAL, "rows of another type than the table's");
    if (a->tokens > kMost || a->dim == 0 || a->dim > kMostWidth || a->vocab == 0 || a->vocab > kMostWidth)
        return fail_free(CKPT_EINVAL, "%llu tokens, %llu wide, %llu words: below 2^31, and 1 to 2^22 each",
                         (unsigned long long)a->tokens, (unsigned long long)a->dim, (unsigned long long)a->vocab);
    if (!std::isfinite((float)a->scale)) return fail_free(CKPT_EINVAL, "scale %g", a->scale);
    if (a->add > 1 || a->reserved || (a->add && !grad)) return fail_free(CKPT_EINVAL, "add is 0 or 1, and the gradient's; reserved is 0");
    return CKPT_OK;
}

// Where everything lies in the workspace.
struct GradPlan {
    bool few = false;
    uint32_t range = 0, chunk = 0;
    uint64_t start = 0, order = 0, word = 0, part = 0, part_ld = 0, join = 0, bytes = 0;
};

GradPlan plan_grad(const ckpt_embed_args* a)
{
    GradPlan l;
    const uint64_t n = a->tokens, columns = 1024 / (a->dtype == CKPT_TYPE_F32 ? 4 : 2), runs = (a->dim + columns - 1) / columns;
    // (A launch's lanes are counted in 32 bits.)
    l.few = n > 0 && n <= kFewRows && (a->vocab + 15) / 16 * runs <= 1u << 23;
    if (l.few) return l;
    // Sorting workgroups: each reads all ids, so no more than the GPU has units, unless LDS holds no more words.
    l.range = (uint32_t)std::min<uint64_t>(std::max<uint64_t>((a->vocab + 255) / 256, 32), kSortRange);
    // Sorted tokens that a wave sums: 64, or fewer down to 8 until each SIMD has two waves (8192 tokens of 4096: 61 us with the
    // table, with four waves 70), or as many as make 1024 chunks of a long batch.  Narrow rows have up to 4096 chunks
    // then (halved until there are 2048 or more), which bounds what is joined for a word that most tokens have.
    uint64_t chunk = std::max<uint64_t>(64, up((n + 1023) / 1024, 64));
    while (chunk > 8 && (n + chunk - 1) / chunk * runs < 2048) chunk /= 2;
    l.chunk = (uint32_t)chunk;
    l.part_ld = up(a->dim, 8);
    uint64_t at = 0;
    const auto take = [&](uint64_t bytes) {
        const uint64_t here = at;
        at += up(bytes, 256);
        return here;
    };
    l.start = take(4 * (a->vocab + 1));
    l.order = take(4 * n);
    l.word = take(4 * n);
    l.part = take(8 * l.part_ld * ((n + chunk - 1) / chunk));
    l.join = take(8 * ((n + chunk - 1) / chunk));
    l.bytes = at;
    return l;
}

ckpt_status check_pointers(const ckpt_embed_args* a, bool grad, int device, Known& known)
{
    const uint64_t e = a->dtype == CKPT_TYPE_F32 ? 4 : 2, te = a->table_dtype == CKPT_TYPE_F32 ? 4 : 2;
    const Given given[] = {{a->ids, a->tokens, 1, 1, 8, "ids"},
                           {a->rows, a->tokens, a->dim, a->rows_stride, e, "rows"},
                           {a->table, a->vocab, a->dim, a->table_stride, te, "table"}};
    for (const Given& g : given)
        if (ckpt_status st = check_given(g, device, known)) return st;
    // One is written while the other is read.
    uint64_t rows = 0, table = 0;
    extent(a->tokens, a->dim, a->rows_stride, e, &rows);
    extent(a->vocab, a->dim, a->table_stride, te, &table);
    const uint64_t r = (uint64_t)(uintptr_t)a->rows, t = (uint64_t)(uintptr_t)a->table;
    if (rows && r < t + table && t < r + rows) return fail_free(CKPT_EINVAL, "rows and table overlap");
    const uint64_t i = (uint64_t)(uintptr_t)a->ids, to = grad ? t : r, bytes = grad ? table : rows;
    if (a->tokens && i < to + bytes && to < i + 8 * a->tokens) return fail_free(CKPT_EINVAL, "ids overlap %s", grad ? "the table" : "rows");
    return CKPT_OK;
}

EmbedArgs embed_args(const ckpt_embed_args* a)
{
    EmbedArgs k = {};
    k.ids = a->ids;
    k.ignore_index = a->ignore_index;
    k.tokens = (uint32_t)a->tokens;
    k.dim = (uint32_t)a->dim;
    k.vocab = (uint32_t)a->vocab;
    k.scale = (float)a->scale;
    k.rows = a->rows;
    k.rows_ld = a->rows_stride;
    k.table = a->table;
    k.table_ld = a->table_stride;
    k.rows_f32 = a->dtype == CKPT_TYPE_F32;
    k.table_f32 = a->table_dtype == CKPT_TYPE_F32;
    k.add = a->add != 0;
    return k;
}

} // namespace
} // namespace ckpt

using namespace ckpt;

extern "C" ckpt_status ckpt_embedding(const ckpt_embed_args* a, int32_t device, void* stream)
{
    clear_free_error();
    if (ckpt_status st = check_embed(a, false)) return st;
    DeviceGuard dg;
    if (ckpt_status st = enter_device(device, dg)) return st;
    Known known;
    if (ckpt_status st = check_pointers(a, false, device, known)) return st;
    const hipError_t err = launch_lookup(embed_args(a), (hipStream_t)stream);
    if (err != hipSuccess) return fail_free(CKPT_EHIP, "lookup: %s", hipGetErrorString(err));
    return CKPT_OK;
}

extern "C" ckpt_status ckpt_embedding_grad_workspace(const ckpt_embed_args* a, uint64_t* bytes)
{
    clear_free_error();
    if (!bytes) return fail_free(CKPT_EINVAL, "null argument");
    if (ckpt_status st = check_embed(a, true)) return st;
    *bytes = plan_grad(a).bytes;
    return CKPT_OK;
}

extern "C" ckpt_status ckpt_embedding_grad(const ckpt_embed_args* a, int32_t device, void* workspace,
                                           uint64_t workspace_bytes, void* stream)
{
    clear_free_error();
    if (ckpt_status st = check_embed(a, true)) return st;
    const GradPlan l = plan_grad(a);
    if (l.bytes && (!workspace || (uintptr_t)workspace % 256)) return fail_free(CKPT_EINVAL, "workspace: null or not 256-byte aligned");
    if (workspace_bytes < l.bytes)
        return fail_free(CKPT_EINVAL, "workspace of %llu bytes needs %llu", (unsigned long long)workspace_bytes,
                         (unsigned long long)l.bytes);
    DeviceGuard dg;
    if (ckpt_status st = enter_device(device, dg)) return st;
    Known known;
    if (ckpt_status st = check_pointers(a, true, device, known)) return st;
    if (l.bytes)
        if (ckpt_status st = check_given({workspace, 1, l.bytes, l.bytes, 1, "workspace"}, device, known)) return st;
    uint8_t* w = (uint8_t*)workspace;
    EmbedArgs k = embed_args(a);
    k.range = l.range;
    k.chunk = l.chunk;
    k.start = (uint32_t*)(w + l.start);
    k.order = (uint32_t*)(w + l.order);
    k.word = (uint32_t*)(w + l.word);
    k.part = (float*)(w + l.part);
    k.part_ld = l.part_ld;
    k.join = (uint2*)(w + l.join);
    hipError_t err = l.few ? launch_few_sums(k, (hipStream_t)stream) : launch_sort(k, (hipStream_t)stream);
    if (err == hipSuccess && !l.few) err = launch_table_sums(k, (hipStream_t)stream);
    if (err != hipSuccess) return fail_free(CKPT_EHIP, "table's gradient: %s", hipGetErrorString(err));
    return CKPT_OK;
}
