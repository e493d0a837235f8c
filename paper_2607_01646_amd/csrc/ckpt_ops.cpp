// ckpt_ops.cpp -- entry points of the training-step operators
// (include/ckpt_ops.h): argument checks, the layout of the caller's workspace,
// the order of launches.  Nothing is allocated and nothing outlives a call.
#include <algorithm>
#include <cmath>

#include "../../include/ckpt_ops.h"
#include "ckpt_host.h"
#include "ops_internal.h"

namespace ckpt {
namespace {

constexpr uint64_t kMost = 0x7fffffffull;  // tokens
constexpr uint64_t kMostWidth = 1ull << 22; // dim, vocab: a tile's rows of an operand stay within 31 bits of bytes
constexpr uint64_t kDefaultPiece = 2ull << 30;
constexpr uint64_t kMostPiece = 1ull << 22; // tokens: a workgroup a row stays below 2^32 lanes
// For so few tokens d_logits has a second bf16 plane: gradients of few terms have no others to average their rounding
// with.  It doubles the gradients' products, in smaller tiles (256 x 4096 x 32000 0.45 ms; 512 tokens with one plane 0.49).
constexpr uint64_t kFewTokens = 256;
// So few tokens' weights are summed again by each workgroup that needs the sum.
constexpr uint64_t kFewSums = 1024;
constexpr uint64_t kAround = 64; // tokens of one small tile (a token's loss does not depend on how many are above that)
constexpr uint64_t kSliceBytes = 256ull << 20; // of the partial sums of a product cut along k

uint64_t up(uint64_t x, uint64_t a) { return (x + a - 1) / a * a; }

// Where everything lies in the workspace, and how the tokens are cut.
struct LossPlan {
    uint32_t planes = 1;      // of hidden and weight
    uint32_t dl_planes = 1;   // of d_logits
    uint64_t dim_pad = 0;     // width of copied operands
    uint64_t vocab_pad = 0;   // width of logits and d_logits
    uint64_t piece = 0;       // tokens in a piece
    uint32_t pieces = 0;
    bool grad = false, teach = false, held = false; // held: a piece's logits are written,
    bool e16 = false;                               // as exponentials in 16 bits where d_logits goes
    bool dots = false;
    bool copy_weight = false, copy_hidden = false, masked_hidden = false;
    bool two_sums = false; // the softmax at 1/temperature has sums of its own
    uint32_t parts = 0;
    uint32_t slices = 1;
    uint64_t row_weight = 0, target_logit = 0, scalars = 0, weight = 0, hidden = 0, part = 0, part_t = 0, logits = 0,
             d_logits = 0, sum = 0, join = 0, bytes = 0;
};

// The bytes of a [rows, cols] operand with rows `ld` elements apart; false where 64 bits do not count them.
bool extent(uint64_t rows, uint64_t cols, uint64_t ld, uint64_t elem, uint64_t* bytes)
{
    *bytes = 0;
    uint64_t last;
    return rows == 0 || (!__builtin_mul_overflow(rows - 1, ld, &last) && !__builtin_add_overflow(last, cols, &last) &&
                         !__builtin_mul_overflow(last, elem, bytes));
}

ckpt_status check_loss(const ckpt_linear_loss_args* a)
{
    if (!a) return fail_free(CKPT_EINVAL, "null argument");
    if (a->dtype != CKPT_TYPE_BF16 && a->dtype != CKPT_TYPE_F32)
        return fail_free(CKPT_EINVAL, "hidden and weight are bf16 or fp32, not type %u", a->dtype);
    if (a->reduction != CKPT_LOSS_MEAN && a->reduction != CKPT_LOSS_SUM)
        return fail_free(CKPT_EINVAL, "no reduction %u", a->reduction);
    if (a->tokens > kMost || a->dim == 0 || a->dim > kMostWidth || a->vocab == 0 || a->vocab > kMostWidth)
        return fail_free(CKPT_EINVAL, "%llu tokens, %llu wide, %llu words: below 2^31, and 1 to 2^22 each",
                         (unsigned long long)a->tokens, (unsigned long long)a->dim, (unsigned long long)a->vocab);
    if (a->topk > 1024) return fail_free(CKPT_EINVAL, "%u teacher entries: at most 1024", a->topk);
    if (a->topk) {
        // The kernels multiply by 1 / T, and by T twice.
        if (!(a->temperature > 0) || !std::isfinite(1 / a->temperature) || !std::isfinite(a->temperature * a->temperature))
            return fail_free(CKPT_EINVAL, "temperature %g: its inverse and its square are fp32 numbers", (double)a->temperature);
        if (!(a->alpha >= 0 && a->alpha <= 1)) return fail_free(CKPT_EINVAL, "alpha %g is not in [0, 1]", (double)a->alpha);
        if (a->teacher_dtype != CKPT_TYPE_BF16 && a->teacher_dtype != CKPT_TYPE_F32)
            return fail_free(CKPT_EINVAL, "teacher logits are bf16 or fp32, not type %u", a->teacher_dtype);
    }
    if (!a->target && (a->topk == 0 || a->alpha < 1) && a->tokens)
        return fail_free(CKPT_EINVAL, "no targets for the cross entropy");
    if (!a->d_hidden != !a->d_weight && a->tokens)
        return fail_free(CKPT_EINVAL, "both gradients or neither");
    const uint64_t e = a->dtype == CKPT_TYPE_F32 ? 4 : 2, te = a->teacher_dtype == CKPT_TYPE_F32 ? 4 : 2;
    const struct {
        uint64_t rows, cols, ld, elem;
        const char* what;
    } each[] = {{a->tokens, a->dim, a->hidden_stride, e, "hidden"},
                {a->vocab, a->dim, a->weight_stride, e, "weight"},
                {a->topk ? a->tokens : 0, a->topk, a->teacher_index_stride, 8, "teacher_index"},
                {a->topk ? a->tokens : 0, a->topk, a->teacher_logits_stride, te, "teacher_logits"},
                {a->d_hidden ? a->tokens : 0, a->dim, a->d_hidden_stride, e, "d_hidden"},
                {a->d_weight ? a->vocab : 0, a->dim, a->d_weight_stride, e, "d_weight"}};
    for (const auto& x : each) {
        uint64_t bytes;
        if (!extent(x.rows, x.cols, x.ld, x.elem, &bytes))
            return fail_free(CKPT_EINVAL, "%s: %llu rows, %llu elements apart, are beyond 64 bits", x.what,
                             (unsigned long long)x.rows, (unsigned long long)x.ld);
    }
    return CKPT_OK;
}

LossPlan plan_loss(const ckpt_linear_loss_args* a)
{
    LossPlan l;
    const bool f32 = a->dtype == CKPT_TYPE_F32;
    const uint64_t n = a->tokens, d = a->dim, v = a->vocab;
    l.planes = f32 ? 3 : 1;
    l.dim_pad = up(d, 64);
    l.vocab_pad = up(v, 64);
    l.grad = a->d_weight != nullptr;
    l.teach = a->topk != 0 && a->alpha > 0;
    l.held = l.grad || l.teach;
    l.two_sums = l.teach && a->temperature != 1;
    l.parts = (uint32_t)(up(v, kPartWords) / kPartWords);
    l.dl_planes = f32 ? 3 : n <= kFewTokens ? 2 : 1;
    l.e16 = l.grad && !l.teach && l.dl_planes == 1 && l.parts <= kE16Parts;
    const auto direct = [&](const void* p, uint64_t ld) { // as it is fit for the loads of a product
        return !f32 && d % 64 == 0 && ld % 8 == 0 && ld <= kMostWidth && (uintptr_t)p % 16 == 0;
    };
    l.dots = n <= kDotTokens || (f32 && !l.grad && n <= kDotTokensF32); // the logits come from the operands as they are
    l.copy_weight = !direct(a->weight, a->weight_stride) && !(l.dots && !l.grad);
    // With gradients the hidden states are copied so that those of rows that do not count are zero: the products over
    // the tokens multiply them by 0, and 0 * NaN is no 0.
    l.masked_hidden = l.grad && direct(a->hidden, a->hidden_stride); // by the row kernel
    l.copy_hidden = !direct(a->hidden, a->hidden_stride) && !(l.dots && !l.grad); // before the logits
    // What a token takes in the workspace: its logits and their gradient, its copy, its statistics, its label's logit.
    const uint64_t row = l.vocab_pad * ((l.held && !l.e16 ? 4 : 0) + (l.grad ? 2 * l.dl_planes : 0)) +
                         (l.copy_hidden || l.masked_hidden ? 2 * l.planes * l.dim_pad : 0) +
                         (l.two_sums ? 12 : 8) * l.parts + 4;
    const uint64_t budget = a->piece_bytes ? a->piece_bytes : kDefaultPiece;
    const auto fit = [&](uint64_t bytes) { // tokens, in whole tiles
        return std::min({n, std::max<uint64_t>(256, bytes / row / 64 * 64), kMostPiece});
    };
    l.piece = fit(budget);
    if (l.grad && n) {
        // The sums of d_hidden's runs are held for a piece's tokens too: room for those that all the tokens that fit would
        // have comes off the piece, at most a quarter of it, and what is left when it is cut bounds them.
        const auto runs = [&](uint64_t bytes) {
            return d_hidden_slices((uint32_t)d, (uint32_t)l.piece, (uint32_t)l.vocab_pad, l.planes, l.dl_planes,
                                   (uint32_t)std::min<uint64_t>(bytes / (4 * l.piece * l.dim_pad), 1u << 20));
        };
        const uint64_t most = std::min(kSliceBytes, budget / 4);
        l.slices = runs(most);
        const uint64_t sums = l.slices > 1 ? 4 * l.piece * l.dim_pad * l.slices : 0;
        if (sums && l.piece * row + sums > budget) {
            l.piece = fit(budget - sums);
            l.slices = runs(std::min(most, budget - std::min(budget, l.piece * row)));
        }
    }
    l.pieces = n ? (uint32_t)((n + l.piece - 1) / l.piece) : 0;
    const uint64_t piece_pad = up(l.piece, 64);

    uint64_t at = 0;
    const auto take = [&](uint64_t bytes) {
        const uint64_t here = at;
        at += up(bytes, 256);
        return here;
    };
    l.scalars = take(256);
    l.row_weight = take(4 * n);
    l.target_logit = take(4 * l.piece);
    if (l.copy_weight) l.weight = take(2ull * l.planes * v * l.dim_pad);
    if (l.copy_hidden || l.masked_hidden) l.hidden = take(2ull * l.planes * piece_pad * l.dim_pad);
    l.part = take(8ull * l.parts * l.piece);
    if (l.two_sums) l.part_t = take(4ull * l.parts * l.piece);
    if (l.held && !l.e16) l.logits = take(4 * l.piece * l.vocab_pad);
    if (l.grad) {
        l.d_logits = take(2ull * l.dl_planes * piece_pad * l.vocab_pad);
        if (l.pieces > 1) l.sum = take(4 * v * d);
        if (l.slices > 1) l.join = take(4 * l.piece * l.dim_pad * l.slices);
    }
    l.bytes = at;
    return l;
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

ckpt_status check_given(const Given& g, int device, Known& known)
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

} // namespace
} // namespace ckpt

using namespace ckpt;

extern "C" ckpt_status ckpt_linear_loss_workspace(const ckpt_linear_loss_args* a, uint64_t* bytes)
{
    clear_free_error();
    if (!bytes) return fail_free(CKPT_EINVAL, "null argument");
    if (ckpt_status st = check_loss(a)) return st;
    *bytes = plan_loss(a).bytes;
    return CKPT_OK;
}

extern "C" ckpt_status ckpt_linear_loss(const ckpt_linear_loss_args* a, int32_t device, void* workspace,
                                        uint64_t workspace_bytes, void* stream)
{
    clear_free_error();
    if (ckpt_status st = check_loss(a)) return st;
    const LossPlan l = plan_loss(a);
    if (!workspace || (uintptr_t)workspace % 256) return fail_free(CKPT_EINVAL, "workspace: null or not 256-byte aligned");
    if (workspace_bytes < l.bytes)
        return fail_free(CKPT_EINVAL, "workspace of %llu bytes needs %llu", (unsigned long long)workspace_bytes,
                         (unsigned long long)l.bytes);
    DeviceGuard dg;
    if (ckpt_status st = enter_device(device, dg)) return st;
    Known known;
    const bool f32 = a->dtype == CKPT_TYPE_F32;
    const uint64_t e = f32 ? 4 : 2, n = a->tokens, d = a->dim, v = a->vocab, k = a->topk;
    const uint64_t te = a->teacher_dtype == CKPT_TYPE_F32 ? 4 : 2;
    const Given given[] = {
        {a->hidden, n, d, a->hidden_stride, e, "hidden"},
        {a->weight, v, d, a->weight_stride, e, "weight"},
        {a->target, a->target ? n : 0, 1, 1, 8, "target"},
        {a->token_weight, a->token_weight ? n : 0, 1, 1, 4, "token_weight"},
        {a->teacher_index, n, k, a->teacher_index_stride, 8, "teacher_index"},
        {a->teacher_logits, n, k, a->teacher_logits_stride, te, "teacher_logits"},
        {a->grad_scale, a->grad_scale ? 1u : 0u, 1, 1, 4, "grad_scale"},
        {a->loss, 1, 1, 1, 4, "loss"},
        {a->token_loss, n, 1, 1, 4, "token_loss"},
        {a->lse, n, 1, 1, 4, "lse"},
        {a->d_hidden, a->d_hidden ? n : 0, d, a->d_hidden_stride, e, "d_hidden"},
        {a->d_weight, a->d_weight ? v : 0, d, a->d_weight_stride, e, "d_weight"},
        {workspace, 1, l.bytes, l.bytes, 1, "workspace"},
    };
    for (const Given& g : given)
        if (ckpt_status st = check_given(g, device, known)) return st;

    hipStream_t s = (hipStream_t)stream;
    uint8_t* w = (uint8_t*)workspace;
    float* scalars = (float*)(w + l.scalars);
    LossRows r = {};
    r.tokens = (uint32_t)n;
    r.vocab = (uint32_t)v;
    r.target = a->target;
    r.ignore_index = a->ignore_index;
    r.token_weight = a->token_weight;
    r.topk = l.teach ? a->topk : 0;
    r.t_index = a->teacher_index;
    r.t_index_ld = a->teacher_index_stride;
    r.t_logits = a->teacher_logits;
    r.t_logits_ld = a->teacher_logits_stride;
    r.t_f32 = a->teacher_dtype == CKPT_TYPE_F32;
    r.temperature = l.teach ? a->temperature : 1.0f;
    r.alpha = l.teach ? a->alpha : 0.0f;
    r.row_weight = (float*)(w + l.row_weight);
    r.token_loss = a->token_loss;
    r.lse = a->lse;
    r.loss = a->loss;
    r.scale = scalars;
    r.grad_scale = a->grad_scale;
    r.mean = a->reduction == CKPT_LOSS_MEAN;

    hipError_t err = hipSuccess;
#define CKPT_STEP(call, what)                                                                                      \
    do {                                                                                                           \
        if ((err = (call)) != hipSuccess) return fail_free(CKPT_EHIP, "%s: %s", what, hipGetErrorString(err));    \
    } while (0)

    Operand W = {(const uint16_t*)a->weight, 0, a->weight_stride, (uint32_t)v, (uint32_t)d};
    if (l.copy_weight && n) {
        const RowCopy c = {a->weight, a->weight_stride, (uint32_t)d, f32, (uint16_t*)(w + l.weight), v * l.dim_pad,
                           (uint32_t)l.dim_pad, (uint32_t)v};
        CKPT_STEP(launch_prepare(nullptr, 0, (uint32_t)v, c, s), "weight copy");
        W = {c.dst, c.plane, l.dim_pad, (uint32_t)v, (uint32_t)l.dim_pad};
    }
    if (l.pieces > 1) { // the gradients' factor has to be there before the last piece's rows are
        CKPT_STEP(launch_prepare(&r, 0, (uint32_t)n, RowCopy(), s), "row weights");
        CKPT_STEP(launch_finish(r, false, s), "scale");
    }
    for (uint32_t piece = 0; piece < l.pieces; ++piece) {
        const uint64_t row0 = piece * l.piece, rows = std::min(l.piece, n - row0), rows_pad = up(rows, 64);
        const uint8_t* h = (const uint8_t*)a->hidden + row0 * a->hidden_stride * e;
        Operand H = {(const uint16_t*)h, 0, a->hidden_stride, (uint32_t)rows, (uint32_t)d};
        RowCopy c = {a->hidden, a->hidden_stride, (uint32_t)d, f32, (uint16_t*)(w + l.hidden), rows_pad * l.dim_pad,
                     (uint32_t)l.dim_pad, (uint32_t)rows_pad};
        const Operand copied = {c.dst, c.plane, l.dim_pad, (uint32_t)rows_pad, (uint32_t)l.dim_pad};
        if (l.copy_hidden) {
            CKPT_STEP(launch_prepare(&r, (uint32_t)row0, (uint32_t)rows, c, s), "rows");
            H = copied;
        }
        if (!l.masked_hidden) c = {};

        LogitsOut lo = {};
        lo.vocab = (uint32_t)v;
        lo.tokens = (uint32_t)rows;
        lo.parts = l.parts;
        lo.target = r.target ? r.target + row0 : nullptr;
        lo.target_logit = (float*)(w + l.target_logit);
        lo.part = (float2*)(w + l.part);
        lo.part_t = l.two_sums ? (float*)(w + l.part_t) : nullptr;
        lo.inv_t = 1 / r.temperature;
        lo.logits = l.held && !l.e16 ? (float*)(w + l.logits) : nullptr;
        lo.e16 = l.e16 ? (uint16_t*)(w + l.d_logits) : nullptr;
        lo.ld = l.vocab_pad;
        if (l.dots)
            CKPT_STEP(launch_dots({a->weight, a->weight_stride}, {a->hidden, a->hidden_stride}, (uint32_t)d, f32, lo, s),
                      "logits");
        else
            CKPT_STEP(launch_logits(W, H, {(uint32_t)v, (uint32_t)rows, (uint32_t)l.dim_pad, 1, n <= kAround}, l.planes, lo, s),
                      "logits");

        LossPiece p = {};
        p.row0 = (uint32_t)row0;
        p.rows = (uint32_t)rows;
        p.parts = l.parts;
        p.part = lo.part;
        p.part_t = lo.part_t;
        p.logits = lo.logits;
        p.ld = l.vocab_pad;
        p.planes = l.dl_planes;
        p.e16 = l.e16;
        if (l.grad) {
            p.d_logits = (uint16_t*)(w + l.d_logits);
            p.dl_ld = l.vocab_pad;
            p.dl_plane = rows_pad * l.vocab_pad;
            p.dl_rows = (uint32_t)rows_pad;
        }
        r.target_logit = lo.target_logit - row0;
        CKPT_STEP(launch_rows(r, p, c, s), "loss rows");
        // Few tokens: one alone was summed with its row, some are summed by what uses their sums.
        const bool few = l.grad && n <= kFewSums && l.pieces == 1;
        if (piece + 1 == l.pieces && n > 1 && !few) CKPT_STEP(launch_finish(r, true, s), "loss");
        if (!l.grad) continue;
        if (l.masked_hidden) H = copied;

        const Operand dl_rows = {p.d_logits, p.dl_plane, l.vocab_pad, (uint32_t)rows_pad, (uint32_t)l.vocab_pad};
        GradOut g = {};
        g.scale = r.scale;
        if (few && n > 1) g.sums = {(uint32_t)n, r.row_weight, r.token_loss, r.grad_scale, r.loss, r.mean};
        g.f32 = f32;
        g.out = (uint8_t*)a->d_hidden + row0 * a->d_hidden_stride * e;
        g.ld = a->d_hidden_stride;
        GradOut gw = g;
        gw.total = few && n > 1;
        gw.out = a->d_weight;
        gw.ld = a->d_weight_stride;
        if (piece > 0) gw.add = (const float*)(w + l.sum), gw.add_ld = d;
        if (piece + 1 < l.pieces) {
            gw.out = w + l.sum;
            gw.ld = d;
            gw.f32 = true;
            gw.scale = nullptr;
        }
        GradOut gh = g;
        if (l.slices > 1) {
            gh = {};
            gh.out = w + l.join;
            gh.f32 = true;
            gh.ld = l.dim_pad;
            gh.slice = rows * l.dim_pad;
        }
        CKPT_STEP(launch_gradients(W, H, l.planes, dl_rows, l.dl_planes,
                                   {(uint32_t)d, (uint32_t)rows, (uint32_t)l.vocab_pad, l.slices, false}, gh,
                                   {(uint32_t)d, (uint32_t)v, (uint32_t)rows_pad, 1, false}, gw, s),
                  "gradients");
        if (l.slices > 1)
            CKPT_STEP(launch_join((const float*)gh.out, gh.slice, (uint32_t)l.dim_pad, l.slices, (uint32_t)d,
                                  (uint32_t)rows, g, s),
                      "d_hidden");
    }
    if (l.pieces == 0) { // no token: a loss of 0, and its gradient
        CKPT_STEP(launch_finish(r, true, s), "loss");
        if (l.grad) CKPT_STEP(launch_zero(a->d_weight, (uint32_t)v, (uint32_t)d, a->d_weight_stride, f32, s), "d_weight");
    }
#undef CKPT_STEP
    return CKPT_OK;
}

namespace {

bool type_bytes(uint32_t type, uint64_t* e)
{
    *e = type == CKPT_TYPE_F32 ? 4 : 2;
    return type == CKPT_TYPE_F32 || type == CKPT_TYPE_BF16;
}

} // namespace

extern "C" ckpt_status ckpt_grad_norm(const ckpt_tensor* grads, uint32_t n, uint32_t dtype, float max_norm, float* out,
                                      void* scratch, int32_t device, void* stream)
{
    clear_free_error();
    uint64_t e = 0;
    if (n && !grads) return fail_free(CKPT_EINVAL, "null argument");
    if (!type_bytes(dtype, &e)) return fail_free(CKPT_EINVAL, "gradients are bf16 or fp32, not type %u", dtype);
    if (std::isnan(max_norm)) return fail_free(CKPT_EINVAL, "max_norm is not a number");
    DeviceGuard dg;
    if (ckpt_status st = enter_device(device, dg)) return st;
    Known known;
    if (ckpt_status st = check_given({out, 1, 2, 2, 4, "out"}, device, known)) return st;
    if (ckpt_status st = check_given({scratch, 1, CKPT_GRAD_NORM_SCRATCH / 8, CKPT_GRAD_NORM_SCRATCH / 8, 8, "scratch"}, device, known)) return st;
    for (uint32_t i = 0; i < n; ++i) {
        if (grads[i].nbytes % e == 0 && (uintptr_t)grads[i].dev_ptr % e == 0 &&
            known.holds((uint64_t)(uintptr_t)grads[i].dev_ptr, grads[i].nbytes))
            continue;
        char what[32];
        snprintf(what, sizeof what, "gradient %u", i);
        if (grads[i].nbytes % e) return fail_free(CKPT_EINVAL, "%s: %llu bytes", what, (unsigned long long)grads[i].nbytes);
        const uint64_t c = grads[i].nbytes / e;
        if (ckpt_status st = check_given({grads[i].dev_ptr, 1, c, c, e, what}, device, known)) return st;
    }
    static_assert(CKPT_GRAD_NORM_SCRATCH == kNormBlocks * 8, "one sum for each workgroup");
    NormArgs a;
    a.count = a.tiles = 0;
    uint64_t total = 0;
    for (uint32_t i = 0; i < n; ++i) total += grads[i].nbytes / e;
    const bool few = n <= kNormFrags && total <= kNormFew;
    const uint64_t tile = few ? kNormFewTile : kNormTile;
    bool fresh = true;
    const auto flush = [&] {
        const hipError_t err = launch_norm(a, e == 4, fresh, (double*)scratch, (hipStream_t)stream);
        a.count = a.tiles = 0;
        fresh = false;
        return err;
    };
    hipError_t err = hipSuccess;
    for (uint32_t i = 0; i < n && err == hipSuccess; ++i) {
        // A fragment of more tiles than a launch counts goes in runs.
        constexpr uint64_t kRun = (uint64_t)kNormTile << 30;
        for (uint64_t at = 0, all = grads[i].nbytes / e; at < all && err == hipSuccess; at += kRun) {
            const uint64_t run = std::min(kRun, all - at), tiles = (run + tile - 1) / tile;
            if (a.count == kNormFrags || a.tiles + tiles > kMost) err = flush();
            a.f[a.count].ptr = (uint64_t)(uintptr_t)grads[i].dev_ptr + at * e;
            a.f[a.count].numel = run;
            a.first[a.count++] = a.tiles;
            a.tiles += (uint32_t)tiles;
        }
    }
    if (few && err == hipSuccess) err = launch_norm_few(a, e == 4, max_norm, out, (hipStream_t)stream);
    if (!few && err == hipSuccess && (a.count || fresh)) err = flush();
    if (!few && err == hipSuccess) err = launch_norm_finish((const double*)scratch, max_norm, out, (hipStream_t)stream);
    if (err != hipSuccess) return fail_free(CKPT_EHIP, "gradient norm: %s", hipGetErrorString(err));
    return CKPT_OK;
}

extern "C" ckpt_status ckpt_adamw(const ckpt_adamw_fragment* f, uint32_t n, uint32_t param_dtype, uint32_t grad_dtype,
                                  uint64_t step, double lr, double beta1, double beta2, double eps, double weight_decay,
                                  const float* grad_scale, int32_t device, void* stream)
{
    clear_free_error();
    uint64_t pe = 0, ge = 0;
    if (n && !f) return fail_free(CKPT_EINVAL, "null argument");
    if (!type_bytes(param_dtype, &pe) || !type_bytes(grad_dtype, &ge))
        return fail_free(CKPT_EINVAL, "parameters and gradients are bf16 or fp32, not types %u and %u", param_dtype, grad_dtype);
    if (step == 0) return fail_free(CKPT_EINVAL, "steps are counted from 1");
    if (!(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1))
        return fail_free(CKPT_EINVAL, "beta1 %g and beta2 %g are not in [0, 1)", beta1, beta2);
    if (!std::isfinite(lr) || !(eps >= 0) || !std::isfinite(eps) || !std::isfinite(weight_decay))
        return fail_free(CKPT_EINVAL, "lr %g, eps %g, weight_decay %g", lr, eps, weight_decay);
    DeviceGuard dg;
    if (ckpt_status st = enter_device(device, dg)) return st;
    Known known;
    if (grad_scale)
        if (ckpt_status st = check_given({grad_scale, 1, 1, 1, 4, "grad_scale"}, device, known)) return st;
    for (uint32_t i = 0; i < n; ++i) {
        const struct {
            const void* p;
            uint64_t e;
            const char* name;
        } part[] = {{f[i].param, pe, "param"}, {f[i].master, 4, "master"}, {f[i].exp_avg, 4, "exp_avg"},
                    {f[i].exp_avg_sq, 4, "exp_avg_sq"}, {f[i].grad, ge, "grad"}};
        if (f[i].numel > (1ull << 60)) return fail_free(CKPT_EINVAL, "fragment %u: %llu elements", i, (unsigned long long)f[i].numel);
        for (const auto& x : part) {
            if ((uintptr_t)x.p % x.e == 0 && known.holds((uint64_t)(uintptr_t)x.p, f[i].numel * x.e)) continue;
            char what[48];
            snprintf(what, sizeof what, "fragment %u, %s", i, x.name);
            if (ckpt_status st = check_given({x.p, 1, f[i].numel, f[i].numel, x.e, what}, device, known)) return st;
        }
    }
    AdamArgs a;
    a.count = a.tiles = 0;
    a.beta1 = (float)beta1;
    a.one_beta1 = (float)(1 - beta1);
    a.beta2 = (float)beta2;
    a.one_beta2 = (float)(1 - beta2);
    a.keep = (float)(1 - lr * weight_decay);
    a.lr = (float)lr;
    a.inv_bc1 = (float)(1 / (1 - std::pow(beta1, (double)step)));
    a.inv_bc2 = (float)(1 / (1 - std::pow(beta2, (double)step)));
    a.eps = (float)eps;
    a.scale = grad_scale;
    hipError_t err = hipSuccess;
    const auto flush = [&] {
        const hipError_t got = a.count ? launch_adamw(a, pe == 4, ge == 4, (hipStream_t)stream) : hipSuccess;
        a.count = a.tiles = 0;
        return got;
    };
    for (uint32_t i = 0; i < n && err == hipSuccess; ++i) {
        constexpr uint64_t kRun = (uint64_t)kAdamTile << 22; // at most 2^23 workgroups of 256 a launch: below 2^32 lanes
        for (uint64_t at = 0; at < f[i].numel && err == hipSuccess; at += kRun) {
            const uint64_t run = std::min(kRun, f[i].numel - at), tiles = (run + kAdamTile - 1) / kAdamTile;
            if (a.count == kAdamFrags || a.tiles + tiles > (1u << 23)) err = flush();
            auto& x = a.f[a.count];
            x.param = (uint64_t)(uintptr_t)f[i].param + at * pe;
            x.master = (uint64_t)(uintptr_t)(f[i].master + at);
            x.m = (uint64_t)(uintptr_t)(f[i].exp_avg + at);
            x.v = (uint64_t)(uintptr_t)(f[i].exp_avg_sq + at);
            x.grad = (uint64_t)(uintptr_t)f[i].grad + at * ge;
            x.numel = run;
            a.first[a.count++] = a.tiles;
            a.tiles += (uint32_t)tiles;
        }
    }
    if (err == hipSuccess) err = flush();
    if (err != hipSuccess) return fail_free(CKPT_EHIP, "optimizer step: %s", hipGetErrorString(err));
    return CKPT_OK;
}
