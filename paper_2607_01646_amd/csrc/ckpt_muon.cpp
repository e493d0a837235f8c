// ckpt_muon.cpp -- entry points of the orthogonalised optimizer step
// (include/ckpt_muon.h): argument checks, groups of matrices that the
// workspace holds, the order of launches.  Nothing is allocated but lists on
// the host, and nothing outlives a call.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "../../include/ckpt_muon.h"
#include "ops_host.h"
#include "ops_internal.h"

namespace ckpt {
namespace {

// Up to this short side it goes step by step, which is 17 launches for 5 steps, by twos (fits_twos) 19, and half the error.
// Above it what is quicker depends on the long side and on how many matrices a launch has (us step by step, by twos: one of
// 512 x 700 153, 167; one of 777 x 1003 177, 209; 32 of 512 x 512 544, 611; 16 of 512 x 1024 424, 419; a GPT's 16 of 512 x 512
// to 2048 693, 606; 2048 x 8192 1757, 1409).  A matrix's own short side decides: its bits may not depend on the others of the
// call, and matrices of two ways in one call would have the launches of both.
constexpr uint64_t kSingly = 448;
// What a short side decides for all matrices of a launch: groups hold matrices of one way alone.
uint32_t way(uint64_t s) { return (s > kSingly) + (s > kMuonAll); }
constexpr uint64_t kDefaultPiece = 4ull << 30; // the matrices of a layer of 4096 x 11008, in one group

// The largest that a singular value becomes, that a step multiplies one by, and that two steps do (NaN and infinity: as
// infinity).  They begin in [0, 1]; the operands' scale has room for 16.
struct Iterates {
    double value = 0, factor = 0, both = 0;
    explicit Iterates(const ckpt_newton_schulz& ns)
    {
        constexpr int kGrid = 128;
        double x[kGrid], before[kGrid] = {};
        for (int k = 0; k < kGrid; ++k) x[k] = (k + 1.0) / kGrid;
        factor = std::fabs(ns.a); // of values near 0
        both = ns.steps > 1 ? ns.a * ns.a : 0;
        bool fine = std::isfinite(ns.a) && std::isfinite(ns.b) && std::isfinite(ns.c);
        for (uint32_t i = 0; i < ns.steps && fine; ++i) {
            for (int k = 0; k < kGrid; ++k) { // side by side: this is part of every call
                const double s = x[k] * x[k], by = ns.a + s * (ns.b + s * ns.c);
                x[k] *= by;
                value = std::max(value, std::fabs(x[k]));
                factor = std::max(factor, std::fabs(by));
                both = std::max(both, std::fabs(by * before[k]));
                before[k] = by;
            }
            fine = value <= 1e3;
        }
        if (!fine) value = factor = both = INFINITY;
    }
};

ckpt_status check_ns(const ckpt_newton_schulz& ns)
{
    if (ns.steps < 1 || ns.steps > 64) return fail_free(CKPT_EINVAL, "%u steps: 1 to 64", ns.steps);
    if (ns.reserved) return fail_free(CKPT_EINVAL, "reserved is not 0");
    if (!(ns.eps >= 1e-30 && ns.eps <= 1)) return fail_free(CKPT_EINVAL, "eps %g is not in [1e-30, 1]", ns.eps);
    const Iterates it(ns);
    const bool fine = it.value <= 2 && it.factor <= 8;
    if (!fine)
        return fail_free(CKPT_EINVAL, "the polynomial %g x + %g x^3 + %g x^5 leaves [-2, 2], or multiplies a value by more than 8",
                         ns.a, ns.b, ns.c);
    return CKPT_OK;
}

// Whether all steps may be made from one Gram matrix in 64 bits: what its roundings leave in the place of a singular value
// of 0 grows by the square of a step's factor.
bool fits_thin(const ckpt_newton_schulz& ns) { return std::pow(Iterates(ns).factor, 2.0 * (ns.steps - 1)) <= 1e7; }

// Whether two steps are made from one Gram matrix: X's next is B A B (all are polynomials of A), and X is multiplied once,
// by the product of both factors.  Of the products with the long side that leaves 9 for 5 steps instead of 15, in units of
// s^2 l, and of those of the short side 11 instead of 5, in units of s^3.  A Gram matrix of X itself sets every other step
// right: 777 x 1003 is 3.1e-6 off, step by step 1.4e-6, by products in fp32 2.7e-6.  (With three from one, what is rounded off
// beside the large singular values grows in the small ones' place until it is all there is.)  The product of both factors has
// to fit the operands' scale.
bool fits_twos(const ckpt_newton_schulz& ns) { return Iterates(ns).both <= 14; }

// A matrix of the call, whichever entry point it is of.
struct Job {
    MuonMatrix m;
    uint64_t s, l;
    bool thin;
    uint64_t x, y, a, b, c, part; // offsets in the workspace
};

// Lays the operands of a matrix out from `at` on; false where 64 bits do not count them.
bool lay_out(Job& j, uint64_t rows, uint64_t cols, uint64_t& at)
{
    j.s = std::min(rows, cols);
    j.l = std::max(rows, cols);
    const uint64_t x = j.thin ? 8 * kThin * kThin : up(4 * j.s * up(j.l, 64), 256); // at most 2^46
    const uint64_t y = j.thin ? 0 : x, a = j.thin ? 0 : up(4 * j.s * up(j.s, 64), 256);
    const uint64_t tiles = ((rows + kMuonRows - 1) / kMuonRows) * ((cols + kMuonCols - 1) / kMuonCols);
    const uint64_t parts = j.thin ? std::min<uint64_t>((j.l + 255) / 256, kThinParts) : tiles;
    j.x = at;
    j.y = j.x + x;
    j.a = j.y + y;
    j.b = j.a + a;
    j.c = j.b + a;
    j.part = j.c + a;
    at = j.part + up(8 * parts * (j.thin ? kThin * kThin : 1), 256);
    j.m.rows = (uint32_t)rows;
    j.m.cols = (uint32_t)cols;
    j.m.part_n = (uint32_t)parts;
    return tiles <= (1u << 23);
}

// The matrices of a call by the way they go, which their own sides decide: a matrix's result does not depend on others.
struct Jobs {
    std::vector<Job> thin;   // short sides up to 16
    std::vector<Job> tiny;   // one launch, no workspace
    std::vector<Job> others;
};
Jobs sorted(const std::vector<Job>& jobs, const ckpt_newton_schulz& ns)
{
    Jobs to;
    const bool thin = fits_thin(ns);
    for (const Job& j : jobs) {
        const uint32_t s = std::min(j.m.rows, j.m.cols), l = std::max(j.m.rows, j.m.cols);
        std::vector<Job>& list = s <= kThin && thin ? to.thin : s <= kTinyShort && l <= kTinyLong ? to.tiny : to.others;
        list.push_back(j);
        list.back().thin = &list == &to.thin;
    }
    const auto of = [](const Job& j) { return way(std::min(j.m.rows, j.m.cols)); };
    std::stable_sort(to.others.begin(), to.others.end(), [&](const Job& x, const Job& y) { return of(x) > of(y); });
    return to;
}

// Cuts the matrices into groups: calls `run(first, last)` for each, and finds the bytes that the largest takes.
template <class F>
ckpt_status grouped(std::vector<Job>& jobs, uint64_t piece_bytes, uint64_t* most, F run)
{
    const uint64_t budget = piece_bytes ? piece_bytes : kDefaultPiece;
    *most = 0;
    for (size_t i = 0; i < jobs.size();) {
        uint64_t at = 0, tiles = 0;
        size_t k = i;
        for (; k < jobs.size() && k - i < kMuonMats; ++k) {
            uint64_t next = at;
            Job j = jobs[k];
            if (!lay_out(j, j.m.rows, j.m.cols, next))
                return fail_free(CKPT_EINVAL, "matrix of %u x %u: too many elements", j.m.rows, j.m.cols);
            tiles += std::max<uint64_t>(j.m.part_n, (j.s + 63) / 64 * ((j.l + 63) / 64)); // of any launch, at most
            if (k > i && (next > budget || tiles > (1u << 23) || way(j.s) != way(jobs[i].s))) break;
            if (tiles > (1u << 23)) return fail_free(CKPT_EINVAL, "matrix of %u x %u: too many elements", j.m.rows, j.m.cols);
            jobs[k] = j;
            at = next;
        }
        *most = std::max(*most, at);
        if (ckpt_status st = run(i, k)) return st;
        i = k;
    }
    return CKPT_OK;
}

ckpt_status nothing(size_t, size_t) { return CKPT_OK; }

// The bytes that all of a call needs: its groups run one behind the other.
ckpt_status needed(Jobs& jobs, uint64_t piece_bytes, uint64_t* bytes)
{
    uint64_t thin = 0;
    if (ckpt_status st = grouped(jobs.thin, piece_bytes, &thin, nothing)) return st;
    if (ckpt_status st = grouped(jobs.others, piece_bytes, bytes, nothing)) return st;
    *bytes = std::max(*bytes, thin);
    return CKPT_OK;
}

ckpt_status sizes(uint64_t rows, uint64_t cols, uint32_t i)
{
    if (rows > kMostWidth || cols > kMostWidth)
        return fail_free(CKPT_EINVAL, "matrix %u: %llu x %llu: at most 2^22 each", i, (unsigned long long)rows,
                         (unsigned long long)cols);
    return CKPT_OK;
}

void add_job(std::vector<Job>& jobs, uint64_t rows, uint64_t cols)
{
    Job j = {};
    j.m.rows = (uint32_t)rows;
    j.m.cols = (uint32_t)cols;
    jobs.push_back(j);
}

// The launches of all groups.  `a`: what they share.
ckpt_status run_all(const std::vector<Job>& all, MuonArgs& a, const ckpt_newton_schulz& ns, void* workspace,
                    uint64_t workspace_bytes, hipStream_t s)
{
    uint64_t need = 0;
    Jobs sides = sorted(all, ns);
    std::vector<Job>& jobs = sides.others;
    if (ckpt_status st = needed(sides, ns.piece_bytes, &need)) return st;
    if (need > workspace_bytes)
        return fail_free(CKPT_EINVAL, "workspace of %llu bytes needs %llu", (unsigned long long)workspace_bytes,
                         (unsigned long long)need);
    a.eps = ns.eps;
    uint8_t* w = (uint8_t*)workspace;
    const MuonPolynomial polynomial = {ns.a, ns.b, ns.c, ns.steps};
    const auto done = [](hipError_t err) {
        return err == hipSuccess ? CKPT_OK : fail_free(CKPT_EHIP, "orthogonalisation: %s", hipGetErrorString(err));
    };
    for (size_t i = 0; i < sides.tiny.size(); i += kMuonMats) {
        a.count = (uint32_t)std::min<size_t>(kMuonMats, sides.tiny.size() - i);
        for (uint32_t k = 0; k < a.count; ++k) a.m[k] = sides.tiny[i + k].m;
        if (ckpt_status st = done(launch_muon_tiny(a, polynomial, s))) return st;
    }
    const ckpt_status thin = grouped(sides.thin, ns.piece_bytes, &need, [&](size_t first, size_t last) {
        a.count = (uint32_t)(last - first);
        for (size_t k = first; k < last; ++k) {
            a.m[k - first] = sides.thin[k].m;
            a.m[k - first].part = (double*)(w + sides.thin[k].part);
            a.m[k - first].x = (uint16_t*)(w + sides.thin[k].x);
        }
        return done(launch_muon_thin(a, polynomial, s));
    });
    if (thin) return thin;
    const bool fits = fits_twos(ns);
    return grouped(jobs, ns.piece_bytes, &need, [&](size_t first, size_t last) {
        const bool twos = fits && jobs[first].s > kSingly;
        a.all = jobs[first].s <= kMuonAll;
        a.count = (uint32_t)(last - first);
        for (size_t k = first; k < last; ++k) {
            a.m[k - first] = jobs[k].m;
            a.m[k - first].part = (double*)(w + jobs[k].part);
            a.m[k - first].x = (uint16_t*)(w + jobs[k].x);
        }
        hipError_t err = launch_muon_first(a, s);
        if (err == hipSuccess) err = launch_muon_pack(a, s);
        const auto k_of = [](uint64_t Job::*p, const Job& j) { return (uint32_t)up(p == &Job::x || p == &Job::y ? j.l : j.s, 64); };
        // out = cb c + cc p q of all matrices, and with `poly` ca I in it.
        const auto tri = [&](uint64_t Job::*p, uint64_t Job::*q, uint64_t Job::*out, bool poly) {
            if (err != hipSuccess) return;
            TriArgs t = {};
            t.count = a.count;
            t.all = a.all;
            t.ca = (float)ns.a;
            t.cb = (float)ns.b;
            t.cc = poly ? (float)ns.c : 1.0f;
            for (size_t k = first; k < last; ++k) {
                const Job& j = jobs[k];
                const auto at = [&](uint64_t Job::*o) { return (uint16_t*)(w + j.*o); };
                const bool gram = p == &Job::x || p == &Job::y;
                const uint32_t k_all = k_of(p, j), chunk = muon_chunk(k_all, gram), s4 = (uint32_t)up(j.s, 4);
                // While the Gram matrix is made the other X holds nothing, and is as large as this one.
                const uint32_t slices = gram && (uint64_t)s4 * up(k_all, chunk) / chunk <= k_all ? (uint32_t)(up(k_all, chunk) / chunk) : 1;
                t.m[k - first] = {at(p), at(q), poly ? at(p) : nullptr, at(out), (uint32_t)j.s, k_all, 0, chunk,
                                  gram ? (float*)at(p == &Job::x ? &Job::y : &Job::x) : nullptr, slices};
            }
            err = launch_muon_tri(t, s);
        };
        uint64_t Job::*x = &Job::x, Job::*y = &Job::y, Job::*f;
        for (uint32_t step = 0; step < ns.steps && err == hipSuccess; std::swap(x, y)) {
            tri(x, x, &Job::a, false);
            tri(&Job::a, &Job::a, &Job::b, true);
            f = &Job::b;
            step += 1;
            if (twos && step < ns.steps) { // the next Gram matrix is B A B, and both factors are one
                tri(&Job::a, &Job::b, &Job::c, false);
                tri(&Job::c, &Job::b, &Job::a, false);
                tri(&Job::a, &Job::a, &Job::c, true);
                tri(&Job::c, &Job::b, &Job::a, false);
                f = &Job::a;
                step += 1;
            }
            if (err != hipSuccess) break;
            for (size_t k = first; k < last; ++k) {
                MuonMatrix& m = a.m[k - first];
                m = jobs[k].m;
                m.x = (uint16_t*)(w + jobs[k].*x);
                m.y = (uint16_t*)(w + jobs[k].*y);
                m.f = (uint16_t*)(w + jobs[k].*f);
            }
            err = launch_muon_apply(a, step == ns.steps, s);
        }
        return done(err);
    });
}

// Bytes [lo, hi): rows of `width`, `pitch` apart.
struct Span {
    uint64_t lo, hi, rows, width, pitch;
    bool written;
    Span(const void* p, uint64_t n, uint64_t cols, uint64_t ld, uint64_t e, bool w)
        : lo((uint64_t)(uintptr_t)p), rows(n), width(cols * e), pitch(ld * e), written(w)
    {
        if (n == 1 || ld == cols) rows = 1, width = pitch = n * cols * e;
        hi = lo + (rows - 1) * pitch + width;
    }
};

// Whether a row of x lies where one of y does; x begins first, and y within it.
bool meet(const Span& x, const Span& y)
{
    if (x.rows == 1 && y.rows == 1) return true;
    if (x.pitch == y.pitch) { // y's rows begin `in` bytes behind those of x from the `skip`-th on
        const uint64_t skip = (y.lo - x.lo) / x.pitch, in = (y.lo - x.lo) % x.pitch;
        return (in < x.width && skip < x.rows) || (in + y.width > x.pitch && skip + 1 < x.rows);
    }
    const Span &few = x.rows < y.rows ? x : y, &many = x.rows < y.rows ? y : x;
    for (uint64_t i = 0; i < few.rows; ++i) {
        const uint64_t lo = few.lo + i * few.pitch, hi = lo + few.width;
        // The first of the others' rows that ends behind lo.
        const uint64_t j = lo < many.lo + many.width ? 0 : (lo - many.lo - many.width) / many.pitch + 1;
        if (j < many.rows && many.lo + j * many.pitch < hi) return true;
    }
    return false;
}

// Whether something written lies where something else does.
bool overlap(std::vector<Span>& spans)
{
    std::sort(spans.begin(), spans.end(), [](const Span& x, const Span& y) { return x.lo < y.lo; });
    std::vector<const Span*> open; // that end behind the beginning of the next
    for (const Span& y : spans) {
        open.erase(std::remove_if(open.begin(), open.end(), [&](const Span* x) { return x->hi <= y.lo; }), open.end());
        for (const Span* x : open)
            if ((x->written || y.written) && meet(*x, y)) return true;
        open.push_back(&y);
    }
    return false;
}

ckpt_status check_workspace(void* workspace, uint64_t bytes, int device, Known& known)
{
    if (!workspace || (uintptr_t)workspace % 256) return fail_free(CKPT_EINVAL, "workspace: null or not 256-byte aligned");
    return check_given({workspace, 1, bytes, bytes, 1, "workspace"}, device, known);
}

ckpt_status orthogonalize_jobs(const ckpt_matrix* m, uint32_t n, const ckpt_newton_schulz* ns, std::vector<Job>& jobs)
{
    if (!ns || (n && !m)) return fail_free(CKPT_EINVAL, "null argument");
    if (ckpt_status st = check_ns(*ns)) return st;
    for (uint32_t i = 0; i < n; ++i) {
        if (ckpt_status st = sizes(m[i].rows, m[i].cols, i)) return st;
        if (m[i].rows && m[i].cols) add_job(jobs, m[i].rows, m[i].cols);
    }
    return CKPT_OK;
}

ckpt_status muon_jobs(const ckpt_muon_matrix* m, uint32_t n, const ckpt_muon_args* args, std::vector<Job>& jobs)
{
    if (!args || (n && !m)) return fail_free(CKPT_EINVAL, "null argument");
    uint64_t e;
    if (!type_bytes(args->param_dtype, &e) || !type_bytes(args->grad_dtype, &e))
        return fail_free(CKPT_EINVAL, "parameters and gradients are bf16 or fp32, not types %u and %u", args->param_dtype,
                         args->grad_dtype);
    if (args->nesterov > 1 || args->reserved) return fail_free(CKPT_EINVAL, "nesterov is 0 or 1, reserved 0");
    if (!(args->momentum >= 0 && args->momentum < 1)) return fail_free(CKPT_EINVAL, "momentum %g is not in [0, 1)", args->momentum);
    if (!std::isfinite(args->lr) || !std::isfinite(args->weight_decay) || !std::isfinite((float)(1 - args->lr * args->weight_decay)))
        return fail_free(CKPT_EINVAL, "lr %g, weight_decay %g", args->lr, args->weight_decay);
    if (ckpt_status st = check_ns(args->ns)) return st;
    for (uint32_t i = 0; i < n; ++i) {
        if (ckpt_status st = sizes(m[i].rows, m[i].cols, i)) return st;
        if (!std::isfinite((float)(args->lr * m[i].scale))) return fail_free(CKPT_EINVAL, "matrix %u: scale %g", i, m[i].scale);
        if (m[i].rows && m[i].cols) add_job(jobs, m[i].rows, m[i].cols);
    }
    return CKPT_OK;
}

// Nothing is thrown past an entry point.
template <class F>
ckpt_status guarded(F f)
{
    clear_free_error();
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return fail_free(CKPT_EINVAL, "no host memory for the list of matrices");
    }
}

} // namespace
} // namespace ckpt

using namespace ckpt;

extern "C" ckpt_status ckpt_orthogonalize_workspace(const ckpt_matrix* m, uint32_t n, const ckpt_newton_schulz* ns,
                                                    uint64_t* bytes)
{
    return guarded([&]() -> ckpt_status {
        std::vector<Job> jobs;
        if (!bytes) return fail_free(CKPT_EINVAL, "null argument");
        if (ckpt_status st = orthogonalize_jobs(m, n, ns, jobs)) return st;
        Jobs sides = sorted(jobs, *ns);
        return needed(sides, ns->piece_bytes, bytes);
    });
}

extern "C" ckpt_status ckpt_orthogonalize(const ckpt_matrix* m, uint32_t n, uint32_t dtype, const ckpt_newton_schulz* ns,
                                          int32_t device, void* workspace, uint64_t workspace_bytes, void* stream)
{
    return guarded([&]() -> ckpt_status {
        std::vector<Job> jobs;
        uint64_t e = 0;
        if (!type_bytes(dtype, &e)) return fail_free(CKPT_EINVAL, "matrices are bf16 or fp32, not type %u", dtype);
        if (ckpt_status st = orthogonalize_jobs(m, n, ns, jobs)) return st;
        DeviceGuard dg;
        if (ckpt_status st = enter_device(device, dg)) return st;
        Known known;
        std::vector<Span> spans;
        size_t at = 0;
        for (uint32_t i = 0; i < n; ++i) {
            const uint64_t rows = m[i].rows, cols = m[i].cols;
            if (!rows || !cols) continue;
            char what[48];
            snprintf(what, sizeof what, "matrix %u", i);
            if (ckpt_status st = check_given({m[i].in, rows, cols, m[i].in_stride, e, what}, device, known)) return st;
            snprintf(what, sizeof what, "matrix %u, its result", i);
            if (ckpt_status st = check_given({m[i].out, rows, cols, m[i].out_stride, e, what}, device, known)) return st;
            spans.emplace_back(m[i].out, rows, cols, m[i].out_stride, e, true);
            if (m[i].in != m[i].out || (rows > 1 && m[i].in_stride != m[i].out_stride))
                spans.emplace_back(m[i].in, rows, cols, m[i].in_stride, e, false);
            MuonMatrix& to = jobs[at++].m;
            to.in = m[i].in;
            to.in_ld = m[i].in_stride;
            to.out = m[i].out;
            to.out_ld = m[i].out_stride;
        }
        if (jobs.empty()) return CKPT_OK;
        if (overlap(spans)) return fail_free(CKPT_EINVAL, "a result overlaps another matrix");
        if (workspace_bytes)
            if (ckpt_status st = check_workspace(workspace, workspace_bytes, device, known)) return st;
        MuonArgs a = {};
        a.in_f32 = a.out_f32 = e == 4;
        return run_all(jobs, a, *ns, workspace, workspace_bytes, (hipStream_t)stream);
    });
}

extern "C" ckpt_status ckpt_muon_workspace(const ckpt_muon_matrix* m, uint32_t n, const ckpt_muon_args* args, uint64_t* bytes)
{
    return guarded([&]() -> ckpt_status {
        std::vector<Job> jobs;
        if (!bytes) return fail_free(CKPT_EINVAL, "null argument");
        if (ckpt_status st = muon_jobs(m, n, args, jobs)) return st;
        Jobs sides = sorted(jobs, args->ns);
        return needed(sides, args->ns.piece_bytes, bytes);
    });
}

extern "C" ckpt_status ckpt_muon(const ckpt_muon_matrix* m, uint32_t n, const ckpt_muon_args* args, int32_t device,
                                 void* workspace, uint64_t workspace_bytes, void* stream)
{
    return guarded([&]() -> ckpt_status {
        std::vector<Job> jobs;
        if (ckpt_status st = muon_jobs(m, n, args, jobs)) return st;
        uint64_t pe = 0, ge = 0;
        type_bytes(args->param_dtype, &pe);
        type_bytes(args->grad_dtype, &ge);
        DeviceGuard dg;
        if (ckpt_status st = enter_device(device, dg)) return st;
        Known known;
        if (args->grad_scale)
            if (ckpt_status st = check_given({args->grad_scale, 1, 1, 1, 4, "grad_scale"}, device, known)) return st;
        std::vector<Span> spans;
        if (args->grad_scale) spans.emplace_back(args->grad_scale, 1, 1, 1, 4, false); // launches behind the first read it again
        size_t at = 0;
        for (uint32_t i = 0; i < n; ++i) {
            const uint64_t all = m[i].rows * m[i].cols;
            if (!all) continue;
            const struct {
                const void* p;
                uint64_t e;
                bool written;
                const char* name;
            } part[] = {{m[i].param, pe, true, "param"}, {m[i].master, 4, true, "master"},
                        {m[i].momentum, 4, true, "momentum"}, {m[i].grad, ge, false, "grad"}};
            for (const auto& x : part) {
                const uint64_t p = (uint64_t)(uintptr_t)x.p;
                if (p % x.e || !known.holds(p, all * x.e)) {
                    char what[48];
                    snprintf(what, sizeof what, "matrix %u, %s", i, x.name);
                    if (ckpt_status st = check_given({x.p, 1, all, all, x.e, what}, device, known)) return st;
                }
                // A parameter in full precision may be its own master copy.
                if (&x == part && m[i].param == (void*)m[i].master && pe == 4) continue;
                spans.emplace_back(x.p, 1, all, all, x.e, x.written);
            }
            MuonMatrix& to = jobs[at++].m;
            to.in = m[i].grad;
            to.momentum = m[i].momentum;
            to.master = m[i].master;
            to.out = m[i].param;
            to.in_ld = to.out_ld = m[i].cols;
            to.scale = (float)(args->lr * m[i].scale);
        }
        if (jobs.empty()) return CKPT_OK;
        if (overlap(spans)) return fail_free(CKPT_EINVAL, "fragments overlap");
        if (workspace_bytes)
            if (ckpt_status st = check_workspace(workspace, workspace_bytes, device, known)) return st;
        MuonArgs a = {};
        a.beta = (float)args->momentum;
        a.one_beta = (float)(1 - args->momentum);
        a.keep = (float)(1 - args->lr * args->weight_decay);
        a.grad_scale = args->grad_scale;
        a.nesterov = args->nesterov != 0;
        a.in_f32 = ge == 4;
        a.out_f32 = pe == 4;
        return run_all(jobs, a, args->ns, workspace, workspace_bytes, (hipStream_t)stream);
    });
}
