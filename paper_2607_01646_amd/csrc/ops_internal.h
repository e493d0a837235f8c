// Internal interface between the training-step operators (ckpt_ops.cpp) and
// their gfx950 kernels.  Not installed; the public ABI is include/ckpt_ops.h.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ckpt {

// ---- products on the matrix cores (loss_kernels.hip) ----

// One operand of out[q][p] = sum_k P(p, k) Q(q, k): bf16, as 1 plane or as the
// 3 whose sum is an fp32 value.  Rows are 16-byte aligned (base and ld), ld is
// at most 2^22.
//   k contiguous:     element (r, k) at base[r * ld + k]; row indices are
//                     clamped below `rows`, k runs to a multiple of 64
//   k across rows:    element (r, k) at base[k * ld + r]; k is clamped below
//                     `rows`, r to `cols`, a multiple of 8
// What a clamp repeats only reaches outputs that are not written, or meets
// zeros of the other operand.
struct Operand {
    const uint16_t* base;
    uint64_t plane; // elements between planes
    uint64_t ld;
    uint32_t rows, cols;
};

struct ProductShape {
    uint32_t p, q, k; // k: a multiple of 64
    uint32_t slices;  // k is cut into this many runs, each a product of its own
    // Each workgroup begins at another value of k.  For few tokens, when the rows of P are a workgroup's own: they lie a
    // power of two apart for most heads, and workgroups at the same place in them wait for the same memory channels.
    bool around;
};

// What becomes of a tile of l = P Q: the logits' statistics.
struct LogitsOut {
    uint32_t vocab, tokens, parts;
    const int64_t* target; // or nullptr
    float* target_logit;   // [tokens], written where the target is a word
    float2* part;          // [tokens][parts]: (max, sum exp(l - max)) over each run of kPartWords words
    float* part_t;         // the same sum at 1/temperature, or nullptr
    float inv_t;
    float* logits; // [tokens][ld], or nullptr
    uint16_t* e16; // [tokens][ld] exp(l - its part's max) in 16 bits, or nullptr
    uint64_t ld;   // a multiple of kPartWords
};
constexpr uint32_t kPartWords = 64;
constexpr uint32_t kE16Parts = 8192; // of a row held in 16 bits: their factors fit in LDS

// Where the factor that all rows share and the loss come from when no launch
// has made them (tokens == 0: one has).
struct LossSums {
    uint32_t tokens;
    const float *row_weight, *token_loss, *grad_scale; // grad_scale or nullptr
    float* loss;
    bool mean;
};

// What becomes of a product that is a gradient (or a slice of one).
struct GradOut {
    LossSums sums;      // with tokens: the factor is made of these, not *scale
    bool total;         // ... and the loss written
    const float* scale; // multiplies the sum; nullptr = 1
    const float* add;   // [q][add_ld] added to the product before the scale, or nullptr
    uint64_t add_ld;
    void* out; // [q][ld]; with slices > 1: fp32 [slices][q][ld]
    uint64_t ld, slice;
    bool f32; // type of out
};

hipError_t launch_logits(const Operand& w, const Operand& h, const ProductShape& s, uint32_t planes,
                         const LogitsOut& o, hipStream_t stream);
// The same for few tokens, from the caller's own operands (any alignment of
// their elements).  Up to kDotTokens; fp32 without gradients, where the
// operands' planes would be made for this product alone, kDotTokensF32 (each 8
// of them read the weight once more: 32000 x 4096 0.12 ms, the planes 0.45 ms).
constexpr uint32_t kDotTokens = 4, kDotTokensF32 = 24;
struct DotOperand {
    const void* base;
    uint64_t ld;
};
hipError_t launch_dots(const DotOperand& w, const DotOperand& h, uint32_t dim, bool f32, const LogitsOut& o,
                       hipStream_t stream);
// Both gradients, in one launch where they are small:
//   d_hidden: P = weight (k = words across rows), Q = d_logits (k contiguous)
//   d_weight: P = hidden, Q = d_logits (both with k = tokens across rows)
// zp, zq: planes of P and Q; (1, 1), (1, 2) or (3, 3).
hipError_t launch_gradients(const Operand& w, const Operand& h, uint32_t zp, const Operand& dl, uint32_t zq,
                            const ProductShape& dh, const GradOut& dho, const ProductShape& dw, const GradOut& dwo,
                            hipStream_t stream);
// out = scale * sum of the n slices (fp32 [n][q][ld_s], `slice` apart; ld_s a multiple of 4)
hipError_t launch_join(const float* slices, uint64_t slice, uint32_t ld_s, uint32_t n, uint32_t p, uint32_t q,
                       const GradOut& o, hipStream_t stream);
hipError_t launch_zero(void* out, uint32_t rows, uint32_t cols, uint64_t ld, bool f32, hipStream_t stream);
// Into how many runs of k to cut d_hidden, at most `most`.
uint32_t d_hidden_slices(uint32_t p, uint32_t q, uint32_t k, uint32_t zp, uint32_t zq, uint32_t most);

// ---- rows of the loss (loss_kernels.hip) ----

struct LossRows {
    uint32_t tokens, vocab;
    const int64_t* target; // or nullptr
    int64_t ignore_index;
    const float* token_weight; // or nullptr
    uint32_t topk;
    const int64_t* t_index;
    uint64_t t_index_ld;
    const void* t_logits;
    uint64_t t_logits_ld;
    bool t_f32;
    float temperature, alpha; // alpha: 0 without a teacher
    float* row_weight;        // [tokens]: the weight of a row that counts, else 0
    float* target_logit;
    float *token_loss, *lse;
    float *loss, *scale; // scalars: the loss; grad_scale over the weights' sum
    const float* grad_scale;
    bool mean;
};

// Copies rows [row0, row0 + rows) of src, fp32 into 3 planes, with zeros to
// the width dst_cols and in rows up to dst_rows; src == nullptr copies
// nothing.  With r != nullptr also computes row_weight of those rows, and
// copies rows that do not count as zeros.
struct RowCopy {
    const void* src;
    uint64_t src_ld;
    uint32_t cols;
    bool f32;
    uint16_t* dst;
    uint64_t plane;
    uint32_t dst_cols, dst_rows;
};
hipError_t launch_prepare(const LossRows* r, uint32_t row0, uint32_t rows, const RowCopy& c, hipStream_t stream);

// From the statistics of `parts` runs of words to row_weight, token_loss and
// lse of rows [row0, row0 + rows); part, part_t and logits are the piece's own.
// With d_logits also writes its rows ([planes][.][dl_ld], dl_rows of them:
// zeros beyond the vocabulary and beyond `rows`); e16: from the exponentials
// that d_logits holds.  With copy.src (bf16, 16-byte aligned rows of dst_cols)
// also copies those rows, zeros for the ones that do not count.
struct LossPiece {
    uint32_t row0, rows, parts;
    const float2* part;
    const float* part_t;
    const float* logits;
    uint64_t ld;
    uint16_t* d_logits;
    uint64_t dl_ld, dl_plane;
    uint32_t dl_rows, planes;
    bool e16;
};
hipError_t launch_rows(const LossRows& r, const LossPiece& p, const RowCopy& copy, hipStream_t stream);
// scale (from row_weight) and, if `total`, the loss.  (launch_rows makes both of
// one token.)
hipError_t launch_finish(const LossRows& r, bool total, hipStream_t stream);

// ---- optimizer (optim_kernels.hip) ----

constexpr uint32_t kAdamFrags = 64; // per launch; their tiles' first numbers fit one wave
struct AdamArgs {
    struct {
        uint64_t param, master, m, v, grad, numel;
    } f[kAdamFrags];
    uint32_t first[kAdamFrags]; // first tile of each fragment
    uint32_t count, tiles;
    float beta1, one_beta1, beta2, one_beta2, keep, lr, inv_bc1, inv_bc2, eps;
    const float* scale;
};
constexpr uint32_t kAdamTile = 1024;
hipError_t launch_adamw(const AdamArgs& a, bool param_f32, bool grad_f32, hipStream_t stream);

constexpr uint32_t kNormFrags = 160;
struct NormArgs {
    struct {
        uint64_t ptr, numel;
    } f[kNormFrags];
    uint32_t first[kNormFrags];
    uint32_t count, tiles;
};
constexpr uint32_t kNormTile = 8192, kNormBlocks = 2048;
// Adds the fragments' squares to part (kNormBlocks sums; `fresh`: stores them).
hipError_t launch_norm(const NormArgs& a, bool f32, bool fresh, double* part, hipStream_t stream);
// All of it, by one workgroup whose 16 waves take a tile of kNormFewTile each at a time: for so few elements that a
// second launch takes longer.
constexpr uint32_t kNormFewTile = 2048, kNormFew = 64 * kNormFewTile;
hipError_t launch_norm_few(const NormArgs& a, bool f32, double max_norm, float* out, hipStream_t stream);
hipError_t launch_norm_finish(const double* part, double max_norm, float* out, hipStream_t stream);

} // namespace ckpt
