// Launchers of the operators at the two ends of a synchronisation and between hidden states and tokens (embedding.hip, grad.hip,
// mx4.hip, norm.hip, distill.hip, verify.hip, adapter.hip); ops_api.cpp
// checks arguments and calls them.  All return a hipError_t as int.
#pragma once

#include <cstddef>
#include <cstdint>

#include "rose_delta.h"

namespace rose {

constexpr int64_t kMostThreads = 0xFFFFFFFF;        // of a launch in one dimension

struct Tokens {
    const void *ids;
    int32_t wide;                       // 64-bit ids
    int64_t n;
    int64_t first_row;
    int64_t rows;                       // ids first_row .. first_row + rows - 1 are this table's
};

struct LookupArgs {
    Tokens tokens;
    const void *table;
    void *out;
    int64_t cols, table_stride, out_stride;
    float scale;
};
int launch_embedding_lookup(const LookupArgs &a, bool table_f32, bool out_f32, void *stream);

struct EmbeddingGradArgs {
    Tokens tokens;
    const void *dy;
    void *grad;
    int64_t cols, dy_stride, grad_stride;
    float scale;
    int32_t accumulate;
    char *workspace;
};
bool embedding_grad_fits(int64_t rows, int64_t cols, int64_t n_tokens, bool grad_f32);      // its sums into launches
size_t embedding_grad_workspace(int64_t rows, int64_t cols, int64_t n_tokens);
int launch_embedding_grad(const EmbeddingGradArgs &a, bool dy_f32, bool grad_f32, void *stream);

struct GradArgs {
    const void *const *grad_ptrs;
    void *const *out_ptrs;
    const int64_t *offsets;
    int32_t n_tensors;
    int64_t piece;                      // elements that a workgroup takes at a time
    double *partials;                   // sum of squares of each workgroup
    int32_t n_partials;
    double *sum;
    float max_norm;
    float *norm;
};
constexpr int kGradPartials = ROSE_GRAD_WORKSPACE_BYTES / 8;
int launch_grad_sum_squares(const GradArgs &a, int64_t total, bool f32, void *stream);
int launch_grad_clip(const GradArgs &a, int64_t total, bool f32, void *stream);
int launch_grad_clip_norm(const GradArgs &a, int64_t total, bool f32, void *stream);

int launch_mx4_quantize(const void *x, bool f32, int64_t rows, int64_t cols, int64_t stride, uint8_t *codes, uint8_t *scales,
                        void *stream);
int launch_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, void *out, bool f32,
                          int64_t stride, void *stream);
struct Mx4ProductArgs {
    const void *x;                      // bf16 activations that are quantised on the way, or null: then a_codes, a_scales
    int64_t x_stride;
    const uint8_t *a_codes, *a_scales, *w_codes, *w_scales;
    void *out;
    int64_t m, n, k, out_stride;
};
// whether a product of this size quantises bf16 activations by itself
bool mx4_product_takes_bf16(int64_t m, int64_t n, int64_t k);
bool mx4_product_fits(int64_t m, int64_t n, int64_t k);        // into launches
int launch_mx4_product(const Mx4ProductArgs &a, bool out_f32, void *stream);

struct NormArgs {
    const void *x, *weight, *bias;      // bias may be null
    void *out;
    int64_t rows, cols, x_stride, out_stride;
    float *mean, *rstd;                 // either may be null
    float eps;
    bool center, w_f32;
};
int launch_layer_norm(const NormArgs &a, bool x_f32, bool out_f32, void *stream);

struct NormGradArgs {
    const void *dy, *x, *weight;
    void *dx;                           // of x's type
    int64_t rows, cols, dy_stride, x_stride, dx_stride;
    const float *mean, *rstd;           // mean null: not centred
    float *dweight, *dbias;             // either may be null
    bool accumulate, w_f32;
    char *workspace;
};
size_t layer_norm_grad_workspace(int64_t rows, int64_t cols);
int launch_layer_norm_grad(const NormGradArgs &a, bool dy_f32, bool x_f32, void *stream);

struct DistillArgs {
    const void *logits;
    int64_t rows, cols, stride;
    const void *ids;
    int32_t wide;                       // 64-bit ids
    const float *teacher;
    int64_t top;
    double temperature;
    const float *d_loss;
    float *loss, *lse;
    void *d_logits;                     // of the logits' type
    int64_t d_stride;
    char *workspace;
    // the launchers': parts of a row that are summed, their columns and sums; chunks of a row whose gradient is written, their columns
    int32_t parts;
    int64_t piece, chunks, chunk;
    double *losses;
    struct Part {
        float most, sum;
    } *partials;
};
size_t distill_workspace(int64_t rows, int64_t cols);
int launch_distill_loss(const DistillArgs &a, bool f32, bool gradient, void *stream);
int launch_distill_grad(const DistillArgs &a, bool f32, void *stream);      // from lse

struct VerifyArgs {
    const void *target, *draft;         // draft may be null
    int64_t cols, target_stride, draft_stride;
    const void *drafted;
    int32_t wide;                       // 64-bit tokens
    int64_t n_drafted;
    const int64_t *offsets;
    int64_t requests;
    const float *uniforms;
    void *tokens;
    int32_t *accepted;
    double *sums;                       // of each part
    int64_t parts, part;                // the launcher's: parts of a row, and their columns
};
bool draft_verify_fits(int64_t requests, int64_t cols);        // into launches
size_t draft_verify_workspace(int64_t requests, int64_t cols);
int launch_draft_verify(const VerifyArgs &a, bool f32, void *stream);

struct bf16_t;
struct AdapterArgs {
    const void *x, *down, *up;
    const float *scales;                // may be null
    const void *chosen;
    int32_t wide;                       // 64-bit numbers of adapters
    void *out;
    int64_t m, n, k, rank, adapters, x_stride, out_stride;
    char *workspace;
    // the launcher's: what lies between the products, [splits][m][ranks]; rows in order of their adapters, and groups of them
    float *h;
    int64_t ranks, splits, share;       // ranks in whole tiles; parts of k, and elements of one
    int64_t columns;                    // of a workgroup
    int64_t units, group;               // groups of rows, at most; rows of one, at most
    bf16_t *cut;                        // scale * h in three numbers of 8 bits
    int32_t *order;
    struct Group {
        int32_t adapter, first, n;
    } *groups;
};
size_t adapter_linear_workspace(int64_t m, int64_t n, int64_t k, int64_t adapters, int64_t rank);
int launch_adapter_linear(const AdapterArgs &a, bool out_f32, void *stream);

}  // namespace rose
