// Launchers of the operators at the two ends of a synchronisation (embedding.hip, grad.hip, mx4.hip); ops_api.cpp
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

}  // namespace rose
