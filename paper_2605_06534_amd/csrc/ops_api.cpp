// C ABI of the operators at the two ends of a synchronisation and between hidden states and tokens: argument checks and hand-off to the launchers.
#include "ops_internal.h"

namespace {

constexpr int64_t kMost = (int64_t)1 << 31;      // tokens, rows and columns are numbered in 31 bits

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

bool known(int32_t dtype) { return dtype == ROSE_DTYPE_BF16 || dtype == ROSE_DTYPE_F32; }

size_t size_of(int32_t dtype) { return dtype == ROSE_DTYPE_F32 ? 4 : 2; }

// A row-major matrix that the call touches if it has any elements.
rose_status check_matrix(const void *p, int32_t dtype, int64_t rows, int64_t cols, int64_t stride) {
    if (!known(dtype) || rows < 0 || cols < 0 || stride < cols) return ROSE_ERR_ARG;
    if (rows >= kMost || cols >= kMost) return ROSE_ERR_UNSUPPORTED;
    if (rows > 0 && cols > 0 && !p) return ROSE_ERR_ARG;
    return aligned(p, size_of(dtype)) ? ROSE_OK : ROSE_ERR_ALIGN;
}

rose_status check_tokens(const void *tokens, int32_t token_bytes, int64_t n, int64_t first_row) {
    if ((token_bytes != 4 && token_bytes != 8) || n < 0 || first_row < 0 || (n > 0 && !tokens)) return ROSE_ERR_ARG;
    if (n >= kMost) return ROSE_ERR_UNSUPPORTED;
    return aligned(tokens, (size_t)token_bytes) ? ROSE_OK : ROSE_ERR_ALIGN;
}

rose_status check_workspace(const void *workspace, size_t bytes, size_t need) {
    if (bytes < need || (need > 0 && !workspace)) return ROSE_ERR_ARG;
    return need == 0 || aligned(workspace, 256) ? ROSE_OK : ROSE_ERR_ALIGN;
}

rose_status check_grads(const void *const *ptrs, const int64_t *offsets, int32_t n_tensors, int64_t total, int32_t dtype) {
    if ((n_tensors > 0 && !ptrs) || !offsets || n_tensors < 0 || total < 0 || !known(dtype)) return ROSE_ERR_ARG;
    return aligned(ptrs, 8) && aligned(offsets, 8) ? ROSE_OK : ROSE_ERR_ALIGN;
}

// A matrix in blocks of 32 that share a scale.
rose_status check_mx4(const void *codes, const void *scales, int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0) return ROSE_ERR_ARG;
    if (rows >= kMost || cols >= kMost) return ROSE_ERR_UNSUPPORTED;
    if (rows > 0 && cols > 0 && (!codes || !scales)) return ROSE_ERR_ARG;
    return aligned(codes, 16) ? ROSE_OK : ROSE_ERR_ALIGN;
}

// What a product can address: a tile of 256 rows within 32 bits of bytes.
constexpr int64_t kMostProductCols = (int64_t)1 << 24;
rose_status check_product(int64_t m, int64_t n, int64_t k) {
    return k < kMostProductCols && rose::mx4_product_fits(m, n, k) ? ROSE_OK : ROSE_ERR_UNSUPPORTED;
}

rose_status status_of(int hip_error) { return hip_error == 0 ? ROSE_OK : ROSE_ERR_HIP; }

int64_t blocks_of(int64_t cols) { return (cols + ROSE_MX4_BLOCK - 1) / ROSE_MX4_BLOCK; }

size_t whole(size_t bytes) { return (bytes + 255) / 256 * 256; }

// The quantised activations of a product, where they go through memory: codes, then scales
size_t linear_workspace(int64_t m, int64_t k) { return whole((size_t)m * blocks_of(k) * 16) + whole((size_t)m * blocks_of(k)); }

}  // namespace

#define ROSE_CHECK(call)                          \
    do {                                          \
        const rose_status check_ = (call);        \
        if (check_ != ROSE_OK) return check_;     \
    } while (0)

extern "C" rose_status rose_embedding_lookup(const void *table, int32_t table_dtype, int64_t rows, int64_t cols,
                                             int64_t table_stride, const void *tokens, int32_t token_bytes, int64_t n_tokens,
                                             int64_t first_row, float scale, void *out, int32_t out_dtype,
                                             int64_t out_stride, void *stream) {
    ROSE_CHECK(check_matrix(table, table_dtype, rows, cols, table_stride));
    ROSE_CHECK(check_tokens(tokens, token_bytes, n_tokens, first_row));
    ROSE_CHECK(check_matrix(out, out_dtype, n_tokens, cols, out_stride));
    rose::LookupArgs a = {{tokens, token_bytes == 8, n_tokens, first_row, rows}, table, out, cols, table_stride, out_stride, scale};
    return status_of(rose::launch_embedding_lookup(a, table_dtype == ROSE_DTYPE_F32, out_dtype == ROSE_DTYPE_F32, stream));
}

extern "C" rose_status rose_embedding_grad_workspace_bytes(int64_t rows, int64_t cols, int64_t n_tokens, size_t *bytes) {
    if (!bytes || rows < 0 || cols < 0 || n_tokens < 0) return ROSE_ERR_ARG;
    if (rows >= kMost || cols >= kMost || n_tokens >= kMost) return ROSE_ERR_UNSUPPORTED;
    *bytes = rose::embedding_grad_workspace(rows, cols, n_tokens);
    return ROSE_OK;
}

extern "C" rose_status rose_embedding_grad(const void *dy, int32_t dy_dtype, int64_t dy_stride, const void *tokens,
                                           int32_t token_bytes, int64_t n_tokens, int64_t first_row, float scale, void *grad,
                                           int32_t grad_dtype, int64_t rows, int64_t cols, int64_t grad_stride,
                                           int32_t accumulate, void *workspace, size_t workspace_bytes, void *stream) {
    ROSE_CHECK(check_matrix(dy, dy_dtype, n_tokens, cols, dy_stride));
    ROSE_CHECK(check_tokens(tokens, token_bytes, n_tokens, first_row));
    ROSE_CHECK(check_matrix(grad, grad_dtype, rows, cols, grad_stride));
    ROSE_CHECK(check_workspace(workspace, workspace_bytes, rose::embedding_grad_workspace(rows, cols, n_tokens)));
    if (!rose::embedding_grad_fits(rows, cols, n_tokens, grad_dtype == ROSE_DTYPE_F32)) return ROSE_ERR_UNSUPPORTED;
    rose::EmbeddingGradArgs a = {{tokens, token_bytes == 8, n_tokens, first_row, rows}, dy, grad, cols, dy_stride, grad_stride,
                                 scale, accumulate != 0, static_cast<char *>(workspace)};
    return status_of(rose::launch_embedding_grad(a, dy_dtype == ROSE_DTYPE_F32, grad_dtype == ROSE_DTYPE_F32, stream));
}

extern "C" rose_status rose_grad_sum_squares(const void *const *grad_ptrs, const int64_t *offsets, int32_t n_tensors,
                                             int64_t total, int32_t dtype, double *sum, void *workspace,
                                             size_t workspace_bytes, void *stream) {
    ROSE_CHECK(check_grads(grad_ptrs, offsets, n_tensors, total, dtype));
    if (!sum) return ROSE_ERR_ARG;
    if (!aligned(sum, 8)) return ROSE_ERR_ALIGN;
    ROSE_CHECK(check_workspace(workspace, workspace_bytes, ROSE_GRAD_WORKSPACE_BYTES));
    rose::GradArgs a = {grad_ptrs, nullptr, offsets, n_tensors, 0, static_cast<double *>(workspace), 0, sum, 0.f, nullptr};
    return status_of(rose::launch_grad_sum_squares(a, total, dtype == ROSE_DTYPE_F32, stream));
}

extern "C" rose_status rose_grad_clip(const void *const *grad_ptrs, const int64_t *offsets, int32_t n_tensors, int64_t total,
                                      int32_t dtype, void *const *out_ptrs, const double *sum, float max_norm, float *norm,
                                      void *stream) {
    ROSE_CHECK(check_grads(grad_ptrs, offsets, n_tensors, total, dtype));
    if ((n_tensors > 0 && !out_ptrs) || !sum || !(max_norm >= 0.f)) return ROSE_ERR_ARG;
    if (!aligned(out_ptrs, 8) || !aligned(sum, 8) || !aligned(norm, 4)) return ROSE_ERR_ALIGN;
    rose::GradArgs a = {grad_ptrs, out_ptrs, offsets, n_tensors, 0, nullptr, 0, const_cast<double *>(sum), max_norm, norm};
    return status_of(rose::launch_grad_clip(a, total, dtype == ROSE_DTYPE_F32, stream));
}

extern "C" rose_status rose_grad_clip_norm(const void *const *grad_ptrs, const int64_t *offsets, int32_t n_tensors,
                                           int64_t total, int32_t dtype, void *const *out_ptrs, float max_norm, float *norm,
                                           void *workspace, size_t workspace_bytes, void *stream) {
    ROSE_CHECK(check_grads(grad_ptrs, offsets, n_tensors, total, dtype));
    if ((n_tensors > 0 && !out_ptrs) || !(max_norm >= 0.f)) return ROSE_ERR_ARG;
    if (!aligned(out_ptrs, 8) || !aligned(norm, 4)) return ROSE_ERR_ALIGN;
    ROSE_CHECK(check_workspace(workspace, workspace_bytes, ROSE_GRAD_WORKSPACE_BYTES));
    rose::GradArgs a = {grad_ptrs, out_ptrs, offsets, n_tensors, 0, static_cast<double *>(workspace), 0, nullptr, max_norm, norm};
    return status_of(rose::launch_grad_clip_norm(a, total, dtype == ROSE_DTYPE_F32, stream));
}

extern "C" rose_status rose_mx4_quantize(const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t stride,
                                         uint8_t *codes, uint8_t *scales, void *stream) {
    ROSE_CHECK(check_matrix(x, dtype, rows, cols, stride));
    ROSE_CHECK(check_mx4(codes, scales, rows, cols));
    return status_of(rose::launch_mx4_quantize(x, dtype == ROSE_DTYPE_F32, rows, cols, stride, codes, scales, stream));
}

extern "C" rose_status rose_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, void *out,
                                           int32_t dtype, int64_t stride, void *stream) {
    ROSE_CHECK(check_mx4(codes, scales, rows, cols));
    ROSE_CHECK(check_matrix(out, dtype, rows, cols, stride));
    return status_of(rose::launch_mx4_dequantize(codes, scales, rows, cols, out, dtype == ROSE_DTYPE_F32, stride, stream));
}

extern "C" rose_status rose_mx4_matmul(const uint8_t *a_codes, const uint8_t *a_scales, int64_t m, const uint8_t *w_codes,
                                       const uint8_t *w_scales, int64_t n, int64_t k, void *out, int32_t out_dtype,
                                       int64_t out_stride, void *stream) {
    ROSE_CHECK(check_mx4(a_codes, a_scales, m, k));
    ROSE_CHECK(check_mx4(w_codes, w_scales, n, k));
    ROSE_CHECK(check_product(m, n, k));
    ROSE_CHECK(check_matrix(out, out_dtype, m, n, out_stride));
    rose::Mx4ProductArgs a = {nullptr, 0, a_codes, a_scales, w_codes, w_scales, out, m, n, k, out_stride};
    return status_of(rose::launch_mx4_product(a, out_dtype == ROSE_DTYPE_F32, stream));
}

extern "C" rose_status rose_mx4_linear_workspace_bytes(int64_t m, int64_t n, int64_t k, size_t *bytes) {
    if (!bytes || m < 0 || n < 0 || k < 0) return ROSE_ERR_ARG;
    if (m >= kMost || n >= kMost || k >= kMost) return ROSE_ERR_UNSUPPORTED;
    *bytes = linear_workspace(m, k);
    return ROSE_OK;
}

extern "C" rose_status rose_mx4_linear(const void *x, int32_t x_dtype, int64_t m, int64_t x_stride, const uint8_t *w_codes,
                                       const uint8_t *w_scales, int64_t n, int64_t k, void *out, int32_t out_dtype,
                                       int64_t out_stride, void *workspace, size_t workspace_bytes, void *stream) {
    ROSE_CHECK(check_matrix(x, x_dtype, m, k, x_stride));
    ROSE_CHECK(check_mx4(w_codes, w_scales, n, k));
    ROSE_CHECK(check_product(m, n, k));
    ROSE_CHECK(check_matrix(out, out_dtype, m, n, out_stride));
    ROSE_CHECK(check_workspace(workspace, workspace_bytes, linear_workspace(m, k)));
    rose::Mx4ProductArgs a = {nullptr, 0, nullptr, nullptr, w_codes, w_scales, out, m, n, k, out_stride};
    if (m == 0 || n == 0) return ROSE_OK;
    if (x_dtype == ROSE_DTYPE_BF16 && rose::mx4_product_takes_bf16(m, n, k)) {
        a.x = x;
        a.x_stride = x_stride;
    } else {
        uint8_t *codes = static_cast<uint8_t *>(workspace), *scales = codes + whole((size_t)m * blocks_of(k) * 16);
        ROSE_CHECK(status_of(rose::launch_mx4_quantize(x, x_dtype == ROSE_DTYPE_F32, m, k, x_stride, codes, scales, stream)));
        a.a_codes = codes;
        a.a_scales = scales;
    }
    return status_of(rose::launch_mx4_product(a, out_dtype == ROSE_DTYPE_F32, stream));
}

extern "C" rose_status rose_layer_norm(const void *x, int32_t x_dtype, int64_t rows, int64_t cols, int64_t x_stride, const void *weight,
                                       const void *bias, int32_t weight_dtype, float eps, int32_t center, void *out, int32_t out_dtype,
                                       int64_t out_stride, float *mean, float *rstd, void *stream) {
    ROSE_CHECK(check_matrix(x, x_dtype, rows, cols, x_stride));
    ROSE_CHECK(check_matrix(out, out_dtype, rows, cols, out_stride));
    ROSE_CHECK(check_matrix(weight, weight_dtype, 1, cols, cols));
    if (cols == 0 || !(eps >= 0.f) || (bias && !center)) return ROSE_ERR_ARG;
    if (!aligned(bias, size_of(weight_dtype)) || !aligned(mean, 4) || !aligned(rstd, 4)) return ROSE_ERR_ALIGN;
    rose::NormArgs a = {x, weight, bias, out, rows, cols, x_stride, out_stride, mean, rstd, eps, center != 0, weight_dtype == ROSE_DTYPE_F32};
    return status_of(rose::launch_layer_norm(a, x_dtype == ROSE_DTYPE_F32, out_dtype == ROSE_DTYPE_F32, stream));
}

extern "C" rose_status rose_layer_norm_grad_workspace_bytes(int64_t rows, int64_t cols, size_t *bytes) {
    if (!bytes || rows < 0 || cols < 0) return ROSE_ERR_ARG;
    if (rows >= kMost || cols >= kMost) return ROSE_ERR_UNSUPPORTED;
    *bytes = rose::layer_norm_grad_workspace(rows, cols);
    return ROSE_OK;
}

extern "C" rose_status rose_layer_norm_grad(const void *dy, int32_t dy_dtype, int64_t dy_stride, const void *x, int32_t x_dtype,
                                            int64_t x_stride, int64_t rows, int64_t cols, const void *weight, int32_t weight_dtype,
                                            const float *mean, const float *rstd, void *dx, int64_t dx_stride, float *dweight,
                                            float *dbias, int32_t accumulate, void *workspace, size_t workspace_bytes, void *stream) {
    ROSE_CHECK(check_matrix(dy, dy_dtype, rows, cols, dy_stride));
    ROSE_CHECK(check_matrix(x, x_dtype, rows, cols, x_stride));
    ROSE_CHECK(check_matrix(dx, x_dtype, rows, cols, dx_stride));
    ROSE_CHECK(check_matrix(weight, weight_dtype, 1, cols, cols));
    if (cols == 0 || (rows > 0 && !rstd)) return ROSE_ERR_ARG;
    if (!aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dweight, 4) || !aligned(dbias, 4)) return ROSE_ERR_ALIGN;
    ROSE_CHECK(check_workspace(workspace, workspace_bytes, rose::layer_norm_grad_workspace(rows, cols)));
    rose::NormGradArgs a = {dy, x, weight, dx, rows, cols, dy_stride, x_stride, dx_stride, mean, rstd, dweight, dbias,
                            accumulate != 0, weight_dtype == ROSE_DTYPE_F32, static_cast<char *>(workspace)};
    return status_of(rose::launch_layer_norm_grad(a, dy_dtype == ROSE_DTYPE_F32, x_dtype == ROSE_DTYPE_F32, stream));
}

namespace {

// What the three forms of the distillation have in common.  (1 / temperature, times log2(e), is a normal number of fp32: infinite or zero it would
// make logits no numbers.)
rose_status check_distill(const void *logits, int32_t dtype, int64_t rows, int64_t cols, int64_t stride, const void *ids, int32_t id_bytes,
                          const float *teacher, int64_t top, double temperature) {
    const rose_status s = check_matrix(logits, dtype, rows, cols, stride);
    if (s != ROSE_OK) return s;
    if ((id_bytes != 4 && id_bytes != 8) || top < 0 || cols == 0 || !(temperature >= 0x1p-126 && temperature <= 0x1p126)) return ROSE_ERR_ARG;
    if (rows >= (1 << 22) || top > ROSE_DISTILL_MOST_TOP) return ROSE_ERR_UNSUPPORTED;
    if (rows > 0 && top > 0 && (!ids || !teacher)) return ROSE_ERR_ARG;
    return aligned(ids, (size_t)id_bytes) && aligned(teacher, 4) ? ROSE_OK : ROSE_ERR_ALIGN;
}

// A list of fp32 numbers that the call touches if it has any rows.
rose_status check_rows(const float *p, int64_t rows) { return rows > 0 && !p ? ROSE_ERR_ARG : aligned(p, 4) ? ROSE_OK : ROSE_ERR_ALIGN; }

}  // namespace

extern "C" rose_status rose_distill_workspace_bytes(int64_t rows, int64_t cols, size_t *bytes) {
    if (!bytes || rows < 0 || cols < 0) return ROSE_ERR_ARG;
    if (rows >= kMost || cols >= kMost) return ROSE_ERR_UNSUPPORTED;
    *bytes = rose::distill_workspace(rows, cols);
    return ROSE_OK;
}

extern "C" rose_status rose_distill_loss(const void *logits, int32_t dtype, int64_t rows, int64_t cols, int64_t stride, const void *ids,
                                         int32_t id_bytes, const float *teacher, int64_t top, double temperature, float *loss, float *lse,
                                         void *workspace, size_t workspace_bytes, void *stream) {
    ROSE_CHECK(check_distill(logits, dtype, rows, cols, stride, ids, id_bytes, teacher, top, temperature));
    ROSE_CHECK(check_rows(loss, rows));
    ROSE_CHECK(check_rows(lse, rows));
    ROSE_CHECK(check_workspace(workspace, workspace_bytes, rose::distill_workspace(rows, cols)));
    rose::DistillArgs a = {logits, rows, cols, stride, ids, id_bytes == 8, teacher, top, temperature, nullptr, loss, lse, nullptr, 0,
                           static_cast<char *>(workspace), 0, 0, 0, 0, nullptr, nullptr};
    return status_of(rose::launch_distill_loss(a, dtype == ROSE_DTYPE_F32, false, stream));
}

extern "C" rose_status rose_distill_loss_grad(const void *logits, int32_t dtype, int64_t rows, int64_t cols, int64_t stride, const void *ids,
                                              int32_t id_bytes, const float *teacher, int64_t top, double temperature, const float *d_loss,
                                              float *loss, float *lse, void *d_logits, int64_t d_stride, void *workspace,
                                              size_t workspace_bytes, void *stream) {
    ROSE_CHECK(check_distill(logits, dtype, rows, cols, stride, ids, id_bytes, teacher, top, temperature));
    ROSE_CHECK(check_matrix(d_logits, dtype, rows, cols, d_stride));
    ROSE_CHECK(check_rows(d_loss, rows));
    ROSE_CHECK(check_rows(loss, rows));
    ROSE_CHECK(check_rows(lse, rows));
    ROSE_CHECK(check_workspace(workspace, workspace_bytes, rose::distill_workspace(rows, cols)));
    rose::DistillArgs a = {logits, rows, cols, stride, ids, id_bytes == 8, teacher, top, temperature, d_loss, loss, lse, d_logits, d_stride,
                           static_cast<char *>(workspace), 0, 0, 0, 0, nullptr, nullptr};
    return status_of(rose::launch_distill_loss(a, dtype == ROSE_DTYPE_F32, true, stream));
}

extern "C" rose_status rose_distill_grad(const void *logits, int32_t dtype, int64_t rows, int64_t cols, int64_t stride, const void *ids,
                                         int32_t id_bytes, const float *teacher, int64_t top, double temperature, const float *lse,
                                         const float *d_loss, void *d_logits, int64_t d_stride, void *stream) {
    ROSE_CHECK(check_distill(logits, dtype, rows, cols, stride, ids, id_bytes, teacher, top, temperature));
    ROSE_CHECK(check_matrix(d_logits, dtype, rows, cols, d_stride));
    ROSE_CHECK(check_rows(lse, rows));
    ROSE_CHECK(check_rows(d_loss, rows));
    rose::DistillArgs a = {logits, rows, cols, stride, ids, id_bytes == 8, teacher, top, temperature, d_loss, nullptr,
                           const_cast<float *>(lse), d_logits, d_stride, nullptr, 0, 0, 0, 0, nullptr, nullptr};
    return status_of(rose::launch_distill_grad(a, dtype == ROSE_DTYPE_F32, stream));
}

extern "C" rose_status rose_draft_verify_workspace_bytes(int64_t requests, int64_t cols, size_t *bytes) {
    if (!bytes || requests < 0 || cols < 0) return ROSE_ERR_ARG;
    if (requests >= kMost || cols >= kMost) return ROSE_ERR_UNSUPPORTED;
    *bytes = rose::draft_verify_workspace(requests, cols);
    return ROSE_OK;
}

extern "C" rose_status rose_draft_verify(const void *target, int64_t target_stride, const void *draft, int64_t draft_stride, int32_t dtype,
                                         int64_t cols, const void *drafted, int32_t token_bytes, int64_t n_drafted, const int64_t *offsets,
                                         int64_t requests, const float *uniforms, void *tokens, int32_t *accepted, void *workspace,
                                         size_t workspace_bytes, void *stream) {
    if (n_drafted < 0 || requests < 0 || cols <= 0) return ROSE_ERR_ARG;
    if (n_drafted >= kMost || requests >= kMost || n_drafted + requests >= kMost) return ROSE_ERR_UNSUPPORTED;
    ROSE_CHECK(check_matrix(target, dtype, requests ? n_drafted + requests : 0, cols, target_stride));
    if (draft) ROSE_CHECK(check_matrix(draft, dtype, n_drafted, cols, draft_stride));
    ROSE_CHECK(check_tokens(drafted, token_bytes, n_drafted, 0));
    if (requests > 0 && (!offsets || !uniforms || !tokens || !accepted)) return ROSE_ERR_ARG;
    if (!aligned(offsets, 8) || !aligned(uniforms, 4) || !aligned(tokens, (size_t)token_bytes) || !aligned(accepted, 4)) return ROSE_ERR_ALIGN;
    ROSE_CHECK(check_workspace(workspace, workspace_bytes, rose::draft_verify_workspace(requests, cols)));
    if (!rose::draft_verify_fits(requests, cols)) return ROSE_ERR_UNSUPPORTED;
    rose::VerifyArgs a = {target, draft, cols, target_stride, draft_stride, drafted, token_bytes == 8, n_drafted, offsets, requests, uniforms,
                          tokens, accepted, static_cast<double *>(workspace), 0, 0};
    return status_of(rose::launch_draft_verify(a, dtype == ROSE_DTYPE_F32, stream));
}

namespace {

rose_status check_adapters(int64_t m, int64_t n, int64_t k, int64_t adapters, int64_t rank) {
    if (m < 0 || n < 0 || k < 0 || adapters < 0 || rank < 0) return ROSE_ERR_ARG;
    // (rows that go in groups of 64: those times pieces of ranks, or of columns, are workgroups)
    if (m > 128 && m >= 32 * adapters && m < (1 << 29) && n < kMost && rank <= ROSE_MOST_RANK) {
        const int64_t groups = m / 64 + adapters + 8;
        if (groups * ((rank + 31) / 32) >= (1 << 24) || groups * ((n + 127) / 128) >= (1 << 24)) return ROSE_ERR_UNSUPPORTED;
    }
    return m < (1 << 29) && n < kMost && k < kMost && adapters <= ROSE_MOST_ADAPTERS && rank <= ROSE_MOST_RANK ? ROSE_OK : ROSE_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" rose_status rose_adapter_linear_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t adapters, int64_t rank, size_t *bytes) {
    if (!bytes) return ROSE_ERR_ARG;
    ROSE_CHECK(check_adapters(m, n, k, adapters, rank));
    *bytes = rose::adapter_linear_workspace(m, n, k, adapters, rank);
    return ROSE_OK;
}

extern "C" rose_status rose_adapter_linear(const void *x, int64_t m, int64_t k, int64_t x_stride, const void *down, const void *up,
                                           const float *scales, int64_t adapters, int64_t rank, const void *chosen, int32_t chosen_bytes,
                                           void *out, int32_t out_dtype, int64_t n, int64_t out_stride, void *workspace,
                                           size_t workspace_bytes, void *stream) {
    ROSE_CHECK(check_adapters(m, n, k, adapters, rank));
    ROSE_CHECK(check_matrix(x, ROSE_DTYPE_BF16, m, k, x_stride));
    ROSE_CHECK(check_matrix(out, out_dtype, m, n, out_stride));
    ROSE_CHECK(check_tokens(chosen, chosen_bytes, m, 0));
    if (adapters > 0 && rank > 0 && ((k > 0 && !down) || (n > 0 && !up))) return ROSE_ERR_ARG;
    if (!aligned(down, 2) || !aligned(up, 2) || !aligned(scales, 4)) return ROSE_ERR_ALIGN;
    ROSE_CHECK(check_workspace(workspace, workspace_bytes, rose::adapter_linear_workspace(m, n, k, adapters, rank)));
    rose::AdapterArgs a = {};
    a.x = x, a.down = down, a.up = up, a.scales = scales, a.chosen = chosen, a.wide = chosen_bytes == 8, a.out = out;
    a.m = m, a.n = n, a.k = k, a.rank = rank, a.adapters = adapters, a.x_stride = x_stride, a.out_stride = out_stride;
    a.workspace = static_cast<char *>(workspace);
    return status_of(rose::launch_adapter_linear(a, out_dtype == ROSE_DTYPE_F32, stream));
}
