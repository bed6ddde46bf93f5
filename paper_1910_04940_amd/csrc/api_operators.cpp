// extern "C" boundary of the operators around the collectives: argument checks.
#include <cmath>

#include "operators_api.hpp"

namespace {

constexpr size_t kMostTokens = 0x7fffffff, kMostDim = size_t{1} << 21, kMostSide = size_t{1} << 20, kMostBatch = 65535;
constexpr int kMostExperts = 1024, kMostSteps = 64;

bool is_token(blink_dtype_t t) { return t == BLINK_INT32 || t == BLINK_INT64; }
// A buffer of elements of `size` bytes; it may be null where it has none.
bool buffer_ok(const void* p, size_t elements, size_t size) { return elements == 0 || (p && blink::aligned(p, size)); }
bool workspace_ok(const void* p, size_t has, size_t needs) { return needs == 0 || (p && has >= needs && blink::aligned(p, 256)); }

// Whether matrices that are written do not overlap: one after the other, or their rows in turn.
bool apart(size_t batch, size_t rows, size_t cols, size_t row_stride, size_t batch_stride) {
    return batch_stride >= (rows - 1) * row_stride + cols || (batch_stride >= cols && row_stride >= (batch - 1) * batch_stride + cols);
}

}  // namespace

extern "C" {

blink_status_t blink_embedding(const void* table, blink_dtype_t table_type, size_t vocab, size_t dim, size_t table_stride, const void* tokens,
                               blink_dtype_t token_type, size_t n_tokens, float scale, void* out, blink_dtype_t out_type, size_t out_stride, void* stream) {
    if (!blink::is_float(table_type) || !blink::is_float(out_type) || !is_token(token_type) || n_tokens > kMostTokens || vocab > kMostTokens ||
        dim > kMostDim || table_stride < dim || out_stride < dim || !buffer_ok(table, vocab * dim, blink::size_of(table_type)) ||
        !buffer_ok(tokens, n_tokens, blink::size_of(token_type)) || !buffer_ok(out, n_tokens * dim, blink::size_of(out_type)))
        return BLINK_EINVAL;
    return blink::embedding(table, table_type, vocab, dim, table_stride, tokens, token_type, n_tokens, scale, out, out_type, out_stride,
                            static_cast<hipStream_t>(stream));
}

size_t blink_embedding_gradient_workspace(size_t n_tokens, size_t vocab, size_t dim) {
    if (n_tokens > kMostTokens || vocab > kMostTokens - 1 || dim > kMostDim) return 0;
    return blink::embedding_gradient_workspace(n_tokens, vocab, dim);
}

blink_status_t blink_embedding_gradient(const void* tokens, blink_dtype_t token_type, size_t n_tokens, const void* grad_out, blink_dtype_t grad_type,
                                        size_t grad_stride, float scale, int accumulate, void* grad_table, blink_dtype_t table_type, size_t vocab, size_t dim,
                                        size_t table_stride, void* workspace, size_t workspace_bytes, void* stream) {
    if (!blink::is_float(table_type) || !blink::is_float(grad_type) || !is_token(token_type) || n_tokens > kMostTokens || vocab > kMostTokens - 1 ||
        dim > kMostDim || table_stride < dim || (grad_stride < dim && grad_stride != 0) || (accumulate != 0 && accumulate != 1) ||
        !buffer_ok(grad_out, n_tokens * dim, blink::size_of(grad_type)) || !buffer_ok(tokens, n_tokens, blink::size_of(token_type)) ||
        !buffer_ok(grad_table, vocab * dim, blink::size_of(table_type)) ||
        !workspace_ok(workspace, workspace_bytes, blink::embedding_gradient_workspace(n_tokens, vocab, dim)))
        return BLINK_EINVAL;
    return blink::embedding_gradient(tokens, token_type, n_tokens, grad_out, grad_type, grad_stride, scale, accumulate == 1, grad_table, table_type, vocab, dim,
                                     table_stride, workspace, static_cast<hipStream_t>(stream));
}

size_t blink_route_workspace(size_t n_tokens, int n_experts) {
    if (n_tokens > kMostTokens || n_experts < 1 || n_experts > kMostExperts) return 0;
    return blink::route_workspace(n_tokens, n_experts);
}

blink_status_t blink_route(const void* logits, blink_dtype_t dtype, size_t n_tokens, int n_experts, size_t stride, const uint8_t* keep, int k, int normalize,
                           int32_t* chosen, float* weights, int32_t* counts, float* sums, void* workspace, size_t workspace_bytes, void* stream) {
    if (!blink::is_float(dtype) || n_tokens > kMostTokens || n_experts < 1 || n_experts > kMostExperts || k < 1 || k > n_experts ||
        stride < static_cast<size_t>(n_experts) || (normalize != 0 && normalize != 1) || !buffer_ok(logits, n_tokens, blink::size_of(dtype)) ||
        !buffer_ok(chosen, n_tokens, 4) || !buffer_ok(weights, n_tokens, 4) || !buffer_ok(counts, 1, 4) || !buffer_ok(sums, 1, 4) ||
        !workspace_ok(workspace, workspace_bytes, blink::route_workspace(n_tokens, n_experts)))
        return BLINK_EINVAL;
    return blink::route(logits, dtype, n_tokens, n_experts, stride, keep, k, normalize == 1, chosen, weights, counts, sums, workspace,
                        static_cast<hipStream_t>(stream));
}

blink_status_t blink_route_loss(const int32_t* counts, const float* sums, int n_experts, int k, float balance, float z, float* loss, void* stream) {
    if (n_experts < 1 || n_experts > kMostExperts || k < 1 || k > n_experts || !buffer_ok(counts, 1, 4) || !buffer_ok(sums, 1, 4) || !buffer_ok(loss, 1, 4))
        return BLINK_EINVAL;
    return blink::route_loss(counts, sums, n_experts, k, balance, z, loss, static_cast<hipStream_t>(stream));
}

blink_status_t blink_route_gradient(const void* logits, blink_dtype_t dtype, size_t n_tokens, int n_experts, size_t stride, const uint8_t* keep, int k,
                                    int normalize, const int32_t* chosen, const float* grad_weights, const int32_t* counts, const float* grad_loss,
                                    float balance, float z, void* grad_logits, size_t grad_stride, void* stream) {
    if (!blink::is_float(dtype) || n_tokens > kMostTokens || n_experts < 1 || n_experts > kMostExperts || k < 1 || k > n_experts ||
        stride < static_cast<size_t>(n_experts) || grad_stride < static_cast<size_t>(n_experts) || (normalize != 0 && normalize != 1) ||
        !buffer_ok(logits, n_tokens, blink::size_of(dtype)) || !buffer_ok(grad_logits, n_tokens, blink::size_of(dtype)) ||
        !buffer_ok(chosen, grad_weights ? n_tokens : 0, 4) || !blink::aligned(grad_weights, 4) || !buffer_ok(counts, 1, 4) || !blink::aligned(grad_loss, 4))
        return BLINK_EINVAL;
    return blink::route_gradient(logits, dtype, n_tokens, n_experts, stride, keep, k, normalize == 1, chosen, grad_weights, counts, grad_loss, balance, z,
                                 grad_logits, grad_stride, static_cast<hipStream_t>(stream));
}

size_t blink_orthogonalize_workspace(size_t batch, size_t rows, size_t cols, blink_dtype_t dtype) {
    if (!blink::is_float(dtype) || batch < 1 || batch > kMostBatch || rows < 1 || rows > kMostSide || cols < 1 || cols > kMostSide) return 0;
    return blink::orthogonalize_workspace(batch, rows, cols, dtype);
}

blink_status_t blink_orthogonalize(const void* matrix, blink_dtype_t dtype, size_t batch, size_t rows, size_t cols, size_t row_stride, size_t batch_stride,
                                   const float* coefficients, int steps, float eps, void* out, size_t out_row_stride, size_t out_batch_stride, void* workspace,
                                   size_t workspace_bytes, void* stream) {
    const size_t needs = blink_orthogonalize_workspace(batch, rows, cols, dtype);
    if (needs == 0 || row_stride < cols || out_row_stride < cols || (batch > 1 && !apart(batch, rows, cols, out_row_stride, out_batch_stride)) || steps < 1 ||
        steps > kMostSteps || !coefficients || !blink::coefficients_fit(coefficients, steps) || !(eps >= 0) || !std::isfinite(eps) ||
        !buffer_ok(matrix, 1, blink::size_of(dtype)) || !buffer_ok(out, 1, blink::size_of(dtype)) || !workspace_ok(workspace, workspace_bytes, needs))
        return BLINK_EINVAL;
    return blink::orthogonalize(matrix, dtype, batch, rows, cols, row_stride, batch_stride, coefficients, steps, eps, out, out_row_stride, out_batch_stride,
                                workspace, static_cast<hipStream_t>(stream));
}

blink_status_t blink_orthogonal_step(const float* weights, float* weights_out, const float* momentum, float* momentum_out, const void* grad,
                                     blink_dtype_t grad_type, size_t batch, size_t rows, size_t cols, float beta, int nesterov, const float* coefficients,
                                     int steps, float eps, float rate, float decay, void* workspace, size_t workspace_bytes, void* stream) {
    const size_t needs = blink_orthogonalize_workspace(batch, rows, cols, BLINK_FP32);
    if (needs == 0 || !blink::is_float(grad_type) || (nesterov != 0 && nesterov != 1) || steps < 1 || steps > kMostSteps || !coefficients ||
        !blink::coefficients_fit(coefficients, steps) || !(eps >= 0) || !std::isfinite(eps) || !buffer_ok(weights, 1, 4) || !buffer_ok(weights_out, 1, 4) ||
        !buffer_ok(momentum, 1, 4) || !buffer_ok(momentum_out, 1, 4) || !buffer_ok(grad, 1, blink::size_of(grad_type)) ||
        !workspace_ok(workspace, workspace_bytes, needs))
        return BLINK_EINVAL;
    return blink::orthogonal_step(weights, weights_out, momentum, momentum_out, grad, grad_type, batch, rows, cols, beta, nesterov == 1, coefficients, steps, eps,
                                  rate, decay, workspace, static_cast<hipStream_t>(stream));
}

}  // extern "C"
