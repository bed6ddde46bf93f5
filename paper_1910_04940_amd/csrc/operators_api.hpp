// What api_operators.cpp checks the arguments for (embedding.hip, route.hip, orthogonal.hip).
#pragma once
#include "operators.hpp"

namespace blink {

blink_status_t embedding(const void* table, blink_dtype_t table_type, size_t vocab, size_t dim, size_t table_stride, const void* tokens,
                         blink_dtype_t token_type, size_t n, float scale, void* out, blink_dtype_t out_type, size_t out_stride, hipStream_t stream);
size_t embedding_gradient_workspace(size_t n, size_t vocab, size_t dim);
blink_status_t embedding_gradient(const void* tokens, blink_dtype_t token_type, size_t n, const void* grad, blink_dtype_t grad_type,
                                  size_t grad_stride, float scale, bool accumulate, void* table, blink_dtype_t table_type, size_t vocab, size_t dim,
                                  size_t table_stride, void* workspace, hipStream_t stream);

size_t route_workspace(size_t tokens, int experts);
blink_status_t route(const void* logits, blink_dtype_t dtype, size_t tokens, int experts, size_t stride, const uint8_t* keep, int k, bool normalize,
                     int32_t* chosen, float* weights, int32_t* counts, float* sums, void* workspace, hipStream_t stream);
blink_status_t route_loss(const int32_t* counts, const float* sums, int experts, int k, float balance, float z, float* loss, hipStream_t stream);
blink_status_t route_gradient(const void* logits, blink_dtype_t dtype, size_t tokens, int experts, size_t stride, const uint8_t* keep, int k,
                              bool normalize, const int32_t* chosen, const float* grad_weights, const int32_t* counts, const float* grad_loss,
                              float balance, float z, void* out, size_t out_stride, hipStream_t stream);

bool coefficients_fit(const float* coefficients, int steps);
size_t orthogonalize_workspace(size_t batch, size_t rows, size_t cols, blink_dtype_t dtype);
blink_status_t orthogonalize(const void* in, blink_dtype_t dtype, size_t batch, size_t rows, size_t cols, size_t in_row, size_t in_batch,
                             const float* coefficients, int steps, float eps, void* out, size_t out_row, size_t out_batch, void* workspace,
                             hipStream_t stream);
blink_status_t orthogonal_step(const float* weights, float* weights_out, const float* momentum, float* momentum_out, const void* grad,
                               blink_dtype_t grad_type, size_t batch, size_t rows, size_t cols, float beta, bool nesterov, const float* coefficients,
                               int steps, float eps, float rate, float decay, void* workspace, hipStream_t stream);

}  // namespace blink
