// extern "C" boundary of the operators around the collectives: argument checks.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "operators_api.hpp"

namespace {

constexpr size_t kMostTokens = 0x7fffffff, kMostDim = size_t{1} << 21, kMostSide = size_t{1} << 20, kMostBatch = 65535;
constexpr size_t kMostElements = size_t{1} << 40;
constexpr int kMostExperts = 1024, kMostGroups = 64, kMostSteps = 64, kMostTensors = 1 << 20;

bool is_token(blink_dtype_t t) { return t == BLINK_INT32 || t == BLINK_INT64; }
// A buffer of elements of `size` bytes; it may be null where it has none.
bool buffer_ok(const void* p, size_t elements, size_t size) { return elements == 0 || (p && blink::aligned(p, size)); }
bool workspace_ok(const void* p, size_t has, size_t needs) { return needs == 0 || (p && has >= needs && blink::aligned(p, 256)); }

// Whether matrices that are written do not overlap: one after the other, or their rows in turn.
bool apart(size_t batch, size_t rows, size_t cols, size_t row_stride, size_t batch_stride) {
    return batch_stride >= (rows - 1) * row_stride + cols || (batch_stride >= cols && row_stride >= (batch - 1) * batch_stride + cols);
}

// One tensor of a list: its addresses, types and numbers.
bool tensor_ok(const blink_update_tensor_t& t) {
    if (!blink::is_float(t.grad_type) || t.elements > kMostElements || !buffer_ok(t.grad, t.elements, blink::size_of(t.grad_type))) return false;
    if (!t.weights) return !t.master && !t.moment1 && !t.moment2 && !t.scale1 && !t.scale2;   // (its gradient counts, it is not stepped)
    const bool eight = t.moment_type == BLINK_FP8;
    if (!blink::is_float(t.weight_type) || (t.moment_type != BLINK_FP32 && !eight) || (t.master && t.weight_type == BLINK_FP32)) return false;
    return blink::aligned(t.weights, blink::size_of(t.weight_type)) && blink::aligned(t.master, 4) && buffer_ok(t.moment1, t.elements, eight ? 1 : 4) &&
           buffer_ok(t.moment2, t.elements, eight ? 1 : 4) && (eight ? buffer_ok(t.scale1, t.elements, 4) && buffer_ok(t.scale2, t.elements, 4) : !t.scale1 && !t.scale2) &&
           std::isfinite(t.rate) && std::isfinite(t.decay);
}
// Whether what a step writes is written by one tensor of the list, and read by no other: their workgroups run at once.
bool tensors_apart(const blink_update_tensor_t* tensors, int n) {
    struct Range {
        uintptr_t from, to;
        bool written;
    };
    std::vector<Range> all;
    const auto add = [&](const void* p, size_t bytes, bool written) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        if (p && bytes) all.push_back({at, at + bytes, written});
    };
    for (int i = 0; i < n; ++i) {
        const blink_update_tensor_t& t = tensors[i];
        const size_t moment = t.moment_type == BLINK_FP8 ? 1 : 4, scales = (t.elements + 255) / 256 * 4;
        add(t.grad, t.elements * blink::size_of(t.grad_type), false);
        if (!t.weights) continue;
        add(t.weights, t.elements * blink::size_of(t.weight_type), true);
        add(t.master, t.elements * 4, true);
        add(t.moment1, t.elements * moment, true);
        add(t.moment2, t.elements * moment, true);
        add(t.scale1, scales, true);
        add(t.scale2, scales, true);
    }
    std::sort(all.begin(), all.end(), [](const Range& a, const Range& b) { return a.from < b.from; });
    uintptr_t read = 0, written = 0;   // where those so far end
    for (const Range& r : all) {
        if (r.from < written || (r.written && r.from < read)) return false;
        uintptr_t& end = r.written ? written : read;
        end = std::max(end, r.to);
    }
    return true;
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

size_t blink_route_biased_workspace(size_t n_tokens, int n_experts) {
    if (n_tokens > kMostTokens || n_experts < 1 || n_experts > kMostExperts) return 0;
    return blink::route_biased_workspace(n_tokens, n_experts);
}

blink_status_t blink_route_biased(const void* logits, blink_dtype_t dtype, size_t n_tokens, int n_experts, size_t stride, const uint8_t* keep, const float* bias,
                                  int k, int groups, int kept_groups, blink_scores_t scores, int normalize, float scale, int32_t* chosen, float* weights,
                                  int32_t* counts, void* workspace, size_t workspace_bytes, void* stream) {
    if (!blink::is_float(dtype) || n_tokens > kMostTokens || n_experts < 1 || n_experts > kMostExperts || groups < 1 || groups > kMostGroups ||
        n_experts % groups != 0 || kept_groups < 1 || kept_groups > groups || k < 1 || k > n_experts / groups * kept_groups ||
        stride < static_cast<size_t>(n_experts) || (scores != BLINK_SIGMOID && scores != BLINK_SOFTMAX) || (normalize != 0 && normalize != 1) ||
        !std::isfinite(scale) || !buffer_ok(logits, n_tokens, blink::size_of(dtype)) || !blink::aligned(bias, 4) || !buffer_ok(chosen, n_tokens, 4) ||
        !buffer_ok(weights, n_tokens, 4) || !buffer_ok(counts, 1, 4) ||
        !workspace_ok(workspace, workspace_bytes, blink::route_biased_workspace(n_tokens, n_experts)))
        return BLINK_EINVAL;
    return blink::route_biased(logits, dtype, n_tokens, n_experts, stride, keep, bias, k, groups, kept_groups, scores == BLINK_SOFTMAX, normalize == 1, scale,
                               chosen, weights, counts, workspace, static_cast<hipStream_t>(stream));
}

blink_status_t blink_route_bias(const int32_t* counts, const float* bias, int n_experts, float rate, float* bias_out, void* stream) {
    if (n_experts < 1 || n_experts > kMostExperts || !std::isfinite(rate) || !buffer_ok(counts, 1, 4) || !buffer_ok(bias, 1, 4) || !buffer_ok(bias_out, 1, 4))
        return BLINK_EINVAL;
    return blink::route_bias(counts, bias, bias_out, n_experts, rate, static_cast<hipStream_t>(stream));
}

blink_status_t blink_route_biased_gradient(const void* logits, blink_dtype_t dtype, size_t n_tokens, int n_experts, size_t stride, const uint8_t* keep, int k,
                                           blink_scores_t scores, int normalize, float scale, const int32_t* chosen, const float* grad_weights,
                                           void* grad_logits, size_t grad_stride, void* stream) {
    if (!blink::is_float(dtype) || n_tokens > kMostTokens || n_experts < 1 || n_experts > kMostExperts || k < 1 || k > n_experts ||
        stride < static_cast<size_t>(n_experts) || grad_stride < static_cast<size_t>(n_experts) || (scores != BLINK_SIGMOID && scores != BLINK_SOFTMAX) ||
        (normalize != 0 && normalize != 1) || !std::isfinite(scale) || !buffer_ok(logits, n_tokens, blink::size_of(dtype)) || !buffer_ok(chosen, n_tokens, 4) ||
        !buffer_ok(grad_weights, n_tokens, 4) || !buffer_ok(grad_logits, n_tokens, blink::size_of(dtype)))
        return BLINK_EINVAL;
    return blink::route_biased_gradient(logits, dtype, n_tokens, n_experts, stride, keep, k, scores == BLINK_SOFTMAX, normalize == 1, scale, chosen,
                                        grad_weights, grad_logits, grad_stride, static_cast<hipStream_t>(stream));
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

blink_status_t blink_make_update(const blink_update_tensor_t* tensors, int n, blink_update_t** out) {
    if (!out) return BLINK_EINVAL;
    *out = nullptr;
    if (!tensors || n < 1 || n > kMostTensors) return BLINK_EINVAL;
    for (int i = 0; i < n; ++i)
        if (!tensor_ok(tensors[i])) return BLINK_EINVAL;
    try {
        if (!tensors_apart(tensors, n)) return BLINK_EINVAL;
        return blink::make_update(tensors, n, out);
    } catch (...) {   // (nothing else throws)
        return BLINK_ENOMEM;
    }
}

void blink_update_free(blink_update_t* u) { blink::free_update(u); }

size_t blink_gradient_norm_workspace(const blink_update_t* u) { return u ? blink::gradient_norm_workspace(*u) : 0; }

blink_status_t blink_gradient_norm(const blink_update_t* u, double max_norm, double factor, float* norm, int32_t* step, void* workspace, size_t workspace_bytes,
                                   void* stream) {
    if (!u || !(max_norm > 0) || !std::isfinite(factor) || !buffer_ok(norm, 1, 4) || !blink::aligned(step, 4) ||
        !workspace_ok(workspace, workspace_bytes, blink::gradient_norm_workspace(*u)))
        return BLINK_EINVAL;
    return blink::gradient_norm(*u, max_norm, factor, norm, step, workspace, static_cast<hipStream_t>(stream));
}

blink_status_t blink_adamw_step(const blink_update_t* u, const int32_t* step, double lr, double beta1, double beta2, double eps, const float* scale,
                                const float* rate, uint32_t seed, void* stream) {
    if (!u || !buffer_ok(step, 1, 4) || !std::isfinite(lr) || !(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1) || !(eps > 0 && std::isfinite(eps)) ||
        !blink::aligned(scale, 4) || !blink::aligned(rate, 4))
        return BLINK_EINVAL;
    return blink::adamw_step(*u, step, lr, beta1, beta2, eps, scale, rate, seed, static_cast<hipStream_t>(stream));
}

}  // extern "C"
