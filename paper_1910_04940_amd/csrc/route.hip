// A router's choice of experts, the loss that keeps the experts evenly used, and the gradient of its logits.
//
//   p = softmax(x) of a token's logits;  chosen: the k largest x, the lowest index first among equals, -inf never
//   w = p of the chosen, or that divided by its sum S over the token's chosen
//   c_e = tokens that chose e;  P_e = sum of p_e;  Z = sum of lse(x)^2;  n = tokens counted
//   loss = balance * E / (k n^2) * sum c_e P_e  +  z / n * Z
//   dx_e = p_e (d_e - sum_f p_f d_f + 2 z lse / n)  with  d_e = balance * E / (k n^2) * c_e + (what the weights' gradient adds)
//
// c, P, Z and n are sums over tokens, so ranks add theirs (c and n as integers) before the loss and its gradient are formed.
// A token is counted if it is kept and not all of its logits are -inf.
//
// L lanes hold a token, N logits each; a wave holds 64 / L tokens and goes through tokens in strides of the grid, so that the
// sums over tokens stay in registers until its end.  Workgroups leave their sums in the workspace, a second kernel adds
// them up in order.  Both kernels over the logits read them once.
#include "operators_api.hpp"

#include <algorithm>
#include <cmath>

namespace blink {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMostGroups = 1024;        // workgroups of the first kernel: 16 waves on a CU
constexpr float kInf = __builtin_inff();

// ---- lanes of a token: L neighbours, L a power of two -----------------------------------------------------------------------
// op(own value, the other half's), for halves of 1, 2, 4 ... lanes, each of which holds one value by then.
template <int L, typename F>
__device__ inline float over_lanes(float x, F op) {
    const auto dpp = [](float v, auto control) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(control)::value, 0xf, 0xf, true));
    };
    if constexpr (L > 1) x = op(x, dpp(x, std::integral_constant<int, 0xB1>()));    // quad_perm 1 0 3 2
    if constexpr (L > 2) x = op(x, dpp(x, std::integral_constant<int, 0x4E>()));    // quad_perm 2 3 0 1
    if constexpr (L > 4) x = op(x, dpp(x, std::integral_constant<int, 0x141>()));   // row_half_mirror
    if constexpr (L > 8) x = op(x, dpp(x, std::integral_constant<int, 0x140>()));   // row_mirror
    if constexpr (L > 16) {
        const unsigned v = __builtin_bit_cast(unsigned, x);
        const auto both = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        x = op(__builtin_bit_cast(float, static_cast<unsigned>(both[0])), __builtin_bit_cast(float, static_cast<unsigned>(both[1])));
    }
    if constexpr (L > 32) {
        const unsigned v = __builtin_bit_cast(unsigned, x);
        const auto both = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        x = op(__builtin_bit_cast(float, static_cast<unsigned>(both[0])), __builtin_bit_cast(float, static_cast<unsigned>(both[1])));
    }
    return x;
}
template <int L>
__device__ inline float lanes_max(float x) {
    return over_lanes<L>(x, [](float a, float b) { return __builtin_fmaxf(a, b); });
}
template <int L>
__device__ inline float lanes_sum(float x) {
    return over_lanes<L>(x, [](float a, float b) { return a + b; });
}
template <int L>
__device__ inline int lanes_min(int x) {   // of numbers below 2^23, as the floats that they are exactly
    return static_cast<int>(over_lanes<L>(static_cast<float>(x), [](float a, float b) { return __builtin_fminf(a, b); }));
}

// Logits [lane * N, lane * N + N) of a token, -inf past the last.  WIDE: 16 bytes at a time.
template <typename T, int N, bool WIDE>
__device__ inline void load_logits(float (&x)[N], const T* row, int first, int experts) {
    if constexpr (WIDE) {
        constexpr int V = 16 / sizeof(T) < N ? 16 / sizeof(T) : N;
#pragma unroll
        for (int i = 0; i < N; i += V) {
            Pack<T, V> y;
            const bool in = first + i < experts;
            if (in) y = *reinterpret_cast<const Pack<T, V>*>(row + first + i);
#pragma unroll
            for (int v = 0; v < V; ++v) x[i + v] = in ? static_cast<float>(y.v[v]) : -kInf;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = first + i < experts ? static_cast<float>(row[first + i]) : -kInf;
    }
}

__device__ inline float power(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }   // e^x, 0 for -inf

// Softmax of a token: x becomes p.  False if all logits are -inf (p is then 0).  A NaN, or +inf, makes p NaN.
template <int L, int N>
__device__ inline bool softmax(float (&x)[N], float* most, float* scale, float* lse) {
    float m = -kInf;
#pragma unroll
    for (int i = 0; i < N; ++i) m = __builtin_fmaxf(m, x[i]);   // (passes over NaN)
    m = lanes_max<L>(m);
    const float from = m == -kInf ? 0.0f : m;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = power(x[i] - from);
        s += x[i];
    }
    s = lanes_sum<L>(s);
    const bool any = s != 0.0f;   // at least 1, or NaN
    const float r = any ? 1.0f / s : 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] *= r;
    *most = from;
    *scale = r;
    *lse = any ? from + logf(s) : 0.0f;
    return any;
}

struct Route {
    const void* logits;
    uint64_t stride;
    const uint8_t* keep;   // null: every token
    uint32_t tokens;
    int experts, k;
    bool normalize;
    int32_t* chosen;
    float* weights;
    int32_t* counts;       // of the result, or [workgroup][experts + 1]
    float* sums;
};

template <typename T, int L, int N, bool WIDE>
__global__ __launch_bounds__(kThreads) void route_choose(const Route a) {
    __shared__ int32_t count[L * N + 1];
    __shared__ float part[kWaves][L * N + 1];
    const int t = threadIdx.x, wave = t >> 6, lane = t & (L - 1), first = lane * N;
    for (int i = t; i <= L * N; i += kThreads) count[i] = 0;
    __syncthreads();
    float total[N] = {}, z = 0.0f;
    int counted = 0;
    const uint32_t step = gridDim.x * (kThreads / L);
    for (uint64_t token = blockIdx.x * (kThreads / L) + t / L; token < a.tokens; token += step) {
        const bool keep = !a.keep || a.keep[token];
        float x[N], free[N];
        if (keep) load_logits<T, N, WIDE>(x, static_cast<const T*>(a.logits) + token * a.stride, first, a.experts);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (!keep) x[i] = -kInf;
            free[i] = x[i] == x[i] ? x[i] : -kInf;   // a NaN is not chosen
        }
        float most, scale, lse;
        const bool any = softmax<L, N>(x, &most, &scale, &lse);
#pragma unroll
        for (int i = 0; i < N; ++i) total[i] += x[i];
        z += lse * lse;
        counted += any;
        // k times the largest that is left; lane j % L keeps the j-th until L are there
        float sum = 0.0f, weight = 0.0f;
        int which = -1;
        for (int j = 0; j < a.k; ++j) {
            float best = -kInf;
#pragma unroll
            for (int i = 0; i < N; ++i) best = __builtin_fmaxf(best, free[i]);
            best = lanes_max<L>(best);
            int at = 1 << 20;
#pragma unroll
            for (int i = N - 1; i >= 0; --i) at = free[i] == best ? first + i : at;
            at = lanes_min<L>(at);
            const bool found = best > -kInf;
#pragma unroll
            for (int i = 0; i < N; ++i) free[i] = first + i == at ? -kInf : free[i];
            const float p = found ? power(best - most) * scale : 0.0f;
            sum += p;
            if (lane == j % L) {
                which = found ? at : -1;
                weight = p;
                if (found) atomicAdd(&count[at], 1);
            }
            if (j % L == L - 1 || j == a.k - 1) {
                const int slot = j / L * L + lane;
                if (slot <= j) {
                    const uint64_t to = token * a.k + slot;
                    a.chosen[to] = which;
                    a.weights[to] = a.normalize && a.k <= L ? (any ? weight / sum : 0.0f) : weight;
                }
            }
        }
        if (a.normalize && a.k > L)
            for (int j = lane; j < a.k; j += L) a.weights[token * a.k + j] = any ? a.weights[token * a.k + j] / sum : 0.0f;
    }
    // the wave's sums, token groups side by side first
#pragma unroll
    for (int d = L; d < 64; d <<= 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) total[i] += __shfl_xor(total[i], d);
        z += __shfl_xor(z, d);
        counted += __shfl_xor(counted, d);
    }
    if ((t & 63) < L)
#pragma unroll
        for (int i = 0; i < N; ++i) part[wave][first + i] = total[i];
    if ((t & 63) == 0) {
        part[wave][L * N] = z;
        atomicAdd(&count[L * N], counted);
    }
    __syncthreads();
    for (int i = t; i <= a.experts; i += kThreads) {
        const int from = i < a.experts ? i : L * N;
        float s = 0.0f;
        for (int w = 0; w < kWaves; ++w) s += part[w][from];
        a.sums[static_cast<uint64_t>(blockIdx.x) * (a.experts + 1) + i] = s;
        a.counts[static_cast<uint64_t>(blockIdx.x) * (a.experts + 1) + i] = count[from];
    }
}

// Adds up what the workgroups left: 64 columns to a workgroup, every wave a part of the rows, in 64 bits.
constexpr int kAddThreads = 1024;
__global__ __launch_bounds__(kAddThreads) void route_add(const int32_t* counts, const float* sums, uint32_t groups, int columns, int32_t* count, float* sum) {
    __shared__ double s[kAddThreads / 64][64];
    __shared__ int32_t c[kAddThreads / 64][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, column = blockIdx.x * 64 + lane;
    double total = 0.0;
    int32_t many = 0;
    if (column < columns)
#pragma unroll 4
        for (uint32_t g = wave; g < groups; g += kAddThreads / 64) {
            total += sums[static_cast<uint64_t>(g) * columns + column];
            many += counts[static_cast<uint64_t>(g) * columns + column];
        }
    s[wave][lane] = total;
    c[wave][lane] = many;
    __syncthreads();
    if (wave != 0 || column >= columns) return;
    for (int w = 1; w < kAddThreads / 64; ++w) {
        total += s[w][lane];
        many += c[w][lane];
    }
    sum[column] = static_cast<float>(total);
    count[column] = many;
}

__global__ __launch_bounds__(64) void route_loss_kernel(const int32_t* counts, const float* sums, int experts, int k, double balance, double z, float* loss) {
    double s = 0.0;
    for (int e = threadIdx.x; e < experts; e += 64) s += static_cast<double>(counts[e]) * sums[e];
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
    if (threadIdx.x != 0) return;
    const double n = counts[experts];
    const double b = n > 0 ? balance * experts / k * s / (n * n) : 0.0, l = n > 0 ? z * sums[experts] / n : 0.0;
    loss[0] = static_cast<float>(b + l);
    loss[1] = static_cast<float>(b);
    loss[2] = static_cast<float>(l);
}

struct RouteGradient {
    const void* logits;
    uint64_t stride;
    const uint8_t* keep;
    uint32_t tokens;
    int experts, k;
    bool normalize;
    const int32_t* chosen;
    const float* grad_weights;   // null: none
    const int32_t* counts;
    const float* grad_loss;      // null: 1
    float balance, z;
    void* out;
    uint64_t out_stride;
};

template <typename T, int L, int N, bool WIDE>
__global__ __launch_bounds__(kThreads) void route_gradient_kernel(const RouteGradient a) {
    __shared__ float by_weight[kThreads / L][L * N];   // what the weights' gradient adds to d, of the token that the lanes hold
    const int t = threadIdx.x, lane = t & (L - 1), first = lane * N;
    float* const add = by_weight[t / L];
    const float up = a.grad_loss ? *a.grad_loss : 1.0f;
    const float n = static_cast<float>(a.counts[a.experts] > 0 ? a.counts[a.experts] : 1);
    float by_p[N];
#pragma unroll
    for (int i = 0; i < N; ++i) by_p[i] = first + i < a.experts ? up * a.balance * a.experts / a.k * (a.counts[first + i] / n) / n : 0.0f;
    const float by_lse = 2.0f * up * a.z / n;
    const uint32_t step = gridDim.x * (kThreads / L);
    for (uint64_t token = blockIdx.x * (kThreads / L) + t / L; token < a.tokens; token += step) {
        const bool keep = !a.keep || a.keep[token];
        const T* const row = static_cast<const T*>(a.logits) + token * a.stride;
        float x[N], d[N];
        if (keep) load_logits<T, N, WIDE>(x, row, first, a.experts);
        if (!keep)
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = -kInf;
        float most, scale, lse;
        const bool any = softmax<L, N>(x, &most, &scale, &lse);
#pragma unroll
        for (int i = 0; i < N; ++i) d[i] = by_p[i];
        if (a.grad_weights && keep) {
            // lanes of a token are lanes of one wave, whose accesses to LDS happen in order
#pragma unroll
            for (int i = 0; i < N; ++i) add[first + i] = 0.0f;
            float sum = 1.0f, dot = 0.0f;
            if (a.normalize) {   // d of the chosen: (g - sum w g) / S
                sum = 0.0f;
                for (int j = lane; j < a.k; j += L) {
                    const int e = a.chosen[token * a.k + j];
                    if (e < 0 || e >= a.experts) continue;
                    const float p = power(static_cast<float>(row[e]) - most) * scale;
                    sum += p;
                    dot += p * a.grad_weights[token * a.k + j];
                }
                sum = lanes_sum<L>(sum);
                dot = lanes_sum<L>(dot) / sum;
            }
            wave_sync();
            for (int j = lane; j < a.k; j += L) {
                const int e = a.chosen[token * a.k + j];
                if (e >= 0 && e < a.experts) add[e] = (a.grad_weights[token * a.k + j] - dot) / sum;
            }
            wave_sync();
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] += add[first + i];
        }
        float dot = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) dot += x[i] * d[i];
        dot = lanes_sum<L>(dot) - by_lse * lse;
        T* const out = static_cast<T*>(a.out) + token * a.out_stride;
        if constexpr (WIDE) {
            constexpr int V = 16 / sizeof(T) < N ? 16 / sizeof(T) : N;
#pragma unroll
            for (int i = 0; i < N; i += V) {
                Pack<T, V> y;
#pragma unroll
                for (int v = 0; v < V; ++v) y.v[v] = static_cast<T>(any ? x[i + v] * (d[i + v] - dot) : 0.0f);
                if (first + i < a.experts) *reinterpret_cast<Pack<T, V>*>(out + first + i) = y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (first + i < a.experts) out[first + i] = static_cast<T>(any ? x[i] * (d[i] - dot) : 0.0f);
        }
    }
}

// ---- host side ----------------------------------------------------------------------------------------------------------------
// Eight logits to a lane (16 where 64 lanes of eight do not hold the token): f is called with the lanes and that number.
template <typename F>
blink_status_t with_lanes(int experts, F f) {
    using std::integral_constant;
    using Eight = integral_constant<int, 8>;
    if (experts <= 8) return f(integral_constant<int, 1>(), Eight());
    if (experts <= 16) return f(integral_constant<int, 2>(), Eight());
    if (experts <= 32) return f(integral_constant<int, 4>(), Eight());
    if (experts <= 64) return f(integral_constant<int, 8>(), Eight());
    if (experts <= 128) return f(integral_constant<int, 16>(), Eight());
    if (experts <= 256) return f(integral_constant<int, 32>(), Eight());
    if (experts <= 512) return f(integral_constant<int, 64>(), Eight());
    return f(integral_constant<int, 64>(), integral_constant<int, 16>());
}

uint32_t lanes_of(int experts) {
    uint32_t l = 1;
    while (l < 64 && static_cast<int>(l * 8) < experts) l <<= 1;
    return l;
}
uint32_t groups_of(size_t tokens, int experts) {
    return static_cast<uint32_t>(std::min<uint64_t>(kMostGroups, ceil_div(tokens, kThreads / lanes_of(experts))));
}

}  // namespace

size_t route_workspace(size_t tokens, int experts) {
    const uint32_t groups = groups_of(tokens, experts);
    Carve c(nullptr);
    if (groups > 1) {
        c.take<float>(static_cast<size_t>(groups) * (experts + 1));
        c.take<int32_t>(static_cast<size_t>(groups) * (experts + 1));
    }
    return c.at;
}

blink_status_t route(const void* logits, blink_dtype_t dtype, size_t tokens, int experts, size_t stride, const uint8_t* keep, int k, bool normalize,
                     int32_t* chosen, float* weights, int32_t* counts, float* sums, void* workspace, hipStream_t stream) {
    const uint32_t groups = std::max(1u, groups_of(tokens, experts));
    Route a{logits, stride, keep, static_cast<uint32_t>(tokens), experts, k, normalize, chosen, weights, counts, sums};
    Carve c(workspace);
    if (groups > 1) {   // one workgroup's sums are the result
        a.sums = c.take<float>(static_cast<size_t>(groups) * (experts + 1));
        a.counts = c.take<int32_t>(static_cast<size_t>(groups) * (experts + 1));
    }
    BLINK_TRY(with_float(dtype, [&](auto type) {
        using T = decltype(type);
        constexpr size_t V = 16 / sizeof(T);
        const bool wide = experts % V == 0 && stride % V == 0 && aligned(logits, 16);
        return with_lanes(experts, [&](auto l, auto n) {
            constexpr int L = decltype(l)::value, N = decltype(n)::value;
            return launch(wide ? route_choose<T, L, N, true> : route_choose<T, L, N, false>, dim3(groups), dim3(kThreads), stream, a);
        });
    }));
    if (groups == 1) return BLINK_OK;
    return launch(route_add, dim3(static_cast<uint32_t>(ceil_div(experts + 1, 64))), dim3(kAddThreads), stream, a.counts, a.sums, groups, experts + 1,
                  counts, sums);
}

blink_status_t route_loss(const int32_t* counts, const float* sums, int experts, int k, float balance, float z, float* loss, hipStream_t stream) {
    return launch(route_loss_kernel, dim3(1), dim3(64), stream, counts, sums, experts, k, static_cast<double>(balance), static_cast<double>(z), loss);
}

blink_status_t route_gradient(const void* logits, blink_dtype_t dtype, size_t tokens, int experts, size_t stride, const uint8_t* keep, int k,
                              bool normalize, const int32_t* chosen, const float* grad_weights, const int32_t* counts, const float* grad_loss,
                              float balance, float z, void* out, size_t out_stride, hipStream_t stream) {
    if (tokens == 0) return BLINK_OK;
    const RouteGradient a{logits, stride, keep, static_cast<uint32_t>(tokens), experts, k, normalize, chosen, grad_weights, counts, grad_loss,
                          balance, z, out, out_stride};
    // no sums are kept from token to token: as many workgroups as there are tokens for, in the end
    const uint32_t groups = static_cast<uint32_t>(std::min<uint64_t>(4 * kMostGroups, ceil_div(tokens, kThreads / lanes_of(experts))));
    return with_float(dtype, [&](auto type) {
        using T = decltype(type);
        constexpr size_t V = 16 / sizeof(T);
        const bool wide = experts % V == 0 && stride % V == 0 && out_stride % V == 0 && aligned(logits, 16) && aligned(out, 16);
        return with_lanes(experts, [&](auto l, auto n) {
            constexpr int L = decltype(l)::value, N = decltype(n)::value;
            return launch(wide ? route_gradient_kernel<T, L, N, true> : route_gradient_kernel<T, L, N, false>, dim3(groups), dim3(kThreads), stream, a);
        });
    });
}

}  // namespace blink
