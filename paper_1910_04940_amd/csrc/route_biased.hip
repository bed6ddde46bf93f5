// A router's choice of experts by scores and a bias, within groups; the gradient of its logits; the bias's own step.
//
//   p = sigmoid(x) of each logit, or softmax(x) of a token's;   a = p + bias, -inf where x is
//   a group's score: the sum of its two largest a (its one, where no other is left);  the `kept` groups with the largest scores stay
//   chosen: the k largest a in them;   the lowest index first among equals, groups and experts alike
//   w = scale * p of the chosen, or scale * p / S, S the sum of p over the token's chosen
//   bias_e moves by rate * sign(mean - c_e), c_e tokens that chose e: no loss, and no gradient, is needed to keep experts evenly used
//
// Gradient of the weights' gradient g, with q = p / S, over the chosen:
//   sigmoid    dx = scale g p (1 - p),                  normalised  scale (g - sum q g) q (1 - p)
//   softmax    dx = p (d - sum p d), d = scale g or 0,  normalised  scale (g - sum q g) q   (softmax of the chosen alone)
//
// The choice is that of scores in 64 bits.  L lanes hold a token, N logits each (see route.hpp).
#include <algorithm>
#include <type_traits>

#include "operators_api.hpp"
#include "route.hpp"

namespace blink {
namespace {

constexpr int kThreads = kRouteThreads;
constexpr int kMostGroups = 1024;        // workgroups: 16 waves on a CU
constexpr double kInf64 = __builtin_inf();

struct Biased {
    const void* logits;
    uint64_t stride;
    const uint8_t* keep;   // null: every token
    const float* bias;     // null: 0
    uint32_t tokens;
    int experts, k, groups, kept;
    bool soft, normalize;
    float scale;
    int32_t* chosen;
    float* weights;
    int32_t* counts;       // of the result, or [workgroup][experts + 1]
};

template <int L>
__device__ inline double lanes_max(double x) {
#pragma unroll
    for (int d = 1; d < L; d <<= 1) x = __builtin_fmax(x, __shfl_xor(x, d));
    return x;
}

// The choice with scores in 64 bits, for a token whose logits are x (-inf: not to be had).  Lane j % L writes and keeps the j-th.
// score: room for a number to each group, the token's own.
template <typename T, int L, int N>
__device__ inline void choose(const Biased& a, const float (&x)[N], int lane, double* score, int32_t* chosen) {
    double v[N];
    if (a.soft) {
        float m = -kInf;
#pragma unroll
        for (int i = 0; i < N; ++i) m = __builtin_fmaxf(m, x[i]);
        m = lanes_max<L>(m);
        const double from = m == -kInf ? 0.0 : m;
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = exp(x[i] - from);
            s += v[i];
        }
        s = lanes_sum<L>(s);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] /= s;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = 1.0 / (1.0 + exp(-static_cast<double>(x[i])));
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = expert_of<T, L>(lane, i);
        const double y = v[i] + (a.bias && e < a.experts ? static_cast<double>(a.bias[e]) : 0.0);
        v[i] = x[i] > -kInf && y > -kInf64 ? y : -kInf64;   // (a bias of -inf or NaN: never)
    }
    if (a.groups > 1) {
        const int size = a.experts / a.groups;
        for (int g = 0; g < a.groups; ++g) {
            double first = -kInf64, second = -kInf64;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int e = expert_of<T, L>(lane, i) - g * size;
                const double y = e >= 0 && e < size ? v[i] : -kInf64;
                second = __builtin_fmax(second, __builtin_fmin(first, y));
                first = __builtin_fmax(first, y);
            }
#pragma unroll
            for (int d = 1; d < L; d <<= 1) {
                const double f = __shfl_xor(first, d), s = __shfl_xor(second, d);
                second = __builtin_fmax(__builtin_fmin(first, f), __builtin_fmax(second, s));
                first = __builtin_fmax(first, f);
            }
            if (lane == 0) score[g] = second > -kInf64 ? first + second : first;
        }
        wave_sync();
        uint32_t low = 0, high = 0;   // the groups that stay
        for (int g = lane; g < a.groups; g += L) {
            const double mine = score[g];
            int before = 0;
            for (int h = 0; h < a.groups; ++h) before += score[h] > mine || (score[h] == mine && h < g);
            const uint32_t bit = before < a.kept ? 1u << (g & 31) : 0;
            low |= g < 32 ? bit : 0;
            high |= g < 32 ? 0 : bit;
        }
        low = lanes_or<L>(low);
        high = lanes_or<L>(high);
        wave_sync();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int g = expert_of<T, L>(lane, i) / size;
            if (!((g < 32 ? low >> (g & 31) : high >> (g & 31)) & 1)) v[i] = -kInf64;
        }
    }
    for (int j = 0; j < a.k; ++j) {
        double best = -kInf64;
        int at = 0x7fffffff;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            at = v[i] > best ? expert_of<T, L>(lane, i) : at;
            best = __builtin_fmax(best, v[i]);
        }
#pragma unroll
        for (int d = 1; d < L; d <<= 1) {
            const double y = __shfl_xor(best, d);
            const int e = __shfl_xor(at, d);
            at = y > best || (y == best && e < at) ? e : at;
            best = __builtin_fmax(best, y);
        }
        const bool found = best > -kInf64;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (found && expert_of<T, L>(lane, i) == at) v[i] = -kInf64;
        if (j % L == lane) chosen[j] = found ? at : -1;
    }
}

// What the weights of a token's chosen are made of: p times a factor that is the same for all of them and keeps them in range.
//   sigmoid: e^(x - c) / (1 + e^x), c the largest chosen x if that is below 0;  softmax: e^(x - c), c the largest
__device__ inline float part_of(bool soft, float x, float c) {
    if (soft) return expf(x - c);
    return x > 0.0f ? 1.0f / (1.0f + expf(-x)) : expf(x - c) / (1.0f + expf(x));
}

template <typename T, int L, int N, int V>
__global__ __launch_bounds__(kThreads) void route_biased_choose(const Biased a) {
    constexpr int kGroups = L * N < 64 ? L * N : 64;
    __shared__ int32_t count[L * N + 1];
    __shared__ double score[kThreads / L][kGroups];
    const int t = threadIdx.x, lane = t & (L - 1);
    for (int i = t; i <= L * N; i += kThreads) count[i] = 0;
    __syncthreads();
    const uint32_t step = gridDim.x * (kThreads / L);
    for (uint64_t token = blockIdx.x * (kThreads / L) + t / L; token < a.tokens; token += step) {
        const bool keep = !a.keep || a.keep[token];
        const T* const row = static_cast<const T*>(a.logits) + token * a.stride;
        int32_t* const chosen = a.chosen + token * a.k;
        float* const weights = a.weights + token * a.k;
        float x[N];
        load_logits<T, L, N, V>(x, row, lane, a.experts);
        bool bad = false;   // a NaN, or with softmax +inf
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = keep ? x[i] : -kInf;
            bad |= a.soft ? !(x[i] < kInf) : x[i] != x[i];
        }
        bad = lanes_or<L>(static_cast<unsigned>(bad));
        if (bad) {
            for (int j = lane; j < a.k; j += L) {
                chosen[j] = -1;
                weights[j] = __builtin_nanf("");
            }
            continue;
        }
        choose<T, L, N>(a, x, lane, score[t / L], chosen);
        const bool whole = a.soft && !a.normalize;   // parts of the token's whole softmax
        float most = -kInf, sum = 0.0f;
        if (whole) {
#pragma unroll
            for (int i = 0; i < N; ++i) most = __builtin_fmaxf(most, x[i]);
            most = lanes_max<L>(most);
#pragma unroll
            for (int i = 0; i < N; ++i) sum += x[i] > -kInf ? power(x[i] - most) : 0.0f;
        } else if (a.normalize) {
            for (int j = lane; j < a.k; j += L)
                if (chosen[j] >= 0) most = __builtin_fmaxf(most, static_cast<float>(row[chosen[j]]));
            most = lanes_max<L>(most);
            if (!a.soft) most = __builtin_fminf(most, 0.0f);
            for (int j = lane; j < a.k; j += L)
                if (chosen[j] >= 0) sum += part_of(a.soft, static_cast<float>(row[chosen[j]]), most);
        }
        sum = whole || a.normalize ? lanes_sum<L>(sum) : 1.0f;
        const float c = whole || a.normalize ? most : 0.0f;
        for (int j = lane; j < a.k; j += L) {
            const int e = chosen[j];
            weights[j] = e < 0 ? 0.0f : a.scale * (part_of(a.soft, static_cast<float>(row[e]), c) / sum);
            if (e >= 0) atomicAdd(&count[e], 1);
            if (e >= 0 && j == 0) atomicAdd(&count[L * N], 1);
        }
    }
    __syncthreads();
    for (int i = t; i <= a.experts; i += kThreads)
        a.counts[static_cast<uint64_t>(blockIdx.x) * (a.experts + 1) + i] = count[i < a.experts ? i : L * N];
}

// Adds up what the workgroups left: eight columns to a workgroup, so that it has many loads under way at once.
constexpr int kAddThreads = 1024, kAddColumns = 8;
__global__ __launch_bounds__(kAddThreads) void route_biased_add(const int32_t* counts, uint32_t groups, int columns, int32_t* count) {
    __shared__ int32_t c[kAddThreads / 64][kAddColumns];
    const int t = threadIdx.x, at = t % kAddColumns, column = blockIdx.x * kAddColumns + at;
    int32_t many = 0;
    if (column < columns)
#pragma unroll 4
        for (uint32_t g = t / kAddColumns; g < groups; g += kAddThreads / kAddColumns) many += counts[static_cast<uint64_t>(g) * columns + column];
    for (int d = kAddColumns; d < 64; d <<= 1) many += __shfl_xor(many, d);
    if ((t & 63) < kAddColumns) c[t >> 6][at] = many;
    __syncthreads();
    if (t >= kAddColumns || column >= columns) return;
    for (int w = 1; w < kAddThreads / 64; ++w) many += c[w][at];
    count[column] = many;
}

constexpr int kBiasThreads = 256;   // at most four experts to a thread
__global__ __launch_bounds__(kBiasThreads) void route_bias_kernel(const int32_t* counts, const float* bias, float* out, int experts, float rate) {
    __shared__ int64_t part[kBiasThreads / 64];
    int32_t c[4];
    int64_t sum = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int e = u * kBiasThreads + threadIdx.x;
        c[u] = e < experts ? counts[e] : 0;
        sum += c[u];
    }
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = 0;
    for (int w = 0; w < kBiasThreads / 64; ++w) sum += part[w];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int e = u * kBiasThreads + threadIdx.x;
        if (e >= experts) break;
        const int64_t off = sum - static_cast<int64_t>(c[u]) * experts;   // experts times (mean - c)
        out[e] = bias[e] + (off > 0 ? rate : off < 0 ? -rate : 0.0f);
    }
}

// ---- gradient -----------------------------------------------------------------------------------------------------------------
struct BiasedGradient {
    const void* logits;
    uint64_t stride;
    const uint8_t* keep;
    uint32_t tokens;
    int experts, k;
    bool soft, normalize;
    float scale;
    const int32_t* chosen;
    const float* grad_weights;
    void* out;
    uint64_t out_stride;
    bool past;
};

template <typename T, int L, int N, int V>
__global__ __launch_bounds__(kThreads) void route_biased_gradient_kernel(const BiasedGradient a) {
    // what the token's chosen get (with a whole softmax: d), 0 wherever no token's are; four neighbours of each lane side by side
    __shared__ __align__(16) float by_expert[kThreads / L][L * N];
    const int t = threadIdx.x, lane = t & (L - 1);
    float* const add = by_expert[t / L];
    constexpr int G = kNeighbours<T>;
    const auto place_at = [](int lane, int i) { return (i / 4 * L + lane) * 4 + i % 4; };
    const auto place = [&](int e) { return place_at(e / G % L, e / (G * L) * G + e % G); };
#pragma unroll
    for (int i = 0; i < N; ++i) add[place_at(lane, i)] = 0.0f;
    const bool whole = a.soft && !a.normalize;
    const uint32_t step = gridDim.x * (kThreads / L);
    for (uint64_t token = blockIdx.x * (kThreads / L) + t / L; token < a.tokens; token += step) {
        const bool keep = !a.keep || a.keep[token];
        const T* const row = static_cast<const T*>(a.logits) + token * a.stride;
        // f(expert, gradient of its weight, its logit) for each of the lane's chosen
        const auto each = [&](auto f) {
            if (!keep) return;
            for (int j = lane; j < a.k; j += L) {
                const int e = a.chosen[token * a.k + j];
                if (e >= 0 && e < a.experts) f(e, a.grad_weights[token * a.k + j], static_cast<float>(row[e]));
            }
        };
        float most = -kInf;
        double sum = 0.0, dot = 0.0;   // in 64 bits: g less its mean may be small
        unsigned any = 0;
        if (a.normalize) {
            each([&](int, float, float x) { most = __builtin_fmaxf(most, x); });
            most = lanes_max<L>(most);
            if (!a.soft) most = __builtin_fminf(most, 0.0f);
            each([&](int, float g, float x) {
                const double p = part_of(a.soft, x, most);
                sum += p;
                dot += p * g;
            });
            sum = lanes_sum<L>(sum);
            dot = lanes_sum<L>(dot) / sum;
        }
        each([&](int e, float g, float x) {
            float d = a.scale * g;
            if (a.normalize) d = static_cast<float>(a.scale * (g - dot) * (part_of(a.soft, x, most) / sum));
            else if (!a.soft) d *= part_of(false, x, 0.0f);
            if (!a.soft) d *= 1.0f / (1.0f + expf(x));
            add[place(e)] = d;
            any = 1;
        });
        wave_sync();
        float d[N];
#pragma unroll
        for (int i = 0; i < N; ++i) d[i] = add[place_at(lane, i)];
        wave_sync();
        each([&](int e, float, float) { add[place(e)] = 0.0f; });
        wave_sync();
        if (whole && lanes_or<L>(any)) {
            float x[N], from, scale, lse;
            load_logits<T, L, N, V>(x, row, lane, a.experts);
            softmax<L, N>(x, &from, &scale, &lse);
            float all = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) all = __builtin_fmaf(x[i], d[i], all);
            all = lanes_sum<L>(all) * scale;
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] = x[i] * scale * (d[i] - all);
        }
        T* const out = static_cast<T*>(a.out) + token * a.out_stride;
#pragma unroll
        for (int i = 0; i < N; i += V) {
            Pack<T, V> y;
#pragma unroll
            for (int v = 0; v < V; ++v) y.v[v] = static_cast<T>(d[i + v]);
            const int e = expert_of<T, L>(lane, i);
            if (e < a.experts) store_result(a.past, reinterpret_cast<Pack<T, V>*>(out + e), y);
        }
    }
}

// ---- host side ----------------------------------------------------------------------------------------------------------------
uint32_t groups_of(size_t tokens, int experts) {
    return static_cast<uint32_t>(std::min<uint64_t>(kMostGroups, ceil_div(tokens, kThreads / lanes_of(experts))));
}

}  // namespace

size_t route_biased_workspace(size_t tokens, int experts) {
    const uint32_t groups = groups_of(tokens, experts);
    return groups > 1 ? static_cast<size_t>(groups) * (experts + 1) * sizeof(int32_t) : 0;
}

blink_status_t route_biased(const void* logits, blink_dtype_t dtype, size_t tokens, int experts, size_t stride, const uint8_t* keep, const float* bias, int k,
                            int expert_groups, int kept_groups, bool soft, bool normalize, float scale, int32_t* chosen, float* weights, int32_t* counts,
                            void* workspace, hipStream_t stream) {
    const uint32_t groups = std::max(1u, groups_of(tokens, experts));
    const Biased a{logits, stride, keep, bias, static_cast<uint32_t>(tokens), experts, k, kept_groups < expert_groups ? expert_groups : 1, kept_groups, soft,
                   normalize, scale, chosen, weights, groups > 1 ? static_cast<int32_t*>(workspace) : counts};
    BLINK_TRY(with_float(dtype, [&](auto type) {
        using T = decltype(type);
        return with_load<T>(experts, stride, logits, stride, logits, [&](auto v) {
            return with_lanes(experts, [&](auto l, auto n) {
                return launch(route_biased_choose<T, decltype(l)::value, decltype(n)::value, decltype(v)::value>, dim3(groups), dim3(kThreads), stream, a);
            });
        });
    }));
    if (groups == 1) return BLINK_OK;
    return launch(route_biased_add, dim3(static_cast<uint32_t>(ceil_div(experts + 1, kAddColumns))), dim3(kAddThreads), stream, a.counts, groups, experts + 1,
                  counts);
}

blink_status_t route_bias(const int32_t* counts, const float* bias, float* out, int experts, float rate, hipStream_t stream) {
    return launch(route_bias_kernel, dim3(1), dim3(kBiasThreads), stream, counts, bias, out, experts, rate);
}

blink_status_t route_biased_gradient(const void* logits, blink_dtype_t dtype, size_t tokens, int experts, size_t stride, const uint8_t* keep, int k, bool soft,
                                     bool normalize, float scale, const int32_t* chosen, const float* grad_weights, void* out, size_t out_stride,
                                     hipStream_t stream) {
    if (tokens == 0) return BLINK_OK;
    const BiasedGradient a{logits, stride, keep, static_cast<uint32_t>(tokens), experts, k, soft, normalize, scale, chosen, grad_weights, out, out_stride,
                           passes_caches(tokens * experts * size_of(dtype))};
    const uint32_t groups = static_cast<uint32_t>(std::min<uint64_t>(4 * kMostGroups, ceil_div(tokens, kThreads / lanes_of(experts))));
    return with_float(dtype, [&](auto type) {
        using T = decltype(type);
        return with_load<T>(experts, stride, logits, out_stride, out, [&](auto v) {
            return with_lanes(experts, [&](auto l, auto n) {
                return launch(route_biased_gradient_kernel<T, decltype(l)::value, decltype(n)::value, decltype(v)::value>, dim3(groups), dim3(kThreads), stream,
                              a);
            });
        });
    });
}

}  // namespace blink
