// Logits of a token in L neighbouring lanes, N to a lane (route.hip, route_biased.hip).
#pragma once
#include <type_traits>

#include "lanes.hpp"
#include "operators.hpp"

namespace blink {

constexpr int kRouteThreads = 256;       // of a workgroup
constexpr float kInf = __builtin_inff();

// The expert whose logit is a lane's i-th: 16 bytes of neighbours to a lane, then the next lane's, so that a load of the wave is one
// piece.  How wide the loads really are changes nothing in it, so that sums do not depend on where a row starts.
template <typename T>
constexpr int kNeighbours = 16 / sizeof(T);
template <typename T, int L>
__device__ inline int expert_of(int lane, int i) {
    return (i / kNeighbours<T> * L + lane) * kNeighbours<T> + i % kNeighbours<T>;
}

// A lane's logits, -inf past the last; V of them at a time.
template <typename T, int L, int N, int V>
__device__ inline void load_logits(float (&x)[N], const T* row, int lane, int experts) {
    const auto load = [&](auto all) {
#pragma unroll
        for (int i = 0; i < N; i += V) {
            Pack<T, V> y;
            const int e = expert_of<T, L>(lane, i);
            const bool in = decltype(all)::value || e < experts;
            if (in) y = *reinterpret_cast<const Pack<T, V>*>(row + e);
#pragma unroll
            for (int v = 0; v < V; ++v) x[i + v] = in ? static_cast<float>(y.v[v]) : -kInf;
        }
    };
    if (experts == L * N) load(std::true_type());
    else load(std::false_type());
}

__device__ inline float power(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }   // e^x, 0 for -inf

// Softmax of a token: x becomes p / scale.  False if all logits are -inf (p is then 0).  A NaN, or +inf, makes p NaN.
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
    *most = from;
    *scale = any ? 1.0f / s : 0.0f;
    *lse = any ? from + logf(s) : 0.0f;
    return any;
}

// Sixteen logits to a lane (eight where they are all): f is called with the lanes and that number.  More lanes with fewer each spend
// more on what they do together.
template <typename F>
blink_status_t with_lanes(int experts, F f) {
    using std::integral_constant;
    using Sixteen = integral_constant<int, 16>;
    if (experts <= 8) return f(integral_constant<int, 1>(), integral_constant<int, 8>());
    if (experts <= 16) return f(integral_constant<int, 1>(), Sixteen());
    if (experts <= 32) return f(integral_constant<int, 2>(), Sixteen());
    if (experts <= 64) return f(integral_constant<int, 4>(), Sixteen());
    if (experts <= 128) return f(integral_constant<int, 8>(), Sixteen());
    if (experts <= 256) return f(integral_constant<int, 16>(), Sixteen());
    if (experts <= 512) return f(integral_constant<int, 32>(), Sixteen());
    return f(integral_constant<int, 64>(), Sixteen());
}

// Calls f with the logits of a load: 16 bytes, 4 where those fit, one.
template <typename T, typename F>
blink_status_t with_load(int experts, size_t stride, const void* p, size_t other_stride, const void* q, F f) {
    const auto fits = [&](size_t v) {
        return experts % v == 0 && stride % v == 0 && other_stride % v == 0 && aligned(p, v * sizeof(T)) && aligned(q, v * sizeof(T));
    };
    constexpr int kWide = 16 / sizeof(T), kTwo = sizeof(T) == 2 ? 2 : 1;
    if (fits(kWide)) return f(std::integral_constant<int, kWide>());
    if (fits(kTwo)) return f(std::integral_constant<int, kTwo>());
    return f(std::integral_constant<int, 1>());
}

inline uint32_t lanes_of(int experts) {
    uint32_t l = 1;
    while (static_cast<int>(l * 16) < experts) l <<= 1;
    return l;
}

}  // namespace blink
