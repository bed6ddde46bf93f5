// What L neighbouring lanes of a wave hold together: their sum, their largest (route.hip, route_biased.hip, update.hip).
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

namespace blink {

// L neighbouring lanes, L a power of two.
// op(own value, the other half's), for halves of 1, 2, 4 ... lanes, each of which holds one value by then.
template <int L, typename X, typename F>
__device__ inline X over_lanes(X x, F op) {
    const auto dpp = [](X v, auto control) {
        return __builtin_bit_cast(X, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(control)::value, 0xf, 0xf, true));
    };
    if constexpr (L > 1) x = op(x, dpp(x, std::integral_constant<int, 0xB1>()));    // quad_perm 1 0 3 2
    if constexpr (L > 2) x = op(x, dpp(x, std::integral_constant<int, 0x4E>()));    // quad_perm 2 3 0 1
    if constexpr (L > 4) x = op(x, dpp(x, std::integral_constant<int, 0x141>()));   // row_half_mirror
    if constexpr (L > 8) x = op(x, dpp(x, std::integral_constant<int, 0x140>()));   // row_mirror
    if constexpr (L > 16) {
        const unsigned v = __builtin_bit_cast(unsigned, x);
        const auto both = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        x = op(__builtin_bit_cast(X, static_cast<unsigned>(both[0])), __builtin_bit_cast(X, static_cast<unsigned>(both[1])));
    }
    if constexpr (L > 32) {
        const unsigned v = __builtin_bit_cast(unsigned, x);
        const auto both = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        x = op(__builtin_bit_cast(X, static_cast<unsigned>(both[0])), __builtin_bit_cast(X, static_cast<unsigned>(both[1])));
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
__device__ inline unsigned lanes_max(unsigned x) {
    return over_lanes<L>(x, [](unsigned a, unsigned b) { return a > b ? a : b; });
}
template <int L>
__device__ inline unsigned lanes_min(unsigned x) {
    return over_lanes<L>(x, [](unsigned a, unsigned b) { return a < b ? a : b; });
}
template <int L>
__device__ inline unsigned lanes_or(unsigned x) {
    return over_lanes<L>(x, [](unsigned a, unsigned b) { return a | b; });
}
template <int L>
__device__ inline int lanes_least(int x) {
    return over_lanes<L>(x, [](int a, int b) { return a < b ? a : b; });
}
template <int L>
__device__ inline double lanes_sum(double x) {
#pragma unroll
    for (int d = 1; d < L; d <<= 1) x += __shfl_xor(x, d);
    return x;
}
// The same over a wave for values of more than 32 bits, whole words of them.
template <typename X, typename F>
__device__ inline X over_wave(X x, F op) {
    constexpr int kWords = sizeof(X) / 4;
    struct Words {
        unsigned w[kWords];
    };
    const auto moved = [&](auto control) {
        Words y = __builtin_bit_cast(Words, x);
#pragma unroll
        for (int i = 0; i < kWords; ++i) y.w[i] = __builtin_amdgcn_update_dpp(0, static_cast<int>(y.w[i]), decltype(control)::value, 0xf, 0xf, true);
        return __builtin_bit_cast(X, y);
    };
    x = op(x, moved(std::integral_constant<int, 0xB1>()));
    x = op(x, moved(std::integral_constant<int, 0x4E>()));
    x = op(x, moved(std::integral_constant<int, 0x141>()));
    x = op(x, moved(std::integral_constant<int, 0x140>()));
    const auto halves = [&](auto swap) {
        const Words y = __builtin_bit_cast(Words, x);
        Words a, b;
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            const auto both = swap(y.w[i]);
            a.w[i] = both[0];
            b.w[i] = both[1];
        }
        x = op(__builtin_bit_cast(X, a), __builtin_bit_cast(X, b));
    };
    halves([](unsigned v) { return __builtin_amdgcn_permlane16_swap(v, v, false, false); });
    halves([](unsigned v) { return __builtin_amdgcn_permlane32_swap(v, v, false, false); });
    return x;
}

}  // namespace blink
