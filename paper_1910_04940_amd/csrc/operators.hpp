// What the operators around the collectives share (embedding.hip, route.hip, orthogonal.hip): element types, wide
// loads, the launch.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>
#include <cstdio>
#include <tuple>
#include <utility>

#include "../../include/blink.h"

namespace blink {

// N elements that are loaded and stored at once; rows of them start on their alignment wherever this is used.
template <typename T, int N>
struct alignas(sizeof(T) * N) Pack {
    T v[N];
};

// Results larger than the eight dies' second-level caches together stream past them, where they would only push out what is read: 131072
// rows of 4 KiB 166 us otherwise, 115 so; logits' gradients of 128 MiB 151 (with the choice), 142.
inline bool passes_caches(uint64_t bytes) { return bytes > (32u << 20); }
template <typename P>
__device__ inline void store_past(P* to, const P& y) {
    typedef unsigned U4 __attribute__((ext_vector_type(4)));
    typedef unsigned U2 __attribute__((ext_vector_type(2)));
    if constexpr (sizeof(P) == 16) __builtin_nontemporal_store(__builtin_bit_cast(U4, y), reinterpret_cast<U4*>(to));
    else if constexpr (sizeof(P) == 8) __builtin_nontemporal_store(__builtin_bit_cast(U2, y), reinterpret_cast<U2*>(to));
    else *to = y;
}
template <typename P>
__device__ inline void store_result(bool past, P* to, const P& y) {
    if (past) {   // (the empty statements keep the compiler from making one ordinary store of the two)
        asm volatile("");
        store_past(to, y);
        asm volatile("");
    } else *to = y;
}

inline size_t size_of(blink_dtype_t t) { return t == BLINK_INT64 ? 8 : t == BLINK_BF16 || t == BLINK_FP16 ? 2 : 4; }
inline bool is_float(blink_dtype_t t) { return t == BLINK_FP32 || t == BLINK_BF16 || t == BLINK_FP16; }
inline bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// Calls f with a value of the C++ type of `t` (a floating one).
template <typename F>
auto with_float(blink_dtype_t t, F f) {
    if (t == BLINK_BF16) return f(__bf16());
    if (t == BLINK_FP16) return f(_Float16());
    return f(float());
}

// hipLaunchKernel returns its own error, not one that somebody else's call left behind.
template <typename... P, size_t... I>
blink_status_t launch_with(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t stream, std::tuple<P...>& args, std::index_sequence<I...>) {
    void* at[] = {static_cast<void*>(&std::get<I>(args))...};
    const hipError_t err = hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, at, 0, stream);
    if (err == hipSuccess) return BLINK_OK;
    std::fprintf(stderr, "blink: kernel launch failed: %s\n", hipGetErrorString(err));
    return err == hipErrorOutOfMemory ? BLINK_ENOMEM : BLINK_EHIP;
}
template <typename... P, typename... A>
blink_status_t launch(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t stream, A... a) {
    std::tuple<P...> args(static_cast<P>(a)...);
    return launch_with(kernel, grid, block, stream, args, std::index_sequence_for<P...>());
}

// Orders a wave's accesses to LDS for the compiler; the wave itself makes them in order.
__device__ inline void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

#define BLINK_TRY(call)                                   \
    do {                                                  \
        const blink_status_t st__ = (call);               \
        if (st__ != BLINK_OK) return st__;                \
    } while (0)

inline uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

// A launch has fewer than 2^32 threads in x.  More workgroups than that go in rows, y of them; block_of is a workgroup's number, which is past
// the last one for some of the last row.
struct Grid {
    uint32_t x, y;
};
inline Grid grid_of(uint64_t groups, uint32_t threads) {
    const uint64_t y = groups == 0 ? 1 : ceil_div(groups, 0xffffffffu / threads);
    return {static_cast<uint32_t>(ceil_div(groups, y)), static_cast<uint32_t>(y)};
}
__device__ inline uint32_t block_of(uint32_t row) { return row * gridDim.x + blockIdx.x; }

// Parts of a workspace, each on a 256-byte line.
struct Carve {
    char* base;
    size_t at = 0;
    explicit Carve(void* p) : base(static_cast<char*>(p)) {}
    template <typename T>
    T* take(size_t n) {
        T* const p = reinterpret_cast<T*>(base + at);
        at += (n * sizeof(T) + 255) / 256 * 256;
        return p;
    }
};

}  // namespace blink
