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
// sums over tokens stay in registers until its end.  Every lane puts its logits in order by a network of exchanges; the k largest are
// then the k largest of the lanes' first ones in turn, at a cost that hardly depends on N.  Workgroups leave their sums in the workspace, a second kernel adds
// them up in order.  Both kernels over the logits read them once.
#include "operators_api.hpp"

#include <algorithm>
#include <type_traits>

namespace blink {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMostGroups = 1024;        // workgroups of the first kernel: 16 waves on a CU
constexpr float kInf = __builtin_inff();

// ---- lanes of a token: L neighbours, L a power of two -----------------------------------------------------------------------
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

// ---- the largest, in order --------------------------------------------------------------------------------------------------
// A logit as a whole number of the same order, above 0 unless it is -inf, a NaN or past the last; equal logits, 0 and -0 among
// them, are in the order of their index.  16-bit logits have room for the index below them, so one number is both.
constexpr uint32_t kLowest = 0x007fffff;   // of -inf, as a 32-bit float

__device__ inline uint32_t ordered(uint32_t bits) { return bits ^ (static_cast<uint32_t>(static_cast<int32_t>(bits) >> 31) | 0x80000000u); }
__device__ inline uint32_t in_order(uint32_t o) { return o >> 31 ? o ^ 0x80000000u : ~o; }   // the bits again

template <typename T>
struct Key {   // a 16-bit logit and its index
    static constexpr bool kBrain = std::is_same<T, __bf16>::value;
    uint32_t v = 0;
    __device__ static Key of(float x, uint32_t index) {
        uint32_t bits;   // (adding 0 makes 0 of -0)
        if constexpr (kBrain) bits = __builtin_bit_cast(uint32_t, x + 0.0f);
        else bits = static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<T>(x + 0.0f))) << 16;
        Key k;
        k.v = (ordered(bits) & 0xffff0000u) | (0xffffu - index);
        return k;
    }
    static constexpr uint32_t kNone = kBrain ? 0x007fffff : 0x03ffffff;   // -inf's, of whatever index
    __device__ bool valid() const { return v > kNone; }
    __device__ uint32_t index() const { return 0xffffu - (v & 0xffffu); }
    __device__ float value() const { return static_cast<float>(__builtin_bit_cast(T, static_cast<uint16_t>(in_order(v & 0xffff0000u | 0xffffu) >> 16))); }
    __device__ static Key pick(bool first, Key a, Key b) {
        a.v = first ? a.v : b.v;
        return a;
    }
    __device__ static void order(Key& a, Key& b) {   // a the larger
        const uint32_t x = a.v, y = b.v;
        a.v = x > y ? x : y;
        b.v = x > y ? y : x;
    }
    template <int L>
    __device__ static Key best(Key mine, bool* won) {
        Key k;
        k.v = lanes_max<L>(mine.v);
        *won = k.v == mine.v;
        return k;
    }
};
template <>
struct Key<float> {
    uint32_t v = 0, i = 0xffffu;
    __device__ static Key of(float x, uint32_t index) {
        Key k;
        k.v = ordered(__builtin_bit_cast(uint32_t, x + 0.0f));
        k.i = index;
        return k;
    }
    __device__ bool valid() const { return v > kLowest; }
    __device__ uint32_t index() const { return i; }
    __device__ float value() const { return __builtin_bit_cast(float, in_order(v)); }
    __device__ static Key pick(bool first, Key a, Key b) {
        a.v = first ? a.v : b.v;
        a.i = first ? a.i : b.i;
        return a;
    }
    __device__ static void order(Key& a, Key& b) {
        const Key x = a, y = b;
        const bool swap = y.v > x.v || (y.v == x.v && y.i < x.i);
        a.v = swap ? y.v : x.v;
        a.i = swap ? y.i : x.i;
        b.v = swap ? x.v : y.v;
        b.i = swap ? x.i : y.i;
    }
    template <int L>
    __device__ static Key best(Key mine, bool* won) {
        Key k;
        k.v = lanes_max<L>(mine.v);
        k.i = lanes_min<L>(mine.v == k.v ? mine.i : 0xffffu);
        *won = k.v == mine.v && k.i == mine.i;
        return k;
    }
};

// Eight keys, the largest first (Batcher's odd-even merge sort, 19 exchanges).
template <typename K>
__device__ inline void sort8(K (&k)[8]) {
    constexpr int pair[19][2] = {{0, 1}, {2, 3}, {4, 5}, {6, 7}, {0, 2}, {1, 3}, {4, 6}, {5, 7}, {1, 2}, {5, 6},
                                 {0, 4}, {1, 5}, {2, 6}, {3, 7}, {2, 4}, {3, 5}, {1, 2}, {3, 4}, {5, 6}};
#pragma unroll
    for (int e = 0; e < 19; ++e) K::order(k[pair[e][0]], k[pair[e][1]]);
}
// The same of eight that rise and then fall, or the other way round (12 exchanges).
template <typename K>
__device__ inline void merge8(K (&k)[8]) {
#pragma unroll
    for (int d = 4; d > 0; d >>= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!(i & d)) K::order(k[i], k[i + d]);
}

// M: how many of its N logits a lane has to know in order, as many as k at the least or all; V logits to a load.  Bound by vector
// instructions: 262144 x 256 bfloat16, k = 8, 62 us, 470 a wave for four tokens.
template <typename T, int L, int N, int M, int V>
__global__ __launch_bounds__(kThreads) void route_choose(const Route a) {
    __shared__ int32_t count[L * N + 1];
    __shared__ float part[kWaves][L * N + 1];
    using K = Key<T>;
    const int t = threadIdx.x, wave = t >> 6, lane = t & (L - 1);
    for (int i = t; i <= L * N; i += kThreads) count[i] = 0;
    __syncthreads();
    float total[N] = {}, z = 0.0f;
    int counted = 0;
    const uint32_t step = gridDim.x * (kThreads / L);
    for (uint64_t token = blockIdx.x * (kThreads / L) + t / L; token < a.tokens; token += step) {
        const bool keep = !a.keep || a.keep[token];
        float x[N];
        load_logits<T, L, N, V>(x, static_cast<const T*>(a.logits) + token * a.stride, lane, a.experts);   // (beside `keep`, not after it)
        if (a.keep)
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = keep ? x[i] : -kInf;
        K own[8], more[8];   // in order, `more` after `own`
        bool nan = false;
#pragma unroll
        for (int i = 0; i < N; i += 2) nan |= __builtin_isunordered(x[i], x[i + 1]);
#pragma unroll
        for (int i = 0; i < 8; ++i) own[i] = K::of(x[i], expert_of<T, L>(lane, i));
        if constexpr (N == 16)
#pragma unroll
            for (int i = 0; i < 8; ++i) more[i] = K::of(x[8 + i], expert_of<T, L>(lane, 8 + i));
        if (nan)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (x[i] != x[i]) (i < 8 ? own : more)[i % 8].v = 0;   // not chosen
        sort8(own);
        if constexpr (N == 16) {
            sort8(more);
#pragma unroll
            for (int i = 0; i < 8; ++i) K::order(own[i], more[7 - i]);
            merge8(own);
            if constexpr (M == 16) merge8(more);
        }
        float most, scale, lse;
        const bool any = softmax<L, N>(x, &most, &scale, &lse);
#pragma unroll
        for (int i = 0; i < N; ++i) total[i] = __builtin_fmaf(x[i], scale, total[i]);
        z += lse * lse;
        counted += any;
        // k times the largest of the lanes' first; lane j % L keeps the j-th
        const auto write = [&](K key, int slot, float p) {
            const bool found = key.valid();
            if (found) atomicAdd(&count[key.index()], 1);
            a.chosen[token * a.k + slot] = found ? static_cast<int32_t>(key.index()) : -1;
            a.weights[token * a.k + slot] = p;
        };
        const auto weight = [&](K key) { return key.valid() ? power(key.value() - most) * scale : 0.0f; };
        if constexpr (M == 8) {   // (k is at most 8: what the j-th leaves behind of a lane's keys gets shorter)
            constexpr int kMine = (8 + L - 1) / L;
            K mine[kMine];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j >= a.k) break;
                bool won;
                const K best = K::template best<L>(own[0], &won);
#pragma unroll
                for (int i = 0; i < 7 - j; ++i) own[i] = K::pick(won, own[i + 1], own[i]);
                mine[j / L] = K::pick(lane == j % L, best, mine[j / L]);
            }
            float p[kMine], sum = 0.0f;
#pragma unroll
            for (int m = 0; m < kMine; ++m) {
                p[m] = m * L + lane < a.k ? weight(mine[m]) : 0.0f;
                sum += p[m];
            }
            const float by = a.normalize && any ? 1.0f / lanes_sum<L>(sum) : 1.0f;
#pragma unroll
            for (int m = 0; m < kMine; ++m)
                if (m * L + lane < a.k) write(mine[m], m * L + lane, p[m] * by);
        } else {
            float sum = 0.0f;
            for (int from = 0; from < a.k; from += L) {
                K mine;
                for (int j = from; j < a.k && j < from + L; ++j) {
                    bool won;
                    const K best = K::template best<L>(own[0], &won);
                    if (won) {
#pragma unroll
                        for (int i = 0; i < 7; ++i) own[i] = own[i + 1];
                        own[7] = more[0];
#pragma unroll
                        for (int i = 0; i < 7; ++i) more[i] = more[i + 1];
                        more[7] = K();
                    }
                    mine = K::pick(lane == j - from, best, mine);
                }
                const float p = from + lane < a.k ? weight(mine) : 0.0f;
                sum += p;
                if (from + lane < a.k) write(mine, from + lane, p);
            }
            if (a.normalize && any) {
                const float by = 1.0f / lanes_sum<L>(sum);
                for (int j = lane; j < a.k; j += L) a.weights[token * a.k + j] *= by;   // (its own)
            }
        }
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
        for (int i = 0; i < N; ++i) part[wave][expert_of<T, L>(lane, i)] = total[i];
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

// Adds up what the workgroups left, in 64 bits: eight columns to a workgroup, so that it has many loads under way at once (1024 x 257
// sums 5 us; 64 columns to a workgroup 11).
constexpr int kAddThreads = 1024, kAddColumns = 8;
__global__ __launch_bounds__(kAddThreads) void route_add(const int32_t* counts, const float* sums, uint32_t groups, int columns, int32_t* count, float* sum) {
    __shared__ double s[kAddThreads / 64][kAddColumns];
    __shared__ int32_t c[kAddThreads / 64][kAddColumns];
    const int t = threadIdx.x, at = t % kAddColumns, column = blockIdx.x * kAddColumns + at;
    double total = 0.0;
    int32_t many = 0;
    if (column < columns)
#pragma unroll 4
        for (uint32_t g = t / kAddColumns; g < groups; g += kAddThreads / kAddColumns) {
            total += sums[static_cast<uint64_t>(g) * columns + column];
            many += counts[static_cast<uint64_t>(g) * columns + column];
        }
    for (int d = kAddColumns; d < 64; d <<= 1) {
        total += __shfl_xor(total, d);
        many += __shfl_xor(many, d);
    }
    if ((t & 63) < kAddColumns) {
        s[t >> 6][at] = total;
        c[t >> 6][at] = many;
    }
    __syncthreads();
    if (t >= kAddColumns || column >= columns) return;
    for (int w = 1; w < kAddThreads / 64; ++w) {
        total += s[w][at];
        many += c[w][at];
    }
    sum[column] = static_cast<float>(total);
    count[column] = many;
}

constexpr int kLossThreads = 256;   // at most four experts to a thread, their loads under way together
__global__ __launch_bounds__(kLossThreads) void route_loss_kernel(const int32_t* counts, const float* sums, int experts, int k, double balance, double z, float* loss) {
    __shared__ double part[kLossThreads / 64];
    const int32_t tokens = counts[experts];
    const float squares = sums[experts];
    double s = 0.0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int e = u * kLossThreads + threadIdx.x;
        if (e < experts) s += static_cast<double>(counts[e]) * sums[e];
    }
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < kLossThreads / 64; ++w) s += part[w];
    const double n = tokens;
    const double b = n > 0 ? balance * experts / k * s / (n * n) : 0.0, l = n > 0 ? z * squares / n : 0.0;
    loss[0] = static_cast<float>(b + l);
    loss[1] = static_cast<float>(b);
    loss[2] = static_cast<float>(l);
}

// The logits are read again: their softmax would have to be written and read.  262144 x 256 bfloat16, k = 8, 67 us, 425 vector instructions a
// wave for four tokens, 268 MB.
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
    bool past;
};

template <typename T, int L, int N, int V>
__global__ __launch_bounds__(kThreads) void route_gradient_kernel(const RouteGradient a) {
    // what the weights' gradient adds to d, of the tokens that the lanes hold; four neighbours of each lane side by side, and 0
    // wherever no token's choice is being added
    __shared__ __align__(16) float by_weight[kThreads / L][L * N];
    const int t = threadIdx.x, lane = t & (L - 1);
    float* const add = by_weight[t / L];
    constexpr int G = kNeighbours<T>;
    const auto place_at = [](int lane, int i) { return (i / 4 * L + lane) * 4 + i % 4; };
    const auto place = [&](int e) { return place_at(e / G % L, e / (G * L) * G + e % G); };
#pragma unroll
    for (int i = 0; i < N; ++i) add[place_at(lane, i)] = 0.0f;
    const float up = a.grad_loss ? *a.grad_loss : 1.0f;
    const float n = static_cast<float>(a.counts[a.experts] > 0 ? a.counts[a.experts] : 1);
    float by_p[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = expert_of<T, L>(lane, i);
        by_p[i] = e < a.experts ? up * a.balance * a.experts / a.k * (a.counts[e] / n) / n : 0.0f;
    }
    const float by_lse = 2.0f * up * a.z / n;
    const uint32_t step = gridDim.x * (kThreads / L);
    for (uint64_t token = blockIdx.x * (kThreads / L) + t / L; token < a.tokens; token += step) {
        const bool keep = !a.keep || a.keep[token];
        const T* const row = static_cast<const T*>(a.logits) + token * a.stride;
        float x[N], d[N];
        // this lane's first choice travels with the logits
        const auto choice = [&](int j, int* e, float* g) {
            *e = j < a.k ? a.chosen[token * a.k + j] : -1;
            *g = j < a.k ? a.grad_weights[token * a.k + j] : 0.0f;
            if (*e >= a.experts) *e = -1;
        };
        int e0 = -1;
        float g0 = 0.0f;
        if (a.grad_weights) choice(lane, &e0, &g0);
        load_logits<T, L, N, V>(x, row, lane, a.experts);
        if (a.keep)
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = keep ? x[i] : -kInf;
        float most, scale, lse;
        const bool any = softmax<L, N>(x, &most, &scale, &lse);
#pragma unroll
        for (int i = 0; i < N; ++i) d[i] = by_p[i];
        if (a.grad_weights && keep) {
            // lanes of a token are lanes of one wave, whose accesses to LDS happen in order
            const auto each = [&](auto f) {
                if (e0 >= 0) f(e0, g0);
                for (int j = lane + L; j < a.k; j += L) {
                    int e;
                    float g;
                    choice(j, &e, &g);
                    if (e >= 0) f(e, g);
                }
            };
            float by = 1.0f, dot = 0.0f;
            if (a.normalize) {   // d of the chosen: (g - sum w g) / S
                float sum = 0.0f;
                each([&](int e, float g) {
                    const float p = power(static_cast<float>(row[e]) - most) * scale;
                    sum += p;
                    dot = __builtin_fmaf(p, g, dot);
                });
                by = 1.0f / lanes_sum<L>(sum);
                dot = lanes_sum<L>(dot) * by;
            }
            each([&](int e, float g) { add[place(e)] = (g - dot) * by; });
            wave_sync();
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] += add[place_at(lane, i)];
            wave_sync();
            each([&](int e, float) { add[place(e)] = 0.0f; });
            wave_sync();
        }
        float dot = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) dot = __builtin_fmaf(x[i], d[i], dot);
        dot = (by_lse * lse - lanes_sum<L>(dot) * scale) * scale;
        T* const out = static_cast<T*>(a.out) + token * a.out_stride;
#pragma unroll
        for (int i = 0; i < N; i += V) {
            Pack<T, V> y;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float z = x[i + v] * __builtin_fmaf(scale, d[i + v], dot);
                y.v[v] = static_cast<T>(any ? z : 0.0f);
            }
            const int e = expert_of<T, L>(lane, i);
            if (e < a.experts) store_result(a.past, reinterpret_cast<Pack<T, V>*>(out + e), y);
        }
    }
}

// ---- host side ----------------------------------------------------------------------------------------------------------------
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

uint32_t lanes_of(int experts) {
    uint32_t l = 1;
    while (static_cast<int>(l * 16) < experts) l <<= 1;
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
        return with_load<T>(experts, stride, logits, stride, logits, [&](auto v) {
            return with_lanes(experts, [&](auto l, auto n) {
                constexpr int L = decltype(l)::value, N = decltype(n)::value, V = decltype(v)::value;
                return launch(k <= 8 ? route_choose<T, L, N, 8, V> : route_choose<T, L, N, N, V>, dim3(groups), dim3(kThreads), stream, a);
            });
        });
    }));
    if (groups == 1) return BLINK_OK;
    return launch(route_add, dim3(static_cast<uint32_t>(ceil_div(experts + 1, kAddColumns))), dim3(kAddThreads), stream, a.counts, a.sums, groups, experts + 1,
                  counts, sums);
}

blink_status_t route_loss(const int32_t* counts, const float* sums, int experts, int k, float balance, float z, float* loss, hipStream_t stream) {
    return launch(route_loss_kernel, dim3(1), dim3(kLossThreads), stream, counts, sums, experts, k, static_cast<double>(balance), static_cast<double>(z), loss);
}

blink_status_t route_gradient(const void* logits, blink_dtype_t dtype, size_t tokens, int experts, size_t stride, const uint8_t* keep, int k,
                              bool normalize, const int32_t* chosen, const float* grad_weights, const int32_t* counts, const float* grad_loss,
                              float balance, float z, void* out, size_t out_stride, hipStream_t stream) {
    if (tokens == 0) return BLINK_OK;
    const RouteGradient a{logits, stride, keep, static_cast<uint32_t>(tokens), experts, k, normalize, chosen, grad_weights, counts, grad_loss,
                          balance, z, out, out_stride, passes_caches(tokens * experts * size_of(dtype))};
    // no sums are kept from token to token: as many workgroups as there are tokens for, in the end
    const uint32_t groups = static_cast<uint32_t>(std::min<uint64_t>(4 * kMostGroups, ceil_div(tokens, kThreads / lanes_of(experts))));
    return with_float(dtype, [&](auto type) {
        using T = decltype(type);
        return with_load<T>(experts, stride, logits, out_stride, out, [&](auto v) {
            return with_lanes(experts, [&](auto l, auto n) {
                constexpr int L = decltype(l)::value, N = decltype(n)::value, V = decltype(v)::value;
                return launch(route_gradient_kernel<T, L, N, V>, dim3(groups), dim3(kThreads), stream, a);
            });
        });
    });
}

}  // namespace blink
