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
    uint32_t* later;       // [workgroup][room]: tokens whose choice in 32 bits is not sure; null: none
    uint32_t* left;        // [workgroup]: how many those are
    uint32_t room;
};

// What the weights of a token's chosen are made of: p times a factor that is the same for all of them and keeps them in range.
//   sigmoid: e^(x - c) / (1 + e^x), c the largest chosen x if that is below 0;  softmax: e^(x - c), c the largest
__device__ inline float part_of(bool soft, float x, float c) {
    if (soft) return expf(x - c);
    return x > 0.0f ? 1.0f / (1.0f + expf(-x)) : expf(x - c) / (1.0f + expf(x));
}

// Weights of a token's chosen, and what they add to the counts; chosen(j): the j-th, for the j of this lane.  most, sum: of the whole softmax.
// count: [experts], then the tokens'.
template <typename T, int L, typename F>
__device__ inline void weigh(const Biased& a, uint64_t token, const T* row, int lane, float most, float sum, int32_t* count, F chosen) {
    float* const weights = a.weights + token * a.k;
    float c = 0.0f, all = 1.0f;
    if (a.normalize) {
        c = -kInf;
        for (int j = lane; j < a.k; j += L) {
            const int e = chosen(j);
            if (e >= 0) c = __builtin_fmaxf(c, static_cast<float>(row[e]));
        }
        c = lanes_max<L>(c);
        if (!a.soft) c = __builtin_fminf(c, 0.0f);
        all = 0.0f;
        for (int j = lane; j < a.k; j += L) {
            const int e = chosen(j);
            if (e >= 0) all += part_of(a.soft, static_cast<float>(row[e]), c);
        }
        all = lanes_sum<L>(all);
    } else if (a.soft) {
        c = most;
        all = sum;
    }
    for (int j = lane; j < a.k; j += L) {
        const int e = chosen(j);
        weights[j] = e < 0 ? 0.0f : a.scale * (part_of(a.soft, static_cast<float>(row[e]), c) / all);
        if (e >= 0) atomicAdd(&count[e], 1);
        if (e >= 0 && j == 0) atomicAdd(&count[a.experts], 1);
    }
}

template <int L, int N>
__device__ inline bool any_nan(const float (&x)[N]) {
    bool nan = false;
#pragma unroll
    for (int i = 0; i < N; i += 2) nan |= __builtin_isunordered(x[i], x[i + 1]);
    return lanes_or<L>(static_cast<unsigned>(nan));
}
template <int L, int N>
__device__ inline float largest(const float (&x)[N]) {
    float m = -kInf;
#pragma unroll
    for (int i = 0; i < N; ++i) m = __builtin_fmaxf(m, x[i]);
    return lanes_max<L>(m);
}
template <int L>
__device__ inline void choose_none(const Biased& a, uint64_t token, int lane) {
    for (int j = lane; j < a.k; j += L) {
        a.chosen[token * a.k + j] = -1;
        a.weights[token * a.k + j] = __builtin_nanf("");
    }
}

// ---- the choice in 64 bits ----------------------------------------------------------------------------------------------------
constexpr int kMostExact = 8;   // tokens of a call that are all chosen this way

__device__ inline double wave_max(double x) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x = __builtin_fmax(x, __shfl_xor(x, d));
    return x;
}

// A wave to a token, N experts to a lane, expert 64 i + lane the i-th: for the tokens that a workgroup of route_biased_choose left in its list, for calls of a
// few tokens and for k above kMostFast.
template <typename T, int N>
__global__ __launch_bounds__(kThreads) void route_biased_exact(const Biased a) {
    __shared__ int32_t count[64 * N + 1];
    const int t = threadIdx.x, lane = t & 63;
    const uint32_t* const list = a.later ? a.later + static_cast<uint64_t>(blockIdx.x) * a.room : nullptr;
    const uint64_t n = list ? a.left[blockIdx.x] : a.tokens;
    if (list && n == 0) return;
    for (int i = t; i <= a.experts; i += kThreads) count[i] = 0;
    __syncthreads();
    const uint64_t wave = (list ? 0 : blockIdx.x) * (kThreads / 64) + t / 64, step = (list ? 1 : gridDim.x) * (kThreads / 64);
    for (uint64_t at = wave; at < n; at += step) {
        const uint64_t token = list ? list[at] : at;
        const bool keep = !a.keep || a.keep[token];
        const T* const row = static_cast<const T*>(a.logits) + token * a.stride;
        int32_t* const chosen = a.chosen + token * a.k;
        float x[N];
        double v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = 64 * i + lane;
            x[i] = keep && e < a.experts ? static_cast<float>(row[e]) : -kInf;
        }
        float most = -kInf, sum = 0.0f;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            most = __builtin_fmaxf(most, x[i]);
            bad |= a.soft ? !(x[i] < kInf) : x[i] != x[i];
        }
        if (__any(bad)) {
            choose_none<64>(a, token, lane);
            continue;
        }
        if (a.soft) {
            most = lanes_max<64>(most);
            const double from = most == -kInf ? 0.0 : most;
            double s = 0.0;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[i] = exp(x[i] - from);
                s += v[i];
            }
            s = lanes_sum<64>(s);
            sum = static_cast<float>(s);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] /= s;
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = 1.0 / (1.0 + exp(-static_cast<double>(x[i])));
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = 64 * i + lane;
            const double y = v[i] + (a.bias && e < a.experts ? static_cast<double>(a.bias[e]) : 0.0);
            v[i] = x[i] > -kInf && y > -kInf64 ? y : -kInf64;   // (a bias of -inf or NaN: never)
        }
        if (a.groups > 1) {
            const int size = a.experts / a.groups;
            double score = -kInf64;   // of group `lane`
            for (int g = 0; g < a.groups; ++g) {
                double first = -kInf64, second = -kInf64;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int e = 64 * i + lane - g * size;
                    const double y = e >= 0 && e < size ? v[i] : -kInf64;
                    second = __builtin_fmax(second, __builtin_fmin(first, y));
                    first = __builtin_fmax(first, y);
                }
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const double f = __shfl_xor(first, d), s = __shfl_xor(second, d);
                    second = __builtin_fmax(__builtin_fmin(first, f), __builtin_fmax(second, s));
                    first = __builtin_fmax(first, f);
                }
                score = lane == g ? (second > -kInf64 ? first + second : first) : score;
            }
            int before = 0;
            for (int h = 0; h < a.groups; ++h) {
                const double other = __shfl(score, h);
                before += other > score || (other == score && h < lane);
            }
            const uint64_t stay = __ballot(lane < a.groups && before < a.kept);
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (!(stay >> ((64 * i + lane) / size & 63) & 1)) v[i] = -kInf64;
        }
        for (int j = 0; j < a.k; ++j) {
            double best = v[0];
#pragma unroll
            for (int i = 1; i < N; ++i) best = __builtin_fmax(best, v[i]);
            best = wave_max(best);
            int at = -1;
#pragma unroll
            for (int i = N - 1; i >= 0; --i) {   // the lowest index
                const uint64_t mask = __ballot(v[i] == best && best > -kInf64);
                if (mask) at = 64 * i + __builtin_ctzll(mask);
            }
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (64 * i + lane == at) v[i] = -kInf64;
            if (j % 64 == lane) chosen[j] = at;
        }
        weigh<T, 64>(a, token, row, lane, most, sum, count, [&](int j) { return chosen[j]; });   // (each lane its own)
    }
    __syncthreads();
    int32_t* const counts = a.counts + static_cast<uint64_t>(blockIdx.x) * (a.experts + 1);
    for (int i = t; i <= a.experts; i += kThreads) counts[i] = (list ? counts[i] : 0) + count[i];
}

// ---- the choice in 32 bits, where it is sure --------------------------------------------------------------------------------
// A score is off by kSigmoidOff at the most: s = 1 / (1 + e), e = e^-x off by (1.5 |x| 2^-24 + 2^-23) of itself, so s by s (1 - s) times that, plus
// 1.5 * 2^-23 s for the sum and the reciprocal; s (1 - s) |x| < 0.224 and s < 1 make 1.92 * 2^-23.
// Of a softmax by kSoftmaxOff times the largest p: 2.5 |x - m| 2^-24 of p for its power, whose p |x - m| is below 0.37 of the largest, and 47 * 2^-24 for
// the sum (1024 numbers, their mean |x - m| at most ln 1024; 22 additions on the way), its reciprocal and product.
// Keys: sums with the bias whose lowest four bits are the place in the lane, and of groups whose lowest six are the group: a key is off by 2^-19, or
// 2^-17, of itself, and no two of a lane, or of a token's groups, are the same.  A token is sure if no two neighbours in the order of its first k + 1, nor the last group
// that stays and the first that does not, are nearer than the sum of all that.
constexpr float kSigmoidOff = 0x1p-21f, kSoftmaxOff = 0x1p-18f;
constexpr float kNone = -1e38f;          // below every key; its sums are numbers still
constexpr float kLargeBias = 1e30f;      // larger ones (but -inf) leave everything to the 64 bits
constexpr int kMostFast = 16;            // k

__device__ inline float key_of(float v, uint32_t bits, uint32_t place) {
    return __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, v) & ~bits) | place);
}
__device__ inline uint32_t place_of(float key, uint32_t bits) { return __builtin_bit_cast(uint32_t, key) & bits; }
__device__ inline float pick(bool first, float a, float b) { return first ? a : b; }   // (of values: of places would keep them in memory)
__device__ inline void order(float& a, float& b) {   // a the larger
    const float x = a, y = b;
    a = __builtin_fmaxf(x, y);
    b = __builtin_fminf(x, y);
}
// Eight, the largest first (Batcher's odd-even merge sort); the same of eight that rise and then fall, or the other way round.
__device__ inline void sort8(float (&k)[8]) {
    constexpr int pair[19][2] = {{0, 1}, {2, 3}, {4, 5}, {6, 7}, {0, 2}, {1, 3}, {4, 6}, {5, 7}, {1, 2}, {5, 6},
                                 {0, 4}, {1, 5}, {2, 6}, {3, 7}, {2, 4}, {3, 5}, {1, 2}, {3, 4}, {5, 6}};
#pragma unroll
    for (int e = 0; e < 19; ++e) order(k[pair[e][0]], k[pair[e][1]]);
}
__device__ inline void merge8(float (&k)[8]) {
#pragma unroll
    for (int d = 4; d > 0; d >>= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!(i & d)) order(k[i], k[i + d]);
}

// The two largest of all that a pair stands for, of this and of other lanes.
struct Two {
    float first = kNone, second = kNone;
    __device__ void add(float y) {
        second = __builtin_amdgcn_fmed3f(first, second, y);
        first = __builtin_fmaxf(first, y);
    }
    __device__ void join(float f, float s) {
        second = __builtin_fmaxf(__builtin_fminf(first, f), __builtin_fmaxf(second, s));
        first = __builtin_fmaxf(first, f);
    }
    template <int CONTROL>
    __device__ void join_lane() {
        const auto dpp = [](float v) {
            return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CONTROL, 0xf, 0xf, true));
        };
        join(dpp(first), dpp(second));
    }
    __device__ float sum() const { return second > kNone ? first + second : first; }
};

template <int L, int N>
struct Shared {   // of a workgroup
    static constexpr int kGroups = L * N < 64 ? L * N : 64;
    int32_t count[L * N + 1];
    uint32_t left;
    union Token {      // one after the other
        struct {
            float group[kGroups];      // keys of groups
            float edge[2];             // of the last that stays, and the first that does not
            float sums[L * N];         // where groups are no runs of a lane's neighbours
        };
        int32_t won[kMostFast];        // places of the chosen
    } token[kThreads / L];
};

// M: how many of its N keys a lane has to know in order, as many as k at the least or all.  Tokens whose choice in 32 bits is not sure are left to
// route_biased_exact.
template <typename T, int L, int N, int M, int V>
__global__ __launch_bounds__(kThreads, 4) void route_biased_choose(const Biased a) {
    using S = Shared<L, N>;
    __shared__ S s;
    if (threadIdx.x == 0) s.left = 0;
    constexpr int NB = kNeighbours<T>, R = N / NB;   // runs of neighbours of a lane
    const int t = threadIdx.x, lane = t & (L - 1);
    for (int i = t; i <= a.experts; i += kThreads) s.count[i] = 0;
    __syncthreads();
    float bias[N], widest = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = expert_of<T, L>(lane, i);
        bias[i] = e >= a.experts ? -kInf : a.bias ? a.bias[e] : 0.0f;
        if (bias[i] > -kInf) widest = __builtin_fmaxf(widest, __builtin_fabsf(bias[i]));
    }
    widest = lanes_max<L>(widest);
    // groups that are runs of P lanes, or not
    const int size = a.experts / a.groups, P = size / NB;
    const bool runs = size % NB == 0 && (P & (P - 1)) == 0 && P <= L && P <= 16;
    const int shift = 31 - __builtin_clz(P | 1);
    typename S::Token& own_slot = s.token[t / L];
    const uint32_t step = gridDim.x * (kThreads / L);
    for (uint64_t token = blockIdx.x * (kThreads / L) + t / L; token < a.tokens; token += step) {
        const bool keep = !a.keep || a.keep[token];
        const T* const row = static_cast<const T*>(a.logits) + token * a.stride;
        float x[N], v[N];
        load_logits<T, L, N, V>(x, row, lane, a.experts);
        if (a.keep)
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = keep ? x[i] : -kInf;
        float most = 0.0f, sum = 0.0f, off = kSigmoidOff;
        if (a.soft) {
            most = largest<L, N>(x);
            const float from = most == -kInf ? 0.0f : most;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[i] = power(x[i] - from);
                sum += v[i];
            }
            sum = lanes_sum<L>(sum);
            const float by = 1.0f / sum;
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] *= by;
            off = by * kSoftmaxOff;
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x[i] * -1.44269504088896341f));
        }
        const bool bad = any_nan<L, N>(x) || (a.soft && most == kInf);
        bool sure = widest <= kLargeBias;
        // sums with the bias, kNone where the logit or the bias is -inf
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = x[i] > -kInf ? __builtin_fmaxf(v[i] + bias[i], kNone) : kNone;
        if (a.groups > 1) {
            float mine[R];        // keys of the groups of a lane's runs
            bool stays[R];
            if (runs) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    Two two;
#pragma unroll
                    for (int i = 0; i < NB; ++i) two.add(v[r * NB + i]);
                    if (P > 1) two.template join_lane<0xB1>();
                    if (P > 2) two.template join_lane<0x4E>();
                    if (P > 4) two.template join_lane<0x141>();
                    if (P > 8) two.template join_lane<0x140>();
                    const int g = (r * L + lane) >> shift;
                    mine[r] = key_of(two.sum(), 63, g & 63);
                    if (g < a.groups) own_slot.group[g] = mine[r];
                }
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) own_slot.sums[expert_of<T, L>(lane, i)] = v[i];
                wave_sync();
                for (int g = lane; g < a.groups; g += L) {
                    Two two;
                    for (int i = 0; i < size; ++i) two.add(own_slot.sums[g * size + i]);
                    own_slot.group[g] = key_of(two.sum(), 63, g);
                }
            }
            wave_sync();
            const auto before = [&](float key) {
                int n = 0;
                for (int h = 0; h < a.groups; ++h) n += own_slot.group[h] > key;
                return n;
            };
            const auto edges = [&](int n, float key) {
                if (n == a.kept - 1) own_slot.edge[0] = key;
                if (n == a.kept) own_slot.edge[1] = key;
            };
            if (runs) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int n = before(mine[r]);
                    stays[r] = n < a.kept;
                    if ((r * L + lane) >> shift < a.groups) edges(n, mine[r]);
#pragma unroll
                    for (int i = 0; i < NB; ++i) v[r * NB + i] = stays[r] ? v[r * NB + i] : kNone;
                }
                wave_sync();
            } else {
                uint32_t low = 0, high = 0;   // the groups that stay
                for (int g = lane; g < a.groups; g += L) {
                    const float key = own_slot.group[g];
                    const int n = before(key);
                    edges(n, key);
                    const uint32_t bit = n < a.kept ? 1u << (g & 31) : 0;
                    low |= g < 32 ? bit : 0;
                    high |= g < 32 ? 0 : bit;
                }
                low = lanes_or<L>(low);
                high = lanes_or<L>(high);
                wave_sync();
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int g = expert_of<T, L>(lane, i) / size;
                    v[i] = (g < 32 ? low >> (g & 31) : high >> (g & 31)) & 1 ? v[i] : kNone;
                }
            }
            const float last = own_slot.edge[0], next = own_slot.edge[1];
            sure &= last < 0.5f * kNone || last - next > __builtin_fabsf(last) * 0x1p-16f + 4.0f * off + (1.0f + widest) * 0x1p-21f;
        }
        // the lane's own in order
        float own[8], more[8], ninth = kNone;   // `more` after `own`; of the lane's ninth at the least how large it is
#pragma unroll
        for (int i = 0; i < 8; ++i) own[i] = key_of(v[i], 15, i);
        sort8(own);
        if constexpr (N == 16) {
#pragma unroll
            for (int i = 0; i < 8; ++i) more[i] = key_of(v[8 + i], 15, 8 + i);
            sort8(more);
#pragma unroll
            for (int i = 0; i < 8; ++i) order(own[i], more[7 - i]);
            merge8(own);
            if constexpr (M == 16) merge8(more);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) ninth = __builtin_fmaxf(ninth, more[i]);
        }
        // k + 1 times the largest of the lanes' first; two lanes may have the same, and then neither is sure
        float last = kInf;
        int found = 0, claimed = 0;
        const auto largest_left = [&](float mine) {
            const float best = lanes_max<L>(mine);
            sure &= best < 0.5f * kNone || last - best > __builtin_fabsf(best) * 0x1.8p-18f + 2.0f * off;
            last = best;
        };
        const auto take = [&](int j, float first) {   // false: not the lane's
            const bool mine = first == last, some = last > 0.5f * kNone;
            found += some;
            claimed += mine && some;
            if (mine) own_slot.won[j] = some ? static_cast<int32_t>(lane << 4 | place_of(last, 15)) : -1;
            return mine;
        };
        wave_sync();
        if constexpr (M == 8) {   // (what the j-th leaves behind of a lane's keys gets shorter)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j >= a.k) break;
                largest_left(own[0]);
                const bool mine = take(j, own[0]);
#pragma unroll
                for (int i = 0; i < 7 && i < 8 - j; ++i) own[i] = pick(mine, own[i + 1], own[i]);
                if (j == 0) own[7] = pick(mine, ninth, own[7]);
            }
        } else {
#pragma unroll 1
            for (int j = 0; j < a.k; ++j) {
                largest_left(own[0]);
                const bool mine = take(j, own[0]);
#pragma unroll
                for (int i = 0; i < 7; ++i) own[i] = pick(mine, own[i + 1], own[i]);
                own[7] = pick(mine, more[0], own[7]);
#pragma unroll
                for (int i = 0; i < 7; ++i) more[i] = pick(mine, more[i + 1], more[i]);
                more[7] = pick(mine, kNone, more[7]);
            }
        }
        largest_left(own[0]);
        wave_sync();
        sure &= lanes_sum<L>(claimed) == found;
        if (bad) {
            choose_none<L>(a, token, lane);
        } else if (!sure) {
            if (lane == 0) a.later[static_cast<uint64_t>(blockIdx.x) * a.room + atomicAdd(&s.left, 1u)] = static_cast<uint32_t>(token);
        } else {
            const auto chosen = [&](int j) {
                const int32_t w = own_slot.won[j];
                const int l = w >> 4, i = w & 15;
                return w < 0 ? -1 : (i / NB * L + l) * NB + i % NB;
            };
            for (int j = lane; j < a.k; j += L) a.chosen[token * a.k + j] = chosen(j);
            weigh<T, L>(a, token, row, lane, most, sum, s.count, chosen);
        }
    }
    __syncthreads();
    for (int i = t; i <= a.experts; i += kThreads) a.counts[static_cast<uint64_t>(blockIdx.x) * (a.experts + 1) + i] = s.count[i];
    if (t == 0) a.left[blockIdx.x] = s.left;
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

// Counts of the workgroups, and the tokens that they leave to the 64 bits; none where those make the whole call, in one workgroup.
struct Plan {
    bool exact;
    uint32_t groups, room = 0;
    int32_t* counts = nullptr;
    uint32_t *later = nullptr, *left = nullptr;
    size_t bytes;
    Plan(size_t tokens, int experts, int k, void* workspace) : exact(tokens <= kMostExact || k > kMostFast) {
        Carve c(workspace);
        groups = exact ? static_cast<uint32_t>(tokens <= kMostExact ? 1 : std::min<uint64_t>(kMostGroups, ceil_div(tokens, kThreads / 64))) : groups_of(tokens, experts);
        if (groups > 1) counts = c.take<int32_t>(static_cast<size_t>(groups) * (experts + 1));
        if (!exact) {
            const uint32_t at_once = kThreads / lanes_of(experts);
            room = static_cast<uint32_t>(ceil_div(tokens, static_cast<uint64_t>(groups) * at_once)) * at_once;
            later = c.take<uint32_t>(static_cast<size_t>(groups) * room);
            left = c.take<uint32_t>(groups);
        }
        bytes = c.at;
    }
};

}  // namespace

size_t route_biased_workspace(size_t tokens, int experts) {
    return std::max(Plan(tokens, experts, 1, nullptr).bytes, Plan(tokens, experts, kMostFast + 1, nullptr).bytes);
}

blink_status_t route_biased(const void* logits, blink_dtype_t dtype, size_t tokens, int experts, size_t stride, const uint8_t* keep, const float* bias, int k,
                            int expert_groups, int kept_groups, bool soft, bool normalize, float scale, int32_t* chosen, float* weights, int32_t* counts,
                            void* workspace, hipStream_t stream) {
    const Plan plan(tokens, experts, k, workspace);
    const Biased a{logits, stride, keep, bias, static_cast<uint32_t>(tokens), experts, k, kept_groups < expert_groups ? expert_groups : 1, kept_groups, soft,
                   normalize, scale, chosen, weights, plan.groups > 1 ? plan.counts : counts, plan.later, plan.left, plan.room};
    BLINK_TRY(with_float(dtype, [&](auto type) {
        using T = decltype(type);
        const auto run = [&](void (*kernel)(Biased)) { return launch(kernel, dim3(plan.groups), dim3(kThreads), stream, a); };
        if (!plan.exact)
            BLINK_TRY(with_load<T>(experts, stride, logits, stride, logits, [&](auto v) {
                return with_lanes(experts, [&](auto l, auto n) {
                    constexpr int L = decltype(l)::value, N = decltype(n)::value, V = decltype(v)::value;
                    if constexpr (N == 16)
                        if (k > 8) return run(route_biased_choose<T, L, N, 16, V>);
                    return run(route_biased_choose<T, L, N, 8, V>);
                });
            }));
        if (experts <= 64) return run(route_biased_exact<T, 1>);
        if (experts <= 256) return run(route_biased_exact<T, 4>);
        return run(route_biased_exact<T, 16>);
    }));
    if (plan.groups == 1) return BLINK_OK;
    return launch(route_biased_add, dim3(static_cast<uint32_t>(ceil_div(experts + 1, kAddColumns))), dim3(kAddThreads), stream, a.counts, plan.groups, experts + 1,
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
