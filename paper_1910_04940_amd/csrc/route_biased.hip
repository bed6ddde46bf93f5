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
//   softmax    dx = scale p (g - sum p g), g = 0 of the others,  normalised  scale (g - sum q g) q   (softmax of the chosen alone)
// Both sums, and g less them, are in 64 bits: where one p is nearly 1 the difference is all there is, (1 - p) g.
//
// The choice is that of scores in 64 bits.  L lanes hold a token, N logits each (see route.hpp).
#include <algorithm>
#include <array>
#include <type_traits>

#include "operators_api.hpp"
#include "route.hpp"

namespace blink {
namespace {

constexpr int kThreads = kRouteThreads;
constexpr int kMostGroups = 1280;        // workgroups: 20 waves on a CU
constexpr double kInf64 = __builtin_inf();

struct Biased {
    const void* logits;
    uint64_t stride;
    const uint8_t* keep;   // null: every token
    const float* bias;     // null: 0
    uint32_t tokens;
    int experts, k, groups, kept;
    int soft, normalize;   // or not
    float scale;
    int32_t* chosen;
    float* weights;
    int32_t* counts;       // of the result, or [workgroup][experts + 1]
    uint32_t* later;       // [workgroup][room]: tokens whose choice in 32 bits is not sure; null: none
    uint32_t* left;        // [workgroup]: how many those are
    uint32_t room, lists;
};

// What the weights of a token's chosen are made of: p times a factor that is the same for all of them and keeps them in range.
//   sigmoid: e^(x - c) / (1 + e^x), c the largest chosen x if that is below 0;  softmax: e^(x - c), c the largest
__device__ inline float part_of(bool soft, float x, float c) {
    const float up = power((x > 0.0f && !soft ? 0.0f : x) - c);
    return soft ? up : up * __builtin_amdgcn_rcpf(1.0f + power(-__builtin_fabsf(x)));
}

// Weights of a token's chosen, and what they add to the counts; chosen(j): the j-th, for the j of this lane.  most, sum: of the whole softmax.
// count: [experts], then the tokens'.
template <typename T, int L, typename F>
__device__ inline void weigh(const Biased& a, uint64_t token, const T* row, int lane, float most, float sum, int32_t* count, F chosen) {
    float* const weights = a.weights + token * a.k;
    const bool one = a.k <= L;   // to a lane
    int e = -1;
    float x = -kInf, part = 0.0f, c = 0.0f, all = 1.0f;
    const auto take = [&](int j) {
        e = j < a.k ? chosen(j) : -1;
        x = e >= 0 ? static_cast<float>(row[e]) : -kInf;
    };
    take(lane);
    if (a.normalize) {
        c = x;
        for (int j = lane + L; j < a.k; j += L) {
            take(j);
            c = __builtin_fmaxf(c, x);
        }
        c = lanes_max<L>(c);
        if (!a.soft) c = __builtin_fminf(c, 0.0f);
        if (!one) take(lane);
        part = e >= 0 ? part_of(a.soft, x, c) : 0.0f;
        all = part;
        for (int j = lane + L; j < a.k; j += L) {
            take(j);
            if (e >= 0) all += part_of(a.soft, x, c);
        }
        all = lanes_sum<L>(all);
    } else if (a.soft) {
        c = most;
        all = sum;
    }
    for (int j = lane; j < a.k; j += L) {
        if (!one) take(j);
        if (!one || !a.normalize) part = part_of(a.soft, x, c);
        weights[j] = e < 0 ? 0.0f : a.scale * (part / all);
        if (e >= 0) atomicAdd(&count[e], 1);
        if (e >= 0 && j == 0) atomicAdd(&count[a.experts], 1);
    }
}

// The same of at most S chosen to a lane, in registers: e[i] the (lane + L i)-th, -1 past the last.
template <typename T, int L, int S>
__device__ inline void weigh_few(const Biased& a, uint64_t token, const T* row, int lane, float most, float sum, int32_t* count,
                                 const int (&e)[S]) {
    float x[S], part[S], c = 0.0f, all = 1.0f;
#pragma unroll
    for (int i = 0; i < S; ++i) x[i] = e[i] >= 0 ? static_cast<float>(row[e[i]]) : -kInf;
    if (a.normalize) {
        c = x[0];
#pragma unroll
        for (int i = 1; i < S; ++i) c = __builtin_fmaxf(c, x[i]);
        c = lanes_max<L>(c);
        if (!a.soft) c = __builtin_fminf(c, 0.0f);
    } else if (a.soft) {
        c = most;
        all = sum;
    }
#pragma unroll
    for (int i = 0; i < S; ++i) part[i] = e[i] >= 0 ? part_of(a.soft, x[i], c) : 0.0f;
    if (a.normalize) {
        all = part[0];
#pragma unroll
        for (int i = 1; i < S; ++i) all += part[i];
        all = lanes_sum<L>(all);
    }
#pragma unroll
    for (int i = 0; i < S; ++i) {
        const int j = lane + i * L;
        if (j >= a.k) break;
        a.chosen[token * a.k + j] = e[i];
        a.weights[token * a.k + j] = e[i] < 0 ? 0.0f : a.scale * (part[i] / all);
        if (e[i] >= 0) atomicAdd(&count[e[i]], 1);
        if (e[i] >= 0 && j == 0) atomicAdd(&count[a.experts], 1);
    }
}

template <int L>
__device__ inline void choose_none(const Biased& a, uint64_t token, int lane) {
    for (int j = lane; j < a.k; j += L) {
        a.chosen[token * a.k + j] = -1;
        a.weights[token * a.k + j] = __builtin_nanf("");
    }
}

// ---- the choice in 64 bits ----------------------------------------------------------------------------------------------------
// A wave for each of the few tokens that two workgroups leave: so all of the kernel's workgroups are there at once (see below for what that measured).
constexpr int kExactThreads = 512;
constexpr uint32_t kLists = 2;
constexpr int kMostExact = 8;        // tokens of a call that are all chosen this way

// The largest of a wave's lanes; the two largest of all that its lanes hold (pairs that stand for different numbers).
__device__ inline double wave_max(double x) {
    return over_wave(x, [](double a, double b) { return __builtin_fmax(a, b); });
}
struct Two64 {
    double first = -kInf64, second = -kInf64;
};
__device__ inline Two64 joined(Two64 a, Two64 b) {
    return {__builtin_fmax(a.first, b.first), __builtin_fmax(__builtin_fmin(a.first, b.first), __builtin_fmax(a.second, b.second))};
}

// A wave to a token, N experts to a lane, expert 64 i + lane the i-th: for the tokens that a workgroup of route_biased_choose left in its list, for calls of a
// few tokens and for k above kMostFast.
// Bound by one token's chain of 64-bit instructions: the tokens that 262144 x 256 leave, 0.8 % of them, 15 us.  Six waves on a SIMD hold all 640 workgroups at
// once; with the registers for five, which hold 512, it was 21, with a workgroup of four waves for each list 25.
template <typename T, int N>
__global__ __launch_bounds__(kExactThreads, N <= 4 ? 6 : 2) void route_biased_exact(const Biased a) {
    __shared__ int32_t count[64 * N + 1];
    __shared__ double sums[kExactThreads / 64][64 * N];
    const int t = threadIdx.x, lane = t & 63;
    const uint32_t first = blockIdx.x * kLists;   // of its lists, whose tokens come one list after the other
    const uint32_t* const list = a.later ? a.later + static_cast<uint64_t>(first) * a.room : nullptr;
    const uint32_t mine = list ? a.left[first] : 0;
    const uint64_t n = list ? mine + (first + 1 < a.lists ? a.left[first + 1] : 0) : a.tokens;
    if (list && n == 0) return;
    int32_t* const counts = a.counts + static_cast<uint64_t>(list ? first : blockIdx.x) * (a.experts + 1);
    for (int i = t; i <= a.experts; i += kExactThreads) count[i] = list ? counts[i] : 0;
    __syncthreads();
    const uint64_t wave = (list ? 0 : blockIdx.x) * (kExactThreads / 64) + t / 64, step = (list ? 1 : gridDim.x) * (kExactThreads / 64);
    for (uint64_t at = wave; at < n; at += step) {
        const uint64_t token = list ? list[at < mine ? at : a.room + (at - mine)] : at;
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
        if (a.soft) most = lanes_max<64>(most);
        const double from = !a.soft || most == -kInf ? 0.0 : most;
        double all = 0.0;
#pragma unroll
        for (int i = 0; i < N; ++i) {   // (one exponential for both: its code is what takes long to come)
            v[i] = exp(a.soft ? x[i] - from : -static_cast<double>(x[i]));
            all += v[i];
        }
        all = a.soft ? lanes_sum<64>(all) : 1.0;
        sum = static_cast<float>(all);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = 64 * i + lane;
            const double p = (a.soft ? v[i] : 1.0) / (a.soft ? all : 1.0 + v[i]);
            const double y = p + (a.bias && e < a.experts ? static_cast<double>(a.bias[e]) : 0.0);
            v[i] = x[i] > -kInf && y > -kInf64 ? y : -kInf64;   // (a bias of -inf or NaN: never)
        }
        if (a.groups > 1) {
            const int size = a.experts / a.groups;
            // Q lanes to a group, which look at its sums in turn
            int Q = 1;
            while (2 * Q * a.groups <= 64) Q *= 2;
#pragma unroll
            for (int i = 0; i < N; ++i) sums[t / 64][64 * i + lane] = v[i];
            wave_sync();
            Two64 two;
            if (lane / Q < a.groups)
                for (int i = lane % Q; i < size; i += Q) two = joined(two, {sums[t / 64][lane / Q * size + i], -kInf64});
            for (int d = 1; d < Q; d *= 2) two = joined(two, {__shfl_xor(two.first, d), __shfl_xor(two.second, d)});
            double score = two.second > -kInf64 ? two.first + two.second : two.first;   // of group lane / Q, then of group `lane`
            score = __shfl(score, lane * Q & 63);
            wave_sync();
            int before = 0;
            for (int h = 0; h < a.groups; ++h) {
                const double other = __shfl(score, h);
                before += other > score || (other == score && h < lane);   // (the same for lanes past the last group, which nobody asks)
            }
            const uint64_t stay = __ballot(lane < a.groups && before < a.kept);
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (!(stay >> ((64 * i + lane) / size & 63) & 1)) v[i] = -kInf64;
        }
        int own = -1;   // the lane-th
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
            own = j == lane ? at : own;
            if (j % 64 == lane) chosen[j] = at;
        }
        weigh<T, 64>(a, token, row, lane, most, sum, count, [&](int j) { return j == lane ? own : chosen[j]; });   // (each lane its own)
    }
    __syncthreads();
    for (int i = t; i <= a.experts; i += kExactThreads) counts[i] = count[i];
}

// ---- the choice in 32 bits, where it is sure --------------------------------------------------------------------------------
// A score is off by kSigmoidOff at the most: s = 1 / (1 + e), e = e^-x off by (1.5 |x| 2^-24 + 2^-23) of itself, so s by s (1 - s) times that, plus
// 1.5 * 2^-23 s for the sum and the reciprocal; s (1 - s) |x| < 0.224 and s < 1 make 1.92 * 2^-23.
// Of a softmax by kSoftmaxOff times the largest p: 2.5 |x - m| 2^-24 of p for its power, whose p |x - m| is below 0.37 of the largest, and 47 * 2^-24 for
// the sum (1024 numbers, their mean |x - m| at most ln 1024; 22 additions on the way), its reciprocal and product.
// The largest |bias|, w, is added to all, so that sums are not negative and compare as whole numbers do; they are off by (1 + 4 w) 2^-24 for that.  Their
// lowest four bits give way to the place in the lane, first places largest (a key is off by 2^-19 of itself), those of groups, sums of two, their lowest six to
// the group (2^-17).
// A token is sure if no two neighbours in the order of its first k + 1, nor the last group that stays and the first that does not, are nearer than the
// sum of all that; two of its first k may be nearer if their logits and biases are the same (16-bit logits often are): among lanes whose keys differ in
// the place only, and so in one run of neighbours, the first one is taken first, and a lane's places are in order.
constexpr float kSigmoidOff = 0x1p-22f, kSoftmaxOff = 0x1p-18f;
constexpr float kLargeBias = 1e37f;      // larger ones (but -inf) leave everything to the 64 bits
constexpr int kMostFast = 16;            // k
// No sum: below 0, and of no two lanes the same, so that one lane has the largest even then.
__device__ inline int32_t none_of(int lane) { return static_cast<int32_t>(0xbf800000u) | lane << 4; }
// A bias that makes it so: what is added to it is lost.
__device__ inline float no_bias(int lane) { return __builtin_bit_cast(float, 0xf0000000u | static_cast<uint32_t>(lane) << 4); }

__device__ inline int32_t bits_of(float x) { return __builtin_bit_cast(int32_t, x); }
__device__ inline float float_of(int32_t x) { return __builtin_bit_cast(float, x); }
__device__ inline int32_t max_of(int32_t a, int32_t b) { return a > b ? a : b; }
__device__ inline int32_t min_of(int32_t a, int32_t b) { return a < b ? a : b; }
__device__ inline int32_t pick(bool first, int32_t a, int32_t b) { return first ? a : b; }   // (of values: of places would keep them in memory)
__device__ inline void order(int32_t& a, int32_t& b) {   // a the larger
    const int32_t x = a, y = b;
    a = max_of(x, y);
    b = min_of(x, y);
}
// Eight, the largest first (Batcher's odd-even merge sort); the same of eight that rise and then fall, or the other way round.
__device__ inline void sort8(int32_t (&k)[8]) {
    constexpr int pair[19][2] = {{0, 1}, {2, 3}, {4, 5}, {6, 7}, {0, 2}, {1, 3}, {4, 6}, {5, 7}, {1, 2}, {5, 6},
                                 {0, 4}, {1, 5}, {2, 6}, {3, 7}, {2, 4}, {3, 5}, {1, 2}, {3, 4}, {5, 6}};
#pragma unroll
    for (int e = 0; e < 19; ++e) order(k[pair[e][0]], k[pair[e][1]]);
}
__device__ inline void merge8(int32_t (&k)[8]) {
#pragma unroll
    for (int d = 4; d > 0; d >>= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!(i & d)) order(k[i], k[i + d]);
}
template <int L>
__device__ inline int32_t lanes_most(int32_t x) {
    return over_lanes<L>(x, [](int32_t a, int32_t b) { return max_of(a, b); });
}

// The two largest of all that a pair stands for, of this and of other lanes.
struct Two {
    int32_t first = none_of(0), second = none_of(0);
    __device__ void add(int32_t y) {
        second = bits_of(__builtin_amdgcn_fmed3f(float_of(first), float_of(second), float_of(y)));
        first = max_of(first, y);
    }
    __device__ void join(int32_t f, int32_t s) {
        second = max_of(min_of(first, f), max_of(second, s));
        first = max_of(first, f);
    }
    template <int CONTROL>
    __device__ void join_lane() {
        const int32_t f = __builtin_amdgcn_update_dpp(0, first, CONTROL, 0xf, 0xf, true), s = __builtin_amdgcn_update_dpp(0, second, CONTROL, 0xf, 0xf, true);
        join(f, s);
    }
    // The group's key; `alone`: what stands for the second of a group that has none, all sums being that much too large.
    __device__ int32_t key(float alone, int32_t g) const {
        const float sum = float_of(first) + (second >= 0 ? float_of(second) : alone);
        return first >= 0 ? (bits_of(sum) & ~63) | g : static_cast<int32_t>(0x80000000u) | g;
    }
};

template <int L, int N>
struct Shared {   // of a workgroup
    static constexpr int kGroups = L * N < 64 ? L * N : 64;
    int32_t count[L * N + 1];
    uint32_t left;
    alignas(8) int32_t lost[kMostFast][2];        // what lanes write that did not win, and nobody reads
    union Token {      // one after the other
        struct {
            alignas(16) int32_t group[kGroups];   // keys of groups
            int32_t edge[2];                      // of the last that stays, and the first that does not
            int32_t sums[L * N];                  // where groups are no runs of a lane's neighbours
        };
        alignas(8) int32_t won[kMostFast][2];     // keys of the chosen, and their lanes
    } token[kThreads / L];
};

// M: how many of its N keys a lane has to know in order, as many as k at the least or all.  Tokens whose choice in 32 bits is not sure are left to
// route_biased_exact.  They are few unless a call is such that all are: logits (or their scores, far above 0) that tie at the end of the choice, as from a router
// of zeros, or a bias so large that nothing is left of the scores' differences: 262144 x 256 then takes 740 to 760 us, 105 otherwise.  So do, with k = 8 and
// sixteen keys to each of four or more lanes, tokens whose eight all come from one lane, which does not know its ninth: groups of eight, of which one
// (or two that share a lane) stays.  262144 x 64 in eight groups: one kept 440 us (k = 7: 39), two 96, four 40.
// Bound by vector instructions: 262144 x 256 bfloat16, eight groups, k = 8, 94 us, 598 a wave for four tokens (32 of them powers and reciprocals at a quarter of
// the rate); all tokens in 64 bits took 630.  Without groups 82 us.  What brought it there: five waves on a SIMD
// (four 103, six, which spill, 110); a lane's chosen in registers, not read from LDS for each of their uses, 2.5 %; the call's numbers asked of for each token
// and winners written without a branch, 9 %: kept as masks of lanes the numbers fill the scalar registers and move to vector registers and back, and both sides of
// the branch moved the lane's keys.  Where groups are no runs of neighbours of 1, 2, 4 .. lanes their sums go through LDS (20011 x 60 in six groups
// 9.8 us, the latency of one pass).
template <typename T, int L, int N, int M, int V>
__global__ __launch_bounds__(kThreads, L >= 8 ? 5 : 4) void route_biased_choose(const Biased args) {
    using S = Shared<L, N>;
    __shared__ S s;
    constexpr int NB = kNeighbours<T>, R = N / NB;   // runs of neighbours of a lane
    constexpr int kSlots = (M + L - 1) / L;          // of a lane's chosen
    const int t = threadIdx.x, lane = t & (L - 1);
    if (t == 0) s.left = 0;
    for (int i = t; i <= args.experts; i += kThreads) s.count[i] = 0;
    __syncthreads();
    float bias[N], widest = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = expert_of<T, L>(lane, i);
        bias[i] = e >= args.experts ? -kInf : args.bias ? args.bias[e] : 0.0f;
        if (bias[i] > -kInf) widest = __builtin_fmaxf(widest, __builtin_fabsf(bias[i]));
    }
    widest = lanes_max<L>(widest);
    const bool fits = widest <= kLargeBias;
    if (!fits) widest = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) bias[i] = bias[i] > -kInf ? bias[i] + widest : no_bias(lane);
    const int32_t none = none_of(lane);
    const float rounded = (1.0f + 4.0f * widest) * 0x1p-23f;
    // groups that are runs of P lanes, or not
    const int size = args.experts / args.groups, P = size / NB;
    const bool runs = size % NB == 0 && (P & (P - 1)) == 0 && P <= L && P <= 16;
    const int shift = 31 - __builtin_clz(P | 1);
    // e / size for e and size below 2^10: e * (2^20 / size, rounded up) is off by less than 2^20
    const uint32_t by_size = ((1u << 20) + size - 1) / size;
    const auto group_of = [&](int e) { return static_cast<int>(e * by_size >> 20); };
    typename S::Token& mine = s.token[t / L];
    const uint32_t step = gridDim.x * (kThreads / L);
    for (uint64_t token = blockIdx.x * (kThreads / L) + t / L; token < args.tokens; token += step) {
        Biased a = args;   // (see above)
        asm volatile("" : "+s"(a.k), "+s"(a.groups), "+s"(a.kept), "+s"(a.soft), "+s"(a.normalize));
        const T* const row = static_cast<const T*>(a.logits) + token * a.stride;
        const bool keep = !a.keep || a.keep[token];
        int here = lane;   // (or what only some calls need of all places, masks and groups, would be kept in registers for all tokens)
        asm volatile("" : "+v"(here));
        float x[N];
        load_logits<T, L, N, V>(x, row, here, a.experts);
        if (a.keep)
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = keep ? x[i] : -kInf;
        float least = x[0];   // (NaN if one is)
#pragma unroll
        for (int i = 1; i < N; ++i) least = __builtin_elementwise_minimum(least, x[i]);
        bool bad = false;
        float most = 0.0f, sum = 0.0f, off = kSigmoidOff;
        int32_t v[N];   // sums with the bias
        {
            float p[N];
            if (a.soft) {
                most = -kInf;
#pragma unroll
                for (int i = 0; i < N; ++i) most = __builtin_fmaxf(most, x[i]);
                most = lanes_max<L>(most);
                const float from = most == -kInf ? 0.0f : most;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    p[i] = power(x[i] - from);
                    sum += p[i];
                }
                sum = lanes_sum<L>(sum);
                const float by = 1.0f / sum;
#pragma unroll
                for (int i = 0; i < N; ++i) p[i] *= by;
                off = by * kSoftmaxOff;
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) p[i] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x[i] * -1.44269504088896341f));
            }
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = bits_of(p[i] + bias[i]);
        }
        if (!(least > -kInf) || (a.soft && most == kInf)) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (!(x[i] > -kInf)) v[i] = none;
                bad |= x[i] != x[i] || (a.soft && x[i] == kInf);
            }
        }
        bad = lanes_or<L>(static_cast<unsigned>(bad));
        bool sure = fits;
        if (a.groups > 1) {
            const auto before = [&](auto keys) {   // how many keys of groups are larger than each of these
                std::array<int, keys.size()> n{};
                const auto look = [&](int32_t other) {
#pragma unroll
                    for (size_t r = 0; r < keys.size(); ++r) n[r] += other > keys[r];
                };
                int h = 0;
                for (; h + 4 <= a.groups; h += 4) {
                    const int4 four = *reinterpret_cast<const int4*>(mine.group + h);
                    look(four.x);
                    look(four.y);
                    look(four.z);
                    look(four.w);
                }
                for (; h < a.groups; ++h) look(mine.group[h]);
                return n;
            };
            const auto edges = [&](int n, int32_t key) {
                if (n == a.kept - 1) mine.edge[0] = key;
                if (n == a.kept) mine.edge[1] = key;
            };
            if (runs) {
                std::array<int32_t, R> key;   // of the groups of the lane's runs
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
                    key[r] = two.key(widest, g & 63);
                    if (g < a.groups) mine.group[g] = key[r];
                }
                wave_sync();
                const auto n = before(key);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    if ((r * L + lane) >> shift < a.groups) edges(n[r], key[r]);
#pragma unroll
                    for (int i = 0; i < NB; ++i) v[r * NB + i] = pick(n[r] < a.kept, v[r * NB + i], none);
                }
                wave_sync();
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) mine.sums[expert_of<T, L>(here, i)] = v[i];
                wave_sync();
                for (int g = lane; g < a.groups; g += L) {
                    Two two;
                    const int32_t* const of = mine.sums + g * size;
                    int i = 0;
                    for (; i + 4 <= size; i += 4) {   // (reads under way together)
                        const int32_t y[4] = {of[i], of[i + 1], of[i + 2], of[i + 3]};
#pragma unroll
                        for (int j = 0; j < 4; ++j) two.add(y[j]);
                    }
                    for (; i < size; ++i) two.add(of[i]);
                    mine.group[g] = two.key(widest, g);
                }
                wave_sync();
                uint32_t low = 0, high = 0;   // the groups that stay
                for (int g = lane; g < a.groups; g += L) {
                    const std::array<int32_t, 1> key{mine.group[g]};
                    const int n = before(key)[0];
                    edges(n, key[0]);
                    const uint32_t bit = n < a.kept ? 1u << (g & 31) : 0;
                    low |= g < 32 ? bit : 0;
                    high |= g < 32 ? 0 : bit;
                }
                low = lanes_or<L>(low);
                high = lanes_or<L>(high);
                wave_sync();
                const uint64_t stay = static_cast<uint64_t>(high) << 32 | low;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int g = group_of(expert_of<T, L>(here, i));
                    v[i] = pick(stay >> (g & 63) & 1, v[i], none);
                }
            }
            const int32_t last = mine.edge[0], next = mine.edge[1];
            sure &= next < 0 || float_of(last) - float_of(next) > float_of(last) * 0x1.2p-16f + 4.0f * (off + rounded);
        }
        // the lane's own in order
        int32_t own[8], more[8], ninth = none;   // `more` after `own`
        constexpr bool kNinth = N == 16 && M == 8 && L <= 2;
#pragma unroll
        for (int i = 0; i < 8; ++i) own[i] = (v[i] & ~15) | (15 - i);
        sort8(own);
        if constexpr (N == 16) {
#pragma unroll
            for (int i = 0; i < 8; ++i) more[i] = (v[8 + i] & ~15) | (7 - i);
            sort8(more);
#pragma unroll
            for (int i = 0; i < 8; ++i) order(own[i], more[7 - i]);
            merge8(own);
            if constexpr (M == 16) merge8(more);
            if constexpr (kNinth)
#pragma unroll
                for (int i = 0; i < 8; ++i) ninth = max_of(ninth, more[i]);
        }
        // k + 1 times the largest of the lanes' first, which leaves its key and its lane
        wave_sync();
        const int there = __popcll(__ballot(lane == 0));
        const auto take = [&](int j, int32_t first) {
            const int32_t key = first & -NB, best = lanes_most<L>(key);
            bool won = key == best;
            if (__popcll(__ballot(won)) != there) {   // some lanes have the same: the first one's
                const int least = lanes_least<L>(won ? lane : L);   // (asked of all lanes)
                won = won && lane == least;
            }
            *reinterpret_cast<int2*>((won ? mine.won : s.lost)[j]) = int2{first, lane};   // (see above)
            return won;
        };
        if constexpr (M == 8) {   // (what the j-th leaves behind of a lane's keys gets shorter)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j >= a.k) break;
                const bool won = take(j, own[0]);
#pragma unroll
                for (int i = 0; i < 7 && i < 8 - j; ++i) own[i] = pick(won, own[i + 1], own[i]);
                // a lane that takes all eight has its eighth once more after it, which is not sure, unless its ninth is there
                if (j == 0 && (kNinth || N == 8)) own[7] = pick(won, ninth, own[7]);
            }
        } else {
#pragma unroll 1
            for (int j = 0; j < a.k; ++j) {
                const bool won = take(j, own[0]);
#pragma unroll
                for (int i = 0; i < 7; ++i) own[i] = pick(won, own[i + 1], own[i]);
                own[7] = pick(won, more[0], own[7]);
#pragma unroll
                for (int i = 0; i < 7; ++i) more[i] = pick(won, more[i + 1], more[i]);
                more[7] = pick(won, none, more[7]);
            }
        }
        const int32_t next = lanes_most<L>(own[0]);
        wave_sync();
        const float near = float_of(max_of(mine.won[0][0], 0)) * 0x1.2p-18f + 2.0f * off + rounded;
        const auto expert_at = [&](int2 w) {
            const int i = 15 - (w.x & 15);
            return w.x < 0 ? -1 : (i / NB * L + w.y) * NB + i % NB;
        };
        const auto at = [&](int j) { return *reinterpret_cast<const int2*>(mine.won[j]); };
        int chosen[kSlots];
#pragma unroll
        for (int i = 0; i < kSlots; ++i) {
            const int j = lane + i * L;
            chosen[i] = -1;
            if (j < a.k) {
                const int2 w = at(j), then = j + 1 < a.k ? at(j + 1) : int2{next, 0};
                chosen[i] = expert_at(w);
                if (!bad && then.x >= 0 && !(float_of(w.x) - float_of(then.x) > near)) {   // (a NaN's keys may stand for no expert)
                    const int e = chosen[i], f = expert_at(then);
                    sure &= j + 1 < a.k && row[e] == row[f] && (!a.bias || a.bias[e] == a.bias[f]);
                }
            }
        }
        sure = !lanes_or<L>(static_cast<unsigned>(!sure));
        if (bad) {
            choose_none<L>(a, token, lane);
        } else if (!sure) {
            if (lane == 0) a.later[static_cast<uint64_t>(blockIdx.x) * a.room + atomicAdd(&s.left, 1u)] = static_cast<uint32_t>(token);
        } else {
            weigh_few<T, L, kSlots>(a, token, row, lane, most, sum, s.count, chosen);
        }
    }
    __syncthreads();
    for (int i = t; i <= args.experts; i += kThreads) args.counts[static_cast<uint64_t>(blockIdx.x) * (args.experts + 1) + i] = s.count[i];
    if (t == 0) args.left[blockIdx.x] = s.left;
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

// Through a whole softmax a row is read once: a lane's powers stay in registers, what its chosen get goes through LDS, and all others get the same.  The 64-bit sums
// take 262144 x 256 bfloat16 from 53 to 55 us, 20011 x 60 from 5.6 to 6.0; in 32 bits the gradient of an expert 16 above all others was mostly error.
// A chosen logit lies in a line of its own, so that nearly all of the logits are read again: 262144 x 256 bfloat16, k = 8, 123 MB read and 134 written, 44 us.
template <typename T, int L, int N, int V>
__global__ __launch_bounds__(kThreads) void route_biased_gradient_kernel(const BiasedGradient a) {
    // what the token's chosen get (with a whole softmax: before p times it), +0 wherever no token's are; four neighbours of each lane side by side
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
        // the lane's first chosen: its expert (-1: none), the gradient of its weight, its logit
        int e0 = -1;
        float g0 = 0.0f, x0 = -kInf;
        const auto chosen = [&](int j, int* e, float* g, float* x) {
            *e = j < a.k && keep ? a.chosen[token * a.k + j] : -1;
            *g = j < a.k ? a.grad_weights[token * a.k + j] : 0.0f;
            if (*e >= a.experts) *e = -1;
            *x = *e >= 0 ? static_cast<float>(row[*e]) : -kInf;
        };
        chosen(lane, &e0, &g0, &x0);
        // f(expert, gradient, logit) for each of the lane's chosen
        const auto each = [&](auto f) {
            if (e0 >= 0) f(e0, g0, x0);
            for (int j = lane + L; j < a.k; j += L) {
                int e;
                float g, x;
                chosen(j, &e, &g, &x);
                if (e >= 0) f(e, g, x);
            }
        };
        float most = -kInf;
        double sum = 0.0, dot = 0.0;
        float x[N], by = 0.0f, others = 0.0f;   // of a whole softmax: powers, 1 / their sum, what logits get that are not chosen
        unsigned any = 0;
        if (whole) each([&](int, float, float) { any = 1; });
        const bool through = lanes_or<L>(any);
        if (through) {
            load_logits<T, L, N, V>(x, row, lane, a.experts);
#pragma unroll
            for (int i = 0; i < N; ++i) most = __builtin_fmaxf(most, x[i]);
            most = lanes_max<L>(most);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                x[i] = power(x[i] - most);
                sum += x[i];
            }
            each([&](int, float g, float x) { dot += static_cast<double>(power(x - most)) * g; });
            sum = 1.0 / lanes_sum<L>(sum);
            dot = lanes_sum<L>(dot) * sum;
            by = static_cast<float>(sum);
            others = static_cast<float>(a.scale * -dot);
        } else if (a.normalize) {
            each([&](int, float, float x) { most = __builtin_fmaxf(most, x); });
            most = lanes_max<L>(most);
            if (!a.soft) most = __builtin_fminf(most, 0.0f);
            each([&](int, float g, float x) {
                const double p = part_of(a.soft, x, most);
                sum += p;
                dot += p * g;
            });
            sum = 1.0 / lanes_sum<L>(sum);
            dot = lanes_sum<L>(dot) * sum;
        }
        each([&](int e, float g, float x) {
            float d = a.scale * g;
            if (whole) {
                d = static_cast<float>(a.scale * (g - dot));
                if (d == 0.0f) d = -0.0f;   // (+0 is no chosen's)
            } else if (a.normalize) {
                d = a.k == 1 ? 0.0f : static_cast<float>(a.scale * (g - dot) * (part_of(a.soft, x, most) * sum));
            } else {
                d *= part_of(false, x, 0.0f);
            }
            if (!a.soft) d *= 1.0f / (1.0f + expf(x));
            add[place(e)] = d;
        });
        wave_sync();
        float d[N];
#pragma unroll
        for (int i = 0; i < N; ++i) d[i] = add[place_at(lane, i)];
        wave_sync();
        if (e0 >= 0) add[place(e0)] = 0.0f;
        for (int j = lane + L; j < a.k; j += L) {
            const int e = a.chosen[token * a.k + j];
            if (e >= 0 && e < a.experts) add[place(e)] = 0.0f;
        }
        wave_sync();
        if (through)
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] = x[i] * by * (bits_of(d[i]) == 0 ? others : d[i]);
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
        groups = exact ? static_cast<uint32_t>(tokens <= kMostExact ? 1 : std::min<uint64_t>(kMostGroups, ceil_div(tokens, kExactThreads / 64))) : groups_of(tokens, experts);
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
                   normalize, scale, chosen, weights, plan.groups > 1 ? plan.counts : counts, plan.later, plan.left, plan.room, plan.groups};
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
        const auto exact = [&](void (*kernel)(Biased)) {
            return launch(kernel, dim3(plan.exact ? plan.groups : static_cast<uint32_t>(ceil_div(plan.groups, kLists))), dim3(kExactThreads), stream, a);
        };
        if (experts <= 64) return exact(route_biased_exact<T, 1>);
        if (experts <= 256) return exact(route_biased_exact<T, 4>);
        return exact(route_biased_exact<T, 16>);
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
