// An optimiser's step over many tensors, and the norm of their gradients that comes before it.
//
//   norm = |factor| * sqrt(sum g^2) over all tensors;   scale = factor * min(1, most / norm)
//   g' = scale g;   m = b1 m + (1 - b1) g';   v = b2 v + (1 - b2) g'^2
//   w = w (1 - lr decay) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
//
// A list of tensors is made once: their records, and one of `Piece` for every 2048 elements of a tensor, lie in device memory, pieces of
// tensors of one kind (types of weights, gradient and moments) one after the other, so that a call is one launch for each kind however
// many tensors there are.  A wave has 256 elements at a time, four neighbours to a lane; tensors start at any element, so loads
// and stores are aligned to elements only.
//
// Moments in 8 bits: m and sqrt(v) as e4m3 numbers (four significant bits down to 2^-6, multiples of 2^-9 below) times the scale of their 256
// elements, which takes the largest to 448.  They are rounded up with the probability of what rounding down would drop: to
// nearest, v, which moves by a thousandth a step, would never leave its number.  A root that is not zero is not stored as zero, which
// would make the next step's divisor vanish.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <limits>
#include <new>
#include <vector>

#include "lanes.hpp"
#include "operators_api.hpp"

namespace blink {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr uint32_t kBlock = 256;                  // elements of a wave at a time, and of a scale
constexpr uint32_t kPieceBlocks = 8, kPiece = kPieceBlocks * kBlock;
constexpr uint32_t kMostGroups = 2048;            // workgroups of the norm, which leave a sum each
constexpr uint64_t kCache = uint64_t{256} << 20;  // the memory-side cache
constexpr uint32_t kHeld = 52 << 10;              // bytes of LDS that let three workgroups onto a compute unit

struct Record {
    void* weights;
    float* master;
    const void* grad;
    void *moment1, *moment2;
    float *scale1, *scale2;
    uint64_t elements;
    double rate, decay;
    uint64_t number;   // in the caller's list
};
struct Piece {
    uint32_t tensor, number;   // its `number`-th 2048 elements
};

// Four elements, wherever they start.  PAST: they come from memory and go there, past the caches.
template <typename T>
struct alignas(sizeof(T)) Four {
    T v[4];
};
template <typename T>
struct Words {   // their bits, as the loads and stores past the caches take them
    typedef uint32_t type __attribute__((ext_vector_type(sizeof(T)), aligned(sizeof(T))));
};
template <>
struct Words<uint8_t> {
    typedef uint32_t type __attribute__((aligned(1)));
};
template <bool PAST, typename T>
__device__ inline Four<T> load4(const T* p) {
    if constexpr (PAST) return __builtin_bit_cast(Four<T>, __builtin_nontemporal_load(reinterpret_cast<const typename Words<T>::type*>(p)));
    else return *reinterpret_cast<const Four<T>*>(p);
}
template <bool PAST, typename T>
__device__ inline void store4(T* p, const Four<T>& y) {
    if constexpr (PAST) __builtin_nontemporal_store(__builtin_bit_cast(typename Words<T>::type, y), reinterpret_cast<typename Words<T>::type*>(p));
    else *reinterpret_cast<Four<T>*>(p) = y;
}
// The same of the last elements of a tensor, `left` of them: zeros past the end.
template <typename T>
__device__ inline Four<T> load_some(const T* p, uint32_t left) {
    Four<T> y;
    for (uint32_t i = 0; i < 4; ++i) y.v[i] = i < left ? p[i] : static_cast<T>(0);
    return y;
}
template <typename T>
__device__ inline void store_some(T* p, const Four<T>& y, uint32_t left) {
    for (uint32_t i = 0; i < 4; ++i)
        if (i < left) p[i] = y.v[i];
}
// How many elements from `at` on a lane has, four at the most.
__device__ inline uint32_t left_of(uint64_t elements, uint64_t at) { return at >= elements ? 0 : elements - at < 4 ? static_cast<uint32_t>(elements - at) : 4; }

// ---- norm -------------------------------------------------------------------------------------------------------------------
struct Norm {
    const Record* tensors;
    const Piece* pieces;
    uint32_t n;            // pieces
    double* sums;          // one to a workgroup
};

template <int WAVES>
__device__ inline double add_up(double s, double (&part)[WAVES]) {   // for thread 0
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0;
    for (int w = 0; w < WAVES; ++w) s += part[w];
    return s;
}

// What a sum of squares makes.
constexpr double kMostLength = 0x1p63;   // of scaled gradients: the square of one, and b2 v + (1 - b2) g^2 of two, stay below 2^127
struct Clip {
    double most, factor;
    float* norm;
    int32_t* step;
    __device__ void finish(double s) const {
        const double length = sqrt(s) * fabs(factor);
        const float scale = static_cast<float>(length > most ? factor * (most / length) : factor);
        // not with an infinite gradient, nor a NaN, nor where the step, in 32 bits, could not scale the gradients or square what that makes of them
        const bool fine = length < __builtin_inf() && fmin(length, most) <= kMostLength && fabsf(scale) < __builtin_inff();
        norm[0] = static_cast<float>(length);
        norm[1] = fine ? scale : __builtin_nanf("");
        if (step && fine) *step += 1;
    }
};

// Squares and their sums in 64 bits: no gradient's square overflows or is lost.  THREADS threads take a piece.
template <typename G, bool PAST, uint32_t THREADS>
__device__ inline double squares_of(const Norm& a, uint32_t piece, uint32_t thread) {
    double s = 0.0;
    const auto add = [&](const Four<G>& g) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const double x = static_cast<float>(g.v[j]);
            s = __builtin_fma(x, x, s);
        }
    };
    constexpr uint32_t kLoads = kPiece / (4 * THREADS);
    const Piece p = a.pieces[piece];
    const Record& r = a.tensors[p.tensor];
    const uint64_t from = static_cast<uint64_t>(p.number) * kPiece;
    const G* const grad = static_cast<const G*>(r.grad) + from;
    if (from + kPiece <= r.elements) {
        Four<G> g[kLoads];
#pragma unroll
        for (uint32_t u = 0; u < kLoads; ++u) g[u] = load4<PAST>(grad + (u * THREADS + thread) * 4);
#pragma unroll
        for (uint32_t u = 0; u < kLoads; ++u) add(g[u]);
    } else {
        for (uint32_t u = 0; u < kLoads; ++u) {
            const uint32_t at = (u * THREADS + thread) * 4;
            add(load_some(grad + at, left_of(r.elements, from + at)));
        }
    }
    return s;
}
// Bound by memory: 151 M fp32 gradients 91 us, 6.6 TB/s; loads past the caches 102, others 109 (168 M).  Gradients that fit the memory-side cache are left
// there for the step.
template <typename G, bool PAST>
__global__ __launch_bounds__(kThreads) void update_squares(const Norm a) {
    __shared__ double part[kWaves];
    double s = 0.0;
    for (uint32_t i = blockIdx.x; i < a.n; i += gridDim.x) s += squares_of<G, PAST, kThreads>(a, i, threadIdx.x);
    s = add_up(s, part);
    if (threadIdx.x == 0) a.sums[blockIdx.x] = s;
}
constexpr int kNormThreads = 1024;   // two sums to each at the most: 330 sums 2.0 us, 2.2 with 256 threads; 2048 behind a list beyond the caches 4.5 to 4.7 either way
__global__ __launch_bounds__(kNormThreads) void update_norm(const double* sums, uint32_t n, const Clip clip) {
    __shared__ double part[kNormThreads / 64];
    double s = 0.0;
#pragma unroll 2
    for (uint32_t i = threadIdx.x; i < n; i += kNormThreads) s += sums[i];
    s = add_up(s, part);
    if (threadIdx.x == 0) clip.finish(s);
}
// Few pieces of one type in one workgroup, a wave to a piece: nine tensors of 5365 elements in all 4.7 us a call, 7.1 as two kernels.
constexpr int kFewThreads = 1024;
constexpr uint32_t kFew = 2 * kFewThreads / 64;
template <typename G>
__global__ __launch_bounds__(kFewThreads) void update_few(const Norm a, const Clip clip) {
    __shared__ double part[kFewThreads / 64];
    double s = 0.0;
    for (uint32_t i = threadIdx.x / 64; i < a.n; i += kFewThreads / 64) s += squares_of<G, false, 64>(a, i, threadIdx.x & 63);
    s = add_up(s, part);
    if (threadIdx.x == 0) clip.finish(s);
}

// ---- step -------------------------------------------------------------------------------------------------------------------
struct Step {
    const Record* tensors;
    const Piece* pieces;
    uint32_t n;                  // pieces
    const int32_t* step;
    const float *scale, *rate;   // null: 1
    double lr, ln1, ln2;         // ln of b1, b2
    float b1, b2, g1, g2, eps;   // g1 = 1 - b1
    uint32_t seed;
};

__device__ inline uint32_t mixed(uint32_t h) {   // the finalizer of MurmurHash3
    h = (h ^ h >> 16) * 0x85ebca6bu;
    h = (h ^ h >> 13) * 0xc2b2ae35u;
    return h ^ h >> 16;
}

// The four numbers of a lane as codes, and the scale of the wave's 256; up: 16 random bits each, in the upper half of a word.  ROOT: y >= 0, and what is not
// zero is not stored as zero.
// The instruction adds the upper 20 of the word's bits to the 20 of a number's 23 that have no place (numbers below 2^-6: to what is left of a
// multiple of 2^-9) and cuts them off; the lower half of the word stands for half of a sixteenth bit, so that all are used alike.  Made of ordinary
// instructions, twenty a number, the 8-bit step of 168 M elements took 590 us, 516 like this.
template <bool ROOT>
__device__ inline uint32_t encode(const float (&y)[4], const uint32_t (&up)[4], float* scale) {
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t size = __builtin_bit_cast(uint32_t, y[j]) & 0x7fffffffu;
        most = size > most ? size : most;
    }
    most = lanes_max<64>(most);
    const float largest = __builtin_bit_cast(float, most);
    if (most >= 0x7f800000u) {   // an infinity or a NaN among them: it shows in all
        *scale = __builtin_nanf("");
        return 0x7f7f7f7fu;
    }
    if (largest < 0x1p-100f) {
        *scale = 0.0f;
        return 0;
    }
    *scale = largest * (1.0f / 448.0f);
    const float by = 1.0f / largest * 448.0f;
    const auto cut = [&](int j) { return static_cast<float>(__builtin_amdgcn_fmed3f(y[j] * by, -448.0f, 448.0f)); };
    uint32_t codes = 0;
    codes = __builtin_amdgcn_cvt_sr_fp8_f32(cut(0), up[0] | 0x8000u, codes, 0);
    codes = __builtin_amdgcn_cvt_sr_fp8_f32(cut(1), up[1] | 0x8000u, codes, 1);
    codes = __builtin_amdgcn_cvt_sr_fp8_f32(cut(2), up[2] | 0x8000u, codes, 2);
    codes = __builtin_amdgcn_cvt_sr_fp8_f32(cut(3), up[3] | 0x8000u, codes, 3);
    if (ROOT && ((codes - 0x01010101u) & ~codes & 0x80808080u)) {   // some are zero
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (!(codes >> (8 * j) & 0xffu) && y[j] * by != 0.0f) codes |= 1u << (8 * j);
    }
    return codes;
}

// Codes that are all 0 are 0 whatever the scale: before the first step nobody has written one.
__device__ inline void decode(uint32_t codes, float scale, float (&y)[4]) {
    scale = codes ? scale : 0.0f;
    const auto low = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), high = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
    y[0] = low[0] * scale;
    y[1] = low[1] * scale;
    y[2] = high[0] * scale;
    y[3] = high[1] * scale;
}

// What a step is for all elements of a tensor.
struct Factors {
    float scale, by_m, by_v, kept, b1, b2, g1, g2, eps;
};
// A lane's four elements of one block of a tensor, as they are in memory.
template <typename W, typename G, bool MASTER, bool EIGHT>
struct Held {
    using M = typename std::conditional<EIGHT, uint8_t, float>::type;
    using C = typename std::conditional<MASTER, float, W>::type;   // of the weights that are stepped
    Four<G> g;
    Four<C> w;
    Four<M> m, v;
    float scale1, scale2;

    template <bool PAST>
    __device__ void load(const Record& r, uint64_t block, uint32_t lane) {
        const uint64_t at = block * kBlock + lane * 4;
        g = load4<PAST>(static_cast<const G*>(r.grad) + at);
        w = load4<PAST>(stepped(r) + at);
        m = load4<PAST>(static_cast<const M*>(r.moment1) + at);
        v = load4<PAST>(static_cast<const M*>(r.moment2) + at);
        scales(r, block);
    }
    __device__ void load(const Record& r, uint64_t block, uint32_t lane, uint32_t left) {
        const uint64_t at = block * kBlock + lane * 4;
        g = load_some(static_cast<const G*>(r.grad) + at, left);
        w = load_some(stepped(r) + at, left);
        m = load_some(static_cast<const M*>(r.moment1) + at, left);
        v = load_some(static_cast<const M*>(r.moment2) + at, left);
        scales(r, block);
    }
    __device__ static C* stepped(const Record& r) {
        if constexpr (MASTER) return r.master;
        else return static_cast<W*>(r.weights);
    }
    __device__ void scales(const Record& r, uint64_t block) {
        if constexpr (EIGHT) {
            scale1 = r.scale1[block];
            scale2 = r.scale2[block];
        }
    }
    // The step, and what it leaves by `store`(place, four elements).
    template <typename F>
    __device__ void step(const Record& r, const Factors& f, uint64_t block, uint32_t lane, uint32_t left, uint32_t key, F store) const {
        float y[4], a[4], b[4], root[4];
        if constexpr (EIGHT) {
            decode(__builtin_bit_cast(uint32_t, m), scale1, a);
            decode(__builtin_bit_cast(uint32_t, v), scale2, b);
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] *= b[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                a[j] = m.v[j];
                b[j] = v.v[j];
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float grad = static_cast<float>(g.v[j]) * f.scale;
            a[j] = f.b1 * a[j] + f.g1 * grad;
            b[j] = f.b2 * b[j] + f.g2 * (grad * grad);
            root[j] = sqrtf(b[j]);
            y[j] = static_cast<float>(w.v[j]) * f.kept - f.by_m * (a[j] / (root[j] * f.by_v + f.eps));
        }
        const uint64_t at = block * kBlock + lane * 4;
        Four<W> to;
#pragma unroll
        for (int j = 0; j < 4; ++j) to.v[j] = static_cast<W>(y[j]);
        store(static_cast<W*>(r.weights) + at, to);
        if constexpr (MASTER) store(r.master + at, Four<float>{{y[0], y[1], y[2], y[3]}});
        if constexpr (EIGHT) {
            const uint32_t mine = mixed(key ^ static_cast<uint32_t>(block));
            uint32_t up1[4], up2[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t h = mixed(mine ^ (lane * 4 + j));
                up1[j] = h << 16;
                up2[j] = h & 0xffff0000u;
                if (static_cast<uint32_t>(j) >= left) a[j] = root[j] = 0.0f;
            }
            float s1, s2;
            const uint32_t c1 = encode<false>(a, up1, &s1), c2 = encode<true>(root, up2, &s2);
            store(static_cast<uint8_t*>(r.moment1) + at, __builtin_bit_cast(Four<uint8_t>, c1));
            store(static_cast<uint8_t*>(r.moment2) + at, __builtin_bit_cast(Four<uint8_t>, c2));
            if (lane == 0) {
                r.scale1[block] = s1;
                r.scale2[block] = s2;
            }
        } else {
            store(static_cast<float*>(r.moment1) + at, Four<float>{{a[0], a[1], a[2], a[3]}});
            store(static_cast<float*>(r.moment2) + at, Four<float>{{b[0], b[1], b[2], b[3]}});
        }
    }
};

// W, G: types of the weights and the gradient; MASTER: weights are the rounding of a copy in 32 bits; EIGHT: moments in 8 bits.  Bound by memory.
// Lists that read more than the memory-side cache holds go past the caches (PAST): 168 M fp32 elements, 4.7 GB, 860 us otherwise, 830 so, and 752 (6.2 TB/s)
// with three workgroups on a unit, which follow one another closely through memory (four 790, two 835).  In 8 bits (16-bit weights with a copy,
// 3.0 GB) there is more to compute, 98 vector instructions an element: as many workgroups as fit, both blocks of a wave loaded
// before either is computed, 506 to 555 us (six TB/s at the best); with LDS for three workgroups 650, one block after the other 600.
// Smaller lists are served by that cache when they were written a step ago: half a piece to a workgroup, 4.9 M elements 19.9 us, a whole one 21.3, past
// the caches 27.
template <typename W, typename G, bool MASTER, bool EIGHT, bool PAST>
__global__ __launch_bounds__(kThreads) void update_adamw(const Step a) {
    if constexpr (PAST && !EIGHT) {   // LDS that nobody uses, so that three workgroups are on a compute unit
        __shared__ volatile uint8_t held[kHeld];
        if (a.n == 0) held[threadIdx.x] = 0;
    }
    // a piece to a workgroup, or where caches serve half a piece: more of them
    constexpr uint32_t kShares = PAST ? 1 : 2, kBlocks = kPieceBlocks / kShares;
    const uint32_t number = block_of(blockIdx.y);
    if (number >= a.n * kShares) return;
    const Piece p = a.pieces[number / kShares];
    const Record r = a.tensors[p.tensor];
    const int32_t t = *a.step;
    const float scale = a.scale ? *a.scale : 1.0f;
    const double rate = a.lr * r.rate * (a.rate ? static_cast<double>(*a.rate) : 1.0);
    if (t < 1 || scale != scale) return;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t first = static_cast<uint64_t>(p.number) * kPieceBlocks + number % kShares * kBlocks;
    using H = Held<W, G, MASTER, EIGHT>;
    const auto factors = [&]() {
        return Factors{scale, static_cast<float>(rate / (1.0 - exp(t * a.ln1))), static_cast<float>(1.0 / sqrt(1.0 - exp(t * a.ln2))),
                       static_cast<float>(1.0 - rate * r.decay), a.b1, a.b2, a.g1, a.g2, a.eps};
    };
    const uint32_t key = mixed(mixed(a.seed + 0x9e3779b9u * static_cast<uint32_t>(t)) ^ static_cast<uint32_t>(r.number));
    if ((first + kBlocks) * kBlock <= r.elements) {
        constexpr uint32_t kTogether = EIGHT && PAST ? 2 : 1;   // blocks of a wave that are under way together
        H h[kTogether];
        const auto load = [&](uint32_t u) {
#pragma unroll
            for (uint32_t i = 0; i < kTogether; ++i) h[i].template load<PAST>(r, first + (u + i) * kWaves + wave, lane);
        };
        load(0);
        const Factors f = factors();
#pragma unroll 1
        for (uint32_t u = 0; u < kBlocks / kWaves; u += kTogether) {
            if (u > 0) load(u);
#pragma unroll
            for (uint32_t i = 0; i < kTogether; ++i)
                h[i].step(r, f, first + (u + i) * kWaves + wave, lane, 4, key, [](auto* to, const auto& y) { store4<PAST>(to, y); });
        }
        return;
    }
    const Factors f = factors();
    for (uint64_t block = first + wave; block < first + kBlocks && block * kBlock < r.elements; block += kWaves) {
        const uint32_t left = left_of(r.elements, block * kBlock + lane * 4);
        H h;
        h.load(r, block, lane, left);
        h.step(r, f, block, lane, left, key, [&](auto* to, const auto& y) { store_some(to, y, left); });
    }
}

// ---- host side ----------------------------------------------------------------------------------------------------------------
struct Kind {   // tensors of the same types, pieces first .. first + n
    blink_dtype_t weights, grad, moments;
    bool master, stepped;
    uint32_t first, n;
    uint64_t bytes;   // that a step reads
};
bool same(const Kind& k, const blink_update_tensor_t& t) {
    const bool stepped = t.weights != nullptr;
    return k.grad == t.grad_type && k.stepped == stepped &&
           (!stepped || (k.weights == t.weight_type && k.moments == t.moment_type && k.master == (t.master != nullptr)));
}

}  // namespace
}  // namespace blink

struct blink_update {
    int device = -1;
    void* block = nullptr;                 // records, then pieces
    const blink::Record* tensors = nullptr;
    const blink::Piece* pieces = nullptr;
    uint64_t bytes = 0;                    // that a step reads
    std::vector<blink::Kind> kinds;        // those of one gradient type next to one another
};

namespace blink {
namespace {

#define BLINK_HIP(call)                                                                  \
    do {                                                                                 \
        const hipError_t err__ = (call);                                                 \
        if (err__ != hipSuccess) {                                                       \
            std::fprintf(stderr, "blink: " #call " failed: %s\n", hipGetErrorString(err__)); \
            return err__ == hipErrorOutOfMemory ? BLINK_ENOMEM : BLINK_EHIP;             \
        }                                                                                \
    } while (0)

blink_status_t on_its_device(const blink_update& u) {
    int device = -1;
    BLINK_HIP(hipGetDevice(&device));
    return device == u.device ? BLINK_OK : BLINK_EMISMATCH;
}

// Calls f(first piece, pieces, gradient type) for each gradient type.
template <typename F>
void each_gradient(const blink_update& u, F f) {
    for (size_t i = 0; i < u.kinds.size();) {
        uint32_t n = 0;
        size_t j = i;
        for (; j < u.kinds.size() && u.kinds[j].grad == u.kinds[i].grad; ++j) n += u.kinds[j].n;
        if (n) f(u.kinds[i].first, n, u.kinds[i].grad);
        i = j;
    }
}
uint32_t groups_of(uint32_t pieces) { return std::min(kMostGroups, pieces); }

}  // namespace

blink_status_t make_update(const blink_update_tensor_t* tensors, int n, blink_update** out) {
    std::vector<Kind> kinds;
    std::vector<std::vector<int>> members;
    uint64_t total = 0;
    for (int i = 0; i < n; ++i) {
        size_t k = 0;
        while (k < kinds.size() && !same(kinds[k], tensors[i])) ++k;
        if (k == kinds.size()) {
            const blink_update_tensor_t& t = tensors[i];
            kinds.push_back({t.weight_type, t.grad_type, t.moment_type, t.master != nullptr, t.weights != nullptr, 0, 0, 0});
            members.emplace_back();
        }
        members[k].push_back(i);
        total += ceil_div(tensors[i].elements, kPiece);
    }
    if (total > 0x7fffffff) return BLINK_EINVAL;
    std::vector<size_t> order(kinds.size());
    for (size_t k = 0; k < order.size(); ++k) order[k] = k;
    std::stable_sort(order.begin(), order.end(), [&](size_t a, size_t b) { return kinds[a].grad < kinds[b].grad; });
    const size_t records = (static_cast<size_t>(n) * sizeof(Record) + 255) / 256 * 256, bytes = records + std::max<uint64_t>(1, total) * sizeof(Piece);
    std::vector<char> host(bytes, 0);
    Record* const record = reinterpret_cast<Record*>(host.data());
    Piece* piece = reinterpret_cast<Piece*>(host.data() + records);
    blink_update* const u = new blink_update;
    struct Drop {
        blink_update* u;
        ~Drop() {
            if (u && u->block) (void)hipFree(u->block);
            delete u;
        }
    } drop{u};
    uint32_t at = 0;
    for (const size_t k : order) {
        Kind kind = kinds[k];
        kind.first = at;
        for (const int i : members[k]) {
            const blink_update_tensor_t& t = tensors[i];
            record[i] = {t.weights, t.master, t.grad, t.moment1, t.moment2, t.scale1, t.scale2, t.elements, t.rate, t.decay, static_cast<uint64_t>(i)};
            kind.bytes += t.elements * (size_of(t.grad_type) + (t.master ? 4 : size_of(t.weight_type)) + (t.moment_type == BLINK_FP8 ? 2 : 8));
            const uint32_t pieces = static_cast<uint32_t>(ceil_div(t.elements, kPiece));
            for (uint32_t j = 0; j < pieces; ++j) piece[at++] = {static_cast<uint32_t>(i), j};
        }
        kind.n = at - kind.first;
        u->kinds.push_back(kind);
    }
    for (const Kind& k : u->kinds) u->bytes += k.stepped ? k.bytes : 0;
    BLINK_HIP(hipGetDevice(&u->device));
    BLINK_HIP(hipMalloc(&u->block, bytes));
    BLINK_HIP(hipMemcpy(u->block, host.data(), bytes, hipMemcpyHostToDevice));
    u->tensors = static_cast<const Record*>(u->block);
    u->pieces = reinterpret_cast<const Piece*>(static_cast<const char*>(u->block) + records);
    *out = u;
    drop.u = nullptr;
    return BLINK_OK;
}

void free_update(blink_update* u) {
    if (!u) return;
    if (u->block) (void)hipFree(u->block);
    delete u;
}

size_t gradient_norm_workspace(const blink_update& u) {
    size_t sums = 0;
    each_gradient(u, [&](uint32_t, uint32_t n, blink_dtype_t) { sums += groups_of(n); });
    return sums * sizeof(double);
}

blink_status_t gradient_norm(const blink_update& u, double most, double factor, float* norm, int32_t* step, void* workspace, hipStream_t stream) {
    BLINK_TRY(on_its_device(u));
    const Clip clip{most, factor, norm, step};
    double* const sums = static_cast<double*>(workspace);
    uint32_t at = 0, types = 0;
    blink_status_t st = BLINK_OK;
    each_gradient(u, [&](uint32_t, uint32_t, blink_dtype_t) { ++types; });
    bool done = false;
    each_gradient(u, [&](uint32_t first, uint32_t n, blink_dtype_t grad) {
        if (types == 1 && n <= kFew) {
            done = true;
            st = with_float(grad, [&](auto g) {
                return launch(update_few<decltype(g)>, dim3(1), dim3(kFewThreads), stream, Norm{u.tensors, u.pieces + first, n, nullptr}, clip);
            });
            return;
        }
        const uint32_t groups = groups_of(n);
        const Norm a{u.tensors, u.pieces + first, n, sums + at};
        at += groups;
        const bool past = static_cast<uint64_t>(n) * kPiece * size_of(grad) > kCache;
        if (st == BLINK_OK) st = with_float(grad, [&](auto g) {
            return launch(past ? update_squares<decltype(g), true> : update_squares<decltype(g), false>, dim3(groups), dim3(kThreads), stream, a);
        });
    });
    if (done || st != BLINK_OK) return st;
    return launch(update_norm, dim3(1), dim3(kNormThreads), stream, sums, at, clip);
}

blink_status_t adamw_step(const blink_update& u, const int32_t* step, double lr, double beta1, double beta2, double eps, const float* scale, const float* rate,
                          uint32_t seed, hipStream_t stream) {
    BLINK_TRY(on_its_device(u));
    // an eps that 32 bits round to 0 would divide 0 by 0 wherever nothing has moved yet
    const float at_least = std::max(static_cast<float>(eps), std::numeric_limits<float>::denorm_min());
    for (const Kind& k : u.kinds) {
        if (!k.stepped || k.n == 0) continue;
        const Step a{u.tensors, u.pieces + k.first, k.n, step, scale, rate, lr, std::log(beta1), std::log(beta2), static_cast<float>(beta1),
                     static_cast<float>(beta2), static_cast<float>(1 - beta1), static_cast<float>(1 - beta2), at_least, seed};
        BLINK_TRY(with_float(k.weights, [&](auto w) {
            return with_float(k.grad, [&](auto g) {
                using W = decltype(w);
                using G = decltype(g);
                const bool beyond = u.bytes > kCache;
                const Grid grid = grid_of(beyond ? k.n : 2 * static_cast<uint64_t>(k.n), kThreads);
                const auto run = [&](void (*here)(Step), void (*past)(Step)) {
                    return launch(beyond ? past : here, dim3(grid.x, grid.y), dim3(kThreads), stream, a);
                };
                if constexpr (!std::is_same<W, float>::value)
                    if (k.master)
                        return k.moments == BLINK_FP32 ? run(update_adamw<W, G, true, false, false>, update_adamw<W, G, true, false, true>)
                                                       : run(update_adamw<W, G, true, true, false>, update_adamw<W, G, true, true, true>);
                return k.moments == BLINK_FP32 ? run(update_adamw<W, G, false, false, false>, update_adamw<W, G, false, false, true>)
                                               : run(update_adamw<W, G, false, true, false>, update_adamw<W, G, false, true, true>);
            });
        }));
    }
    return BLINK_OK;
}

}  // namespace blink
