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

// Four elements, wherever they start.
template <typename T>
struct alignas(sizeof(T)) Four {
    T v[4];
};
template <typename T>
__device__ inline Four<T> load4(const T* p, uint32_t left) {   // zeros past the end
    if (left >= 4) return *reinterpret_cast<const Four<T>*>(p);
    Four<T> y;
    for (uint32_t i = 0; i < 4; ++i) y.v[i] = i < left ? p[i] : static_cast<T>(0);
    return y;
}
template <typename T>
__device__ inline void store4(T* p, uint32_t left, const Four<T>& y) {
    if (left >= 4) {
        *reinterpret_cast<Four<T>*>(p) = y;
        return;
    }
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

__device__ inline double add_up(double s, double (&part)[kWaves]) {   // for thread 0
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0;
    for (int w = 0; w < kWaves; ++w) s += part[w];
    return s;
}

// Squares and their sums in 64 bits: no gradient's square overflows or is lost.
template <typename G>
__global__ __launch_bounds__(kThreads) void update_squares(const Norm a) {
    __shared__ double part[kWaves];
    double s = 0.0;
    for (uint32_t i = blockIdx.x; i < a.n; i += gridDim.x) {
        const Piece p = a.pieces[i];
        const Record& r = a.tensors[p.tensor];
        const uint64_t from = static_cast<uint64_t>(p.number) * kPiece;
        const G* const grad = static_cast<const G*>(r.grad);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint64_t at = from + (u * kThreads + threadIdx.x) * 4;
            const uint32_t left = left_of(r.elements, at);
            const Four<G> g = load4(grad + at, left);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const double x = static_cast<float>(g.v[j]);
                s = __builtin_fma(x, x, s);
            }
        }
    }
    s = add_up(s, part);
    if (threadIdx.x == 0) a.sums[blockIdx.x] = s;
}

__global__ __launch_bounds__(kThreads) void update_norm(const double* sums, uint32_t n, double most, double factor, float* norm, int32_t* step) {
    __shared__ double part[kWaves];
    double s = 0.0;
    for (uint32_t i = threadIdx.x; i < n; i += kThreads) s += sums[i];
    s = add_up(s, part);
    if (threadIdx.x != 0) return;
    const bool fine = s < __builtin_inf();   // (not with an infinite gradient, nor with a NaN)
    const double length = sqrt(s) * fabs(factor);
    norm[0] = static_cast<float>(length);
    norm[1] = fine ? static_cast<float>(length > most ? factor * (most / length) : factor) : __builtin_nanf("");
    if (step && fine) *step += 1;
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

// |z| <= 448, given by its bits, as an e4m3 number; `up`: 16 random bits.
__device__ inline uint32_t to_eight(uint32_t z, uint32_t up) {
    constexpr uint32_t kNormal = 0x3c800000u;   // 2^-6
    const float y = __builtin_bit_cast(float, z);
    const uint32_t large = ((z + (up << 4 | 8)) >> 20) - 960;             // (exponents differ by 120, 3 bits of 23 stay)
    const float units = y * 512.0f;                                       // exact, as is what is left of it
    const uint32_t down = static_cast<uint32_t>(units);
    const uint32_t small = down + (units - static_cast<float>(down) >= 1.0f - (static_cast<float>(up) + 0.5f) * 0x1p-16f);
    const uint32_t code = z >= kNormal ? large : small;
    return code > 0x7e ? 0x7e : code;
}

// The four numbers of a lane as codes, and the scale of the wave's 256.  ROOT: y >= 0, and what is not zero is not stored as zero.
template <bool ROOT>
__device__ inline uint32_t encode(const float (&y)[4], const uint32_t (&up)[4], float* scale) {
    uint32_t bits[4], most = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        bits[j] = __builtin_bit_cast(uint32_t, y[j]);
        const uint32_t size = bits[j] & 0x7fffffffu;
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
    uint32_t codes = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float z = __builtin_fminf(__builtin_fabsf(y[j]) * by, 448.0f);
        uint32_t c = to_eight(__builtin_bit_cast(uint32_t, z), up[j]);
        if (ROOT) c = c == 0 && z != 0.0f ? 1 : c;
        else c |= bits[j] >> 24 & 0x80u;
        codes |= c << (8 * j);
    }
    return codes;
}

__device__ inline void decode(uint32_t codes, float scale, float (&y)[4]) {
    const auto low = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), high = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
    y[0] = low[0] * scale;
    y[1] = low[1] * scale;
    y[2] = high[0] * scale;
    y[3] = high[1] * scale;
}

// W, G: types of the weights and the gradient; MASTER: weights are the rounding of a copy in 32 bits; EIGHT: moments in 8 bits.
template <typename W, typename G, bool MASTER, bool EIGHT>
__global__ __launch_bounds__(kThreads) void update_adamw(const Step a) {
    const uint32_t number = block_of(blockIdx.y);
    if (number >= a.n) return;
    const Piece p = a.pieces[number];
    const Record r = a.tensors[p.tensor];
    const int32_t t = *a.step;
    const float scale = a.scale ? *a.scale : 1.0f;
    const double rate = a.lr * r.rate * (a.rate ? static_cast<double>(*a.rate) : 1.0);
    if (t < 1 || scale != scale) return;
    const float by_m = static_cast<float>(rate / (1.0 - exp(t * a.ln1))), by_v = static_cast<float>(1.0 / sqrt(1.0 - exp(t * a.ln2)));
    const float kept = static_cast<float>(1.0 - rate * r.decay);
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t key = mixed(mixed(a.seed + 0x9e3779b9u * static_cast<uint32_t>(t)) ^ static_cast<uint32_t>(r.number));
    for (uint32_t u = wave; u < kPieceBlocks; u += kWaves) {
        const uint64_t block = static_cast<uint64_t>(p.number) * kPieceBlocks + u, from = block * kBlock;
        if (from >= r.elements) return;
        const uint64_t at = from + lane * 4;
        const uint32_t left = left_of(r.elements, at);
        const Four<G> g4 = load4(static_cast<const G*>(r.grad) + at, left);
        float w[4], m[4], v[4];
        if constexpr (MASTER) {
            const Four<float> y = load4(r.master + at, left);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = y.v[j];
        } else {
            const Four<W> y = load4(static_cast<const W*>(r.weights) + at, left);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = static_cast<float>(y.v[j]);
        }
        if constexpr (EIGHT) {
            const Four<uint8_t> c1 = load4(static_cast<const uint8_t*>(r.moment1) + at, left), c2 = load4(static_cast<const uint8_t*>(r.moment2) + at, left);
            decode(__builtin_bit_cast(uint32_t, c1), r.scale1[block], m);
            decode(__builtin_bit_cast(uint32_t, c2), r.scale2[block], v);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] *= v[j];
        } else {
            const Four<float> y1 = load4(static_cast<const float*>(r.moment1) + at, left), y2 = load4(static_cast<const float*>(r.moment2) + at, left);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                m[j] = y1.v[j];
                v[j] = y2.v[j];
            }
        }
        float root[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float g = static_cast<float>(g4.v[j]) * scale;
            m[j] = a.b1 * m[j] + a.g1 * g;
            v[j] = a.b2 * v[j] + a.g2 * (g * g);
            root[j] = sqrtf(v[j]);
            w[j] = w[j] * kept - by_m * (m[j] / (root[j] * by_v + a.eps));
        }
        Four<W> w4;
#pragma unroll
        for (int j = 0; j < 4; ++j) w4.v[j] = static_cast<W>(w[j]);
        store4(static_cast<W*>(r.weights) + at, left, w4);
        if constexpr (MASTER) store4(r.master + at, left, Four<float>{{w[0], w[1], w[2], w[3]}});
        if constexpr (EIGHT) {
            const uint32_t mine = mixed(key ^ static_cast<uint32_t>(block));
            uint32_t up1[4], up2[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t h = mixed(mine ^ (lane * 4 + j));
                up1[j] = h & 0xffffu;
                up2[j] = h >> 16;
                if (static_cast<uint32_t>(j) >= left) m[j] = root[j] = 0.0f;
            }
            float s1, s2;
            const uint32_t c1 = encode<false>(m, up1, &s1), c2 = encode<true>(root, up2, &s2);
            store4(static_cast<uint8_t*>(r.moment1) + at, left, __builtin_bit_cast(Four<uint8_t>, c1));
            store4(static_cast<uint8_t*>(r.moment2) + at, left, __builtin_bit_cast(Four<uint8_t>, c2));
            if (lane == 0) {
                r.scale1[block] = s1;
                r.scale2[block] = s2;
            }
        } else {
            store4(static_cast<float*>(r.moment1) + at, left, Four<float>{{m[0], m[1], m[2], m[3]}});
            store4(static_cast<float*>(r.moment2) + at, left, Four<float>{{v[0], v[1], v[2], v[3]}});
        }
    }
}

// ---- host side ----------------------------------------------------------------------------------------------------------------
struct Kind {   // tensors of the same types, pieces first .. first + n
    blink_dtype_t weights, grad, moments;
    bool master, stepped;
    uint32_t first, n;
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
    uint32_t n_pieces = 0;
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
            kinds.push_back({t.weight_type, t.grad_type, t.moment_type, t.master != nullptr, t.weights != nullptr, 0, 0});
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
            const uint32_t pieces = static_cast<uint32_t>(ceil_div(t.elements, kPiece));
            for (uint32_t j = 0; j < pieces; ++j) piece[at++] = {static_cast<uint32_t>(i), j};
        }
        kind.n = at - kind.first;
        u->kinds.push_back(kind);
    }
    u->n_pieces = at;
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
    double* const sums = static_cast<double*>(workspace);
    uint32_t at = 0;
    blink_status_t st = BLINK_OK;
    each_gradient(u, [&](uint32_t first, uint32_t n, blink_dtype_t grad) {
        const uint32_t groups = groups_of(n);
        const Norm a{u.tensors, u.pieces + first, n, sums + at};
        at += groups;
        if (st == BLINK_OK) st = with_float(grad, [&](auto g) { return launch(update_squares<decltype(g)>, dim3(groups), dim3(kThreads), stream, a); });
    });
    BLINK_TRY(st);
    return launch(update_norm, dim3(1), dim3(kThreads), stream, sums, at, most, factor, norm, step);
}

blink_status_t adamw_step(const blink_update& u, const int32_t* step, double lr, double beta1, double beta2, double eps, const float* scale, const float* rate,
                          uint32_t seed, hipStream_t stream) {
    BLINK_TRY(on_its_device(u));
    for (const Kind& k : u.kinds) {
        if (!k.stepped || k.n == 0) continue;
        const Step a{u.tensors, u.pieces + k.first, k.n, step, scale, rate, lr, std::log(beta1), std::log(beta2), static_cast<float>(beta1),
                     static_cast<float>(beta2), static_cast<float>(1 - beta1), static_cast<float>(1 - beta2), static_cast<float>(eps), seed};
        BLINK_TRY(with_float(k.weights, [&](auto w) {
            return with_float(k.grad, [&](auto g) {
                using W = decltype(w);
                using G = decltype(g);
                const Grid grid = grid_of(k.n, kThreads);
                const auto run = [&](void (*kernel)(Step)) { return launch(kernel, dim3(grid.x, grid.y), dim3(kThreads), stream, a); };
                if constexpr (!std::is_same<W, float>::value)
                    if (k.master) return k.moments == BLINK_FP32 ? run(update_adamw<W, G, true, false>) : run(update_adamw<W, G, true, true>);
                return k.moments == BLINK_FP32 ? run(update_adamw<W, G, false, false>) : run(update_adamw<W, G, false, true>);
            });
        }));
    }
    return BLINK_OK;
}

}  // namespace blink
