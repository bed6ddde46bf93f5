// Orthogonalised updates: the iteration of Newton and Schulz, which moves a matrix's singular values towards 1.
//
//   X = U / (|U| + eps)     (Frobenius norm; the transpose where U is tall, so that X is m x n with m <= n)
//   then for every step (a, b, c):  A = X X',  B = a I + b A + c A A,  X <- B X
//
// Bound by matrix products: m^2 n + m^3 + 2 m^2 n multiplications and additions a step, A and B being symmetric: of
// those only the tiles on and below the diagonal are computed.
//
// Numerics.  The products run on the 16-bit matrix instructions with sums in 32 bits.  X, A and B of every type of matrix are kept as
// pairs of 16-bit floats, hi = round(x) and lo = round(x - hi), 22 bits together, and a product is the sum of three: hi hi + hi lo + lo hi.  An
// error in A or B is relative to X and stays so; one in X lies across the small singular values, which a step makes up to a times
// larger.  Against 64 bits, five steps: 16 of 1024 x 1024 2.1e-6 of the result's norm, with 32-bit floats throughout 3.1e-6.  Single 16-bit A and
// B would do for no type: 9e-4 by themselves, more than half of what rounding the result to bfloat16's 8 bits adds (1.7e-3).  Everything is scaled
// by powers of two, so that what is stored lies in the middle of the 16-bit range.
//
// Layout.  All three products are sums over the contiguous index of both operands: A = X X', A A = A A', X B' with B'
// = B, so X is kept both ways round (X for the first, its transpose for the third).  A row of pairs is a sequence of groups of 128
// bytes, 32 hi and then their 32 lo, so one stage of a tile's row is one line of memory.  Sizes are rounded up to whole tiles with
// zeros, which the iteration keeps, and only the first and the last pass see the caller's sizes and strides.
#include "operators_api.hpp"

#include <algorithm>
#include <cmath>

namespace blink {
namespace {

using Half = _Float16;
typedef Half Half8 __attribute__((ext_vector_type(8)));
typedef float Float16v __attribute__((ext_vector_type(16)));

// Powers of two: |X| <= 2 (singular values of what the caller's coefficients allow, see coefficients_fit), |A| <= 4, |B| < 8.
constexpr float kScaleX = 16384.0f, kScaleA = 16384.0f, kScaleB = 8192.0f;

enum Last { kNone = 0, kMatrix, kWeights };   // what the last product writes: the matrix, or weights updated by it

// The caller's side: what is read at the start and written at the end.
struct Outer {
    const void* in;          // U, or the gradient
    uint64_t in_row, in_batch;
    const float* momentum;   // null: U is `in`
    float* momentum_out;
    float beta;
    bool nesterov;
    uint32_t rows, cols;
    const float* weights;
    float* weights_out;
    void* out;
    uint64_t out_row, out_batch;
    float rate, keep;        // weights' = keep * weights - rate * result
};

// U's element from the gradient's and the new momentum's; from the caller's buffers.
__device__ inline float update_of(const Outer& o, float g, float m) { return o.nesterov ? __builtin_fmaf(o.beta, m, g) : m; }
template <typename In>
__device__ inline float update_at(const Outer& o, uint64_t batch, uint32_t r, uint32_t c) {
    const float g = static_cast<float>(static_cast<const In*>(o.in)[batch * o.in_batch + r * o.in_row + c]);
    return o.momentum ? update_of(o, g, o.momentum_out[(batch * o.rows + r) * o.cols + c]) : g;
}

// ---- the norm, and the momentum ------------------------------------------------------------------------------------------
// A workgroup per part of a matrix; squares are added in 64 bits, where no 32-bit float's overflows or vanishes.  V neighbours to a
// thread at a time.  Bound by memory: a step's 8192 x 4096 of 32 bits 69 us, 5.8 TB/s.
constexpr int kNormThreads = 256, kNormMost = 1024;
template <typename In, int V>
__global__ __launch_bounds__(kNormThreads) void ortho_norm(const Outer o, double* parts) {
    __shared__ double wave_sum[kNormThreads / 64];
    const uint64_t batch = blockIdx.y, all = static_cast<uint64_t>(o.rows) * o.cols;
    const uint32_t packs = o.cols / V;   // of a row
    const uint64_t units = static_cast<uint64_t>(o.rows) * packs, step = static_cast<uint64_t>(gridDim.x) * kNormThreads;
    double s = 0.0;
#pragma unroll 4
    for (uint64_t e = blockIdx.x * static_cast<uint64_t>(kNormThreads) + threadIdx.x; e < units; e += step) {
        const uint32_t r = static_cast<uint32_t>(units >> 32 ? e / packs : static_cast<uint32_t>(e) / packs), c = static_cast<uint32_t>(e - static_cast<uint64_t>(r) * packs) * V;
        const Pack<In, V> g = *reinterpret_cast<const Pack<In, V>*>(static_cast<const In*>(o.in) + batch * o.in_batch + r * o.in_row + c);
        float u[V];
#pragma unroll
        for (int v = 0; v < V; ++v) u[v] = static_cast<float>(g.v[v]);
        if (o.momentum) {
            const uint64_t at = batch * all + static_cast<uint64_t>(r) * o.cols + c;
            Pack<float, V> m = *reinterpret_cast<const Pack<float, V>*>(o.momentum + at);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                m.v[v] = __builtin_fmaf(o.beta, m.v[v], u[v]);
                u[v] = update_of(o, u[v], m.v[v]);
            }
            *reinterpret_cast<Pack<float, V>*>(o.momentum_out + at) = m;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) s = __builtin_fma(static_cast<double>(u[v]), static_cast<double>(u[v]), s);
    }
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) wave_sum[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kNormThreads / 64; ++w) s += wave_sum[w];
        parts[batch * gridDim.x + blockIdx.x] = s;
    }
}

// ---- 16-bit storage ----------------------------------------------------------------------------------------------------------
// Sixteen values of a row from column j (a multiple of 16) on.
__device__ inline void store16(Half* row, uint32_t j, const float (&v)[16]) {
    Half8 h[2], l[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const Half hi = static_cast<Half>(v[i]);
        h[i / 8][i % 8] = hi;
        l[i / 8][i % 8] = static_cast<Half>(v[i] - static_cast<float>(hi));
    }
    Half* const at = row + (j >> 5) * 64 + (j & 31);
    *reinterpret_cast<Half8*>(at) = h[0];
    *reinterpret_cast<Half8*>(at + 8) = h[1];
    *reinterpret_cast<Half8*>(at + 32) = l[0];
    *reinterpret_cast<Half8*>(at + 40) = l[1];
}
__device__ inline void load16(float (&v)[16], const Half* row, uint32_t j) {
    const Half* const at = row + (j >> 5) * 64 + (j & 31);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const Half8 h = *reinterpret_cast<const Half8*>(at + 8 * q), l = *reinterpret_cast<const Half8*>(at + 32 + 8 * q);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[8 * q + i] = static_cast<float>(h[i]) + static_cast<float>(l[i]);
    }
}

// ---- X and its transpose from U ------------------------------------------------------------------------------------------------
// 64 x 64 of X to a workgroup.  Bound by memory: 8192 x 4096 of 32 bits 136
// us, 3.9 TB/s.
constexpr int kFirstThreads = 256;
template <typename In>
__global__ __launch_bounds__(kFirstThreads) void ortho_first(const Outer o, bool tall, const double* parts, uint32_t n_parts, float eps, uint32_t mp, uint32_t np,
                                                             Half* x, Half* xt) {
    __shared__ float tile[64][65];
    __shared__ double wave_sum[kFirstThreads / 64];
    const int t = threadIdx.x;
    const uint64_t batch = blockIdx.z;
    const uint32_t i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;
    // along the caller's contiguous index: X's columns, or its rows where U is tall
    const uint32_t r0 = tall ? j0 : i0, c0 = tall ? i0 : j0;
    float u[16];
#pragma unroll
    for (int q = 0; q < 16; ++q) {
        const uint32_t r = r0 + q * 4 + t / 64, c = c0 + t % 64;
        u[q] = r < o.rows && c < o.cols ? update_at<In>(o, batch, r, c) : 0.0f;
    }
    static_assert(kNormMost % kFirstThreads == 0, "every part once");
    double s = 0.0;
#pragma unroll
    for (uint32_t p = 0; p < kNormMost; p += kFirstThreads) s += p + t < n_parts ? parts[batch * n_parts + p + t] : 0.0;
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
    if (t % 64 == 0) wave_sum[t / 64] = s;
#pragma unroll
    for (int q = 0; q < 16; ++q) {
        const uint32_t r = q * 4 + t / 64, c = t % 64;
        if (tall) tile[c][r] = u[q];
        else tile[r][c] = u[q];
    }
    __syncthreads();
    double sum = 0.0;
    for (int w = 0; w < kFirstThreads / 64; ++w) sum += wave_sum[w];
    // a matrix of zeros, its norm and eps both 0, stays one; f may be past the range of 32-bit floats, its products with elements are in it
    const double norm = sqrt(sum) + eps, f = norm == 0.0 ? 0.0 : kScaleX / norm;
    const uint32_t row = t / 4, col = t % 4 * 16;
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = static_cast<float>(tile[row][col + i] * f);
    store16(x + (batch * mp + i0 + row) * np * 2, j0 + col, v);
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = static_cast<float>(tile[col + i][row] * f);
    store16(xt + (batch * np + j0 + row) * mp * 2, i0 + col, v);
}

// ---- the products --------------------------------------------------------------------------------------------------------------
enum Product { kGram, kSquare, kApply, kApplyLast };   // A = X X', B of A, X <- B X, the result

struct Factors {
    const Half *p, *q;     // out[i][j] = sum over k of p[i][k] q[j][k]
    uint32_t mp, np;       // rows of p and q
    uint32_t k;            // a multiple of the stage
    uint32_t tiles, tiles_n;
    const Half* a;         // kSquare: A itself
    Half *out, *out_t;     // what is written, and its transpose (kApply); A and B are their own transposes
    float c0, c1, c2;      // factors of I, of A, of the product
    uint32_t part;         // stages of a part of a long sum (tiles of 128 and 64)
};

// A workgroup's tile is TM x TN, its waves' WM x WN of 32 x 32 blocks each; a stage is 32 of k, a row of it 128 bytes.  Stages are copied to
// LDS by the loads themselves, one ahead of the stage that is multiplied, three where a stage takes less time than its copy (tiles of 128
// and 64; with one ahead 2048 x 2048 took 742 us in tiles of 128, with three 663).  The sixteen 16-byte parts of 256 bytes lie in the order part ^
// (line % 16), so that any 16 of a block's rows, read part by part, fall on all banks (in eights, 128 bytes a line: half of the LDS cycles were
// conflicts).
constexpr int kStage = 32;   // of k
constexpr int kLine = 128;   // bytes of a row's stage
template <int TM, int TN, int WAVES_M, int WAVES_N>
struct Tile {
    static constexpr int kThreads = WAVES_M * WAVES_N * 64;
    static constexpr int kBytesP = TM * kLine, kBytes = kBytesP + TN * kLine;
    static constexpr int kWM = TM / WAVES_M, kWN = TN / WAVES_N, kBM = kWM / 32, kBN = kWN / 32;
    static constexpr int kCopies = kBytes / 16 / kThreads;            // of a thread, for a stage
    static constexpr int kAhead = TM <= 128 ? 3 : 1;                  // stages on their way while one is multiplied
    static constexpr int kBlock = 32 * 33 * 4;                        // bytes of a wave's block at the end
    static_assert(WAVES_M * WAVES_N * kBlock <= 2 * kBytes, "the blocks fit the stages");
};

constexpr uint32_t kRows = 256 / kLine, kParts = kLine / 16;        // of 256 bytes; of a row
__device__ inline uint32_t slot_of(uint32_t row, uint32_t part) {   // byte offset of a part of a row
    const uint32_t line = row / kRows, at = row % kRows * kParts + part;
    return line * 256 + ((at ^ (line & 15)) * 16);
}

// Copies a stage of ROWS rows: every thread 16 bytes at a time, in the order of LDS, each from where its part is.  A thread's places
// in the rounds are a whole number of sixteens of lines apart, so one offset serves them all.
__device__ inline uint32_t first_offset(uint32_t pitch) {
    const uint32_t t = threadIdx.x, line = t >> 4, at = (t & 15) ^ (line & 15), row = line * kRows + at / kParts, part = at % kParts;
    return row * pitch + part * 16;
}
template <int ROWS, int THREADS>
__device__ inline void copy_stage(__amdgpu_buffer_rsrc_t from, uint32_t offset, uint32_t pitch, uint32_t k_bytes, char* to) {
    constexpr int kTimes = ROWS * kLine / 16 / THREADS, kRound = ROWS / kTimes;   // rounds, rows of one
    static_assert(kTimes * THREADS * 16 == ROWS * kLine && THREADS % 256 == 0, "whole rounds");
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int u = 0; u < kTimes; ++u)   // (a wave's lanes follow one another in LDS)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)(to + (u * THREADS + wave * 64) * 16), 16, offset,
                                                 k_bytes + u * kRound * pitch, 0, 0);
}

template <int TM, int TN, int WAVES_M, int WAVES_N>
__device__ inline void multiply_stage(const char* at, Float16v (&acc)[TM / WAVES_M / 32][TN / WAVES_N / 32],
                                      Float16v (&low)[TM / WAVES_M / 32][TN / WAVES_N / 32], int wm, int wn) {
    using S = Tile<TM, TN, WAVES_M, WAVES_N>;
    const int lane = threadIdx.x & 63, row = lane & 31, half = lane >> 5;
    const char* const p = at;
    const char* const q = at + S::kBytesP;
#pragma unroll
    for (int ks = 0; ks < kStage / 16; ++ks) {   // 16 of k: two parts of 8
        const uint32_t part = ks * 2 + half;
        Half8 ph[S::kBM], pl[S::kBM], qh[S::kBN], ql[S::kBN];
#pragma unroll
        for (int i = 0; i < S::kBM; ++i) {
            const uint32_t r = wm * S::kWM + i * 32 + row;
            ph[i] = *reinterpret_cast<const Half8*>(p + slot_of(r, part));
            pl[i] = *reinterpret_cast<const Half8*>(p + slot_of(r, part + 4));
        }
#pragma unroll
        for (int j = 0; j < S::kBN; ++j) {
            const uint32_t r = wn * S::kWN + j * 32 + row;
            qh[j] = *reinterpret_cast<const Half8*>(q + slot_of(r, part));
            ql[j] = *reinterpret_cast<const Half8*>(q + slot_of(r, part + 4));
        }
        // the same sums again only after all the others
#pragma unroll
        for (int term = 0; term < 3; ++term)
#pragma unroll
            for (int i = 0; i < S::kBM; ++i)
#pragma unroll
                for (int j = 0; j < S::kBN; ++j) {
                    if (term == 0) low[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph[i], ql[j], low[i][j], 0, 0, 0);
                    if (term == 1) low[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl[i], qh[j], low[i][j], 0, 0, 0);
                    if (term == 2) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph[i], qh[j], acc[i][j], 0, 0, 0);
                }
    }
}

// The tile of a product that a place in the grid stands for.
struct Place {
    uint64_t batch;
    uint32_t ti, tj;
};
template <bool SYMMETRIC>
__device__ inline Place place_of(uint32_t place, uint32_t tiles, uint32_t tiles_n) {
    Place r;
    r.batch = place / tiles;
    const uint32_t tile = place - static_cast<uint32_t>(r.batch) * tiles;
    if (SYMMETRIC) {   // rows of the triangle: row i has i + 1 tiles
        uint32_t i = static_cast<uint32_t>((sqrtf(8.0f * tile + 1.0f) - 1.0f) * 0.5f);
        while (i * (i + 1) / 2 > tile) --i;
        while ((i + 1) * (i + 2) / 2 <= tile) ++i;
        r.ti = i;
        r.tj = tile - i * (i + 1) / 2;
    } else {
        // eight rows of tiles at a time, column by column: the tiles that a die has at a time share few rows of both operands
        const uint32_t tm = tiles / tiles_n, eights = tile / (8 * tiles_n), rows = min(8u, tm - eights * 8), in = tile - eights * 8 * tiles_n;
        r.tj = in / rows;
        r.ti = eights * 8 + in - r.tj * rows;
    }
    return r;
}
// Workgroups go round the eight dies in turn: each die gets a run of neighbouring places.
__device__ inline uint32_t die_run() {
    const uint32_t per = gridDim.x >> 3, bid = blockIdx.x;
    return bid < per * 8 ? (bid & 7) * per + (bid >> 3) : bid;
}

// Adds stages [from, to) of a tile's product to acc.
template <int TM, int TN, int WAVES_M, int WAVES_N>
__device__ inline void accumulate(const Factors& f, const Place& at, uint32_t from, uint32_t to, char* buf0, char* buf1, char* buf2, char* buf3,
                                  Float16v (&acc)[TM / WAVES_M / 32][TN / WAVES_N / 32], int wm, int wn) {
    using S = Tile<TM, TN, WAVES_M, WAVES_N>;
    const uint32_t pitch = f.k * 4;   // bytes of a row of pairs
    const auto rows_of = [pitch](const Half* first, uint64_t row, int rows) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(reinterpret_cast<const char*>(first)) + row * pitch, 0, rows * pitch, 0x00020000);
    };
    const auto p = rows_of(f.p, at.batch * f.mp + at.ti * TM, TM), q = rows_of(f.q, at.batch * f.np + at.tj * TN, TN);
    const uint32_t offset = first_offset(pitch);
    const auto copy = [&](uint32_t stage, char* to_buf) {
        copy_stage<TM, S::kThreads>(p, offset, pitch, stage * kLine, to_buf);
        copy_stage<TN, S::kThreads>(q, offset, pitch, stage * kLine, to_buf + S::kBytesP);
    };
    // The stage that is due has arrived, of this wave's copies and then of everybody's, and everybody has read the one before; `later` stages may
    // still be on their way, for which __syncthreads would wait.
    const auto arrived = [](auto later) {
        constexpr int kMany = decltype(later)::value * S::kCopies;
        static_assert(kMany < 64, "what the counter counts");
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070 | (kMany & 15) | (kMany >> 4 << 14));   // (copies in flight at most; no LDS access of its own)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // Where there are registers for it the products with a lo, which are small, are summed apart from the others: a matrix instruction rounds its
    // sum, and three in a row for every 16 of a long k left the step's result (2025 x 22) 4.2e-6 off, 2.5 times as far as 32-bit products do.
    Float16v low[S::kBM][S::kBN] = {};
    const auto stage = [&](uint32_t s, char* now, char* free) {   // (past the last stage that one is copied again, so that the count stays; nobody reads it)
        arrived(std::integral_constant<int, S::kAhead - 1>());
        copy(min(s + S::kAhead, to - 1), free);
        if constexpr (S::kAhead == 1) {
            asm volatile("" ::: "memory");   // on their way before anything is read: the compiler would send them last
            multiply_stage<TM, TN, WAVES_M, WAVES_N>(now, acc, acc, wm, wn);
        } else
            multiply_stage<TM, TN, WAVES_M, WAVES_N>(now, acc, low, wm, wn);
    };
    copy(from, buf0);
    uint32_t s = from;
    if constexpr (S::kAhead == 1) {
        for (; s + 1 < to; s += 2) {
            stage(s, buf0, buf1);
            stage(s + 1, buf1, buf0);
        }
        if (s < to) stage(s, buf0, buf1);
    } else {
        copy(min(from + 1, to - 1), buf1);
        copy(min(from + 2, to - 1), buf2);
        for (; s + 3 < to; s += 4) {
            stage(s, buf0, buf3);
            stage(s + 1, buf1, buf0);
            stage(s + 2, buf2, buf1);
            stage(s + 3, buf3, buf2);
        }
        if (s < to) stage(s, buf0, buf3);
        if (s + 1 < to) stage(s + 1, buf1, buf0);
        if (s + 2 < to) stage(s + 2, buf2, buf1);
#pragma unroll
        for (int b = 0; b < S::kBM * S::kBN; ++b) acc[b / S::kBN][b % S::kBN] += low[b / S::kBN][b % S::kBN];
    }
    arrived(std::integral_constant<int, 0>());
}

// Writes 32 x 32 of a product from row i and column j on, through 32 x 33 floats of LDS that are the wave's own, so that rows are written whole in both
// directions.  mirrored: the tile has another one on the other side of the diagonal (A and B).
template <Product WHAT, Last LAST, typename Out>
__device__ inline void write_block(const Factors& f, const Outer& o, bool tall, uint64_t batch, uint32_t i, uint32_t j, bool mirrored, const Float16v& acc, float* block) {
    constexpr bool kSymmetric = WHAT == kGram || WHAT == kSquare;
    const int lane = threadIdx.x & 63;
    // what has to be read travels while the block goes through LDS
    float old[16];
    const uint32_t r = lane >> 1, c = (lane & 1) * 16;
    if constexpr (WHAT == kSquare) load16(old, f.a + (batch * f.mp + i + r) * f.np * 2, j + c);
    const uint32_t row0 = (tall ? j : i) + (lane >> 5), col = (tall ? i : j) + (lane & 31);   // of the caller's matrix
    if constexpr (LAST == kWeights)
#pragma unroll
        for (int u = 0; u < 16; ++u)
            old[u] = row0 + u * 2 < o.rows && col < o.cols ? o.weights[(batch * o.rows + row0 + u * 2) * o.cols + col] : 0.0f;
    wave_sync();
#pragma unroll
    for (int r = 0; r < 16; ++r) block[(8 * (r / 4) + 4 * (lane >> 5) + r % 4) * 33 + (lane & 31)] = acc[r] * f.c2;
    wave_sync();
    if constexpr (WHAT == kApplyLast) {
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            const uint32_t r = u * 2 + (lane >> 5), c = lane & 31, row = row0 + u * 2;
            const float v = tall ? block[c * 33 + r] : block[r * 33 + c];
            if (row < o.rows && col < o.cols) {
                if constexpr (LAST == kWeights) {
                    o.weights_out[(batch * o.rows + row) * o.cols + col] = __builtin_fmaf(-o.rate, v, o.keep * old[u]);
                } else {
                    static_cast<Out*>(o.out)[batch * o.out_batch + row * o.out_row + col] = static_cast<Out>(v);
                }
            }
        }
    } else {
        float v[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) v[u] = block[r * 33 + c + u];
        if constexpr (WHAT == kSquare) {
#pragma unroll
            for (int u = 0; u < 16; ++u) {
                v[u] = __builtin_fmaf(f.c1, old[u], v[u]) + (i + r == j + c + u ? f.c0 : 0.0f);
                block[r * 33 + c + u] = v[u];
            }
            wave_sync();
        }
        store16(f.out + (batch * f.mp + i + r) * f.np * 2, j + c, v);
        if (!kSymmetric || mirrored) {
#pragma unroll
            for (int u = 0; u < 16; ++u) v[u] = block[(c + u) * 33 + r];
            if constexpr (kSymmetric) store16(f.out + (batch * f.mp + j + r) * f.np * 2, i + c, v);
            else store16(f.out_t + (batch * f.np + j + r) * f.mp * 2, i + c, v);
        }
    }
}

// A tile of a product to a workgroup.  Tiles of 256 are bound by the matrix instructions at
// the clock that power allows: B X of 8192 x 4096 pairs 706 us, 1.17 PFLOP/s of products, 68 % busy at 1.64 GHz (16-bit library product
// of 8192 cubed 1.39); small ones by latency, 3 to 10 us.
template <int TM, int TN, int WAVES_M, int WAVES_N, Product WHAT, Last LAST, typename Out>
__global__ __launch_bounds__(WAVES_M * WAVES_N * 64) void ortho_product(const Factors f, const Outer o, bool tall) {
    using S = Tile<TM, TN, WAVES_M, WAVES_N>;
    // (arrays of their own, so that the compiler knows which loads a read has to wait for)
    __shared__ __align__(1024) char buf0[S::kBytes], buf1[S::kBytes];
    __shared__ __align__(1024) char buf2[S::kAhead > 1 ? S::kBytes : 16], buf3[S::kAhead > 1 ? S::kBytes : 16];
    constexpr bool kSymmetric = WHAT == kGram || WHAT == kSquare;
    static_assert(!kSymmetric || TM == TN, "square tiles");
    const int wave = threadIdx.x >> 6, wm = wave / WAVES_N, wn = wave % WAVES_N;
    const Place at = place_of<kSymmetric>(die_run(), f.tiles, f.tiles_n);
    Float16v acc[S::kBM][S::kBN] = {};
    const uint32_t stages = f.k / kStage;
    accumulate<TM, TN, WAVES_M, WAVES_N>(f, at, 0, S::kAhead == 1 ? stages : min(f.part, stages), buf0, buf1, buf2, buf3, acc, wm, wn);
    if constexpr (S::kAhead > 1)   // (parts of a long sum, as `low` is one)
        for (uint32_t from = f.part; from < stages; from += f.part) {
            Float16v part[S::kBM][S::kBN] = {};
            accumulate<TM, TN, WAVES_M, WAVES_N>(f, at, from, min(from + f.part, stages), buf0, buf1, buf2, buf3, part, wm, wn);
#pragma unroll
            for (int b = 0; b < S::kBM * S::kBN; ++b) acc[b / S::kBN][b % S::kBN] += part[b / S::kBN][b % S::kBN];
        }
    constexpr int kFits = S::kBytes / S::kBlock;
    float* const block = reinterpret_cast<float*>((wave < kFits ? buf0 : buf1) + (wave < kFits ? wave : wave - kFits) * S::kBlock);
#pragma unroll
    for (int bi = 0; bi < S::kBM; ++bi)
#pragma unroll
        for (int bj = 0; bj < S::kBN; ++bj)
            write_block<WHAT, LAST, Out>(f, o, tall, at.batch, at.ti * TM + wm * S::kWM + bi * 32, at.tj * TN + wn * S::kWN + bj * 32, at.ti != at.tj, acc[bi][bj],
                                             block);
}

// ---- symmetric products with fewer tiles than compute units -------------------------------------------------------------------
// The stages of all tiles in one line, an equal run of them to every workgroup (never longer than a tile, so it touches two at most); a
// run's sums go to the workspace in 32 bits, and a second kernel adds a tile's together in order.  136 tiles of 256 stages: 500 us a tile to
// a workgroup, 360 + 36 in runs.
constexpr uint32_t kRuns = 256;
constexpr size_t kPartFloats = 256 * 256;   // a run has two of them
struct Runs {
    float* parts;
    uint32_t stages, tiles;   // stages of a tile, tiles of all matrices
    __host__ __device__ uint64_t begin(uint32_t run) const { return static_cast<uint64_t>(run) * stages * tiles / kRuns; }
};
using Whole = Tile<256, 256, 2, 4>;
constexpr int kPartBlocks = 64;             // of 32 x 32

__global__ __launch_bounds__(Whole::kThreads) void ortho_runs(const Factors f, const Runs runs) {
    using S = Whole;
    __shared__ __align__(1024) char buf0[S::kBytes], buf1[S::kBytes];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = wave / 4, wn = wave % 4;
    const uint32_t run = die_run();
    uint64_t u = runs.begin(run);
    const uint64_t end = runs.begin(run + 1);
    for (uint32_t part = run * 2; u < end; ++part) {
        const uint32_t tile = static_cast<uint32_t>(u / runs.stages), from = static_cast<uint32_t>(u - static_cast<uint64_t>(tile) * runs.stages);
        const uint32_t to = static_cast<uint32_t>(min(static_cast<uint64_t>(runs.stages), from + (end - u)));
        Float16v acc[S::kBM][S::kBN] = {};
        accumulate<256, 256, 2, 4>(f, place_of<true>(tile, f.tiles, f.tiles_n), from, to, buf0, buf1, buf0, buf1, acc, wm, wn);
        Pack<float, 4>* const out = reinterpret_cast<Pack<float, 4>*>(runs.parts + part * kPartFloats) + wave * (S::kBM * S::kBN * 256) + lane;
#pragma unroll
        for (int b = 0; b < S::kBM * S::kBN; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                Pack<float, 4> y;
#pragma unroll
                for (int v = 0; v < 4; ++v) y.v[v] = acc[b / S::kBN][b % S::kBN][r * 4 + v];
                out[(b * 4 + r) * 64] = y;
            }
        u += to - from;
    }
}

constexpr int kGatherThreads = 256;
template <Product WHAT>
__global__ __launch_bounds__(kGatherThreads) void ortho_gather(const Factors f, const Runs runs) {
    using S = Whole;
    __shared__ float blocks[kGatherThreads / 64][32 * 33];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const uint32_t tile = blockIdx.x / (kPartBlocks / (kGatherThreads / 64)), b = blockIdx.x % (kPartBlocks / (kGatherThreads / 64)) * (kGatherThreads / 64) + wave;
    const Place at = place_of<true>(tile, f.tiles, f.tiles_n);
    const uint64_t first = static_cast<uint64_t>(tile) * runs.stages, last = first + runs.stages - 1;
    uint32_t run = static_cast<uint32_t>(first * kRuns / (static_cast<uint64_t>(runs.stages) * runs.tiles));
    while (runs.begin(run) > first) --run;
    while (runs.begin(run + 1) <= first) ++run;
    Float16v acc = {};
    for (; run < kRuns && runs.begin(run) <= last; ++run) {
        if (runs.begin(run) == runs.begin(run + 1)) continue;        // (more runs than stages)
        const uint32_t part = run * 2 + (runs.begin(run) < first);   // a run's second tile is one that it began before
        const Pack<float, 4>* const in = reinterpret_cast<const Pack<float, 4>*>(runs.parts + part * kPartFloats) + b * 256 + lane;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const Pack<float, 4> y = in[r * 64];
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[r * 4 + v] += y.v[v];
        }
    }
    const uint32_t w = b / (S::kBM * S::kBN), in_wave = b % (S::kBM * S::kBN);   // in the order of ortho_runs
    write_block<WHAT, kNone, float>(f, Outer{}, false, at.batch, at.ti * 256 + w / 4 * S::kWM + in_wave / S::kBN * 32, at.tj * 256 + w % 4 * S::kWN + in_wave % S::kBN * 32,
                                        at.ti != at.tj, acc, blocks[wave]);
}

// ---- host side ------------------------------------------------------------------------------------------------------------------
struct Sizes {
    uint32_t m, n, mp, np, tile;
    uint32_t norm_parts;
};

// Tiles of 256 keep the matrix instructions busiest, if there are about as many as compute units (a symmetric product that has fewer is done
// in runs); tiles of 128 if the symmetric products have half as many.  us, 32-bit, tiles of 64 / 128 / 256: 1024 x 4096 388 / 559 /
// 702, 1536 x 1536 432 / 443 / 813, 4 of 1024 x 1024 429 / 401 / 739, 2048 x 4096 1253 / 1043 / 1237, 4096 x 4096 5735 / 4306 / 3747.
// Both only where rounding a side up to them adds no more than a third: what is added is multiplied and stored too.  us, 32-bit,
// as here / in tiles that do not fill: 16 of 16 x 8192 431 / 877, 16 of 64 x 4096 236 / 527, 32 of 128 x 2048 247 / 562, 200 of 16 x 16
// 86 / 488, 128 of 64 x 64 81 / 141, 48 of 180 x 1000 284 / 543, 16 of 320 x 4096 690 / 1285, 96 of 250 x 300 445 / 512.  But A of few narrow
// and very long matrices has hardly a workgroup in small tiles, and runs of large ones share its sums (tiles of 64 / runs in tiles of 256 not
// filled): 64 x 49152 1556 / 923, 128 x 100000 3205 / 1215, 2 of 128 x 24600 893 / 689, 4 of 16 x 16000 668 / 610, but 3 of 64 x 16600 604 / 607,
// 4 of 64 x 12288 475 / 554, 8 of 16 x 16000 705 / 903.
Sizes sizes_of(size_t batch, size_t rows, size_t cols) {
    Sizes z;
    z.m = static_cast<uint32_t>(std::min(rows, cols));
    z.n = static_cast<uint32_t>(std::max(rows, cols));
    const auto tiles = [&](uint64_t t) { return batch * ceil_div(z.m, t) * ceil_div(z.n, t); };
    const uint64_t side = ceil_div(z.m, 128);
    const auto fills = [&](uint64_t t) { return 3 * ceil_div(z.m, t) * t <= 4 * uint64_t{z.m} && 3 * ceil_div(z.n, t) * t <= 4 * uint64_t{z.n}; };
    const bool long_sums = batch <= 4 && z.n > 16384;
    z.tile = (fills(256) || long_sums) && tiles(256) >= 192 ? 256 : fills(128) && batch * side * (side + 1) / 2 >= 128 ? 128 : 64;
    z.mp = static_cast<uint32_t>(ceil_div(z.m, z.tile) * z.tile);
    z.np = static_cast<uint32_t>(ceil_div(z.n, z.tile) * z.tile);
    // parts of 1024 elements at the least, four to a thread, and about 4096 workgroups in all at the most
    const uint64_t parts = std::min<uint64_t>(ceil_div(static_cast<uint64_t>(rows) * cols, 1024), std::max<uint64_t>(16, 4096 / batch));
    z.norm_parts = static_cast<uint32_t>(std::min<uint64_t>(kNormMost, parts));
    return z;
}

// Whether a symmetric product over k is done in runs: the compute units that its tiles leave idle gain (256 - tiles) / 256 of a tile's
// stages at about 2 us each, the sums that go through the workspace cost about 0.13 us for each run and tile.
bool in_runs(const Sizes& z, uint64_t batch, uint64_t k) {
    const uint64_t side = z.mp / 256, tiles = batch * side * (side + 1) / 2, stages = k / kStage;
    return z.tile == 256 && tiles <= kRuns && (kRuns - tiles) * stages > 17 * (kRuns + tiles);
}

struct Space {
    float* sums;
    double* parts;
    Half *x, *xt[2], *a, *b;   // a null: shared
    size_t bytes;
};
// A of 16-bit matrices lies in the copy of X' that the step has yet to write and nobody reads any more: A is not needed once B is there, and
// mp <= np.  That takes back from their workspace most of what pairs cost it.
Space space_of(const Sizes& z, size_t batch, bool shared, void* workspace) {
    Space s;
    Carve c(workspace);
    const size_t mn = batch * z.mp * z.np * 2, mm = batch * z.mp * z.mp * 2;
    s.sums = c.take<float>(in_runs(z, batch, z.np) ? kRuns * 2 * kPartFloats : 0);   // (if the square is, which is over fewer, so is A)
    s.parts = c.take<double>(batch * z.norm_parts);
    s.x = c.take<Half>(mn);
    for (Half*& t : s.xt) t = c.take<Half>(mn);
    s.a = shared ? nullptr : c.take<Half>(mm);
    s.b = c.take<Half>(mm);
    s.bytes = c.at;
    return s;
}

// T: the tile's edge.
template <int T, Product WHAT, Last LAST, typename Out>
blink_status_t run_product(const Factors& f, const Outer& o, bool tall, size_t batch, hipStream_t stream) {
    constexpr int kM = 2, kN = T >= 128 ? 4 : 2;
    Factors g = f;
    const uint32_t tm = f.mp / T, tn = f.np / T;
    g.tiles_n = tn;
    g.tiles = WHAT == kGram || WHAT == kSquare ? tm * (tm + 1) / 2 : tm * tn;
    const uint64_t groups = static_cast<uint64_t>(g.tiles) * batch;
    if (groups * (kM * kN * 64) > 0xffffffff) return BLINK_EINVAL;   // (threads of a launch; a workspace beyond any memory)
    return launch(ortho_product<T, T, kM, kN, WHAT, LAST, Out>, dim3(static_cast<uint32_t>(groups)), dim3(kM * kN * 64), stream, g, o, tall);
}

// A or B, of tiles of T.
template <int T, Product WHAT>
blink_status_t run_symmetric(const Sizes& z, const Space& s, const Factors& f, size_t batch, hipStream_t stream) {
    if constexpr (T == 256)
        if (in_runs(z, batch, f.k)) {
            Factors g = f;
            g.tiles_n = f.mp / 256;
            g.tiles = g.tiles_n * (g.tiles_n + 1) / 2;
            const Runs runs{s.sums, f.k / kStage, static_cast<uint32_t>(g.tiles * batch)};
            BLINK_TRY(launch(ortho_runs, dim3(kRuns), dim3(Whole::kThreads), stream, g, runs));
            return launch(ortho_gather<WHAT>, dim3(runs.tiles * (kPartBlocks / (kGatherThreads / 64))), dim3(kGatherThreads), stream, g, runs);
        }
    return run_product<T, WHAT, kNone, float>(f, Outer{}, false, batch, stream);
}

template <int T, Last LAST, typename Out>
blink_status_t iterate(const Sizes& z, const Space& s, const Outer& o, bool tall, size_t batch, const float* co, int steps, hipStream_t stream) {
    for (int step = 0; step < steps; ++step, co += 3) {
        Factors f{};
        Half* const a = s.a ? s.a : s.xt[~step & 1];
        f.p = f.q = s.x;
        f.mp = f.np = z.mp;
        f.k = z.np;
        f.out = a;
        f.c2 = kScaleA / (kScaleX * kScaleX);
        f.part = z.m < 64 ? 16 : 64;   // of few rows an element of A weighs more in the result
        BLINK_TRY((run_symmetric<T, kGram>(z, s, f, batch, stream)));
        f.p = f.q = f.a = a;
        f.k = z.mp;
        f.out = s.b;
        f.c0 = co[0] * kScaleB;
        f.c1 = co[1] * (kScaleB / kScaleA);
        f.c2 = co[2] * (kScaleB / (kScaleA * kScaleA));
        BLINK_TRY((run_symmetric<T, kSquare>(z, s, f, batch, stream)));
        f.p = s.b;
        f.q = s.xt[step & 1];
        f.np = z.np;
        f.out = s.x;
        f.out_t = s.xt[~step & 1];
        if (step < steps - 1) {
            f.c2 = 1.0f / kScaleB;
            BLINK_TRY((run_product<T, kApply, kNone, float>(f, o, tall, batch, stream)));
        } else {
            f.c2 = 1.0f / (kScaleB * kScaleX);
            BLINK_TRY((run_product<T, kApplyLast, LAST, Out>(f, o, tall, batch, stream)));
        }
    }
    return BLINK_OK;
}

template <typename In, Last LAST, typename Out>
blink_status_t run_all(const Sizes& z, size_t batch, const Outer& o, const float* co, int steps, float eps, void* workspace, hipStream_t stream) {
    const Space s = space_of(z, batch, sizeof(Out) == 2, workspace);
    const bool tall = o.rows > o.cols;
    constexpr size_t V = 16 / sizeof(float);
    const bool wide = o.cols % V == 0 && o.in_row % V == 0 && (batch == 1 || o.in_batch % V == 0) && aligned(o.in, V * sizeof(In)) && aligned(o.momentum, 16) &&
                      aligned(o.momentum_out, 16);
    BLINK_TRY(launch(wide ? ortho_norm<In, V> : ortho_norm<In, 1>, dim3(z.norm_parts, static_cast<uint32_t>(batch)), dim3(kNormThreads), stream, o, s.parts));
    BLINK_TRY(launch(ortho_first<In>, dim3(z.np / 64, z.mp / 64, static_cast<uint32_t>(batch)), dim3(kFirstThreads), stream, o, tall, s.parts, z.norm_parts, eps,
                     z.mp, z.np, s.x, s.xt[0]));
    if (z.tile == 256) return iterate<256, LAST, Out>(z, s, o, tall, batch, co, steps, stream);
    if (z.tile == 128) return iterate<128, LAST, Out>(z, s, o, tall, batch, co, steps, stream);
    return iterate<64, LAST, Out>(z, s, o, tall, batch, co, steps, stream);
}

}  // namespace

// Whether the iteration keeps singular values below 2 and the polynomial's below 8 for all that start in [0, 1].
bool coefficients_fit(const float* co, int steps) {
    double most = 1.0;
    for (int i = 0; i < steps; ++i, co += 3) {
        if (!std::isfinite(co[0]) || !std::isfinite(co[1]) || !std::isfinite(co[2])) return false;
        double next = 0.0;
        for (int u = 0; u <= 1024; ++u) {
            const double x = most * u / 1024, p = co[0] + x * x * (co[1] + x * x * co[2]);
            if (std::fabs(p) > 7.75) return false;
            next = std::max(next, std::fabs(x * p));
        }
        most = next * 1.001;
        if (most > 1.95) return false;
    }
    return true;
}

size_t orthogonalize_workspace(size_t batch, size_t rows, size_t cols, blink_dtype_t dtype) {
    return space_of(sizes_of(batch, rows, cols), batch, dtype != BLINK_FP32, nullptr).bytes;
}

blink_status_t orthogonalize(const void* in, blink_dtype_t dtype, size_t batch, size_t rows, size_t cols, size_t in_row, size_t in_batch, const float* co,
                             int steps, float eps, void* out, size_t out_row, size_t out_batch, void* workspace, hipStream_t stream) {
    Outer o{};
    o.in = in;
    o.in_row = in_row;
    o.in_batch = in_batch;
    o.rows = static_cast<uint32_t>(rows);
    o.cols = static_cast<uint32_t>(cols);
    o.out = out;
    o.out_row = out_row;
    o.out_batch = out_batch;
    const Sizes z = sizes_of(batch, rows, cols);
    return with_float(dtype, [&](auto type) {
        using T = decltype(type);
        return run_all<T, kMatrix, T>(z, batch, o, co, steps, eps, workspace, stream);
    });
}

blink_status_t orthogonal_step(const float* weights, float* weights_out, const float* momentum, float* momentum_out, const void* grad,
                               blink_dtype_t grad_type, size_t batch, size_t rows, size_t cols, float beta, bool nesterov, const float* co, int steps,
                               float eps, float rate, float decay, void* workspace, hipStream_t stream) {
    Outer o{};
    o.in = grad;
    o.in_row = cols;
    o.in_batch = rows * cols;
    o.momentum = momentum;
    o.momentum_out = momentum_out;
    o.beta = beta;
    o.nesterov = nesterov;
    o.rows = static_cast<uint32_t>(rows);
    o.cols = static_cast<uint32_t>(cols);
    o.weights = weights;
    o.weights_out = weights_out;
    o.rate = rate;
    o.keep = 1.0f - decay;
    const Sizes z = sizes_of(batch, rows, cols);
    return with_float(grad_type, [&](auto type) {
        return run_all<decltype(type), kWeights, float>(z, batch, o, co, steps, eps, workspace, stream);
    });
}

}  // namespace blink
