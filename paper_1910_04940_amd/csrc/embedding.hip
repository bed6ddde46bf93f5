// Rows of an embedding table for tokens, and the gradient of the table.
//
//   rows      out[i] = scale * table[token[i]]
//   gradient  table'[v] = scale * sum of grad[i] over the i with token[i] = v, in the order of i
//
// A token outside [0, vocab) is padding: its row is zero and its gradient goes nowhere.
//
// Both are bound by memory.  The gradient is formed without atomics on numbers, so that it is the same every time: the
// tokens are sorted with their positions (a stable radix sort), and the sorted list is merged with the table's rows:
// "row ends" and "positions" form one sequence in which position j of the sorted list has the place j + token[j] and the
// end of row v the place v + (tokens up to v).  Every wave takes an equal stretch of that sequence and walks it, so a
// row named by thousands of tokens and a thousand rows named by none cost what they move, every row is written once,
// and a stretch's start is found by a search over the sorted list.  What a stretch has of a row that it does not begin
// or does not end goes to the workspace in 32 bits; a second kernel joins those in order, one workgroup all parts of a row.
#include "operators_api.hpp"

#include <algorithm>

namespace blink {
namespace {

// ---- rows ---------------------------------------------------------------------------------------------------------------
constexpr int kRowThreads = 256;
constexpr int kRowUnits = 2;   // packs of one thread, their loads under way together (131072 x 2048: 115 us, 4 packs 119, 8 121)

// A pack is V elements; a row has `packs` of them.  Places go out pack by pack through all rows, so short and long rows
// fill the waves alike.  Bound by memory: 131072 rows of 2048 bfloat16 118 us, 6.8 TB/s with the table partly in the memory-side cache; one row 2.0 us.
template <typename In, typename Out, typename Token, typename Unit, int V>
__global__ __launch_bounds__(kRowThreads) void embedding_rows(const In* table, uint64_t vocab, uint64_t table_stride, const Token* tokens,
                                                              Unit units, uint32_t packs, float scale, Out* out, uint64_t out_stride, bool past) {
    const uint32_t block = sizeof(Unit) == 8 ? block_of(blockIdx.y) : blockIdx.x;
    const Unit first = static_cast<Unit>(block) * (kRowThreads * kRowUnits) + threadIdx.x;   // (a Unit holds the grid's places)
    int64_t token[kRowUnits];
    uint64_t row[kRowUnits];
    uint32_t at[kRowUnits];
#pragma unroll
    for (int u = 0; u < kRowUnits; ++u) {
        const Unit unit = first + u * kRowThreads;
        row[u] = unit / packs;
        at[u] = static_cast<uint32_t>(unit - row[u] * packs) * V;
        token[u] = unit < units ? static_cast<int64_t>(tokens[row[u]]) : -1;
    }
    Pack<In, V> x[kRowUnits];
#pragma unroll
    for (int u = 0; u < kRowUnits; ++u) {
        x[u] = Pack<In, V>{};
        if (static_cast<uint64_t>(token[u]) < vocab)
            x[u] = *reinterpret_cast<const Pack<In, V>*>(table + static_cast<uint64_t>(token[u]) * table_stride + at[u]);
    }
#pragma unroll
    for (int u = 0; u < kRowUnits; ++u) {
        Pack<Out, V> y;
#pragma unroll
        for (int i = 0; i < V; ++i) {   // (a padding token's row is +0 whatever the scale)
            float z = scale * static_cast<float>(x[u].v[i]);
            if constexpr (sizeof(Out) < 4) asm("" : "+v"(z));   // a 32-bit product: the mixed 16-bit one rounds it otherwise
            y.v[i] = static_cast<uint64_t>(token[u]) < vocab ? static_cast<Out>(z) : static_cast<Out>(0.0f);
        }
        if (first + u * kRowThreads < units) store_result(past, reinterpret_cast<Pack<Out, V>*>(out + row[u] * out_stride + at[u]), y);
    }
}

// ---- sorting tokens with their positions ------------------------------------------------------------------------------------
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;

// Ranks the items of a wave by digit, 64 at a time in order: counts[digit] goes up by the wave's items with that digit,
// the result is an item's place among them.  Items of lanes that are not `in` count nowhere.
__device__ inline uint32_t rank_in_wave(uint32_t digit, bool in, int bits, volatile uint32_t* counts) {
    const uint32_t lane = threadIdx.x & 63;
    unsigned long long same = __ballot(in);
    for (int b = 0; b < bits; ++b) {
        const bool one = digit >> b & 1;
        const unsigned long long ones = __ballot(one);
        same &= one ? ones : ~ones;
    }
    const uint32_t below = __popcll(same & ((1ull << lane) - 1));
    uint32_t before = 0;
    if (in) {
        before = counts[digit];
        if (below == 0) counts[digit] = before + __popcll(same);
    }
    return before + below;
}

// From counts[wave][digit]: begin[digit] becomes the sum of all smaller digits' items, counts[wave][digit] those of the digit in the waves
// before.  Of a workgroup with a thread to a digit at least.
__device__ inline void scan_counts(uint32_t (*counts)[kDigits], int digits, uint32_t* begin, uint32_t* wave_sum) {
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, waves = blockDim.x >> 6;
    uint32_t total = 0;
    if (t < digits)
        for (int w = 0; w < waves; ++w) {
            const uint32_t c = counts[w][t];
            counts[w][t] = total;
            total += c;
        }
    uint32_t sum = total;
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t other = __shfl_up(sum, d);
        if (lane >= d) sum += other;
    }
    if (lane == 63) wave_sum[wave] = sum;
    __syncthreads();
    for (int w = 0; w < wave; ++w) sum += wave_sum[w];
    if (t < digits) begin[t] = sum - total;
    __syncthreads();
}

template <typename Token>
__device__ inline uint32_t key_of(Token token, uint32_t vocab) {
    return static_cast<uint64_t>(static_cast<int64_t>(token)) < vocab ? static_cast<uint32_t>(token) : vocab;
}

// A token's place is the number of tokens that come before it.  Up to 2048 tokens are counted against one another, 64 tokens to a
// workgroup, a part of the list to each of its waves: no passes that wait for one another (509 tokens 4.8 us, two passes of the next kernel 8.1).
constexpr int kFewThreads = 256, kFewMost = 2048;
template <typename Token>
__global__ __launch_bounds__(kFewThreads) void embedding_sort_few(const Token* tokens, uint32_t n, uint32_t vocab, uint32_t* key_out, uint32_t* pos_out) {
    constexpr int kWaves = kFewThreads / 64;
    __shared__ __align__(16) uint32_t keys[kFewMost];
    __shared__ uint32_t before[kWaves][64];
    const uint32_t t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), i = blockIdx.x * 64 + lane;
    const uint32_t up = (n + 63) / 64 * 64;
    for (uint32_t j = t; j < up; j += kFewThreads) keys[j] = j < n ? key_of(tokens[j], vocab) : ~0u;
    __syncthreads();
    const uint32_t key = keys[i];
    uint32_t many = 0;
    for (uint32_t block = wave; block < up / 64; block += kWaves) {
        if (block == blockIdx.x) {
#pragma unroll 16
            for (uint32_t j = 0; j < 64; ++j) many += keys[block * 64 + j] < key + (j < lane);
        } else {   // an equal one counts if it is in a block before
            const uint32_t least = key + (block < blockIdx.x);
#pragma unroll 16
            for (uint32_t j = 0; j < 64; ++j) many += keys[block * 64 + j] < least;
        }
    }
    before[wave][lane] = many;
    __syncthreads();
    if (wave != 0 || i >= n) return;
    for (int w = 1; w < kWaves; ++w) many += before[w][lane];
    key_out[many] = key;
    pos_out[many] = i;
}

// More: one workgroup, the list in LDS from pass to pass.
constexpr int kOneThreads = 1024, kOneItems = 8, kOneMost = kOneThreads * kOneItems;
template <typename Token>
__global__ __launch_bounds__(kOneThreads) void embedding_sort_one(const Token* tokens, uint32_t n, uint32_t vocab, int bits, int passes, uint32_t* key_out,
                                                              uint32_t* pos_out) {
    __shared__ uint32_t counts[kOneThreads / 64][kDigits];
    __shared__ uint32_t begin[kDigits], wave_sum[kOneThreads / 64];
    __shared__ uint32_t keys[kOneMost], places[kOneMost];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, digits = 1 << bits;
    // every wave has a run of whole 64s, as few as hold them all
    const uint32_t rounds = (n + kOneThreads - 1) / kOneThreads;
    const uint32_t first = wave * rounds * 64 + lane;
    uint32_t key[kOneItems], pos[kOneItems], rank[kOneItems];
#pragma unroll
    for (int j = 0; j < kOneItems; ++j)
        if (j < static_cast<int>(rounds)) {
            const uint32_t i = first + j * 64;
            key[j] = i < n ? key_of(tokens[i], vocab) : 0;
            pos[j] = i;
        }
    for (int pass = 0, shift = 0; pass < passes; ++pass, shift += bits) {
        for (int d = lane; d < digits; d += 64) counts[wave][d] = 0;   // (a wave's counts are its own until the scan)
        wave_sync();
#pragma unroll
        for (int j = 0; j < kOneItems; ++j)
            if (j < static_cast<int>(rounds)) {
                const uint32_t i = first + j * 64;
                if (pass > 0 && i < n) {
                    key[j] = keys[i];
                    pos[j] = places[i];
                }
                rank[j] = rank_in_wave(key[j] >> shift & (digits - 1), i < n, bits, counts[wave]);
            }
        __syncthreads();
        scan_counts(counts, digits, begin, wave_sum);
#pragma unroll
        for (int j = 0; j < kOneItems; ++j)
            if (j < static_cast<int>(rounds) && first + j * 64 < n) {
                const uint32_t digit = key[j] >> shift & (digits - 1);
                const uint32_t to = begin[digit] + counts[wave][digit] + rank[j];
                (pass == passes - 1 ? key_out : keys)[to] = key[j];
                (pass == passes - 1 ? pos_out : places)[to] = pos[j];
            }
        __syncthreads();
    }
}

// More tokens: at most kMostChunks chunks of whole tiles, a workgroup to each.  A pass counts the digits of every chunk, then
// every workgroup adds up what it needs of the counts (two launches a pass; a third that scans them cost 4.5 us), and moves its items.
// Bound by latency: 65536 tokens, two passes of 64 chunks, 4.6 us to count and 6.9 to move each.
// (Counting the next digits while moving, by atomics on all chunks' counts, takes longer than the launch it saves: frequent tokens share a count.)
constexpr int kTileThreads = 512, kTileItems = 2, kTile = kTileThreads * kTileItems, kMostChunks = 256;
static_assert(kDigits <= kTileThreads, "a thread per digit");

template <typename Token>
__global__ __launch_bounds__(kTileThreads) void embedding_sort_count(const Token* tokens, const uint32_t* keys, uint32_t n, uint32_t vocab, uint32_t chunk,
                                                                     int shift, int bits, uint32_t* counts) {
    __shared__ uint32_t count[kDigits];
    const uint32_t t = threadIdx.x;
    count[t] = 0;
    __syncthreads();
    const uint64_t from = static_cast<uint64_t>(blockIdx.x) * chunk, to = from + chunk < n ? from + chunk : n;
#pragma unroll 2
    for (uint64_t i = from + t; i < to; i += kTileThreads)
        atomicAdd(&count[(tokens ? key_of(tokens[i], vocab) : keys[i]) >> shift & ((1u << bits) - 1)], 1u);
    __syncthreads();
    if (t < 1u << bits) counts[(blockIdx.x << bits) + t] = count[t];
}

template <typename Token>
__global__ __launch_bounds__(kTileThreads) void embedding_sort_move(const Token* tokens, const uint32_t* keys, const uint32_t* places, uint32_t n,
                                                                    uint32_t vocab, uint32_t chunk, int shift, int bits, const uint32_t* all_counts,
                                                                    uint32_t* key_out, uint32_t* pos_out) {
    __shared__ uint32_t counts[kTileThreads / 64][kDigits];
    __shared__ uint32_t begin[kDigits], wave_sum[kTileThreads / 64];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, digits = 1 << bits;
    const uint64_t from = static_cast<uint64_t>(blockIdx.x) * chunk, end = from + chunk < n ? from + chunk : n;
    uint64_t first = from + wave * (64 * kTileItems) + lane;
    uint32_t key[kTileItems], pos[kTileItems], rank[kTileItems];
    const auto load = [&] {
#pragma unroll
        for (int j = 0; j < kTileItems; ++j) {
            const uint64_t i = first + j * 64;
            const bool in = i < end;
            key[j] = !in ? 0 : tokens ? key_of(tokens[i], vocab) : keys[i];
            pos[j] = !in ? 0 : tokens ? static_cast<uint32_t>(i) : places[i];
        }
    };
    load();
    // where each digit begins: after the smaller digits of all chunks and its own of the chunks before
    uint32_t own = 0, ahead = 0;
    if (t < digits)
#pragma unroll 32
        for (uint32_t c = 0; c < gridDim.x; ++c) {
            const uint32_t many = all_counts[(c << bits) + t];
            own += many;
            ahead += c < blockIdx.x ? many : 0;
        }
    uint32_t sum = own;
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t other = __shfl_up(sum, d);
        if (lane >= d) sum += other;
    }
    if (lane == 63) wave_sum[wave] = sum;
    __syncthreads();
    for (int w = 0; w < wave; ++w) sum += wave_sum[w];
    begin[t] = sum - own + ahead;
    for (uint64_t tile = from; tile < end; tile += kTile, first += kTile) {
        if (tile != from) load();
        for (int d = lane; d < digits; d += 64) counts[wave][d] = 0;
        wave_sync();
#pragma unroll
        for (int j = 0; j < kTileItems; ++j) rank[j] = rank_in_wave(key[j] >> shift & (digits - 1), first + j * 64 < end, bits, counts[wave]);
        __syncthreads();
        uint32_t total = 0;
        if (t < digits)
            for (int w = 0; w < kTileThreads / 64; ++w) {
                const uint32_t c = counts[w][t];
                counts[w][t] = total;
                total += c;
            }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kTileItems; ++j)
            if (first + j * 64 < end) {
                const uint32_t digit = key[j] >> shift & (digits - 1), to = begin[digit] + counts[wave][digit] + rank[j];
                key_out[to] = key[j];
                pos_out[to] = pos[j];
            }
        __syncthreads();
        if (t < digits) begin[t] += total;
    }
}

// ---- the sums ---------------------------------------------------------------------------------------------------------------
// How many of the sorted positions, from the first on, are `before`.  A wave's 64 lanes probe 64 of them at a time.
template <typename F>
__device__ inline uint32_t search(uint32_t n, F before) {
    const uint32_t lane = threadIdx.x & 63;
    uint32_t lo = 0, hi = n;   // the answer is in [lo, hi]
    while (lo < hi) {
        const uint32_t step = (hi - lo + 63) / 64;
        const uint64_t j = lo + static_cast<uint64_t>(step) * lane;
        const int many = __popcll(__ballot(j < hi && before(j)));
        if (many == 0) return lo;
        const uint64_t top = static_cast<uint64_t>(lo) + static_cast<uint64_t>(step) * many;
        lo += step * (many - 1) + 1;
        hi = static_cast<uint32_t>(top < hi ? top : hi);
    }
    return lo;
}
// Those that come before place `d`: all j with j + key[j] < d (ALL), or d itself where rows that no token names are left alone and
// only positions have places.
template <bool ALL>
__device__ inline uint32_t positions_before(const uint32_t* keys, uint32_t n, uint64_t d) {
    if (!ALL) return static_cast<uint32_t>(d < n ? d : n);
    return search(n, [=](uint64_t j) { return j + keys[j] < d; });
}

struct Sums {
    const void* grad;
    uint64_t grad_stride;
    const uint32_t *keys, *places;
    uint32_t n, vocab, dim;
    float scale;
    void* table;
    uint64_t table_stride;
    uint32_t stretch;         // places of a wave, at most 64
    uint32_t stretches, columns;   // waves beside one another on a row
    float *head, *tail;       // [stretch][dim]: what a stretch has of a row that began before it, of one that does not end in it
    uint32_t* joined;         // [stretch]: the row that began before the stretch and ends in it, or kNoRow
    uint32_t dim_up;          // elements of a row of head and tail
    bool past;
};
constexpr uint32_t kNoRow = ~0u;

template <typename T, int V>
__device__ inline void load_up(float (&x)[V], const T* p) {
    const Pack<T, V> y = *reinterpret_cast<const Pack<T, V>*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = static_cast<float>(y.v[i]);
}
// The row's final sum: scaled, added to `y`, what is there, where ADD, rounded once.
template <typename T, int V, bool ADD>
__device__ inline void store_row(bool past, T* p, Pack<T, V> y, const float (&sum)[V], float scale) {
#pragma unroll
    for (int i = 0; i < V; ++i) y.v[i] = static_cast<T>(ADD ? __builtin_fmaf(scale, sum[i], static_cast<float>(y.v[i])) : scale * sum[i]);
    store_result(past, reinterpret_cast<Pack<T, V>*>(p), y);
}

constexpr int kSumThreads = 256;
constexpr int kSumAhead = 8;   // rows of a sum whose loads are under way together

// A wave: 64 V columns of the rows of its stretch, V to a lane; the next wave has the columns after them, so that a workgroup
// writes rows in one piece.  ALL: rows that no token names are written as zeros, else (ADD too) left alone.
// Bound by memory: 65536 rows of 1024 bfloat16 into 131072 of 32-bit floats 117 us, 5.7 TB/s; added to 5003 x 1001, 509 tokens, 7.1 us, latency.
template <typename Grad, typename T, int V, bool ADD>
__global__ __launch_bounds__(kSumThreads) void embedding_sums(const Sums s) {
    constexpr bool ALL = !ADD;
    const uint32_t place_of = __builtin_amdgcn_readfirstlane(block_of(blockIdx.y) * (kSumThreads / 64) + (threadIdx.x >> 6));
    const uint32_t w = place_of / s.columns, column = place_of - w * s.columns;
    if (w >= s.stretches) return;
    const uint32_t lane = threadIdx.x & 63, col = (column * 64 + lane) * V;
    const bool in = col < s.dim;
    const Grad* const grad = static_cast<const Grad*>(s.grad) + (in ? col : 0);
    T* const table = static_cast<T*>(s.table) + (in ? col : 0);
    const uint64_t places = static_cast<uint64_t>(s.n) + (ALL ? s.vocab : 0), d0 = static_cast<uint64_t>(w) * s.stretch;
    const uint64_t d1 = d0 + s.stretch < places ? d0 + s.stretch : places;
    const uint32_t p = __builtin_amdgcn_readfirstlane(positions_before<ALL>(s.keys, s.n, d0));
    // the stretch's positions lie in the 64 from p on
    const bool there_is = p + lane < s.n;
    const uint32_t key = there_is ? s.keys[p + lane] : s.vocab, place = there_is ? s.places[p + lane] : 0;
    const uint32_t last = p > 0 ? s.keys[p - 1] : kNoRow;
    const uint32_t many = __popcll(__ballot(there_is && (ALL ? p + lane + static_cast<uint64_t>(key) < d1 : p + lane < d1))), end = p + many;
    const uint32_t real = __popcll(__ballot(lane < many && key < s.vocab));   // padding comes last
    const uint32_t next = !ALL && end < s.n ? s.keys[end] : kNoRow;             // the next stretch's first row
    const uint32_t r_end = static_cast<uint32_t>(ALL ? d1 - end : s.vocab);   // rows below it end here (ALL)
    uint32_t r = static_cast<uint32_t>(ALL ? d0 - p : __builtin_amdgcn_readfirstlane(key));
    bool begun = p > 0 && r < s.vocab && __builtin_amdgcn_readfirstlane(last) == r;   // the row has positions in an earlier stretch
    bool any = false;                                                                          // and in this one
    float sum[V] = {};
    Pack<T, V> there;   // what the row holds (ADD)
    uint32_t joins = kNoRow;
    const auto finish = [&] {   // row r ends
        if (begun) joins = r;
        if (in) {
            if (begun) *reinterpret_cast<Pack<float, V>*>(s.head + static_cast<uint64_t>(w) * s.dim_up + col) = *reinterpret_cast<Pack<float, V>*>(sum);
            else if (ALL || any) store_row<T, V, ADD>(s.past, table + static_cast<uint64_t>(r) * s.table_stride, there, sum, s.scale);
        }
        begun = any = false;
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] = 0.0f;
    };
    const auto finish_up_to = [&](uint32_t next) {
        if (!ALL) {
            if (r != next) finish();
            r = next;
        } else
            for (; r < next; ++r) finish();
    };
    for (uint32_t j = 0; j < real; j += kSumAhead) {
        float x[kSumAhead][V];
        Pack<T, V> held[kSumAhead];   // (a row's every time, so that none is waited for at its end)
#pragma unroll
        for (int a = 0; a < kSumAhead; ++a)
            if (j + a < real) {
                const uint32_t row = __builtin_amdgcn_readlane(place, j + a), to = __builtin_amdgcn_readlane(key, j + a);
                if (in) load_up<Grad, V>(x[a], grad + static_cast<uint64_t>(row) * s.grad_stride);
                if (ADD && in) held[a] = *reinterpret_cast<const Pack<T, V>*>(table + static_cast<uint64_t>(to) * s.table_stride);
            }
#pragma unroll
        for (int a = 0; a < kSumAhead; ++a)
            if (j + a < real) {
                finish_up_to(__builtin_amdgcn_readlane(key, j + a));
                any = true;
                if (ADD && in) there = held[a];
                if (in)
#pragma unroll
                    for (int i = 0; i < V; ++i) sum[i] += x[a][i];
            }
    }
    if (ALL) finish_up_to(r_end);
    if (any) {
        if (!ALL && __builtin_amdgcn_readfirstlane(next) != r) finish();
        else if (in) *reinterpret_cast<Pack<float, V>*>(s.tail + static_cast<uint64_t>(w) * s.dim_up + col) = *reinterpret_cast<Pack<float, V>*>(sum);
    }
    if (column == 0 && lane == 0) s.joined[w] = joins;
}

// Rows that several stretches share: their sums, joined in the order of the stretches.  A wave looks at the row that ends in its
// stretch, if one does, and adds up a few parts by itself; the waves of a workgroup share the parts of longer rows.  Bound by latency: 10 us
// for a batch's gradient as above, where the most frequent token has 120 parts.  A row that most of a long list names takes longer than its
// sums: 1 Mi tokens into 131072 x 1024 762 us spread, 1526 all the same.
constexpr int kJoinThreads = 256, kJoinWaves = kJoinThreads / 64;
constexpr uint32_t kJoinAlone = 16;
template <typename T, int V, bool ADD>
__global__ __launch_bounds__(kJoinThreads) void embedding_join(const Sums s) {
    constexpr bool ALL = !ADD;
    __shared__ Pack<float, V> part[kJoinWaves][64];
    __shared__ uint32_t row_of[kJoinWaves], from_of[kJoinWaves];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t col = (blockIdx.y * 64 + lane) * V, w0 = block_of(blockIdx.z) * kJoinWaves;
    const bool in = col < s.dim;
    const auto add_up = [&](float (&sum)[V], uint32_t a, uint32_t b) {
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] = 0.0f;
        if (in)
#pragma unroll 8
            for (uint32_t i = a; i < b; ++i) {
                float x[V];
                load_up<float, V>(x, s.tail + static_cast<uint64_t>(i) * s.dim_up + col);
#pragma unroll
                for (int v = 0; v < V; ++v) sum[v] += x[v];
            }
    };
    const auto finish = [&](float (&sum)[V], uint32_t w, uint32_t r) {
        if (!in) return;
        float x[V];
        load_up<float, V>(x, s.head + static_cast<uint64_t>(w) * s.dim_up + col);
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] += x[v];
        T* const to = static_cast<T*>(s.table) + static_cast<uint64_t>(r) * s.table_stride + col;
        Pack<T, V> there;
        if (ADD) there = *reinterpret_cast<const Pack<T, V>*>(to);
        store_row<T, V, ADD>(s.past, to, there, sum, s.scale);
    };
    float sum[V];
    uint32_t r = w0 + wave < s.stretches ? __builtin_amdgcn_readfirstlane(s.joined[w0 + wave]) : kNoRow, from = 0;
    if (r != kNoRow) {
        const uint32_t first = search(s.n, [&](uint64_t j) { return s.keys[j] < r; });
        from = static_cast<uint32_t>((static_cast<uint64_t>(first) + (ALL ? r : 0)) / s.stretch);
        if (w0 + wave - from <= kJoinAlone) {
            add_up(sum, from, w0 + wave);
            finish(sum, w0 + wave, r);
            r = kNoRow;
        }
    }
    if (lane == 0) {
        row_of[wave] = r;
        from_of[wave] = from;
    }
    __syncthreads();
    for (int q = 0; q < kJoinWaves; ++q) {
        const uint32_t row = row_of[q], begin = from_of[q], many = w0 + q - begin, each = (many + kJoinWaves - 1) / kJoinWaves;
        if (row == kNoRow) continue;
        add_up(sum, begin + min(many, wave * each), begin + min(many, (wave + 1) * each));
#pragma unroll
        for (int v = 0; v < V; ++v) part[wave][lane].v[v] = sum[v];
        __syncthreads();
        if (wave == 0) {
            for (int o = 1; o < kJoinWaves; ++o)
#pragma unroll
                for (int v = 0; v < V; ++v) sum[v] += part[o][lane].v[v];
            finish(sum, w0 + q, row);
        }
        __syncthreads();
    }
}

// ---- host side ----------------------------------------------------------------------------------------------------------------
// What the sort and the sums need of a call, by its sizes alone.
struct GradientPlan {
    int bits = 0, passes = 0;
    uint32_t chunk = 0, chunks = 0, stretch = 0, stretches_all = 0, stretches_add = 0, dim_up = 0;
    size_t bytes = 0;
    uint32_t *key[2], *place[2], *counts;
    float *head, *tail;
    uint32_t* joined;
};

GradientPlan plan_gradient(size_t n, size_t vocab, size_t dim, void* workspace) {
    GradientPlan g;
    int all = 1;   // keys are 0 ... vocab, the last for padding
    while (vocab >> all) ++all;
    g.passes = (all + kDigitBits - 1) / kDigitBits;
    g.bits = (all + g.passes - 1) / g.passes;
    g.chunk = static_cast<uint32_t>(ceil_div(ceil_div(n, kMostChunks), kTile) * kTile);
    g.chunks = n <= kOneMost ? 1 : static_cast<uint32_t>(ceil_div(n, g.chunk));
    g.dim_up = static_cast<uint32_t>((dim + 7) / 8 * 8);
    // 32 places to a stretch (65536 tokens, 131072 x 1024 rows: 16 151 us, 32 153, 64 161, 128 165); fewer where that leaves the GPU
    // without waves, at least 8 (below that the joining costs more)
    const uint64_t columns = ceil_div(dim, 256);
    g.stretch = static_cast<uint32_t>(std::min<uint64_t>(32, std::max<uint64_t>(8, (n + vocab) * columns / 8192)));
    g.stretches_all = static_cast<uint32_t>(ceil_div(n + vocab, g.stretch));
    g.stretches_add = static_cast<uint32_t>(ceil_div(n, g.stretch));
    Carve c(workspace);
    for (int i = 0; i < 2; ++i) {
        g.key[i] = c.take<uint32_t>(n);
        g.place[i] = c.take<uint32_t>(n);
    }
    g.counts = c.take<uint32_t>(g.chunks > 1 ? static_cast<size_t>(g.chunks) << g.bits : 0);
    // only stretches that a token's position lies in have such rows, but any may
    const size_t rows = n > 0 ? static_cast<size_t>(g.stretches_all) * g.dim_up : 0;
    g.head = c.take<float>(rows);
    g.tail = c.take<float>(rows);
    g.joined = c.take<uint32_t>(g.stretches_all);
    g.bytes = c.at;
    return g;
}

template <typename Token>
blink_status_t sort_tokens(const Token* tokens, uint32_t n, uint32_t vocab, const GradientPlan& g, hipStream_t stream, int* where) {
    if (n <= kOneMost) {
        *where = 0;
        if (n <= kFewMost)
            return launch(embedding_sort_few<Token>, dim3(static_cast<uint32_t>(ceil_div(n, 64))), dim3(kFewThreads), stream, tokens, n, vocab, g.key[0], g.place[0]);
        return launch(embedding_sort_one<Token>, dim3(1), dim3(kOneThreads), stream, tokens, n, vocab, g.bits, g.passes, g.key[0], g.place[0]);
    }
    for (int pass = 0; pass < g.passes; ++pass) {
        const Token* const from = pass == 0 ? tokens : nullptr;
        const int shift = pass * g.bits, in = (pass + 1) & 1, out = pass & 1;
        BLINK_TRY(launch(embedding_sort_count<Token>, dim3(g.chunks), dim3(kTileThreads), stream, from, g.key[in], n, vocab, g.chunk, shift, g.bits, g.counts));
        BLINK_TRY(launch(embedding_sort_move<Token>, dim3(g.chunks), dim3(kTileThreads), stream, from, g.key[in], g.place[in], n, vocab, g.chunk, shift, g.bits,
                         g.counts, g.key[out], g.place[out]));
        *where = out;
    }
    return BLINK_OK;
}

template <typename Grad, typename T, int V>
blink_status_t run_sums(Sums s, bool add, hipStream_t stream) {
    s.columns = static_cast<uint32_t>(ceil_div(s.dim, 64 * V));
    const uint64_t groups = ceil_div(static_cast<uint64_t>(s.stretches) * s.columns, kSumThreads / 64);
    if (groups > 0x3fffff00) return BLINK_EINVAL;   // (the waves' numbers have 32 bits)
    const Grid grid = grid_of(groups, kSumThreads);
    BLINK_TRY(launch(add ? embedding_sums<Grad, T, V, true> : embedding_sums<Grad, T, V, false>, dim3(grid.x, grid.y), dim3(kSumThreads), stream, s));
    // no row lies in two stretches: one position alone has one place, but next to that a row's end has one of its own where all rows are written
    if (s.n < (add ? 2u : 1u) || s.stretches < 2) return BLINK_OK;
    const Grid join = grid_of(ceil_div(s.stretches, kJoinWaves), kJoinThreads);
    return launch(add ? embedding_join<T, V, true> : embedding_join<T, V, false>, dim3(join.x, s.columns, join.y), dim3(kJoinThreads), stream, s);
}

}  // namespace

size_t embedding_gradient_workspace(size_t n, size_t vocab, size_t dim) { return plan_gradient(n, vocab, dim, nullptr).bytes; }

blink_status_t embedding(const void* table, blink_dtype_t table_type, size_t vocab, size_t dim, size_t table_stride, const void* tokens,
                         blink_dtype_t token_type, size_t n, float scale, void* out, blink_dtype_t out_type, size_t out_stride, hipStream_t stream) {
    if (n == 0 || dim == 0) return BLINK_OK;
    return with_float(table_type, [&](auto in) {
        return with_float(out_type, [&](auto to) -> blink_status_t {
            using In = decltype(in);
            using Out = decltype(to);
            constexpr int kMost = 16 / static_cast<int>(sizeof(In) > sizeof(Out) ? sizeof(In) : sizeof(Out));
            const auto fits = [&](size_t v) {
                return dim % v == 0 && table_stride % v == 0 && out_stride % v == 0 && aligned(table, v * sizeof(In)) && aligned(out, v * sizeof(Out));
            };
            const int v = fits(kMost) ? kMost : 1;
            const uint64_t packs = dim / v, units = n * packs, blocks = ceil_div(units, kRowThreads * kRowUnits);
            if (blocks > 0xfffff000) return BLINK_EINVAL;   // (2^41 elements at the least)
            const Grid grid = grid_of(blocks, kRowThreads);
            const auto with_token = [&](auto token) {
                using Token = decltype(token);
                const auto go = [&](auto kernel) {
                    return launch(kernel, dim3(grid.x, grid.y), dim3(kRowThreads), stream, static_cast<const In*>(table), vocab, table_stride,
                                  static_cast<const Token*>(tokens), units, static_cast<uint32_t>(packs), scale, static_cast<Out*>(out), out_stride,
                                  passes_caches(n * dim * sizeof(Out)));
                };
                if (blocks * kRowThreads * kRowUnits >> 32)
                    return v == kMost ? go(embedding_rows<In, Out, Token, uint64_t, kMost>) : go(embedding_rows<In, Out, Token, uint64_t, 1>);
                return v == kMost ? go(embedding_rows<In, Out, Token, uint32_t, kMost>) : go(embedding_rows<In, Out, Token, uint32_t, 1>);
            };
            return token_type == BLINK_INT64 ? with_token(int64_t()) : with_token(int32_t());
        });
    });
}

blink_status_t embedding_gradient(const void* tokens, blink_dtype_t token_type, size_t n, const void* grad, blink_dtype_t grad_type,
                                  size_t grad_stride, float scale, bool accumulate, void* table, blink_dtype_t table_type, size_t vocab, size_t dim,
                                  size_t table_stride, void* workspace, hipStream_t stream) {
    if (vocab == 0 || dim == 0 || (n == 0 && accumulate)) return BLINK_OK;
    const GradientPlan g = plan_gradient(n, vocab, dim, workspace);
    int where = 0;
    const uint32_t n32 = static_cast<uint32_t>(n), v32 = static_cast<uint32_t>(vocab);
    if (n > 0) {
        BLINK_TRY(token_type == BLINK_INT64 ? sort_tokens(static_cast<const int64_t*>(tokens), n32, v32, g, stream, &where)
                                            : sort_tokens(static_cast<const int32_t*>(tokens), n32, v32, g, stream, &where));
    }
    Sums s;
    s.grad = grad;
    s.grad_stride = grad_stride;
    s.keys = g.key[where];
    s.places = g.place[where];
    s.n = n32;
    s.vocab = v32;
    s.dim = static_cast<uint32_t>(dim);
    s.scale = scale;
    s.table = table;
    s.table_stride = table_stride;
    s.stretch = g.stretch;
    s.stretches = accumulate ? g.stretches_add : g.stretches_all;
    s.head = g.head;
    s.tail = g.tail;
    s.joined = g.joined;
    s.dim_up = g.dim_up;
    s.past = !accumulate && passes_caches(vocab * dim * size_of(table_type));
    return with_float(grad_type, [&](auto from) {
        return with_float(table_type, [&](auto to) -> blink_status_t {
            using Grad = decltype(from);
            using T = decltype(to);
            constexpr int kMost = 16 / static_cast<int>(sizeof(Grad) > sizeof(T) ? sizeof(Grad) : sizeof(T));
            const bool wide = dim % kMost == 0 && grad_stride % kMost == 0 && table_stride % kMost == 0 && aligned(grad, kMost * sizeof(Grad)) &&
                              aligned(table, kMost * sizeof(T));
            return wide ? run_sums<Grad, T, kMost>(s, accumulate, stream) : run_sums<Grad, T, 1>(s, accumulate, stream);
        });
    });
}

}  // namespace blink
