// gem_embed.hip -- rows of an embedding for tokens, and the embedding's gradient, for gfx950.
//
// The gradient of a table's row is the sum of the gradients of the places that its token stands
// at.  Places are sorted by token (stably, so that every sum has one order, whatever runs
// first), and each row is then summed and written by its own lanes: the table's gradient is written
// once, the places' read once, no atomics.  Bytes bound both.  A token that stands at many places (in
// language the likeliest makes up a tenth) is summed in chunks of the sorted places first.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gem_ops.hpp"
#include "gem_ops_device.hpp"

namespace gemk {
namespace {

constexpr int kThreads = 256;
constexpr int kCols = 4;                   // columns of a lane: 16 bytes of binary32, next to its neighbours'

// ---- four elements at any address of their own alignment --------------------------------------

template <class T> struct Vec;
template <> struct Vec<float> {
    using Type = uint32_t __attribute__((ext_vector_type(4), aligned(4)));
    static __device__ __forceinline__ void widen(const Type& r, float (&v)[kCols])
    {
#pragma unroll
        for (int i = 0; i < kCols; ++i) v[i] = __uint_as_float(r[i]);
    }
    static __device__ __forceinline__ Type narrow(const float (&v)[kCols])
    {
        return Type{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    }
};
template <> struct Vec<uint16_t> {
    using Type = uint32_t __attribute__((ext_vector_type(2), aligned(2)));
    static __device__ __forceinline__ void widen(const Type& r, float (&v)[kCols])
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            v[2 * i] = __uint_as_float(r[i] << 16);
            v[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ Type narrow(const float (&v)[kCols])
    {
        return Type{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
    }
};

// A lane's columns of a row of `dim`: [c, c + kCols), of which it stores those from `from` on.  Past
// the row's end it has the last ones again, so that loads are whole and stand in no branch; FEW: the
// row has fewer than kCols.
struct Cols {
    int c, from, dim;
    Cols() = default;
    __device__ Cols(int at, int dim_) : c(at), from(at), dim(dim_)
    {
        if (c + kCols > dim) c = dim > kCols ? dim - kCols : 0;
    }
    __device__ bool any() const { return from < dim; }
};
template <class T, bool FEW> __device__ __forceinline__ typename Vec<T>::Type fetch(const T* row, const Cols& o)
{
    if constexpr (!FEW) return *reinterpret_cast<const typename Vec<T>::Type*>(row + o.c);
    typename Vec<T>::Type r{};
    T* e = reinterpret_cast<T*>(&r);
#pragma unroll
    for (int i = 0; i < kCols; ++i) e[i] = row[i < o.dim ? i : o.dim - 1];
    return r;
}
// Non-temporal: 32768 x 2048 rows looked up 48 us instead of 52, their gradient 2% less.
template <class T> __device__ __forceinline__ void put(T* row, const Cols& o, const float (&v)[kCols])
{
    if (o.from + kCols <= o.dim) {
        __builtin_nontemporal_store(Vec<T>::narrow(v), reinterpret_cast<typename Vec<T>::Type*>(row + o.c));
    } else {
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            if (o.c + i >= o.from && o.c + i < o.dim) store(row, o.c + i, v[i]);
    }
}

// ---- lanes over rows ------------------------------------------------------------------------

// Rows, or groups of them, are taken in pieces of Q x `lanes` (a power of two, at most 64) x kCols
// columns, by as many lanes.
struct Pieces {
    int lanes, of_row;
    int64_t rows;
};
__device__ __forceinline__ int64_t first_piece(const Pieces& p)
{
    return (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) / p.lanes;
}
__device__ __forceinline__ int64_t piece_step(const Pieces& p) { return static_cast<int64_t>(gridDim.x) * (kThreads / p.lanes); }
// The lane's q-th columns in a piece of Q.
template <int Q> __device__ __forceinline__ Cols piece_cols(const Pieces& p, int piece, int q, int dim)
{
    return Cols(((piece * Q + q) * p.lanes + static_cast<int>(threadIdx.x) % p.lanes) * kCols, dim);
}

// ---- forward -------------------------------------------------------------------------------

// ROWS places a piece, all in flight: many for the rate (32768 x 2048 bfloat16 of 65536 binary32 rows, tokens as
// frequent as words, 48 us, 5.6 TB/s), one where there are few places (64 x 4096 4.9 us, the launch).
template <class T, class TO, int ROWS, bool FEW>
__global__ __launch_bounds__(kThreads) void lookup_kernel(const EmbedArgs a, const Pieces p)
{
    const int64_t n = p.rows * p.of_row;
    for (int64_t i = first_piece(p); i < n; i += piece_step(p)) {
        const int64_t group = i / p.of_row, t = group * ROWS;
        const Cols o = piece_cols<1>(p, static_cast<int>(i - group * p.of_row), 0, a.e.dim);
        if (!o.any()) continue;
        int token[ROWS];
        typename Vec<T>::Type raw[ROWS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) token[u] = a.e.tokens[t + u < a.e.count ? t + u : a.e.count - 1];
#pragma unroll
        for (int u = 0; u < ROWS; ++u)         // padding: row 0, which is not used
            raw[u] = fetch<T, FEW>(static_cast<const T*>(a.e.table) + (token[u] >= 0 && token[u] < a.e.vocab ? token[u] : 0) * a.e.stride, o);
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            float v[kCols];
            Vec<T>::widen(raw[u], v);
            const bool there = token[u] >= 0 && token[u] < a.e.vocab;
#pragma unroll
            for (int k = 0; k < kCols; ++k) v[k] = there ? v[k] * a.e.scale : 0.0f;
            if (t + u < a.e.count) put(static_cast<TO*>(a.rows) + (t + u) * a.rows_stride, o, v);
        }
    }
}

// ---- places sorted by token ------------------------------------------------------------------

// A token outside the vocabulary (padding) comes last.
__device__ __forceinline__ int key_of(int token, int vocab) { return token >= 0 && token < vocab ? token : vocab; }

struct Segment {
    int lo, hi;                // a token's places among the sorted ones
};

__device__ __forceinline__ void clear(Segment* seg, int vocab)
{
    if (!seg) return;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < vocab;
         i += static_cast<int64_t>(gridDim.x) * blockDim.x)
        seg[i] = Segment{0, 0};
}

// Few places: each one's rank, by comparing it with all.  A block has 64 of them, a lane each, and
// its sixteen waves a sixteenth of all to compare with.  2047 places take 8 us and 8192, 64 M comparisons, 19.
// The gradient of n x 64 bfloat16 into 50021 rows, us, ranked and sorted: 4096 22, 29; 8192 30, 31; 12288 38, 34.
// (The blocks clear the segments too, 18 of the 20 us that one block takes for 64 places of 160000 tokens.)
constexpr int kRankMost = 8192, kRankThreads = 1024;

__global__ __launch_bounds__(kRankThreads) void rank_kernel(const int32_t* tokens, int n, int vocab, int32_t* keys, int32_t* places,
                                                            Segment* seg)
{
    constexpr int kWaves = kRankThreads / 64;
    __shared__ __align__(16) int all[kRankMost];
    __shared__ int ranks[64];
    clear(seg, vocab);
    const int padded = (n + 63) / 64 * 64;
    for (int i = threadIdx.x; i < padded; i += kRankThreads) all[i] = i < n ? key_of(tokens[i], vocab) : INT32_MAX - 1;
    if (threadIdx.x < 64) ranks[threadIdx.x] = 0;
    __syncthreads();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int b0 = blockIdx.x * 64, me = b0 + lane, key = all[me];
    const int part = (padded / 4 + kWaves - 1) / kWaves * 4;
    const int from = wave * part, to = from + part < padded ? from + part : padded;
    const int4* quads = reinterpret_cast<const int4*>(all);
    int rank = 0;
    // Ahead of it are smaller keys, and equal ones of earlier places: below the block's those are
    // the keys under key + 1, behind it those under key.
    const auto count = [&](int s, int e, int limit) {
        for (; s < e; s += 4) {
            const int4 q = quads[s / 4];
            rank += (q.x < limit) + (q.y < limit) + (q.z < limit) + (q.w < limit);
        }
    };
    const auto least = [](int x, int y) { return x < y ? x : y; };
    const auto most = [](int x, int y) { return x > y ? x : y; };
    count(from, least(to, b0), key + 1);
    for (int s = most(from, b0); s < least(to, b0 + 64); ++s) rank += all[s] < key + (s < me);
    count(most(from, b0 + 64), to, key);
    atomicAdd(&ranks[lane], rank);
    __syncthreads();
    if (wave == 0 && me < n) {
        keys[ranks[lane]] = key;
        places[ranks[lane]] = me;
    }
}

// More places: a radix sort, least digits first, of nine bits or fewer a pass.  A block has a tile
// of the places; each pass counts every tile's digits (count_kernel), and scatters behind what the
// counts say stands ahead (scatter_kernel).
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
constexpr int kSortThreads = kDigits, kSortWaves = kSortThreads / 64;
constexpr int kHeld = 4, kShare = 64 * kHeld;      // places of a lane and a wave at a time

struct Pass {
    const int32_t* keys;       // null: of the tokens
    const int32_t* places;     // null: in order
    const int32_t* tokens;
    int32_t* to_keys;
    int32_t* to_places;
    uint32_t* counts;          // [tiles][kDigits]
    int n, vocab, tile, tiles, shift, bits;

    __device__ int key(int i) const { return keys ? keys[i] : key_of(tokens[i], vocab); }
    __device__ int digit(int key) const { return key >> shift & ((1 << bits) - 1); }
};

__global__ __launch_bounds__(kSortThreads) void count_kernel(const Pass p, Segment* seg)
{
    __shared__ uint32_t counts[kDigits];
    const int tid = threadIdx.x;
    if (static_cast<int>(blockIdx.x) < p.tiles) {
        counts[tid] = 0;
        __syncthreads();
        const int64_t from = static_cast<int64_t>(blockIdx.x) * p.tile;
        const int64_t to = from + p.tile < p.n ? from + p.tile : p.n;
        for (int64_t base = from; base < to; base += kHeld * kSortThreads) {
            int key[kHeld];
#pragma unroll
            for (int u = 0; u < kHeld; ++u) {
                const int64_t i = base + u * kSortThreads + tid;
                key[u] = p.key(static_cast<int>(i < to ? i : to - 1));
            }
#pragma unroll
            for (int u = 0; u < kHeld; ++u)
                if (base + u * kSortThreads + tid < to) atomicAdd(&counts[p.digit(key[u])], 1u);
        }
        __syncthreads();
        p.counts[static_cast<int64_t>(blockIdx.x) * kDigits + tid] = counts[tid];
    }
    clear(seg, p.vocab);
}

__global__ __launch_bounds__(kSortThreads) void scatter_kernel(const Pass p)
{
    __shared__ uint32_t next[kSortWaves][kDigits];     // where each wave's next place of a digit goes
    __shared__ uint32_t waves[kSortWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tid = threadIdx.x;
    const int share = p.tile / kSortWaves;
    const int64_t from = static_cast<int64_t>(blockIdx.x) * p.tile + static_cast<int64_t>(wave) * share;
    const int64_t to = from + share < p.n ? from + share : p.n;
    int key[kHeld], place[kHeld];
    const auto hold = [&](int64_t base) {
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            const int64_t i = base + u * 64 + lane;
            const int at = static_cast<int>(i < to ? i : to - 1);
            key[u] = p.key(at);
            place[u] = p.places ? p.places[at] : at;
        }
    };
    if (from < to) hold(from);
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) next[w][tid] = 0;
    // Of the thread's digit: the places in earlier tiles, and in all.
    uint32_t before = 0, all = 0;
    const int mine = blockIdx.x;
#pragma unroll 16
    for (int t = 0; t < p.tiles; ++t) {
        const uint32_t c = p.counts[static_cast<int64_t>(t) * kDigits + tid];
        before += t < mine ? c : 0u;
        all += c;
    }
    uint32_t sum = all;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        const uint32_t add = __shfl_up(sum, s);
        sum += lane >= s ? add : 0u;
    }
    if (lane == 63) waves[wave] = sum;
    __syncthreads();
    for (int64_t base = from; base < to; base += kShare) {
        if (base > from) hold(base);
#pragma unroll
        for (int u = 0; u < kHeld; ++u)
            if (base + u * 64 + lane < to) atomicAdd(&next[wave][p.digit(key[u])], 1u);
    }
    if (share > kShare && from < to) hold(from);
    __syncthreads();
    uint32_t at = sum - all + before;
    for (int w = 0; w < wave; ++w) at += waves[w];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t c = next[w][tid];
        next[w][tid] = at;
        at += c;
    }
    __syncthreads();
    for (int64_t base = from; base < to; base += kShare) {
        if (base > from) hold(base);
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            const bool in = base + u * 64 + lane < to;
            const int digit = p.digit(key[u]);
            uint64_t same = __ballot(in);          // of the lane's digit
            for (int b = 0; b < p.bits; ++b) {
                const uint64_t set = __ballot(in && (digit >> b & 1));
                same &= digit >> b & 1 ? set : ~set;
            }
            const int first = __builtin_ctzll(same);
            uint32_t start = 0;
            if (in && lane == first) start = atomicAdd(&next[wave][digit], static_cast<uint32_t>(__builtin_popcountll(same)));
            start = __shfl(start, first);
            const uint32_t dest = start + __builtin_popcountll(same & ((uint64_t{1} << lane) - 1));
            if (in) {
                p.to_keys[dest] = key[u];
                p.to_places[dest] = place[u];
            }
        }
    }
}

// ---- sums ------------------------------------------------------------------------------------

// Chunks of kChunk sorted places that all have one token are summed ahead, and kChunk of such
// chunks again, so that a row adds fewer than 2 kChunk places, as many chunks, and chunks of chunks.
// 32768 x 2048 into 65536 rows, tokens as frequent as words: 165 us, 171 with chunks of 32.
constexpr int kChunk = 16;
constexpr int kTake = 16, kFew = 4;        // rows in flight
constexpr int kGroup = 4;                  // rows of the table that lanes take together
using Few = int32_t __attribute__((ext_vector_type(kFew), aligned(4)));

struct Sums {
    const int32_t* keys;
    const int32_t* places;
    Segment* seg;
    float* chunks;             // [n / kChunk][dim]
    float* big;                // [n / kChunk / kChunk][dim], null: not taken
    int n;
};

// v += rows [from, to) of T, in their order, TAKE in flight; row(i) is where one begins.
template <class T, bool FEW, int Q, int TAKE, class F>
__device__ __forceinline__ void add_batches(float (&v)[Q][kCols], int& i, int to, const Cols (&o)[Q], F row)
{
    for (; i + (TAKE == kFew ? 1 : TAKE) <= to; i += TAKE) {
        const T* at[TAKE];
        typename Vec<T>::Type raw[TAKE][Q];
#pragma unroll
        for (int u = 0; u < TAKE; ++u) at[u] = row(TAKE > kFew || i + u < to ? i + u : to - 1);
#pragma unroll
        for (int u = 0; u < TAKE; ++u)
#pragma unroll
            for (int q = 0; q < Q; ++q) raw[u][q] = fetch<T, FEW>(at[u], o[q]);
#pragma unroll
        for (int u = 0; u < TAKE; ++u)
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                float x[kCols];
                Vec<T>::widen(raw[u][q], x);
#pragma unroll
                for (int k = 0; k < kCols; ++k) v[q][k] += TAKE > kFew || i + u < to ? x[k] : 0.0f;
            }
    }
}
// The last few with the very last again where there are fewer than kFew.
template <class T, bool FEW, int Q, class F>
__device__ __forceinline__ void add_rows(float (&v)[Q][kCols], int from, int to, const Cols (&o)[Q], F row)
{
    if constexpr (Q == 1) add_batches<T, FEW, Q, kTake>(v, from, to, o, row);
    add_batches<T, FEW, Q, kFew>(v, from, to, o, row);
}

template <class T, bool FEW>
__global__ __launch_bounds__(kThreads) void chunk_kernel(const EmbedArgs a, const Pieces p, const Sums s)
{
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < s.n; i += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int key = s.keys[i];
        if (key >= a.e.vocab) continue;
        if (i == 0 || s.keys[i - 1] != key) s.seg[key].lo = static_cast<int>(i);
        if (i == s.n - 1 || s.keys[i + 1] != key) s.seg[key].hi = static_cast<int>(i) + 1;
    }
    const int64_t n = p.rows * p.of_row;
    for (int64_t i = first_piece(p); i < n; i += piece_step(p)) {
        const int c = static_cast<int>(i / p.of_row);
        const Cols o[1] = {piece_cols<1>(p, static_cast<int>(i - static_cast<int64_t>(c) * p.of_row), 0, a.e.dim)};
        const int from = c * kChunk, key = s.keys[from], last = s.keys[from + kChunk - 1];
        if (!o[0].any() || key >= a.e.vocab || last != key) continue;
        float v[1][kCols] = {};
        add_rows<T, FEW>(v, from, from + kChunk, o,
                         [&](int j) { return static_cast<const T*>(a.rows) + s.places[j] * a.rows_stride; });
        put(s.chunks + static_cast<int64_t>(c) * a.e.dim, o[0], v[0]);
    }
}

template <bool FEW>
__global__ __launch_bounds__(kThreads) void big_chunk_kernel(const EmbedArgs a, const Pieces p, const Sums s)
{
    const int64_t n = p.rows * p.of_row;
    for (int64_t i = first_piece(p); i < n; i += piece_step(p)) {
        const int c = static_cast<int>(i / p.of_row);
        const Cols o[1] = {piece_cols<1>(p, static_cast<int>(i - static_cast<int64_t>(c) * p.of_row), 0, a.e.dim)};
        const int from = c * kChunk * kChunk, key = s.keys[from], last = s.keys[from + kChunk * kChunk - 1];
        if (!o[0].any() || key >= a.e.vocab || last != key) continue;
        float v[1][kCols] = {};
        add_rows<float, FEW>(v, c * kChunk, (c + 1) * kChunk, o,
                             [&](int j) { return s.chunks + static_cast<int64_t>(j) * a.e.dim; });
        put(s.big + static_cast<int64_t>(c) * a.e.dim, o[0], v[0]);
    }
}

// A token's whole chunks [c0, c1); none if c0 >= c1.
struct Whole {
    int c0, c1;
    __device__ explicit Whole(const Segment& g) : c0((g.lo + kChunk - 1) / kChunk), c1(g.hi / kChunk) {}
    __device__ bool any() const { return c0 < c1; }
};

// v += the sorted places of a token with whole chunks, in their order.
template <class T, bool FEW>
__device__ __forceinline__ void add_long(float (&v)[1][kCols], const EmbedArgs& a, const Sums& s, const Segment& g, const Cols (&o)[1])
{
    const auto place = [&](int j) { return static_cast<const T*>(a.rows) + s.places[j] * a.rows_stride; };
    const auto chunk = [&](int j) { return s.chunks + static_cast<int64_t>(j) * a.e.dim; };
    const Whole w(g);
    const int b0 = (w.c0 + kChunk - 1) / kChunk, b1 = w.c1 / kChunk;
    const bool big = s.big && b0 < b1;
    add_rows<T, FEW>(v, g.lo, w.c0 * kChunk, o, place);
    add_rows<float, FEW>(v, w.c0, big ? b0 * kChunk : w.c1, o, chunk);
    if (big) {
        add_rows<float, FEW>(v, b0, b1, o, [&](int j) { return s.big + static_cast<int64_t>(j) * a.e.dim; });
        add_rows<float, FEW>(v, b1 * kChunk, w.c1, o, chunk);
    }
    add_rows<T, FEW>(v, w.c1 * kChunk, g.hi, o, place);
}

template <class TG, bool FEW, bool ADD, int Q>
__device__ __forceinline__ void write(TG* to, const Cols (&o)[Q], float (&v)[Q][kCols], float scale)
{
    float x[Q][kCols] = {};
    if constexpr (ADD) {
#pragma unroll
        for (int q = 0; q < Q; ++q) Vec<TG>::widen(fetch<TG, FEW>(to, o[q]), x[q]);
    }
#pragma unroll
    for (int q = 0; q < Q; ++q) {
#pragma unroll
        for (int k = 0; k < kCols; ++k) v[q][k] = v[q][k] * scale + x[q][k];
        put(to, o[q], v[q]);
    }
}

// The first `ahead` blocks: rows of tokens with whole chunks, each by the lanes that find the first
// of them.  The others: all rows, or (ADD: added to what is there) those of tokens that occur, each
// of which goes to the first of its sorted places.  kGroup rows are taken by the same lanes, and
// the zeros of tokens that do not occur, which are most, are on their way before the first sum.
// 32768 x 2048 bfloat16 into 65536 binary32 rows 124 us (5.0 TB/s); writing zeros alone takes 98.
template <class T, class TG, bool FEW, bool ADD, int Q>
__global__ __launch_bounds__(kThreads) void rows_kernel(const EmbedArgs a, const Pieces p, const Pieces ahead, int blocks_ahead, const Sums s)
{
    if (static_cast<int>(blockIdx.x) < blocks_ahead) {
        const int64_t n = ahead.rows * ahead.of_row, step = static_cast<int64_t>(blocks_ahead) * (kThreads / ahead.lanes);
        for (int64_t i = first_piece(ahead); i < n; i += step) {
            const int c = static_cast<int>(i / ahead.of_row);
            const Cols o[1] = {piece_cols<1>(ahead, static_cast<int>(i - static_cast<int64_t>(c) * ahead.of_row), 0, a.e.dim)};
            const int from = c * kChunk, key = s.keys[from], last = s.keys[from + kChunk - 1];
            if (!o[0].any() || key >= a.e.vocab || last != key) continue;
            const Segment g = s.seg[key];
            if (Whole(g).c0 != c) continue;
            float v[1][kCols] = {};
            add_long<T, FEW>(v, a, s, g, o);
            write<TG, FEW, ADD>(static_cast<TG*>(a.grad) + key * a.grad_stride, o, v, a.e.scale);
        }
        return;
    }
    const int64_t n = p.rows * p.of_row, behind = static_cast<int64_t>(blocks_ahead) * (kThreads / p.lanes);
    for (int64_t i = first_piece(p) - behind; i < n; i += piece_step(p) - behind) {
        const int64_t group = i / p.of_row;
        Cols o[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) o[q] = piece_cols<Q>(p, static_cast<int>(i - group * p.of_row), q, a.e.dim);
        const int64_t rows = ADD ? s.n : a.e.vocab;
        Segment g[kGroup];
        int token[kGroup];
#pragma unroll
        for (int u = 0; u < kGroup; ++u) {
            const int64_t at = group * kGroup + u;
            g[u] = Segment{0, 0};
            token[u] = static_cast<int>(at);
            if (at >= rows || !s.n) continue;
            if (ADD) {
                token[u] = s.keys[at];
                if (token[u] >= a.e.vocab || (at > 0 && s.keys[at - 1] == token[u])) continue;
            }
            g[u] = s.seg[token[u]];
        }
        // The first places of each row, on their way together.
        Few places[kGroup];
#pragma unroll
        for (int u = 0; u < kGroup; ++u)
            if (s.n) places[u] = *reinterpret_cast<const Few*>(s.places + g[u].lo);
        const float none[kCols] = {};
#pragma unroll
        for (int u = 0; u < kGroup; ++u)
            if (!ADD && group * kGroup + u < rows && g[u].hi == g[u].lo) {
#pragma unroll
                for (int q = 0; q < Q; ++q) put(static_cast<TG*>(a.grad) + token[u] * a.grad_stride, o[q], none);
            }
        const auto place = [&](int j) { return static_cast<const T*>(a.rows) + s.places[j] * a.rows_stride; };
#pragma unroll
        for (int u = 0; u < kGroup; ++u) {
            if (g[u].hi == g[u].lo || Whole(g[u]).any()) continue;
            float v[Q][kCols] = {};
            // The last again where there are fewer than kFew.
            const int m = g[u].hi - g[u].lo;
            const T* at[kFew];
#pragma unroll
            for (int i = 0; i < kFew; ++i) at[i] = static_cast<const T*>(a.rows) + (i < m ? places[u][i] : places[u][0]) * a.rows_stride;
            typename Vec<T>::Type raw[kFew][Q];
#pragma unroll
            for (int i = 0; i < kFew; ++i)
#pragma unroll
                for (int q = 0; q < Q; ++q) raw[i][q] = fetch<T, FEW>(at[i], o[q]);
#pragma unroll
            for (int i = 0; i < kFew; ++i)
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    float x[kCols];
                    Vec<T>::widen(raw[i][q], x);
#pragma unroll
                    for (int k = 0; k < kCols; ++k) v[q][k] += i < m ? x[k] : 0.0f;
                }
            add_rows<T, FEW>(v, g[u].lo + kFew, g[u].hi, o, place);
            write<TG, FEW, ADD>(static_cast<TG*>(a.grad) + token[u] * a.grad_stride, o, v, a.e.scale);
        }
    }
}

// ---- launches -------------------------------------------------------------------------------

int64_t over(int64_t n, int64_t part) { return (n + part - 1) / part; }

Pieces pieces_of(int64_t rows, int dim, int quads = 1)
{
    Pieces p;
    p.lanes = 1;
    while (p.lanes < 64 && p.lanes * kCols < dim) p.lanes *= 2;
    p.of_row = static_cast<int>(over(dim, quads * p.lanes * kCols));
    p.rows = rows;
    return p;
}
// Blocks that loop over what is left.
constexpr int64_t kBlocksMost = int64_t{1} << 20;
dim3 grid_of(const Pieces& p)
{
    const int64_t blocks = over(p.rows * p.of_row, kThreads / p.lanes);
    return dim3(static_cast<unsigned>(blocks < 1 ? 1 : blocks < kBlocksMost ? blocks : kBlocksMost));
}

int bits_of(int vocab)         // of keys up to vocab
{
    int b = 1;
    while (vocab >> b) ++b;
    return b;
}

// Places of a block in a pass of the sort: no more tiles than kTilesMost, since every block reads
// all tiles' counts.
constexpr int64_t kTileLeast = kSortWaves * kShare, kTilesMost = 512;
int64_t tile_of(int64_t n) { return over(over(n, kTilesMost) + (n == 0), kTileLeast) * kTileLeast; }

// The parts of the scratch, in this order: two sorts' keys and places, counts, segments, chunks.
struct Layout {
    int64_t order, counts, seg, chunks, big, bytes;

    Layout(int64_t n, int64_t vocab, int64_t dim)
    {
        const auto up = [](int64_t b) { return over(b, 256) * 256; };
        order = up((n + kFew) * 4);            // a row's first places are read as kFew
        counts = 4 * order;
        const int64_t tiles = over(n, kTileLeast);
        seg = counts + up((tiles < kTilesMost ? tiles : kTilesMost) * kDigits * 4);
        chunks = seg + up(vocab * static_cast<int64_t>(sizeof(Segment)));
        big = chunks + up(n / kChunk * dim * 4);
        bytes = big + up(n / kChunk / kChunk * dim * 4);
        if (n == 0) bytes = 0;
    }
};

// From this many places on chunks of chunks are worth a launch: n x 1024 bfloat16 into 32768 rows, tokens as frequent as
// words, us, with them and without: 8192 56, 53; 16384 64, 60; 32768 64, 65; 131072 124, 136.
constexpr int kBigLeast = 1 << 14;

template <class T, class TO, bool FEW> hipError_t forward(const EmbedArgs& a, hipStream_t stream)
{
    constexpr int ROWS = 4;
    const Pieces each = pieces_of(a.e.count, a.e.dim), p = pieces_of(over(a.e.count, ROWS), a.e.dim);
    // Enough pieces of several rows for four waves a SIMD.
    if (p.rows * p.of_row * p.lanes >= int64_t{64} * 4096)
        hipLaunchKernelGGL((lookup_kernel<T, TO, ROWS, FEW>), grid_of(p), dim3(kThreads), 0, stream, a, p);
    else
        hipLaunchKernelGGL((lookup_kernel<T, TO, 1, FEW>), grid_of(each), dim3(kThreads), 0, stream, a, each);
    return hipGetLastError();
}

// Leaves the sorted keys and places in s.
void sort(const EmbedArgs& a, const Layout& l, char* scratch, Sums& s, hipStream_t stream)
{
    int32_t* order[4];
    for (int i = 0; i < 4; ++i) order[i] = reinterpret_cast<int32_t*>(scratch + i * l.order);
    Segment* seg = a.add ? nullptr : s.seg;
    s.keys = order[0];
    s.places = order[1];
    if (s.n <= kRankMost) {
        const unsigned blocks = static_cast<unsigned>(over(s.n, 64));
        hipLaunchKernelGGL(rank_kernel, dim3(blocks), dim3(kRankThreads), 0, stream, a.e.tokens, s.n, a.e.vocab, order[0], order[1], seg);
        return;
    }
    Pass p{};
    p.tokens = a.e.tokens;
    p.counts = reinterpret_cast<uint32_t*>(scratch + l.counts);
    p.n = s.n;
    p.vocab = a.e.vocab;
    p.tile = static_cast<int>(tile_of(s.n));
    p.tiles = static_cast<int>(over(s.n, p.tile));
    const int bits = bits_of(a.e.vocab), passes = static_cast<int>(over(bits, kDigitBits));
    for (int i = 0, at = 0; i < passes; ++i, at ^= 1) {
        p.bits = static_cast<int>(over(bits - p.shift, passes - i));
        p.to_keys = order[2 * at];
        p.to_places = order[2 * at + 1];
        const int64_t clears = i == 0 && seg ? over(a.e.vocab, kSortThreads) : 0;
        hipLaunchKernelGGL(count_kernel, dim3(static_cast<unsigned>(clears > p.tiles ? clears : p.tiles)), dim3(kSortThreads), 0,
                           stream, p, i == 0 ? seg : nullptr);
        hipLaunchKernelGGL(scatter_kernel, dim3(static_cast<unsigned>(p.tiles)), dim3(kSortThreads), 0, stream, p);
        p.shift += p.bits;
        p.keys = s.keys = p.to_keys;
        p.places = s.places = p.to_places;
    }
}

template <class T, class TG, bool FEW, bool ADD, int Q>
void rows(const EmbedArgs& a, const Sums& s, hipStream_t stream)
{
    const Pieces p = pieces_of(over(ADD ? s.n : a.e.vocab, kGroup), a.e.dim, Q), ahead = pieces_of(s.n / kChunk, a.e.dim);
    const unsigned first = ahead.rows ? grid_of(ahead).x : 0;
    hipLaunchKernelGGL((rows_kernel<T, TG, FEW, ADD, Q>), dim3(grid_of(p).x + first), dim3(kThreads), 0, stream, a, p, ahead,
                       static_cast<int>(first), s);
}

template <class T, class TG, bool FEW> hipError_t backward(const EmbedArgs& a, const OpsDevice& d, hipStream_t stream)
{
    const Layout l(a.e.count, a.e.vocab, a.e.dim);
    char* scratch = static_cast<char*>(d.scan);
    Sums s{};
    s.n = static_cast<int>(a.e.count);
    if (s.n > 0) {
        s.seg = reinterpret_cast<Segment*>(scratch + l.seg);
        s.chunks = reinterpret_cast<float*>(scratch + l.chunks);
        sort(a, l, scratch, s, stream);
        const Pieces chunks = pieces_of(s.n / kChunk, a.e.dim);
        const int64_t places = over(s.n, kThreads), blocks = grid_of(chunks).x;
        hipLaunchKernelGGL((chunk_kernel<T, FEW>), dim3(static_cast<unsigned>(blocks > places ? blocks : places)), dim3(kThreads), 0,
                           stream, a, chunks, s);
        if (s.n >= kBigLeast) {
            s.big = reinterpret_cast<float*>(scratch + l.big);
            const Pieces big = pieces_of(s.n / kChunk / kChunk, a.e.dim);
            hipLaunchKernelGGL((big_chunk_kernel<FEW>), grid_of(big), dim3(kThreads), 0, stream, a, big, s);
        }
    } else if (a.add) {
        return hipSuccess;
    }
    constexpr int Q = FEW ? 1 : 4;
    if (FEW || a.e.dim <= 64 * kCols) {
        if (a.add) rows<T, TG, FEW, true, 1>(a, s, stream);
        else rows<T, TG, FEW, false, 1>(a, s, stream);
    } else {
        if (a.add) rows<T, TG, FEW, true, Q>(a, s, stream);
        else rows<T, TG, FEW, false, Q>(a, s, stream);
    }
    return hipGetLastError();
}

template <class T, class TR> hipError_t forward_of(const EmbedArgs& a, hipStream_t stream)
{
    return a.e.dim < kCols ? forward<T, TR, true>(a, stream) : forward<T, TR, false>(a, stream);
}
template <class T, class TR> hipError_t backward_of(const EmbedArgs& a, const OpsDevice& d, hipStream_t stream)
{
    return a.e.dim < kCols ? backward<TR, T, true>(a, d, stream) : backward<TR, T, false>(a, d, stream);
}

}  // namespace

int64_t embed_scratch_bytes(int64_t count, int64_t vocab, int64_t dim) { return Layout(count, vocab, dim).bytes; }

hipError_t launch_embed_forward(const EmbedArgs& a, bool bf16, bool rows_bf16, hipStream_t stream)
{
    if (rows_bf16) return bf16 ? forward_of<uint16_t, uint16_t>(a, stream) : forward_of<float, uint16_t>(a, stream);
    return bf16 ? forward_of<uint16_t, float>(a, stream) : forward_of<float, float>(a, stream);
}

hipError_t launch_embed_backward(const EmbedArgs& a, bool bf16, bool rows_bf16, const OpsDevice& d, hipStream_t stream)
{
    if (rows_bf16) return bf16 ? backward_of<uint16_t, uint16_t>(a, d, stream) : backward_of<float, uint16_t>(a, d, stream);
    return bf16 ? backward_of<uint16_t, float>(a, d, stream) : backward_of<float, float>(a, d, stream);
}

}  // namespace gemk
