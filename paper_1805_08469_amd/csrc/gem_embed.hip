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
constexpr int kCols = 8;                   // columns of a lane

// ---- eight elements at any address of their own alignment ------------------------------------

template <class T> using Raw = uint32_t __attribute__((ext_vector_type(4), aligned(sizeof(T))));

__device__ __forceinline__ void load8(const float* p, float (&v)[kCols])
{
    const Raw<float> a = reinterpret_cast<const Raw<float>*>(p)[0], b = reinterpret_cast<const Raw<float>*>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = __uint_as_float(a[i]);
        v[4 + i] = __uint_as_float(b[i]);
    }
}
__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[kCols])
{
    const Raw<uint16_t> a = *reinterpret_cast<const Raw<uint16_t>*>(p);
    unpack(u32x4{a[0], a[1], a[2], a[3]}, v);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[kCols])
{
#pragma unroll
    for (int h = 0; h < 2; ++h)
        reinterpret_cast<Raw<float>*>(p)[h] = Raw<float>{__float_as_uint(v[4 * h]), __float_as_uint(v[4 * h + 1]),
                                                         __float_as_uint(v[4 * h + 2]), __float_as_uint(v[4 * h + 3])};
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[kCols])
{
    const u32x4 r = pack(v);
    *reinterpret_cast<Raw<uint16_t>*>(p) = Raw<uint16_t>{r[0], r[1], r[2], r[3]};
}
// The first n of them.
template <class T> __device__ __forceinline__ void fetch(const T* p, int n, float (&v)[kCols])
{
    if (n >= kCols) {
        load8(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < kCols; ++i) v[i] = i < n ? load(p, i) : 0.0f;
    }
}
template <class T> __device__ __forceinline__ void put(T* p, int n, const float (&v)[kCols])
{
    if (n >= kCols) {
        store8(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            if (i < n) store(p, i, v[i]);
    }
}

// ---- lanes over rows ------------------------------------------------------------------------

// Rows are taken in pieces of `lanes` (a power of two, at most 64) x 8 columns, by as many lanes.
struct Pieces {
    int lanes, of_row;
    int64_t rows;
};
__device__ __forceinline__ int64_t first_piece(const Pieces& p)
{
    return (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) / p.lanes;
}
__device__ __forceinline__ int64_t piece_step(const Pieces& p) { return static_cast<int64_t>(gridDim.x) * (kThreads / p.lanes); }
__device__ __forceinline__ int piece_col(const Pieces& p, int piece) { return (piece * p.lanes + static_cast<int>(threadIdx.x) % p.lanes) * kCols; }

// ---- forward -------------------------------------------------------------------------------

template <class T, class TO>
__global__ __launch_bounds__(kThreads) void lookup_kernel(const EmbedArgs a, const Pieces p)
{
    const int64_t n = p.rows * p.of_row;
    for (int64_t i = first_piece(p); i < n; i += piece_step(p)) {
        const int64_t t = i / p.of_row;
        const int col = piece_col(p, static_cast<int>(i - t * p.of_row)), left = a.e.dim - col;
        if (left <= 0) continue;
        const int token = a.e.tokens[t];
        float v[kCols] = {};
        if (token >= 0 && token < a.e.vocab) {
            fetch(static_cast<const T*>(a.e.table) + token * a.e.stride + col, left, v);
#pragma unroll
            for (int k = 0; k < kCols; ++k) v[k] *= a.e.scale;
        }
        put(static_cast<TO*>(a.rows) + t * a.rows_stride + col, left, v);
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
// its sixteen waves a sixteenth of all to compare with.  8192 places: 64 M comparisons.
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
constexpr int kSortWaves = kThreads / 64;

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

__global__ __launch_bounds__(kThreads) void count_kernel(const Pass p, Segment* seg)
{
    __shared__ uint32_t counts[kDigits];
    clear(seg, p.vocab);
    for (int d = threadIdx.x; d < kDigits; d += kThreads) counts[d] = 0;
    __syncthreads();
    if (static_cast<int>(blockIdx.x) >= p.tiles) return;
    const int64_t from = static_cast<int64_t>(blockIdx.x) * p.tile;
    const int to = from + p.tile < p.n ? static_cast<int>(from + p.tile) : p.n;
    for (int64_t i = from + threadIdx.x; i < to; i += kThreads) atomicAdd(&counts[p.digit(p.key(static_cast<int>(i)))], 1u);
    __syncthreads();
    for (int d = threadIdx.x; d < kDigits; d += kThreads) p.counts[blockIdx.x * kDigits + d] = counts[d];
}

__global__ __launch_bounds__(kThreads) void scatter_kernel(const Pass p)
{
    __shared__ uint32_t next[kSortWaves][kDigits];     // where each wave's next place of a digit goes
    __shared__ uint32_t totals[kThreads];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tid = threadIdx.x;
    const int share = p.tile / kSortWaves;
    const int64_t from = static_cast<int64_t>(blockIdx.x) * p.tile + static_cast<int64_t>(wave) * share;
    const int to = from + share < p.n ? static_cast<int>(from + share) : p.n;
    for (int i = tid; i < kSortWaves * kDigits; i += kThreads) next[i / kDigits][i % kDigits] = 0;
    __syncthreads();
    for (int64_t i = from + lane; i < to; i += 64) atomicAdd(&next[wave][p.digit(p.key(static_cast<int>(i)))], 1u);
    // Of a thread's two digits: the places in earlier tiles, and in all.
    uint32_t before[2] = {}, all[2] = {};
    const uint2* rows = reinterpret_cast<const uint2*>(p.counts) + tid;
    const int mine = blockIdx.x;
#pragma unroll 8
    for (int t = 0; t < p.tiles; ++t) {
        const uint2 c = rows[static_cast<int64_t>(t) * (kDigits / 2)];
        before[0] += t < mine ? c.x : 0u;
        before[1] += t < mine ? c.y : 0u;
        all[0] += c.x;
        all[1] += c.y;
    }
    totals[tid] = all[0] + all[1];
    __syncthreads();
    for (int s = 1; s < kThreads; s *= 2) {
        const uint32_t add = tid >= s ? totals[tid - s] : 0u;
        __syncthreads();
        totals[tid] += add;
        __syncthreads();
    }
    uint32_t at = totals[tid] - all[0] - all[1];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        uint32_t base = at + before[k];
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = next[w][2 * tid + k];
            next[w][2 * tid + k] = base;
            base += c;
        }
        at += all[k];
    }
    __syncthreads();
    for (int64_t base = from; base < to; base += 64) {
        const int64_t i = base + lane;
        const bool in = i < to;
        const int key = in ? p.key(static_cast<int>(i)) : 0, digit = p.digit(key);
        uint64_t same = __ballot(in);
        for (int b = 0; b < p.bits; ++b) {
            const uint64_t set = __ballot(in && (digit >> b & 1));
            same &= digit >> b & 1 ? set : ~set;
        }
        if (!in) continue;
        const int first = __builtin_ctzll(same);
        uint32_t start = 0;
        if (lane == first) start = atomicAdd(&next[wave][digit], static_cast<uint32_t>(__builtin_popcountll(same)));
        start = __shfl(start, first);
        const uint32_t dest = start + __builtin_popcountll(same & ((uint64_t{1} << lane) - 1));
        p.to_keys[dest] = key;
        p.to_places[dest] = p.places ? p.places[i] : static_cast<int>(i);
    }
}

// ---- sums ------------------------------------------------------------------------------------

// Chunks of kChunk sorted places that all have one token are summed ahead, and kChunk of such
// chunks again, so that a row adds at most 2 kChunk places, as many chunks, and chunks of chunks.
constexpr int kChunk = 32;
constexpr int kTake = 8;                   // rows in flight

struct Sums {
    const int32_t* keys;
    const int32_t* places;
    Segment* seg;
    float* chunks;             // [n / kChunk][dim]
    float* big;                // [n / kChunk / kChunk][dim], null: not taken
    int n;
};

// v += rows [from, to) of f's, in their order.
template <class F> __device__ __forceinline__ void add_rows(float (&v)[kCols], int from, int to, F f)
{
    int i = from;
    for (; i + kTake <= to; i += kTake) {
        float x[kTake][kCols];
#pragma unroll
        for (int u = 0; u < kTake; ++u) f(i + u, x[u]);
#pragma unroll
        for (int u = 0; u < kTake; ++u)
#pragma unroll
            for (int k = 0; k < kCols; ++k) v[k] += x[u][k];
    }
    for (; i < to; ++i) {
        float x[kCols];
        f(i, x);
#pragma unroll
        for (int k = 0; k < kCols; ++k) v[k] += x[k];
    }
}

template <class T> struct Places {
    const T* rows;
    int64_t stride;
    const int32_t* places;
    int col, left;

    __device__ void operator()(int i, float (&x)[kCols]) const { fetch(rows + places[i] * stride + col, left, x); }
};
struct Chunks {
    const float* rows;
    int dim, col, left;

    __device__ void operator()(int i, float (&x)[kCols]) const { fetch(rows + static_cast<int64_t>(i) * dim + col, left, x); }
};

template <class T>
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
        const int col = piece_col(p, static_cast<int>(i - static_cast<int64_t>(c) * p.of_row)), left = a.e.dim - col;
        const int from = c * kChunk, key = s.keys[from];
        if (left <= 0 || key >= a.e.vocab || s.keys[from + kChunk - 1] != key) continue;
        float v[kCols] = {};
        add_rows(v, from, from + kChunk, Places<T>{static_cast<const T*>(a.rows), a.rows_stride, s.places, col, left});
        put(s.chunks + static_cast<int64_t>(c) * a.e.dim + col, left, v);
    }
}

__global__ __launch_bounds__(kThreads) void big_chunk_kernel(const EmbedArgs a, const Pieces p, const Sums s)
{
    const int64_t n = p.rows * p.of_row;
    for (int64_t i = first_piece(p); i < n; i += piece_step(p)) {
        const int c = static_cast<int>(i / p.of_row);
        const int col = piece_col(p, static_cast<int>(i - static_cast<int64_t>(c) * p.of_row)), left = a.e.dim - col;
        const int from = c * kChunk * kChunk, key = s.keys[from];
        if (left <= 0 || key >= a.e.vocab || s.keys[from + kChunk * kChunk - 1] != key) continue;
        float v[kCols] = {};
        add_rows(v, c * kChunk, (c + 1) * kChunk, Chunks{s.chunks, a.e.dim, col, left});
        put(s.big + static_cast<int64_t>(c) * a.e.dim + col, left, v);
    }
}

// v += the sorted places [lo, hi), in their order, from whole chunks where there are any.
template <class T>
__device__ __forceinline__ void add_segment(float (&v)[kCols], const EmbedArgs& a, const Sums& s, int lo, int hi, int col, int left)
{
    const Places<T> places{static_cast<const T*>(a.rows), a.rows_stride, s.places, col, left};
    const int c0 = (lo + kChunk - 1) / kChunk, c1 = hi / kChunk;
    if (c0 >= c1) {
        add_rows(v, lo, hi, places);
        return;
    }
    add_rows(v, lo, c0 * kChunk, places);
    const Chunks chunks{s.chunks, a.e.dim, col, left};
    const int b0 = (c0 + kChunk - 1) / kChunk, b1 = c1 / kChunk;
    if (!s.big || b0 >= b1) {
        add_rows(v, c0, c1, chunks);
    } else {
        add_rows(v, c0, b0 * kChunk, chunks);
        add_rows(v, b0, b1, Chunks{s.big, a.e.dim, col, left});
        add_rows(v, b1 * kChunk, c1, chunks);
    }
    add_rows(v, c1 * kChunk, hi, places);
}

// Every row of the table's gradient, or (ADD) those of tokens that occur, added to what is there:
// a row then goes to the first of its sorted places.
template <class T, class TG, bool ADD>
__global__ __launch_bounds__(kThreads) void rows_kernel(const EmbedArgs a, const Pieces p, const Sums s)
{
    const int64_t n = p.rows * p.of_row;
    for (int64_t i = first_piece(p); i < n; i += piece_step(p)) {
        const int row = static_cast<int>(i / p.of_row);
        const int col = piece_col(p, static_cast<int>(i - static_cast<int64_t>(row) * p.of_row)), left = a.e.dim - col;
        if (left <= 0) continue;
        int token = row;
        if (ADD) {
            token = s.keys[row];
            if (token >= a.e.vocab || (row > 0 && s.keys[row - 1] == token)) continue;
        }
        TG* to = static_cast<TG*>(a.grad) + token * a.grad_stride + col;
        const Segment g = s.n ? s.seg[token] : Segment{0, 0};
        float v[kCols] = {};
        if (g.hi > g.lo) {
            add_segment<T>(v, a, s, g.lo, g.hi, col, left);
#pragma unroll
            for (int k = 0; k < kCols; ++k) v[k] *= a.e.scale;
            if (ADD) {
                float x[kCols];
                fetch(to, left, x);
#pragma unroll
                for (int k = 0; k < kCols; ++k) v[k] += x[k];
            }
        }
        put(to, left, v);
    }
}

// ---- launches -------------------------------------------------------------------------------

int64_t over(int64_t n, int64_t part) { return (n + part - 1) / part; }

Pieces pieces_of(int64_t rows, int dim)
{
    Pieces p;
    p.lanes = 1;
    while (p.lanes < 64 && p.lanes * kCols < dim) p.lanes *= 2;
    p.of_row = static_cast<int>(over(dim, p.lanes * kCols));
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

// Places of a block in a pass of the sort: each wave has at least kShare, and there are no more
// tiles than kTilesMost, since every block reads all tiles' counts.
constexpr int64_t kShare = 512, kTilesMost = 512;
int64_t tile_of(int64_t n)
{
    const int64_t least = kSortWaves * kShare, part = over(over(n, kTilesMost), kThreads) * kThreads;
    return part > least ? part : least;
}

// The parts of the scratch, in this order: two sorts' keys and places, counts, segments, chunks.
struct Layout {
    int64_t order, counts, seg, chunks, big, bytes;

    Layout(int64_t n, int64_t vocab, int64_t dim)
    {
        const auto up = [](int64_t b) { return over(b, 256) * 256; };
        order = up(n * 4);
        counts = 4 * order;
        const int64_t tiles = over(n, kSortWaves * kShare);
        seg = counts + up((tiles < kTilesMost ? tiles : kTilesMost) * kDigits * 4);
        chunks = seg + up(vocab * static_cast<int64_t>(sizeof(Segment)));
        big = chunks + up(n / kChunk * dim * 4);
        bytes = big + up(n / kChunk / kChunk * dim * 4);
        if (n == 0) bytes = 0;
    }
};

// From this many places on chunks of chunks are worth a launch.
constexpr int kBigLeast = 1 << 14;

template <class T> hipError_t forward(const EmbedArgs& a, bool out_bf16, hipStream_t stream)
{
    const Pieces p = pieces_of(a.e.count, a.e.dim);
    if (out_bf16) hipLaunchKernelGGL((lookup_kernel<T, uint16_t>), grid_of(p), dim3(kThreads), 0, stream, a, p);
    else hipLaunchKernelGGL((lookup_kernel<T, float>), grid_of(p), dim3(kThreads), 0, stream, a, p);
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
        hipLaunchKernelGGL(count_kernel, dim3(static_cast<unsigned>(p.tiles)), dim3(kThreads), 0, stream, p, i == 0 ? seg : nullptr);
        hipLaunchKernelGGL(scatter_kernel, dim3(static_cast<unsigned>(p.tiles)), dim3(kThreads), 0, stream, p);
        p.shift += p.bits;
        p.keys = s.keys = p.to_keys;
        p.places = s.places = p.to_places;
    }
}

template <class T, class TG> hipError_t backward(const EmbedArgs& a, const OpsDevice& d, hipStream_t stream)
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
        hipLaunchKernelGGL((chunk_kernel<T>), dim3(static_cast<unsigned>(blocks > places ? blocks : places)), dim3(kThreads), 0, stream,
                           a, chunks, s);
        if (s.n >= kBigLeast) {
            s.big = reinterpret_cast<float*>(scratch + l.big);
            const Pieces big = pieces_of(s.n / kChunk / kChunk, a.e.dim);
            hipLaunchKernelGGL(big_chunk_kernel, grid_of(big), dim3(kThreads), 0, stream, a, big, s);
        }
    } else if (a.add) {
        return hipSuccess;
    }
    const Pieces p = pieces_of(a.add ? s.n : a.e.vocab, a.e.dim);
    if (a.add) hipLaunchKernelGGL((rows_kernel<T, TG, true>), grid_of(p), dim3(kThreads), 0, stream, a, p, s);
    else hipLaunchKernelGGL((rows_kernel<T, TG, false>), grid_of(p), dim3(kThreads), 0, stream, a, p, s);
    return hipGetLastError();
}

}  // namespace

int64_t embed_scratch_bytes(int64_t count, int64_t vocab, int64_t dim) { return Layout(count, vocab, dim).bytes; }

hipError_t launch_embed_forward(const EmbedArgs& a, bool bf16, bool rows_bf16, hipStream_t stream)
{
    return bf16 ? forward<uint16_t>(a, rows_bf16, stream) : forward<float>(a, rows_bf16, stream);
}

hipError_t launch_embed_backward(const EmbedArgs& a, bool bf16, bool rows_bf16, const OpsDevice& d, hipStream_t stream)
{
    if (rows_bf16) return bf16 ? backward<uint16_t, uint16_t>(a, d, stream) : backward<uint16_t, float>(a, d, stream);
    return bf16 ? backward<float, uint16_t>(a, d, stream) : backward<float, float>(a, d, stream);
}

}  // namespace gemk
