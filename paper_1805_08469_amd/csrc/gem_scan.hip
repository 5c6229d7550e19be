// gem_scan.hip -- the gated linear recurrence and its backward pass for gfx950.
//
// h_t = a_t h_{t-1} + (1 - a_t) x_t is a chain along the tokens, but any run of tokens
// is one map h -> A h + B, and maps compose.  A block takes a tile of 128 tokens by 64
// channels: each thread runs through 4 tokens of 4 channels, the threads' maps are
// joined over lanes and waves, and the tiles of one slice of channels are joined in
// token order by the blocks themselves, through words in memory: a tile leaves its map
// as soon as it has it and its state as soon as it knows it, and a tile that waits takes
// the nearest state before it through the maps in between.  So every array is read once
// and written once, in one launch, whatever the number and lengths of the sequences
// (a sequence's first token is a map that ignores h), and its bytes bound the pass.
//
// The values do not depend on which state a tile finds: every state is the one before it
// through one map, whoever computes it.
//
// Blocks draw their tiles in order from a counter, all tiles of one run of tokens before
// any of the next, so the tiles that a waiting block needs are always held by blocks that
// run and that wait for none but earlier ones: the wait ends.
//
// Eight waves of a block move data; a ninth draws the next tile, finds the sequences that
// begin or end in it, and waits for the state: its polls would otherwise queue behind the
// others' loads and stores.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gem_ops.hpp"
#include "gem_ops_device.hpp"

namespace gemk {
namespace {

constexpr int kWaves = 8;                  // waves that move data
constexpr int kThreads = (kWaves + 1) * 64;
constexpr int kChan = 4;                   // channels of a thread
constexpr int kLanes = 16;                 // threads side by side
constexpr int kSlice = kChan * kLanes;     // channels of a tile
constexpr int kSteps = 4;                  // tokens of a thread
constexpr int kSubs = 64 / kLanes;         // runs of tokens of a wave
static_assert(kWaves * kSubs * kSteps == kScanTile, "a tile's tokens");
static_assert(kSlice == 64, "the ninth wave has a lane a channel");

// ---- elements ----------------------------------------------------------------------

// Four channels of a row, at any address of the elements' own alignment.
template <class T> struct Raw;
template <> struct Raw<float> {
    using Type = u32x4 __attribute__((aligned(4)));
};
template <> struct Raw<uint16_t> {
    using Type = uint32_t __attribute__((ext_vector_type(2), aligned(2)));
};
__device__ __forceinline__ void widen(const Raw<float>::Type& r, float (&v)[kChan])
{
#pragma unroll
    for (int i = 0; i < kChan; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void widen(const Raw<uint16_t>::Type& r, float (&v)[kChan])
{
    v[0] = __uint_as_float(r[0] << 16);
    v[1] = __uint_as_float(r[0] & 0xFFFF0000u);
    v[2] = __uint_as_float(r[1] << 16);
    v[3] = __uint_as_float(r[1] & 0xFFFF0000u);
}

// Channels [c, c + 4) of row p, those below `channels`.
template <class T>
__device__ __forceinline__ typename Raw<T>::Type fetch(const T* p, int c, int channels)
{
    using R = typename Raw<T>::Type;
    if (c + kChan <= channels) return *reinterpret_cast<const R*>(p + c);
    R r{};
    T* e = reinterpret_cast<T*>(&r);
#pragma unroll
    for (int i = 0; i < kChan; ++i)
        if (c + i < channels) e[i] = p[c + i];
    return r;
}

__device__ __forceinline__ Raw<float>::Type narrow(const float (&v)[kChan], const float*)
{
    return Raw<float>::Type{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
}
__device__ __forceinline__ Raw<uint16_t>::Type narrow(const float (&v)[kChan], const uint16_t*)
{
    return Raw<uint16_t>::Type{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
}

template <class T>
__device__ __forceinline__ void put(T* p, int c, int channels, const float (&v)[kChan])
{
    const typename Raw<T>::Type r = narrow(v, p);
    if (c + kChan <= channels) {
        *reinterpret_cast<typename Raw<T>::Type*>(p + c) = r;
    } else {
        const T* e = reinterpret_cast<const T*>(&r);
#pragma unroll
        for (int i = 0; i < kChan; ++i)
            if (c + i < channels) p[c + i] = e[i];
    }
}

// a = sigmoid(g) and b = 1 - a, each to full precision whatever its size: with
// E = exp(-|g|) <= 1 the smaller is E / (1 + E), and the larger is one minus it, rounded
// once (an error of a's last bit grows with the tokens that a state lives).
__device__ __forceinline__ void gates(float g, float& a, float& b)
{
    const float E = __builtin_amdgcn_exp2f(__builtin_fabsf(g) * -kLog2e);
    const float small = E * __builtin_amdgcn_rcpf(1.0f + E);
    const float big = 1.0f - small;
    a = g >= 0.0f ? big : small;
    b = g >= 0.0f ? small : big;
}

// ---- maps ----------------------------------------------------------------------------

// h -> A h + B on a thread's channels.  A map that ignores h (a sequence begins) has
// A = -0: gates are not negative, so no product of them is, and 0 h would be NaN where h
// is infinite.
struct Map {
    float A[kChan], B[kChan];
};

// One channel: (A, B) after (A0, B0).  CUTS: sequences begin in the tile.
template <bool CUTS>
__device__ __forceinline__ void after(float& A, float& B, float A0, float B0)
{
    const float b = __builtin_fmaf(A, B0, B), a = A * A0;
    if constexpr (CUTS) {
        const bool cut = __float_as_int(A) < 0;
        B = cut ? B : b;
        A = cut ? A : a;
    } else {
        B = b;
        A = a;
    }
}
template <bool CUTS>
__device__ __forceinline__ float through(float A, float B, float h)
{
    const float r = __builtin_fmaf(A, h, B);
    if constexpr (CUTS) return __float_as_int(A) < 0 ? B : r;
    return r;
}

// A tile's map of each wave, [map of forward or backward][wave][channel].
struct WaveMaps {
    float A[kWaves][kSlice], B[kWaves][kSlice];
};

// Joins the maps of a wave's four runs of tokens; in order (UP) or from the last.  m
// becomes the map of all tokens before the thread's (beyond them), and the whole wave's
// goes to w.
template <bool CUTS, bool UP>
__device__ __forceinline__ void join_lanes(Map& m, WaveMaps& w, int wave, int lane)
{
    const int run = UP ? lane / kLanes : kSubs - 1 - lane / kLanes;
#pragma unroll
    for (int s = 1; s < kSubs; s *= 2) {
#pragma unroll
        for (int c = 0; c < kChan; ++c) {
            const float A0 = UP ? __shfl_up(m.A[c], s * kLanes) : __shfl_down(m.A[c], s * kLanes);
            const float B0 = UP ? __shfl_up(m.B[c], s * kLanes) : __shfl_down(m.B[c], s * kLanes);
            if (run >= s) after<CUTS>(m.A[c], m.B[c], A0, B0);
        }
    }
    if (run == kSubs - 1) {
        const int c = lane % kLanes * kChan;
#pragma unroll
        for (int i = 0; i < kChan; ++i) {
            w.A[wave][c + i] = m.A[i];
            w.B[wave][c + i] = m.B[i];
        }
    }
#pragma unroll
    for (int c = 0; c < kChan; ++c) {
        const float A0 = UP ? __shfl_up(m.A[c], kLanes) : __shfl_down(m.A[c], kLanes);
        const float B0 = UP ? __shfl_up(m.B[c], kLanes) : __shfl_down(m.B[c], kLanes);
        m.A[c] = run ? A0 : 1.0f;
        m.B[c] = run ? B0 : 0.0f;
    }
}

// The state that reaches a thread: the tile's through the maps of the waves before its
// own, then through m.
template <bool CUTS, bool UP>
__device__ __forceinline__ void reach(float (&h)[kChan], const Map& m, const WaveMaps& w, int wave, int c0)
{
    if constexpr (UP) {
        for (int k = 0; k < wave; ++k)
#pragma unroll
            for (int i = 0; i < kChan; ++i) h[i] = through<CUTS>(w.A[k][c0 + i], w.B[k][c0 + i], h[i]);
    } else {
        for (int k = kWaves - 1; k > wave; --k)
#pragma unroll
            for (int i = 0; i < kChan; ++i) h[i] = through<CUTS>(w.A[k][c0 + i], w.B[k][c0 + i], h[i]);
    }
#pragma unroll
    for (int i = 0; i < kChan; ++i) h[i] = through<CUTS>(m.A[i], m.B[i], h[i]);
}

// ---- tiles of a slice, joined through memory ---------------------------------------------

// Counters of a handle's recurrences: zero between launches but for the number of
// launches, which marks the words that a launch writes (older ones have older marks).
struct ScanCounters {
    uint32_t drawn, done, launches;
};

// A channel's words of a tile: its map's A and B, its state; each with the launch's mark
// in its upper half.
struct TileWords {
    uint64_t A[kSlice], B[kSlice], h[kSlice];
};
// What a tile has left so far: 1 its map, 2 its state (with the mark).  Only a hint where
// to look: the words' own marks say whether they are there.
enum : uint32_t { kHasMap = 1, kHasState = 2 };

struct Chain {
    ScanCounters* counters;
    uint64_t* hints;             // [slices][tiles]
    TileWords* words;            // [tiles][slices]
    int tiles, slices;
    int64_t total;               // tiles * slices
};

__device__ __forceinline__ uint64_t peek(const uint64_t* w)
{
    return __hip_atomic_load(w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void leave(uint64_t* w, uint32_t mark, uint32_t v)
{
    __hip_atomic_store(w, (static_cast<uint64_t>(mark) << 32) | v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// A word of each lane, once all lanes' are there.
__device__ __forceinline__ float await(const uint64_t* w, uint32_t mark)
{
    uint64_t v = peek(w);
    while (__ballot(static_cast<uint32_t>(v >> 32) != mark)) {
        __builtin_amdgcn_s_sleep(1);
        v = peek(w);
    }
    return __uint_as_float(static_cast<uint32_t>(v));
}

// The state that reaches tile `at` (at >= 1, in the order of the chain); a lane a channel.
// Some tile at most 64 before it has left its state or will.
__device__ __forceinline__ float state_before(const Chain& ch, int slice, int at, uint32_t mark, int lane)
{
    const uint64_t* hints = ch.hints + static_cast<int64_t>(slice) * ch.tiles;
    int far;                                   // tiles back, less one
    for (;;) {
        const int t = at - 1 - lane;
        const uint64_t hint = t >= 0 ? peek(hints + t) : 0;
        const bool mine = static_cast<uint32_t>(hint >> 32) == mark;
        const uint64_t states = __ballot(mine && static_cast<uint32_t>(hint) == kHasState);
        const uint64_t maps = __ballot(mine);
        if (states) {
            far = __builtin_ctzll(states);
            const uint64_t between = (uint64_t{1} << far) - 1;
            if ((maps & between) == between) break;
        }
        __builtin_amdgcn_s_sleep(2);
    }
    const auto words = [&](int t) { return ch.words + static_cast<int64_t>(t) * ch.slices + slice; };
    float h = await(&words(at - 1 - far)->h[lane], mark);
    constexpr int kAhead = 4;
    for (int i = far; i > 0; i -= kAhead) {    // maps of tiles at - i, at - i + 1, ...
        uint64_t A[kAhead], B[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int t = at - (i - u > 0 ? i - u : 1);
            A[u] = peek(&words(t)->A[lane]);
            B[u] = peek(&words(t)->B[lane]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i - u <= 0) continue;
            const bool there = static_cast<uint32_t>(A[u] >> 32) == mark && static_cast<uint32_t>(B[u] >> 32) == mark;
            float a = __uint_as_float(static_cast<uint32_t>(A[u])), b = __uint_as_float(static_cast<uint32_t>(B[u]));
            if (__ballot(!there)) {
                a = await(&words(at - i + u)->A[lane], mark);
                b = await(&words(at - i + u)->B[lane], mark);
            }
            h = __builtin_fmaf(a, h, b);
        }
    }
    return h;
}

// ---- sequences in a tile -----------------------------------------------------------------

// For each token of a tile the sequence that begins or ends with it, or -1; any: there
// is one.
struct Ends {
    int first[kScanTile], last[kScanTile];
    int any;
};

// The least b in [0, n] with offsets[b] >= t, by one wave (whatever the offsets hold, a
// number in that range).
__device__ __forceinline__ int lower_bound(const int64_t* offsets, int n, int64_t t, int lane)
{
    int lo = 0, hi = n;                        // the answer is in [lo, hi]
    while (hi > lo) {
        const int step = (hi - lo + 63) / 64;
        const int64_t at = static_cast<int64_t>(lo) + static_cast<int64_t>(lane) * step;
        const bool less = at < hi && offsets[at] < t;
        const uint64_t m = __ballot(less);
        // Probes lo, lo + step, ...: the answer lies behind the last that is less, up to the next.
        const int k = m == 0 ? 0 : 64 - __builtin_clzll(m);
        const int64_t below = static_cast<int64_t>(lo) + static_cast<int64_t>(k - 1) * step;
        const int64_t above = static_cast<int64_t>(lo) + static_cast<int64_t>(k) * step;
        if (k == 0) return lo;
        hi = above < hi ? static_cast<int>(above) : hi;
        lo = static_cast<int>(below) + 1;
    }
    return lo;
}

// Fills e for the tile of tokens from t0, by one wave.  empty(b) is called, by every
// lane, for each empty sequence b that lies in it.
template <class F>
__device__ __forceinline__ void find_ends(Ends& e, const gem_scan& s, int64_t t0, int lane, F empty)
{
    const int64_t end = t0 + kScanTile;
    if (!s.offsets) {
        const uint32_t len = static_cast<uint32_t>(s.tokens / s.sequences);
        const uint32_t in = static_cast<uint32_t>(t0) % len;         // tokens > 0, so len > 0
        const bool any = in == 0 || in + kScanTile >= len;
        if (lane == 0) e.any = any;
        if (!any) return;
        for (int i = lane; i < kScanTile; i += 64) {
            const uint32_t t = static_cast<uint32_t>(t0) + i, q = t / len, r = t - q * len;
            const bool in_all = t0 + i < s.tokens;
            e.first[i] = in_all && r == 0 ? static_cast<int>(q) : -1;
            e.last[i] = in_all && r == len - 1 ? static_cast<int>(q) : -1;
        }
        return;
    }
    for (int i = lane; i < kScanTile; i += 64) e.first[i] = e.last[i] = -1;
    // Sequences from the one that reaches into the tile to the last that begins in it; the
    // last tile takes the empty ones behind all tokens too.
    const int64_t stop = end >= s.tokens ? INT64_MAX : end;
    int b = lower_bound(s.offsets, s.sequences, t0, lane) - 1;
    if (b < 0) b = 0;
    bool any = false;
    for (;; b += 64) {
        const int q = b + lane;
        const bool in = q < s.sequences;
        const int64_t from = in ? s.offsets[q] : INT64_MAX, to = in ? s.offsets[q + 1] : INT64_MAX;
        const bool here = in && from < stop;
        if (here && to > from) {
            if (from >= t0 && from < end && from < s.tokens) {
                e.first[from - t0] = q;
                any = true;
            }
            if (to > t0 && to <= end && to <= s.tokens) {
                e.last[to - 1 - t0] = q;
                any = true;
            }
        }
        uint64_t none = __ballot(here && to <= from && from >= t0);
        while (none) {
            empty(b + __builtin_ctzll(none));
            none &= none - 1;
        }
        if (__ballot(!here)) break;
    }
    const bool some = __ballot(any) != 0;
    if (lane == 0) e.any = some;
}

// ---- forward ---------------------------------------------------------------------------

template <class T> struct ForwardTile {
    typename Raw<T>::Type x[kSteps], g[kSteps];

    // Rows from token t on; past the last the last is read again.
    __device__ void load(const gem_scan& s, int64_t t, int c)
    {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int64_t r = t + i < s.tokens ? t + i : s.tokens - 1;
            x[i] = fetch(static_cast<const T*>(s.x) + r * s.x_stride, c, s.channels);
            g[i] = fetch(static_cast<const T*>(s.gate) + r * s.gate_stride, c, s.channels);
        }
    }
};

struct ForwardLds {
    WaveMaps maps[2];
    Ends ends[3];
    float carry[kSlice];
    int64_t next[2];
};

// A thread's tokens: A[i], B[i] the map of tokens up to i.
template <bool CUTS, class T>
__device__ __forceinline__ void forward_local(const ScanArgs& a, const ForwardTile<T>& d, const Ends& e, int64_t t, int i0,
                                              int c, float (&A)[kSteps][kChan], float (&B)[kSteps][kChan])
{
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        float x[kChan], g[kChan];
        widen(d.x[i], x);
        widen(d.g[i], g);
        const bool in = t + i < a.s.tokens;
        const int q = CUTS ? e.first[i0 + i] : -1;
#pragma unroll
        for (int k = 0; k < kChan; ++k) {
            float keep, take;
            gates(g[k], keep, take);
            float add = take * x[k];
            if (!in) {
                keep = 1.0f;
                add = 0.0f;
            }
            A[i][k] = i == 0 ? keep : A[i ? i - 1 : 0][k] * keep;
            B[i][k] = i == 0 ? add : __builtin_fmaf(keep, B[i ? i - 1 : 0][k], add);
            if (CUTS && q >= 0) {
                const float h0 = a.s.h0 && c + k < a.s.channels ? a.s.h0[static_cast<int64_t>(q) * a.s.channels + c + k] : 0.0f;
                A[i][k] = -0.0f;
                B[i][k] = __builtin_fmaf(keep, h0, add);
            }
        }
    }
}

template <bool CUTS, class T>
__device__ __forceinline__ void forward_out(const ScanArgs& a, const Ends& e, int64_t t, int i0, int c,
                                            const float (&A)[kSteps][kChan], const float (&B)[kSteps][kChan],
                                            const float (&h)[kChan])
{
    if (c >= a.s.channels) return;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        float y[kChan];
#pragma unroll
        for (int k = 0; k < kChan; ++k) y[k] = through<CUTS>(A[i][k], B[i][k], h[k]);
        if (t + i < a.s.tokens) put(static_cast<T*>(a.y) + (t + i) * a.y_stride, c, a.s.channels, y);
        if (CUTS && a.h_last && e.last[i0 + i] >= 0)
            put(a.h_last + static_cast<int64_t>(e.last[i0 + i]) * a.s.channels, c, a.s.channels, y);
    }
}

// The ninth wave's part of a tile: the tile's map from the waves', left for later tiles,
// and the state that reaches it.  cuts: the map ignores that state; apart: so does every
// token.
template <bool UP>
__device__ __forceinline__ float join_tile(const Chain& ch, const WaveMaps& w, bool cuts, bool apart, int slice, int at,
                                           uint32_t mark, int lane)
{
    float A = 1.0f, B = 0.0f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
        const int v = UP ? k : kWaves - 1 - k;
        float a = w.A[v][lane], b = w.B[v][lane];
        after<true>(a, b, A, B);
        A = a;
        B = b;
    }
    const bool chained = ch.tiles > 1;
    TileWords* words = ch.words + static_cast<int64_t>(at) * ch.slices + slice;
    uint64_t* hint = ch.hints + static_cast<int64_t>(slice) * ch.tiles + at;
    const bool known = at == 0 || cuts;        // the tile's own state needs none before it
    const bool last = at == ch.tiles - 1;
    if (chained && !last) {
        if (known) {
            leave(&words->h[lane], mark, __float_as_uint(B));
        } else {
            leave(&words->A[lane], mark, __float_as_uint(A));
            leave(&words->B[lane], mark, __float_as_uint(B));
        }
        if (lane == 0) leave(hint, mark, known ? kHasState : kHasMap);
    }
    if (at == 0 || apart) return 0.0f;
    const float h = state_before(ch, slice, at, mark, lane);
    if (!known && !last) {
        leave(&words->h[lane], mark, __float_as_uint(__builtin_fmaf(A, h, B)));
        if (lane == 0) leave(hint, mark, kHasState);
    }
    return h;
}

// The ninth wave draws the next tile.
__device__ __forceinline__ int64_t draw(const Chain& ch, int lane)
{
    if (ch.tiles == 1) return ch.total;        // a block a tile
    uint32_t k = 0;
    if (lane == 0)
        k = __hip_atomic_fetch_add(&ch.counters->drawn, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return __shfl(k, 0);
}

// A block is through: the last one sets the counters for the next launch.
__device__ __forceinline__ void finish(const Chain& ch)
{
    if (ch.tiles == 1) return;
    const uint32_t before = __hip_atomic_fetch_add(&ch.counters->done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (before == gridDim.x - 1) {
        __hip_atomic_store(&ch.counters->drawn, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(&ch.counters->done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_fetch_add(&ch.counters->launches, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

// A sequence of no tokens: what reached it leaves it, channels of one slice.
__device__ __forceinline__ void pass_empty(const float* from, float* to, int64_t q, int channels, int c)
{
    if (to && c < channels) to[q * channels + c] = from ? from[q * channels + c] : 0.0f;
}

template <class T>
__global__ __launch_bounds__(kThreads) void forward_kernel(const ScanArgs a, const Chain ch)
{
    __shared__ ForwardLds l;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool control = wave == kWaves;
    const int i0 = (wave * kSubs + lane / kLanes) * kSteps;    // the thread's first token in a tile
    const int c0 = lane % kLanes * kChan;                      // and its first channel in a slice
    uint32_t mark = 0;
    const auto ends_of = [&](Ends& e, int64_t k) {
        const int slice = static_cast<int>(k % ch.slices);
        find_ends(e, a.s, k / ch.slices * kScanTile, lane,
                  [&](int q) { pass_empty(a.s.h0, a.h_last, q, a.s.channels, slice * kSlice + lane); });
    };
    if (control) {
        if (ch.tiles > 1)
            mark = 1 + __hip_atomic_load(&ch.counters->launches, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const int64_t k = ch.tiles == 1 ? blockIdx.x : draw(ch, lane);
        if (k < ch.total) ends_of(l.ends[0], k);
        if (lane == 0) l.next[1] = k;
    }
    __syncthreads();
    int64_t k = l.next[1];
    ForwardTile<T> d;
    if (!control && k < ch.total)
        d.load(a.s, k / ch.slices * kScanTile + i0, static_cast<int>(k % ch.slices) * kSlice + c0);
    // Words that a tile's last phase reads are not written in the next tile's first: there are
    // two sets of maps, and three of ends, which are found a tile ahead.
    for (int n = 0; k < ch.total; ++n) {
        const int turn = n & 1;
        const int slice = static_cast<int>(k % ch.slices), at = static_cast<int>(k / ch.slices);
        const int64_t t = static_cast<int64_t>(at) * kScanTile + i0;
        const int c = slice * kSlice + c0;
        const Ends& e = l.ends[n % 3];
        const bool cuts = e.any;
        float A[kSteps][kChan], B[kSteps][kChan];
        Map m;
        if (control) {
            const int64_t next = draw(ch, lane);
            if (next < ch.total) ends_of(l.ends[(n + 1) % 3], next);
            if (lane == 0) l.next[turn] = next;
        } else {
            if (cuts) forward_local<true>(a, d, e, t, i0, c, A, B);
            else forward_local<false>(a, d, e, t, i0, c, A, B);
#pragma unroll
            for (int i = 0; i < kChan; ++i) {
                m.A[i] = A[kSteps - 1][i];
                m.B[i] = B[kSteps - 1][i];
            }
            if (cuts) join_lanes<true, true>(m, l.maps[turn], wave, lane);
            else join_lanes<false, true>(m, l.maps[turn], wave, lane);
        }
        __syncthreads();
        const int64_t next = l.next[turn];
        if (control) {
            bool begins = false;
            if (cuts)
                for (int i = lane; i < kScanTile; i += 64) begins |= e.first[i] >= 0;
            const float h = join_tile<true>(ch, l.maps[turn], __ballot(begins) != 0, cuts && e.first[0] >= 0, slice, at, mark,
                                            lane);
            l.carry[lane] = h;
            if (a.states && slice * kSlice + lane < a.s.channels)
                a.states[static_cast<int64_t>(at) * a.s.channels + slice * kSlice + lane] = h;
        } else if (next < ch.total) {
            d.load(a.s, next / ch.slices * kScanTile + i0, static_cast<int>(next % ch.slices) * kSlice + c0);
        }
        __syncthreads();
        if (!control) {
            float h[kChan];
#pragma unroll
            for (int i = 0; i < kChan; ++i) h[i] = l.carry[c0 + i];
            if (cuts) {
                reach<true, true>(h, m, l.maps[turn], wave, c0);
                forward_out<true, T>(a, e, t, i0, c, A, B, h);
            } else {
                reach<false, true>(h, m, l.maps[turn], wave, c0);
                forward_out<false, T>(a, e, t, i0, c, A, B, h);
            }
        }
        k = next;
    }
    if (threadIdx.x == kWaves * 64) finish(ch);
}

// ---- backward ------------------------------------------------------------------------------

// With e_t = a_t r_t, what a token hands to the one before it, e_t = a_t e_{t+1} + a_t dy_t
// is the same kind of chain from the last token to the first; h is formed again inside each
// tile from the state that forward kept for it.
template <class T> struct BackwardTile {
    typename Raw<T>::Type x[kSteps], g[kSteps], dy[kSteps];
    float state[kChan];

    __device__ void load(const ScanBackArgs& a, int at, int64_t t, int c)
    {
        const gem_scan& s = a.s;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int64_t r = t + i < s.tokens ? t + i : s.tokens - 1;
            g[i] = fetch(static_cast<const T*>(s.gate) + r * s.gate_stride, c, s.channels);
            x[i] = fetch(static_cast<const T*>(s.x) + r * s.x_stride, c, s.channels);
            dy[i] = fetch(static_cast<const T*>(a.dy) + r * a.dy_stride, c, s.channels);
        }
        const auto h = fetch(a.states + static_cast<int64_t>(at) * s.channels, c, s.channels);
        widen(h, state);
    }
};

struct BackwardLds {
    WaveMaps up[2], down[2];
    Ends ends[3];
    float carry[kSlice];
    int64_t next[2];
};

// A thread's gates, and its maps in both directions.
template <bool CUTS, class T>
__device__ __forceinline__ void backward_local(const ScanBackArgs& a, const BackwardTile<T>& d, const Ends& e, int64_t t,
                                               int i0, int c, float (&keep)[kSteps][kChan], float (&take)[kSteps][kChan],
                                               Map& up, Map& down)
{
    const int64_t D = a.s.channels;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        float x[kChan], g[kChan];
        widen(d.x[i], x);
        widen(d.g[i], g);
        const bool in = t + i < a.s.tokens;
        const int q = CUTS ? e.first[i0 + i] : -1;
#pragma unroll
        for (int k = 0; k < kChan; ++k) {
            gates(g[k], keep[i][k], take[i][k]);
            if (!in) {
                keep[i][k] = 1.0f;
                take[i][k] = 0.0f;
            }
            const float add = take[i][k] * x[k];
            up.A[k] = i == 0 ? keep[i][k] : up.A[k] * keep[i][k];
            up.B[k] = i == 0 ? add : __builtin_fmaf(keep[i][k], up.B[k], add);
            if (CUTS && q >= 0) {
                const float h0 = a.s.h0 && c + k < D ? a.s.h0[q * D + c + k] : 0.0f;
                up.A[k] = -0.0f;
                up.B[k] = __builtin_fmaf(keep[i][k], h0, add);
            }
        }
    }
#pragma unroll
    for (int i = kSteps - 1; i >= 0; --i) {
        float dy[kChan];
        widen(d.dy[i], dy);
        const bool in = t + i < a.s.tokens;
        const int q = CUTS ? e.last[i0 + i] : -1;
#pragma unroll
        for (int k = 0; k < kChan; ++k) {
            const float add = in ? keep[i][k] * dy[k] : 0.0f;
            const float kp = keep[i][k];
            down.A[k] = i == kSteps - 1 ? kp : down.A[k] * kp;
            down.B[k] = i == kSteps - 1 ? add : __builtin_fmaf(kp, down.B[k], add);
            if (CUTS && q >= 0) {
                const float end = a.dh_last && c + k < D ? a.dh_last[q * D + c + k] : 0.0f;
                down.A[k] = -0.0f;
                down.B[k] = __builtin_fmaf(kp, end, add);
            }
        }
    }
}

// From the state h before the thread's tokens, and what the tokens behind them hand down.
template <bool CUTS, class T>
__device__ __forceinline__ void backward_out(const ScanBackArgs& a, const BackwardTile<T>& d, const Ends& e, int64_t t, int i0,
                                             int c, const float (&keep)[kSteps][kChan], const float (&take)[kSteps][kChan],
                                             float (&h)[kChan], float (&back)[kChan], const float (&diff)[kSteps][kChan])
{
    const int64_t D = a.s.channels;
#pragma unroll
    for (int i = kSteps - 1; i >= 0; --i) {
        float dy[kChan], dx[kChan], dg[kChan];
        widen(d.dy[i], dy);
        const bool in = t + i < a.s.tokens;
        const int ql = CUTS ? e.last[i0 + i] : -1, qf = CUTS ? e.first[i0 + i] : -1;
#pragma unroll
        for (int k = 0; k < kChan; ++k) {
            if (CUTS && ql >= 0) back[k] = a.dh_last && c + k < D ? a.dh_last[ql * D + c + k] : 0.0f;
            const float r = in ? dy[k] + back[k] : back[k];
            dx[k] = take[i][k] * r;
            dg[k] = keep[i][k] * take[i][k] * diff[i][k] * r;
            back[k] = keep[i][k] * r;
        }
        if (c < D && in) {
            put(static_cast<T*>(a.dx) + (t + i) * a.dx_stride, c, a.s.channels, dx);
            put(static_cast<T*>(a.dgate) + (t + i) * a.dgate_stride, c, a.s.channels, dg);
            if (CUTS && a.dh0 && qf >= 0) put(a.dh0 + qf * D, c, a.s.channels, back);
        }
    }
}

// h_{t-1} - x_t for each of the thread's tokens.
template <bool CUTS, class T>
__device__ __forceinline__ void differences(const ScanBackArgs& a, const BackwardTile<T>& d, const Ends& e, int i0, int c,
                                            const float (&keep)[kSteps][kChan], const float (&take)[kSteps][kChan],
                                            float (&h)[kChan], float (&diff)[kSteps][kChan])
{
    const int64_t D = a.s.channels;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        float x[kChan];
        widen(d.x[i], x);
        const int q = CUTS ? e.first[i0 + i] : -1;
#pragma unroll
        for (int k = 0; k < kChan; ++k) {
            if (CUTS && q >= 0) h[k] = a.s.h0 && c + k < D ? a.s.h0[q * D + c + k] : 0.0f;
            diff[i][k] = h[k] - x[k];
            h[k] = __builtin_fmaf(keep[i][k], h[k], take[i][k] * x[k]);
        }
    }
}

template <class T>
__global__ __launch_bounds__(kThreads) void backward_kernel(const ScanBackArgs a, const Chain ch)
{
    __shared__ BackwardLds l;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool control = wave == kWaves;
    const int i0 = (wave * kSubs + lane / kLanes) * kSteps;
    const int c0 = lane % kLanes * kChan;
    uint32_t mark = 0;
    // The chain's tile `at` is the tokens' tile ch.tiles - 1 - at.
    const auto tile_of = [&](int64_t k) { return ch.tiles - 1 - static_cast<int>(k / ch.slices); };
    const auto ends_of = [&](Ends& e, int64_t k) {
        const int slice = static_cast<int>(k % ch.slices);
        find_ends(e, a.s, static_cast<int64_t>(tile_of(k)) * kScanTile, lane,
                  [&](int q) { pass_empty(a.dh_last, a.dh0, q, a.s.channels, slice * kSlice + lane); });
    };
    if (control) {
        if (ch.tiles > 1)
            mark = 1 + __hip_atomic_load(&ch.counters->launches, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const int64_t k = ch.tiles == 1 ? blockIdx.x : draw(ch, lane);
        if (k < ch.total) ends_of(l.ends[0], k);
        if (lane == 0) l.next[1] = k;
    }
    __syncthreads();
    int64_t k = l.next[1];
    // Words that a tile's last phase reads are not written in the next tile's first: there are
    // two sets of maps, and three of ends, which are found a tile ahead.
    for (int n = 0; k < ch.total; ++n) {
        const int turn = n & 1;
        const int slice = static_cast<int>(k % ch.slices), at = static_cast<int>(k / ch.slices), tile = tile_of(k);
        const int64_t t = static_cast<int64_t>(tile) * kScanTile + i0;
        const int c = slice * kSlice + c0;
        const Ends& e = l.ends[n % 3];
        const bool cuts = e.any;
        BackwardTile<T> d;
        float keep[kSteps][kChan], take[kSteps][kChan], diff[kSteps][kChan], h[kChan];
        Map up, down;
        if (control) {
            const int64_t next = draw(ch, lane);
            if (next < ch.total) ends_of(l.ends[(n + 1) % 3], next);
            if (lane == 0) l.next[turn] = next;
        } else {
            d.load(a, tile, t, c);
            if (cuts) {
                backward_local<true>(a, d, e, t, i0, c, keep, take, up, down);
                join_lanes<true, true>(up, l.up[turn], wave, lane);
                join_lanes<true, false>(down, l.down[turn], wave, lane);
            } else {
                backward_local<false>(a, d, e, t, i0, c, keep, take, up, down);
                join_lanes<false, true>(up, l.up[turn], wave, lane);
                join_lanes<false, false>(down, l.down[turn], wave, lane);
            }
        }
        __syncthreads();
        const int64_t next = l.next[turn];
        if (control) {
            bool ends = false;
            if (cuts)
                for (int i = lane; i < kScanTile; i += 64) ends |= e.last[i] >= 0;
            l.carry[lane] = join_tile<false>(ch, l.down[turn], __ballot(ends) != 0, cuts && e.last[kScanTile - 1] >= 0, slice,
                                             at, mark, lane);
        } else {
#pragma unroll
            for (int i = 0; i < kChan; ++i) h[i] = d.state[i];
            if (cuts) {
                reach<true, true>(h, up, l.up[turn], wave, c0);
                differences<true>(a, d, e, i0, c, keep, take, h, diff);
            } else {
                reach<false, true>(h, up, l.up[turn], wave, c0);
                differences<false>(a, d, e, i0, c, keep, take, h, diff);
            }
        }
        __syncthreads();
        if (!control) {
            float back[kChan];
#pragma unroll
            for (int i = 0; i < kChan; ++i) back[i] = l.carry[c0 + i];
            if (cuts) {
                reach<true, false>(back, down, l.down[turn], wave, c0);
                backward_out<true, T>(a, d, e, t, i0, c, keep, take, h, back, diff);
            } else {
                reach<false, false>(back, down, l.down[turn], wave, c0);
                backward_out<false, T>(a, d, e, t, i0, c, keep, take, h, back, diff);
            }
        }
        k = next;
    }
    if (threadIdx.x == kWaves * 64) finish(ch);
}

// ---- single tokens, no tokens ----------------------------------------------------------------

// One token a sequence: no chain.
constexpr int kStepThreads = 256;

template <class T>
__global__ __launch_bounds__(kStepThreads) void step_kernel(const ScanArgs a, int groups)
{
    const int D = a.s.channels;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kStepThreads + threadIdx.x; i < a.s.tokens * groups;
         i += static_cast<int64_t>(gridDim.x) * kStepThreads) {
        const int64_t t = i / groups;
        const int c = static_cast<int>(i - t * groups) * kChan;
        float x[kChan], g[kChan], h[kChan] = {}, y[kChan];
        widen(fetch(static_cast<const T*>(a.s.x) + t * a.s.x_stride, c, D), x);
        widen(fetch(static_cast<const T*>(a.s.gate) + t * a.s.gate_stride, c, D), g);
        if (a.s.h0) widen(fetch(a.s.h0 + t * D, c, D), h);
#pragma unroll
        for (int k = 0; k < kChan; ++k) {
            float keep, take;
            gates(g[k], keep, take);
            y[k] = __builtin_fmaf(keep, h[k], take * x[k]);
        }
        put(static_cast<T*>(a.y) + t * a.y_stride, c, D, y);
        if (a.h_last) put(a.h_last + t * D, c, D, y);
    }
}

// A launch's most blocks of elementwise kernels, which loop over the rest.
constexpr int64_t kStepBlocks = int64_t{1} << 20;

// No tokens at all: what reaches each sequence leaves it.
__global__ __launch_bounds__(kStepThreads) void empty_kernel(const float* from, float* to, int64_t n)
{
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kStepThreads + threadIdx.x; i < n;
         i += static_cast<int64_t>(gridDim.x) * kStepThreads)
        to[i] = from ? from[i] : 0.0f;
}

hipError_t pass_all(const gem_scan& s, const float* from, float* to, hipStream_t stream)
{
    const int64_t n = static_cast<int64_t>(s.sequences) * s.channels;
    if (!to || from == to) return hipSuccess;
    const int64_t blocks = (n + kStepThreads - 1) / kStepThreads;
    hipLaunchKernelGGL(empty_kernel, dim3(static_cast<unsigned>(blocks < kStepBlocks ? blocks : kStepBlocks)), dim3(kStepThreads), 0,
                       stream, from, to, n);
    return hipGetLastError();
}

int64_t tiles_of(int64_t tokens) { return (tokens + kScanTile - 1) / kScanTile; }
int64_t slices_of(int64_t channels) { return (channels + kSlice - 1) / kSlice; }

Chain chain_of(const gem_scan& s, const OpsDevice& d)
{
    Chain ch;
    ch.tiles = static_cast<int>(tiles_of(s.tokens));
    ch.slices = static_cast<int>(slices_of(s.channels));
    ch.total = static_cast<int64_t>(ch.tiles) * ch.slices;
    ch.counters = static_cast<ScanCounters*>(d.counters);
    ch.words = static_cast<TileWords*>(d.scan);
    ch.hints = reinterpret_cast<uint64_t*>(ch.words + ch.total);
    return ch;
}

unsigned blocks_of(const Chain& ch, const OpsDevice& d, int per_cu)
{
    if (ch.tiles == 1) return static_cast<unsigned>(ch.total);
    const int64_t most = static_cast<int64_t>(d.cus) * per_cu;
    return static_cast<unsigned>(ch.total < most ? ch.total : most);
}

}  // namespace

int64_t scan_tiles(int64_t tokens, int64_t channels) { return tiles_of(tokens) * slices_of(channels); }

int64_t scan_scratch_bytes(int64_t tokens, int64_t channels)
{
    const int64_t tiles = tiles_of(tokens);
    return tiles <= 1 ? 0 : tiles * slices_of(channels) * static_cast<int64_t>(sizeof(TileWords) + 8);
}

hipError_t launch_scan_forward(const ScanArgs& a, bool bf16, const OpsDevice& d, hipStream_t stream)
{
    if (a.s.tokens == 0) return pass_all(a.s, a.s.h0, a.h_last, stream);
    if (!a.s.offsets && a.s.tokens == a.s.sequences) {
        const int groups = (a.s.channels + kChan - 1) / kChan;
        const int64_t blocks = (a.s.tokens * groups + kStepThreads - 1) / kStepThreads;
        const dim3 grid(static_cast<unsigned>(blocks < kStepBlocks ? blocks : kStepBlocks));
        if (bf16) hipLaunchKernelGGL((step_kernel<uint16_t>), grid, dim3(kStepThreads), 0, stream, a, groups);
        else hipLaunchKernelGGL((step_kernel<float>), grid, dim3(kStepThreads), 0, stream, a, groups);
        return hipGetLastError();
    }
    const Chain ch = chain_of(a.s, d);
    const dim3 grid(blocks_of(ch, d, 2));
    if (bf16) hipLaunchKernelGGL((forward_kernel<uint16_t>), grid, dim3(kThreads), 0, stream, a, ch);
    else hipLaunchKernelGGL((forward_kernel<float>), grid, dim3(kThreads), 0, stream, a, ch);
    return hipGetLastError();
}

hipError_t launch_scan_backward(const ScanBackArgs& a, bool bf16, const OpsDevice& d, hipStream_t stream)
{
    if (a.s.tokens == 0) return pass_all(a.s, a.dh_last, a.dh0, stream);
    const Chain ch = chain_of(a.s, d);
    const dim3 grid(blocks_of(ch, d, 2));
    if (bf16) hipLaunchKernelGGL((backward_kernel<uint16_t>), grid, dim3(kThreads), 0, stream, a, ch);
    else hipLaunchKernelGGL((backward_kernel<float>), grid, dim3(kThreads), 0, stream, a, ch);
    return hipGetLastError();
}

}  // namespace gemk
