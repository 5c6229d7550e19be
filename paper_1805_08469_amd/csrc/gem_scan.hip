// gem_scan.hip -- the gated linear recurrence and its backward pass for gfx950.
//
// h_t = a_t h_{t-1} + (1 - a_t) x_t is a chain along the tokens, but any run of tokens is
// one map h -> A h + B, and maps compose.  The tokens are cut into runs; a row of 32 lanes
// (256 bytes of channels, 8 a lane) walks through one run with its state in registers.
// Three launches: the maps of all runs; their composition, which gives the state that
// reaches each run; and the walk again from that state, which writes the outputs.  So the
// inputs are read twice, the second time partly from the Infinity Cache, and nothing waits
// inside a launch: no row needs another's result.  Bytes bound it.
//
// (One launch that reads everything once, its blocks handing states to each other through
// memory, was slower: 168 us where this takes 137, 32768 x 2048 bfloat16 forward.  A
// state travels along a slice of channels at 4 tiles of 112 tokens a microsecond, by polls
// that each take about one.)
//
// A sequence's first token is a map that ignores h, so sequences of any number and lengths
// are runs like any other.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gem_ops.hpp"
#include "gem_ops_device.hpp"
#include "gem_rows_device.hpp"

namespace gemk {
namespace {

// A map that ignores h (a sequence begins in the run) has A = -0: gates are not negative, so
// no product of them is, and 0 h would be NaN where h is infinite.
constexpr float kCut = -0.0f;
__device__ __forceinline__ bool is_cut(float A) { return __float_as_int(A) < 0; }

// (A, B) after (A0, B0).
__device__ __forceinline__ void after(float& A, float& B, float A0, float B0)
{
    const bool cut = is_cut(A);
    B = cut ? B : __builtin_fmaf(A, B0, B);
    A = cut ? A : A * A0;
}
__device__ __forceinline__ float through(float A, float B, float h) { return is_cut(A) ? B : __builtin_fmaf(A, h, B); }

// ---- sequences ---------------------------------------------------------------------------

// A sequence of no tokens: what reached it leaves it.
template <int N>
__device__ __forceinline__ void pass_empty(const float* from, float* to, int64_t q, int channels, const Channels& o)
{
    if (!to) return;
    float v[N];
    fetch_or_zero(from, q, o, v);
    put_f32(to + q * channels, o, v);
}

// ---- a launch's rows ------------------------------------------------------------------

struct Runs {
    int len;                   // tokens of a run
    int count, slices;
    float* maps;               // [count][2][channels]: A, B
    float* reach;              // [count][channels]: the state before (behind) each run
    // h_last is h0's memory: a state that belongs there replaces the one that reached its run,
    // since the rows of the sequence's first tokens may still have to read h0 (ends_kernel).
    bool in_place;
};

struct Row {
    int run, slice;
    int t0, t1;                // its tokens
};
__device__ __forceinline__ bool row_of(const Runs& r, int tokens, Row& out)
{
    const uint32_t i = blockIdx.x * kRows + threadIdx.x / kLanes, run = i / static_cast<uint32_t>(r.slices);
    if (run >= static_cast<uint32_t>(r.count)) return false;
    out.run = static_cast<int>(run);
    out.slice = static_cast<int>(i - run * r.slices);
    out.t0 = out.run * r.len;
    out.t1 = tokens - out.t0 > r.len ? out.t0 + r.len : tokens;
    return true;
}

// kStep rows of an array from token t.  Steps of fewer tokens, and those in which a sequence
// begins or ends, are walked token by token, each row fetched as it comes: one path of
// unrolled loads and gates keeps the registers that two would share.
template <class T, int KIND>
__device__ __forceinline__ void fetch_rows(Raw<T> (&r)[kStep], const void* array, int64_t stride, int t, const Channels& o)
{
    const T* p = static_cast<const T*>(array) + t * stride;
#pragma unroll
    for (int i = 0; i < kStep; ++i) r[i] = fetch<T, KIND>(p + i * stride, o);
}

template <class T, int KIND>
__device__ __forceinline__ void fetch_row(float (&v)[kChan<T>], const void* array, int64_t stride, int t, const Channels& o)
{
    const Raw<T> r = fetch<T, KIND>(static_cast<const T*>(array) + t * stride, o);
    widen(r[0], r[1], v);
}

// ---- forward ---------------------------------------------------------------------------

// OUT: the outputs, from the states that reach the runs; else the runs' maps.  32768 x 2048
// bfloat16 in eight sequences: the maps 53 us (5.1 TB/s).
template <class T, bool OUT, int KIND>
__global__ __launch_bounds__(kThreads) void forward_kernel(const ScanArgs a, const Runs runs, const Bounds bound)
{
    constexpr int C = kChan<T>;
    Row row;
    if (!row_of(runs, static_cast<int>(a.s.tokens), row)) return;
    const int D = a.s.channels;
    const Channels o = channels_of<T>(D, row.slice);
    if (idle<T>(o)) return;
    const bool all = whole<T>(o);
    float A[C], B[C];          // the map of the tokens so far, or (B alone) the state
#pragma unroll
    for (int k = 0; k < C; ++k) A[k] = 1.0f;
    Raw<T> x[kStep], g[kStep];
    const auto load = [&](int t) {
        if (t + kStep > row.t1) return;
        fetch_rows<T, KIND>(x, a.s.x, a.s.x_stride, t, o);
        fetch_rows<T, KIND>(g, a.s.gate, a.s.gate_stride, t, o);
    };
    load(row.t0);
    fetch_or_zero(OUT && row.run > 0 ? runs.reach : nullptr, row.run, o, B);
    // The sequence of the current token, and where the next begins (here, with the first).
    int q = bound.at(row.t0);
    bool begins = bound(q) == row.t0;
    int next = begins ? row.t0 : bound(q + 1);
    float* end_of_first = OUT && a.h_last ? a.h_last + static_cast<int64_t>(q) * D : nullptr;
    if (OUT && runs.in_place && !begins) end_of_first = runs.reach + static_cast<int64_t>(row.run) * D;
    const int first = q;
    if (OUT && begins)
        for (int e = q - 1; e >= 0 && bound(e) >= row.t0; --e) pass_empty<C>(a.s.h0, a.h_last, e, D, o);
    const auto token = [&](const float (&xi)[C], const float (&gi)[C]) {
#pragma unroll
        for (int k = 0; k < C; ++k) {
            float keep, take;
            gates(gi[k], keep, take);
            B[k] = __builtin_fmaf(keep, B[k], take * xi[k]);
            if (!OUT) A[k] *= keep;
        }
    };
    for (int t = row.t0; t < row.t1; t += kStep) {
        if (OUT && a.states) put_f32(a.states + static_cast<int64_t>(t / kStateTokens) * D, o, B);
        T* y = static_cast<T*>(a.y) + t * a.y_stride;
        if (next > t + kStep && t + kStep <= row.t1) {     // nothing begins or ends here
            Raw<T> out[kStep];
#pragma unroll
            for (int i = 0; i < kStep; ++i) {
                float xi[C], gi[C];
                widen(x[i][0], x[i][1], xi);
                widen(g[i][0], g[i][1], gi);
                token(xi, gi);
                if (OUT) out[i] = narrow<T>(B);
            }
            load(t + kStep);
            if (OUT)
#pragma unroll
                for (int i = 0; i < kStep; ++i) put<T, KIND>(y + i * a.y_stride, o, all, out[i]);
            continue;
        }
        const int end = t + kStep < row.t1 ? t + kStep : row.t1;
#pragma unroll 1
        for (int u = t; u < end; ++u) {
            float xi[C], gi[C];
            fetch_row<T, KIND>(xi, a.s.x, a.s.x_stride, u, o);
            fetch_row<T, KIND>(gi, a.s.gate, a.s.gate_stride, u, o);
            if (u == next) {
                const int old = q;
                while (!begins && q + 1 < bound.n && bound(q + 1) <= u) ++q;
                if (OUT)
                    for (int e = old + 1; e < q; ++e) pass_empty<C>(a.s.h0, a.h_last, e, D, o);
                begins = false;
                next = bound(q + 1);
                fetch_or_zero(a.s.h0, q, o, B);
#pragma unroll
                for (int k = 0; k < C; ++k) A[k] = kCut;
            }
            token(xi, gi);
            if (OUT) {
                put<T, KIND>(y + (u - t) * a.y_stride, o, all, narrow<T>(B));
                if (a.h_last && u + 1 == next)
                    put_f32(q == first ? end_of_first : a.h_last + static_cast<int64_t>(q) * D, o, B);
            }
        }
        load(t + kStep);
    }
    if (!OUT) {
        put_f32(runs.maps + (static_cast<int64_t>(row.run) * 2) * D, o, A);
        put_f32(runs.maps + (static_cast<int64_t>(row.run) * 2 + 1) * D, o, B);
    } else if (row.t1 == a.s.tokens) {
        for (int e = q + 1; e < bound.n; ++e)
            if (bound(e) >= row.t1) pass_empty<C>(a.s.h0, a.h_last, e, D, o);
    }
}

// The ends of sequences that began in an earlier run, which forward_kernel left in the place of
// the states that reached their last runs.
__global__ __launch_bounds__(kThreads) void ends_kernel(const Runs r, const Bounds bound, int channels, float* h_last)
{
    const int64_t n = static_cast<int64_t>(bound.n) * channels;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n;
         i += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int q = static_cast<int>(i / channels);
        const int begin = bound(q), end = bound(q + 1);
        if (end <= begin) continue;
        const int run = (end - 1) / r.len;
        if (run < r.count && begin / r.len < run)
            h_last[i] = r.reach[static_cast<int64_t>(run) * channels + (i - static_cast<int64_t>(q) * channels)];
    }
}

// ---- the states between runs ---------------------------------------------------------------

// Block: 16 channels; a thread takes kFold consecutive runs of one channel in registers, 64
// threads a channel, so one round covers 512 runs; UP in order, else from the last.
constexpr int kFoldChan = 16, kFoldParts = 64, kFold = 8;
constexpr int kFoldThreads = kFoldChan * kFoldParts;

template <bool UP>
__global__ __launch_bounds__(kFoldThreads) void fold_kernel(const Runs r, int channels)
{
    __shared__ float sA[kFoldParts][kFoldChan], sB[kFoldParts][kFoldChan];
    const int c = blockIdx.x * kFoldChan + threadIdx.x % kFoldChan, part = threadIdx.x / kFoldChan;
    const bool in = c < channels;
    float h = 0.0f;            // the state that reaches the round
    for (int base = 0; base < r.count; base += kFoldParts * kFold) {
        float A[kFold], B[kFold];
#pragma unroll
        for (int i = 0; i < kFold; ++i) {
            const int at = base + part * kFold + i;        // in the order of the chain
            const int64_t run = UP ? at : r.count - 1 - at;
            const bool there = in && at < r.count;
            A[i] = there ? r.maps[run * 2 * channels + c] : 1.0f;
            B[i] = there ? r.maps[(run * 2 + 1) * channels + c] : 0.0f;
        }
        float a = A[0], b = B[0];
#pragma unroll
        for (int i = 1; i < kFold; ++i) {
            float a1 = A[i], b1 = B[i];
            after(a1, b1, a, b);
            a = a1;
            b = b1;
        }
        // Join the parts: each round doubles what a part's map covers.
        for (int s = 1; s < kFoldParts; s *= 2) {
            sA[part][threadIdx.x % kFoldChan] = a;
            sB[part][threadIdx.x % kFoldChan] = b;
            __syncthreads();
            if (part >= s) after(a, b, sA[part - s][threadIdx.x % kFoldChan], sB[part - s][threadIdx.x % kFoldChan]);
            __syncthreads();
        }
        sA[part][threadIdx.x % kFoldChan] = a;
        sB[part][threadIdx.x % kFoldChan] = b;
        __syncthreads();
        float now = part ? through(sA[part - 1][threadIdx.x % kFoldChan], sB[part - 1][threadIdx.x % kFoldChan], h) : h;
        h = through(sA[kFoldParts - 1][threadIdx.x % kFoldChan], sB[kFoldParts - 1][threadIdx.x % kFoldChan], h);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kFold; ++i) {
            const int at = base + part * kFold + i;
            const int64_t run = UP ? at : r.count - 1 - at;
            if (in && at < r.count) r.reach[run * channels + c] = now;
            now = through(A[i], B[i], now);
        }
    }
}

// ---- backward ------------------------------------------------------------------------------

// With e_t = a_t r_t, what a token hands to the one before it, e_t = a_t e_{t+1} + a_t dy_t
// is the same kind of chain from the last token to the first.
template <class T, int KIND>
__global__ __launch_bounds__(kThreads) void backward_map_kernel(const ScanBackArgs a, const Runs runs, const Bounds bound)
{
    constexpr int C = kChan<T>;
    Row row;
    if (!row_of(runs, static_cast<int>(a.s.tokens), row)) return;
    const int D = a.s.channels;
    const Channels o = channels_of<T>(D, row.slice);
    if (idle<T>(o)) return;
    float A[C], B[C];
#pragma unroll
    for (int k = 0; k < C; ++k) {
        A[k] = 1.0f;
        B[k] = 0.0f;
    }
    int t = row.t0 + (row.t1 - 1 - row.t0) / kStep * kStep;
    Raw<T> g[kStep], dy[kStep];
    const auto load = [&](int t) {
        if (t < row.t0 || t + kStep > row.t1) return;
        fetch_rows<T, KIND>(g, a.s.gate, a.s.gate_stride, t, o);
        fetch_rows<T, KIND>(dy, a.dy, a.dy_stride, t, o);
    };
    load(t);
    // The sequence of the current token, and where it ends.
    int q = bound.at(row.t1 - 1);
    int begin = bound(q), end = bound(q + 1);
    const auto token = [&](const float (&gi)[C], const float (&di)[C]) {
#pragma unroll
        for (int k = 0; k < C; ++k) {
            float keep, take;
            gates(gi[k], keep, take);
            B[k] = keep * (di[k] + B[k]);
            A[k] *= keep;
        }
    };
    for (; t >= row.t0; t -= kStep) {
        if (begin <= t && end > t + kStep && t + kStep <= row.t1) {
#pragma unroll
            for (int i = kStep - 1; i >= 0; --i) {
                float gi[C], di[C];
                widen(g[i][0], g[i][1], gi);
                widen(dy[i][0], dy[i][1], di);
                token(gi, di);
            }
            load(t - kStep);
            continue;
        }
#pragma unroll 1
        for (int u = (t + kStep < row.t1 ? t + kStep : row.t1) - 1; u >= t; --u) {
            float gi[C], di[C];
            fetch_row<T, KIND>(gi, a.s.gate, a.s.gate_stride, u, o);
            fetch_row<T, KIND>(di, a.dy, a.dy_stride, u, o);
            if (u < begin) {
                end = begin;
                while (q > 0 && begin > u) begin = bound(--q);
            }
            if (u + 1 == end) {
                fetch_or_zero(a.dh_last, q, o, B);
#pragma unroll
                for (int k = 0; k < C; ++k) A[k] = kCut;
            }
            token(gi, di);
        }
        load(t - kStep);
    }
    put_f32(runs.maps + (static_cast<int64_t>(row.run) * 2) * D, o, A);
    put_f32(runs.maps + (static_cast<int64_t>(row.run) * 2 + 1) * D, o, B);
}

// The gradients, kStep tokens at a time from the run's last: h from the state that forward
// kept for them, then e from behind.  Keeping every eighth state costs a sixteenth of the
// traffic, and saves walking from the run's first token or keeping h in the inputs' type.
// Forward and backward of 32768 x 2048 bfloat16 take 337 us in their six launches (the bytes
// alone, with x read three times and the gate four, 266 us at a copy's rate).
template <class T, int KIND>
__global__ __launch_bounds__(kThreads, 2) void backward_kernel(const ScanBackArgs a, const Runs runs, const Bounds bound)
{
    constexpr int C = kChan<T>;
    __shared__ float before[kStep][C][kThreads];       // h_{t-1} of a step walked token by token
    Row row;
    if (!row_of(runs, static_cast<int>(a.s.tokens), row)) return;
    const int D = a.s.channels;
    const Channels o = channels_of<T>(D, row.slice);
    if (idle<T>(o)) return;
    const bool all = whole<T>(o);
    float back[C];
    fetch_or_zero(row.run + 1 < runs.count ? runs.reach : nullptr, row.run, o, back);
    int q = bound.at(row.t1 - 1);
    int begin = bound(q), end = bound(q + 1);
    if (row.t1 == a.s.tokens)
        for (int e = q + 1; e < bound.n; ++e)
            if (bound(e) >= row.t1) pass_empty<C>(a.dh_last, a.dh0, e, D, o);
    for (int t = row.t0 + (row.t1 - 1 - row.t0) / kStep * kStep; t >= row.t0; t -= kStep) {
        float h[C];
        fetch_f32(a.states + static_cast<int64_t>(t / kStateTokens) * D, o, h);
        T* px = static_cast<T*>(a.dx) + t * a.dx_stride;
        T* pg = static_cast<T*>(a.dgate) + t * a.dgate_stride;
        if (begin < t && end > t + kStep && t + kStep <= row.t1) {     // nothing begins or ends here
            Raw<T> x[kStep], g[kStep], dy[kStep];
            // f: a_t (1 - a_t) (h_{t-1} - x_t)
            float keep[kStep][C], take[kStep][C], f[kStep][C];
            fetch_rows<T, KIND>(g, a.s.gate, a.s.gate_stride, t, o);
            fetch_rows<T, KIND>(x, a.s.x, a.s.x_stride, t, o);
            fetch_rows<T, KIND>(dy, a.dy, a.dy_stride, t, o);
#pragma unroll
            for (int i = 0; i < kStep; ++i) {
                float xi[C], gi[C];
                widen(x[i][0], x[i][1], xi);
                widen(g[i][0], g[i][1], gi);
#pragma unroll
                for (int k = 0; k < C; ++k) {
                    gates(gi[k], keep[i][k], take[i][k]);
                    f[i][k] = keep[i][k] * take[i][k] * (h[k] - xi[k]);
                    h[k] = __builtin_fmaf(keep[i][k], h[k], take[i][k] * xi[k]);
                }
            }
#pragma unroll
            for (int i = kStep - 1; i >= 0; --i) {
                float di[C], dx[C], dg[C];
                widen(dy[i][0], dy[i][1], di);
#pragma unroll
                for (int k = 0; k < C; ++k) {
                    const float r = di[k] + back[k];
                    dx[k] = take[i][k] * r;
                    dg[k] = f[i][k] * r;
                    back[k] = keep[i][k] * r;
                }
                put<T, KIND>(px + i * a.dx_stride, o, all, narrow<T>(dx));
                put<T, KIND>(pg + i * a.dgate_stride, o, all, narrow<T>(dg));
            }
            continue;
        }
        const int stop = t + kStep < row.t1 ? t + kStep : row.t1;
        // The sequence of token t, and where the next begins (here, with the first).
        int s = q, from = begin;
        while (s > 0 && from > t) from = bound(--s);
        bool begins = from == t;
        int next = begins ? t : bound(s + 1);
#pragma unroll 1
        for (int u = t; u < stop; ++u) {
            float xi[C], gi[C];
            fetch_row<T, KIND>(gi, a.s.gate, a.s.gate_stride, u, o);
            fetch_row<T, KIND>(xi, a.s.x, a.s.x_stride, u, o);
            if (u == next) {
                while (!begins && s + 1 < bound.n && bound(s + 1) <= u) ++s;
                begins = false;
                next = bound(s + 1);
                fetch_or_zero(a.s.h0, s, o, h);
            }
#pragma unroll
            for (int k = 0; k < C; ++k) {
                float keep, take;
                gates(gi[k], keep, take);
                before[u - t][k][threadIdx.x] = h[k];
                h[k] = __builtin_fmaf(keep, h[k], take * xi[k]);
            }
        }
#pragma unroll 1
        for (int u = stop - 1; u >= t; --u) {
            float xi[C], gi[C], di[C], dx[C], dg[C];
            fetch_row<T, KIND>(gi, a.s.gate, a.s.gate_stride, u, o);
            fetch_row<T, KIND>(xi, a.s.x, a.s.x_stride, u, o);
            fetch_row<T, KIND>(di, a.dy, a.dy_stride, u, o);
            if (u < begin) {
                const int old = q;
                end = begin;
                while (q > 0 && begin > u) begin = bound(--q);
                for (int e = q + 1; e < old; ++e) pass_empty<C>(a.dh_last, a.dh0, e, D, o);
            }
            if (u + 1 == end) fetch_or_zero(a.dh_last, q, o, back);
#pragma unroll
            for (int k = 0; k < C; ++k) {
                float keep, take;
                gates(gi[k], keep, take);
                const float r = di[k] + back[k];
                dx[k] = take * r;
                dg[k] = keep * take * (before[u - t][k][threadIdx.x] - xi[k]) * r;
                back[k] = keep * r;
            }
            put<T, KIND>(px + (u - t) * a.dx_stride, o, all, narrow<T>(dx));
            put<T, KIND>(pg + (u - t) * a.dgate_stride, o, all, narrow<T>(dg));
            if (a.dh0 && u == begin) put_f32(a.dh0 + static_cast<int64_t>(q) * D, o, back);
        }
    }
    // Empty sequences ahead of one that begins with the run.
    if (begin == row.t0)
        for (int e = q - 1; e >= 0 && bound(e) >= row.t0; --e) pass_empty<C>(a.dh_last, a.dh0, e, D, o);
}

// ---- single tokens, no tokens ----------------------------------------------------------------

// One token a sequence: no chain, one launch, which is what it costs (64 x 4096 bfloat16 5.5 us).
template <class T, int KIND>
__global__ __launch_bounds__(kThreads) void step_kernel(const ScanArgs a, int slices)
{
    constexpr int C = kChan<T>;
    const int D = a.s.channels;
    const int64_t rows = a.s.tokens * slices;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / kLanes; i < rows;
         i += static_cast<int64_t>(gridDim.x) * kRows) {
        const int64_t t = i / slices;
        const Channels o = channels_of<T>(D, static_cast<int>(i - t * slices));
        if (idle<T>(o)) continue;
        float x[C], g[C], h[C];
        const Raw<T> rx = fetch<T, KIND>(static_cast<const T*>(a.s.x) + t * a.s.x_stride, o);
        const Raw<T> rg = fetch<T, KIND>(static_cast<const T*>(a.s.gate) + t * a.s.gate_stride, o);
        fetch_or_zero(a.s.h0, t, o, h);
        if (a.states && t % kStateTokens == 0) put_f32(a.states + t / kStateTokens * D, o, h);
        widen(rx[0], rx[1], x);
        widen(rg[0], rg[1], g);
#pragma unroll
        for (int k = 0; k < C; ++k) {
            float keep, take;
            gates(g[k], keep, take);
            h[k] = __builtin_fmaf(keep, h[k], take * x[k]);
        }
        put<T, KIND>(static_cast<T*>(a.y) + t * a.y_stride, o, whole<T>(o), narrow<T>(h));
        if (a.h_last) put_f32(a.h_last + t * D, o, h);
    }
}

// No tokens at all: what reaches each sequence leaves it.
__global__ __launch_bounds__(kThreads) void empty_kernel(const float* from, float* to, int64_t n)
{
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n;
         i += static_cast<int64_t>(gridDim.x) * kThreads)
        to[i] = from ? from[i] : 0.0f;
}

// ---- launches ----------------------------------------------------------------------

hipError_t pass_all(const gem_scan& s, const float* from, float* to, hipStream_t stream)
{
    const int64_t n = static_cast<int64_t>(s.sequences) * s.channels;
    if (!to || from == to) return hipSuccess;
    hipLaunchKernelGGL(empty_kernel, loop_grid(over(n, kThreads)), dim3(kThreads), 0, stream, from, to, n);
    return hipGetLastError();
}

// Tokens of a run: the most, up to 128, that leave the launches `least` rows of 32 lanes (eight
// to a compute unit at 2048).  Longer runs have fewer maps to write, join and read; fewer rows
// leave compute units idle.  us, by runs of 128 / 64 / 32: 32768 x 2048 bfloat16, both
// directions, 336 / 346 / 378; 65536 x 512 binary32 315 / 333 / 347; 16384 x 512 bfloat16 in
// two sequences 151 / 103 / 85 (512, 1024 and 2048 rows).  Forward, packed sequences are
// better with twice the rows, since a row in which they begin is walked token by token: 24 of
// 16384 x 2048 98 / 92 / 92 (2048, 4096 and 8192 rows); both directions of 8192 x 4096 are 188
// with 2048 rows, 205 with 4096, and 193 as it is.
constexpr int64_t kForwardRows = 4096, kBackwardRows = 2048;
constexpr int kRunMost = 128, kRunLeast = 16;
int run_len(int64_t tokens, int64_t slices, int64_t least)
{
    int len = kRunMost;
    while (len > kRunLeast && over(tokens, len) * slices < least) len /= 2;
    return len;
}
static_assert(kRunLeast % kStateTokens == 0, "runs begin where states are kept");

template <class T> Runs runs_of(const gem_scan& s, const OpsDevice& d, int64_t least)
{
    Runs r;
    r.slices = static_cast<int>(over(s.channels, kSlice<T>));
    r.len = run_len(s.tokens, r.slices, least);
    r.count = static_cast<int>(over(s.tokens, r.len));
    r.maps = static_cast<float*>(d.scan);
    r.reach = r.maps + static_cast<int64_t>(r.count) * 2 * s.channels;
    r.in_place = false;
    return r;
}
Bounds bounds_of(const gem_scan& s) { return {s.offsets, s.offsets ? 0 : s.tokens / s.sequences, s.sequences}; }
dim3 grid_of(const Runs& r) { return dim3(static_cast<unsigned>(over(static_cast<int64_t>(r.count) * r.slices, kRows))); }

template <bool UP> void fold(const Runs& r, int channels, hipStream_t stream)
{
    hipLaunchKernelGGL((fold_kernel<UP>), dim3(static_cast<unsigned>(over(channels, kFoldChan))), dim3(kFoldThreads), 0, stream,
                       r, channels);
}

template <class T, int KIND>
hipError_t forward(const ScanArgs& a, const OpsDevice& d, hipStream_t stream)
{
    Runs r = runs_of<T>(a.s, d, kForwardRows);
    if (!a.s.offsets && a.s.tokens == a.s.sequences) {
        hipLaunchKernelGGL((step_kernel<T, KIND>), loop_grid(over(a.s.tokens * r.slices, kRows)), dim3(kThreads), 0, stream, a,
                           r.slices);
        return hipGetLastError();
    }
    const Bounds b = bounds_of(a.s);
    if (r.count > 1) {
        hipLaunchKernelGGL((forward_kernel<T, false, KIND>), grid_of(r), dim3(kThreads), 0, stream, a, r, b);
        fold<true>(r, a.s.channels, stream);
    }
    r.in_place = r.count > 1 && a.h_last && a.h_last == a.s.h0;
    hipLaunchKernelGGL((forward_kernel<T, true, KIND>), grid_of(r), dim3(kThreads), 0, stream, a, r, b);
    if (r.in_place) {
        const int64_t n = static_cast<int64_t>(a.s.sequences) * a.s.channels;
        hipLaunchKernelGGL(ends_kernel, loop_grid(over(n, kThreads)), dim3(kThreads), 0, stream, r, b, a.s.channels, a.h_last);
    }
    return hipGetLastError();
}

template <class T, int KIND>
hipError_t backward(const ScanBackArgs& a, const OpsDevice& d, hipStream_t stream)
{
    const Runs r = runs_of<T>(a.s, d, kBackwardRows);
    const Bounds b = bounds_of(a.s);
    if (r.count > 1) {
        hipLaunchKernelGGL((backward_map_kernel<T, KIND>), grid_of(r), dim3(kThreads), 0, stream, a, r, b);
        fold<false>(r, a.s.channels, stream);
    }
    hipLaunchKernelGGL((backward_kernel<T, KIND>), grid_of(r), dim3(kThreads), 0, stream, a, r, b);
    return hipGetLastError();
}

struct Forward {
    template <class T, int KIND> static hipError_t launch(const ScanArgs& a, const OpsDevice& d, hipStream_t stream)
    {
        return forward<T, KIND>(a, d, stream);
    }
};
struct Backward {
    template <class T, int KIND> static hipError_t launch(const ScanBackArgs& a, const OpsDevice& d, hipStream_t stream)
    {
        return backward<T, KIND>(a, d, stream);
    }
};

template <class T, class F, class A> hipError_t by_channels(const A& a, const OpsDevice& d, hipStream_t stream)
{
    if (a.s.channels < kChan<T>) return F::template launch<T, kFew>(a, d, stream);
    if (a.s.channels % kChan<T>) return F::template launch<T, kOdd>(a, d, stream);
    return F::template launch<T, kEven>(a, d, stream);
}

}  // namespace

// The most rows of a launch (of the type with the narrower slices).
int64_t scan_rows(int64_t tokens, int64_t channels)
{
    const int64_t slices = over(channels, kSlice<float>);
    return over(tokens, run_len(tokens, slices, kForwardRows)) * slices;
}

// A run's A, B and state, of each channel.
constexpr int64_t kRunBytes = 3 * static_cast<int64_t>(sizeof(float));

// For the most runs: of the type with the wider slices, in the direction with the shorter runs.
int64_t scan_bytes(int64_t tokens, int64_t channels)
{
    const int64_t runs = over(tokens, run_len(tokens, over(channels, kSlice<uint16_t>), kForwardRows));
    return runs <= 1 ? 0 : runs * channels * kRunBytes;
}

// Enough for these sizes and all smaller ones.  Fewer tokens can have more runs, since those get
// shorter where the rows would be too few; but with runs of less than 128 tokens twice as long
// ones would leave less than kForwardRows rows, so that the runs' channels are fewer than those of
// 2 kForwardRows slices.
int64_t scan_scratch_bytes(int64_t tokens, int64_t channels)
{
    if (tokens <= kRunLeast) return 0;
    const int64_t longest = over(tokens, kRunMost) * channels, shortest = over(tokens, kRunLeast) * channels;
    const int64_t most = 2 * kForwardRows * kSlice<uint16_t>;
    const int64_t capped = shortest < most ? shortest : most;
    return (longest > capped ? longest : capped) * kRunBytes;
}

hipError_t launch_scan_forward(const ScanArgs& a, bool bf16, const OpsDevice& d, hipStream_t stream)
{
    if (a.s.tokens == 0) return pass_all(a.s, a.s.h0, a.h_last, stream);
    return bf16 ? by_channels<uint16_t, Forward>(a, d, stream) : by_channels<float, Forward>(a, d, stream);
}

hipError_t launch_scan_backward(const ScanBackArgs& a, bool bf16, const OpsDevice& d, hipStream_t stream)
{
    if (a.s.tokens == 0) return pass_all(a.s, a.dh_last, a.dh0, stream);
    return bf16 ? by_channels<uint16_t, Backward>(a, d, stream) : by_channels<float, Backward>(a, d, stream);
}

}  // namespace gemk
