// gem_conv.hip -- the short causal convolution of each channel along the tokens, with its
// activation, and its backward pass, for gfx950.
//
// c_t = bias + sum_j w_j x_{t-W+1+j}, y = c or c sigmoid(c).  A row of 32 lanes (256 bytes of
// channels, 8 a lane) walks through a run of tokens with the last W - 1 inputs in registers, so x is
// read once but for those ahead of a run.  Backward walks from a run's last token to its first with the
// last W - 1 of g_t = dy_t act'(c_t) in registers: dx_t = sum_k w_{W-1-k} g_{t+k}; the weights' gradients
// are sums over a run's tokens, which a second launch adds up.  Bytes bound both.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gem_ops.hpp"
#include "gem_ops_device.hpp"
#include "gem_rows_device.hpp"

namespace gemk {
namespace {

struct Runs {
    int len, count, slices;
    float* sums;               // [count][W + 1][channels]: the weights' gradients, the bias's
};
struct Row {
    int run, slice, t0, t1;
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

template <int W, int C> struct Weights {
    float w[W][C], bias[C];

    __device__ Weights(const gem_conv& s, const Channels& o)
    {
#pragma unroll
        for (int k = 0; k < C; ++k) {
            const int64_t c = o.c + k < s.channels ? o.c + k : s.channels - 1;
#pragma unroll
            for (int j = 0; j < W; ++j) w[j][k] = s.weight[c * W + j];
            bias[k] = s.bias ? s.bias[c] : 0.0f;
        }
    }
};

// What one token gives: x holds the inputs of its taps.
template <int W, int C, class X> __device__ __forceinline__ void convolve(const Weights<W, C>& w, X x, float (&c)[C])
{
#pragma unroll
    for (int k = 0; k < C; ++k) {
        c[k] = w.bias[k];
#pragma unroll
        for (int j = 0; j < W; ++j) c[k] = __builtin_fmaf(w.w[j][k], x(j)[k], c[k]);
    }
}
template <int C> __device__ __forceinline__ void activate(bool act, float (&c)[C])
{
    if (!act) return;
#pragma unroll
    for (int k = 0; k < C; ++k) {
        float s, t;
        gates(c[k], s, t);
        c[k] *= s;
    }
}
// dy times the activation's derivative, s + c s (1 - s).
template <int C> __device__ __forceinline__ void slope(bool act, const float (&c)[C], float (&g)[C])
{
    if (!act) return;
#pragma unroll
    for (int k = 0; k < C; ++k) {
        float s, t;
        gates(c[k], s, t);
        g[k] *= __builtin_fmaf(c[k] * t, s, s);
    }
}

// The sequence of a token, as far as the taps need it: its first token (none behind u) and the next
// one's.
struct Place {
    int q, begin, end;
};
__device__ __forceinline__ Place place_of(const Bounds& bound, int q, int u)
{
    Place p{q, bound(q), bound(q + 1)};
    if (p.begin > u) p.begin = u;
    if (p.end <= u) p.end = INT32_MAX;
    return p;
}

// Input s of a sequence; those ahead of it are in `before`.
template <class T, int KIND, int W>
__device__ __forceinline__ void input(const gem_conv& a, const Place& p, int s, const Channels& o, float (&v)[kChan<T>])
{
    if (s >= p.begin) {
        const Raw<T> r = fetch<T, KIND>(static_cast<const T*>(a.x) + s * a.x_stride, o);
        widen(r[0], r[1], v);
        return;
    }
    const int i = W - 1 + s - p.begin;
#pragma unroll
    for (int k = 0; k < kChan<T>; ++k) v[k] = 0.0f;
    if (!a.before || i < 0) return;
    const Raw<T> r = fetch<T, KIND>(static_cast<const T*>(a.before) + (static_cast<int64_t>(p.q) * (W - 1) + i) * a.channels, o);
    widen(r[0], r[1], v);
}

// ---- forward ---------------------------------------------------------------------------

// 32768 x 2048 bfloat16 in eight sequences, four taps: 54 us (5.1 TB/s).
template <class T, int KIND, int W>
__global__ __launch_bounds__(kThreads) void forward_kernel(const ConvArgs a, const Runs runs, const Bounds bound)
{
    constexpr int C = kChan<T>;
    Row row;
    if (!row_of(runs, static_cast<int>(a.s.tokens), row)) return;
    const Channels o = channels_of<T>(a.s.channels, row.slice);
    if (idle<T>(o)) return;
    const bool all = whole<T>(o);
    const T* x = static_cast<const T*>(a.s.x);
    T* y = static_cast<T*>(a.y);
    Raw<T> next[kStep];
    const auto load = [&](int t) {
        if (t + kStep > row.t1) return;
#pragma unroll
        for (int i = 0; i < kStep; ++i) next[i] = fetch<T, KIND>(x + (t + i) * a.s.x_stride, o);
    };
    load(row.t0);
    const Weights<W, C> w(a.s, o);
    float past[W][C];          // the inputs of the last W - 1 tokens, and one more
    Place p = place_of(bound, bound.at(row.t0), row.t0);
    const auto begin = [&](int u) {
#pragma unroll
        for (int j = 0; j + 1 < W; ++j) input<T, KIND, W>(a.s, p, u - (W - 1) + j, o, past[j]);
    };
    const auto token = [&](float (&c)[C]) {
        convolve(w, [&](int j) { return past[j]; }, c);
        activate(a.s.act != 0, c);
#pragma unroll
        for (int j = 0; j + 1 < W; ++j)
#pragma unroll
            for (int k = 0; k < C; ++k) past[j][k] = past[j + 1][k];
    };
    const auto advance = [&](int u) {
        int q = p.q;
        while (q + 1 < bound.n && bound(q + 1) <= u) ++q;
        p = place_of(bound, q, u);
        begin(u);
    };
    begin(row.t0);
    for (int t = row.t0; t < row.t1; t += kStep) {
        if (p.end <= t) advance(t);
        if (p.end >= t + kStep && t + kStep <= row.t1) {       // no sequence begins behind the first
            Raw<T> cur[kStep];
#pragma unroll
            for (int i = 0; i < kStep; ++i) cur[i] = next[i];
            load(t + kStep);
#pragma unroll
            for (int i = 0; i < kStep; ++i) {
                float c[C];
                widen(cur[i][0], cur[i][1], past[W - 1]);
                token(c);
                put<T, KIND>(y + (t + i) * a.y_stride, o, all, narrow<T>(c));
            }
            continue;
        }
        const int end = t + kStep < row.t1 ? t + kStep : row.t1;
#pragma unroll 1
        for (int u = t; u < end; ++u) {
            if (p.end <= u) advance(u);
            float c[C];
            const Raw<T> r = fetch<T, KIND>(x + u * a.s.x_stride, o);
            widen(r[0], r[1], past[W - 1]);
            token(c);
            put<T, KIND>(y + u * a.y_stride, o, all, narrow<T>(c));
        }
        load(t + kStep);
    }
}

// One token a sequence, with the inputs that stay behind it, in one launch, which is what it costs (64 x 4096
// bfloat16 5.5 us).
template <class T, int KIND, int W>
__global__ __launch_bounds__(kThreads) void step_kernel(const ConvArgs a, int slices)
{
    constexpr int C = kChan<T>;
    const int64_t rows = a.s.tokens * slices;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / kLanes; i < rows;
         i += static_cast<int64_t>(gridDim.x) * kRows) {
        const int64_t t = i / slices;
        const Channels o = channels_of<T>(a.s.channels, static_cast<int>(i - t * slices));
        if (idle<T>(o)) continue;
        const Weights<W, C> w(a.s, o);
        const T* before = static_cast<const T*>(a.s.before) + t * (W - 1) * a.s.channels;
        T* last = static_cast<T*>(a.last) + t * (W - 1) * a.s.channels;
        Raw<T> r[W];
#pragma unroll
        for (int j = 0; j + 1 < W; ++j) r[j] = a.s.before ? fetch<T, KIND>(before + j * a.s.channels, o) : Raw<T>{};
        r[W - 1] = fetch<T, KIND>(static_cast<const T*>(a.s.x) + t * a.s.x_stride, o);
        float x[W][C], c[C];
#pragma unroll
        for (int j = 0; j < W; ++j) widen(r[j][0], r[j][1], x[j]);
        convolve(w, [&](int j) { return x[j]; }, c);
        activate(a.s.act != 0, c);
        put<T, KIND>(static_cast<T*>(a.y) + t * a.y_stride, o, whole<T>(o), narrow<T>(c));
        if (a.last)
#pragma unroll
            for (int j = 0; j + 1 < W; ++j) put<T, KIND>(last + j * a.s.channels, o, whole<T>(o), r[j + 1]);
    }
}

// ---- what stays behind the sequences, and what is ahead of them ---------------------------

// A sequence's first token and the tokens it has.
struct Span {
    int64_t begin, len;
    __device__ Span(const Bounds& bound, int q, int64_t tokens) : begin(bound(q))
    {
        int64_t end = bound(q + 1);
        if (end > tokens) end = tokens;
        len = end > begin ? end - begin : 0;
    }
};

// Input i of [before, x] of a sequence, as its bits.
template <class T> __device__ __forceinline__ T bits_at(const gem_conv& s, const Span& p, int q, int W, int64_t i, int c)
{
    if (i >= W - 1) return static_cast<const T*>(s.x)[(p.begin + i - (W - 1)) * s.x_stride + c];
    return s.before ? static_cast<const T*>(s.before)[(static_cast<int64_t>(q) * (W - 1) + i) * s.channels + c] : T{};
}

// A thread's channel of a sequence: `last` may be `before`, whose inputs are read in front of where
// they are written.
template <class T>
__global__ __launch_bounds__(kThreads) void last_kernel(const ConvArgs a, const Bounds bound)
{
    const int W = a.s.width;
    const int64_t n = static_cast<int64_t>(a.s.sequences) * a.s.channels;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int q = static_cast<int>(i / a.s.channels), c = static_cast<int>(i - static_cast<int64_t>(q) * a.s.channels);
        const Span p(bound, q, a.s.tokens);
        T* to = static_cast<T*>(a.last) + static_cast<int64_t>(q) * (W - 1) * a.s.channels + c;
        for (int j = 0; j < W - 1; ++j) to[static_cast<int64_t>(j) * a.s.channels] = bits_at<T>(a.s, p, q, W, p.len + j, c);
    }
}

// The gradient of `before`: sum_j w_j g_{i-j} over the sequence's first tokens, whose g are formed again,
// and what `last` hands on where the sequence is shorter than that.
template <class T>
__global__ __launch_bounds__(kThreads) void before_kernel(const ConvBackArgs a, const Bounds bound)
{
    const int W = a.s.width;
    const int64_t n = static_cast<int64_t>(a.s.sequences) * a.s.channels;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int q = static_cast<int>(i / a.s.channels), c = static_cast<int>(i - static_cast<int64_t>(q) * a.s.channels);
        const Span p(bound, q, a.s.tokens);
        const float* w = a.s.weight + static_cast<int64_t>(c) * W;
        const int64_t at = static_cast<int64_t>(q) * (W - 1) * a.s.channels + c;
        for (int k = 0; k < W - 1; ++k) {
            float sum = 0.0f;
            if (a.dlast && k >= p.len) sum = load(static_cast<const T*>(a.dlast), at + (k - p.len) * a.s.channels);
            for (int t = 0; t <= k && t < p.len; ++t) {
                float v[1] = {a.s.bias ? a.s.bias[c] : 0.0f};
                for (int j = 0; j < W; ++j) {
                    const T x = bits_at<T>(a.s, p, q, W, t + j, c);
                    v[0] = __builtin_fmaf(w[j], load(&x, 0), v[0]);
                }
                float g[1] = {load(static_cast<const T*>(a.dy), (p.begin + t) * a.dy_stride + c)};
                slope(a.s.act != 0, v, g);
                sum = __builtin_fmaf(w[k - t], g[0], sum);
            }
            store(static_cast<T*>(a.dbefore), at + static_cast<int64_t>(k) * a.s.channels, sum);
        }
    }
}

// ---- backward ------------------------------------------------------------------------------

// The same sizes: 106 us, 4.0 TB/s; its vector instructions, 39 an element, take 73 of that.
// Tokens of a step: with eight the registers leave two waves a SIMD (32768 x 2048 bfloat16, both
// directions, 173 us; 164 with four).
constexpr int kBack = 4;

template <class T, int KIND, int W>
__global__ __launch_bounds__(kThreads, 3) void backward_kernel(const ConvBackArgs a, const Runs runs, const Bounds bound)
{
    constexpr int C = kChan<T>;
    Row row;
    if (!row_of(runs, static_cast<int>(a.s.tokens), row)) return;
    const int D = a.s.channels;
    const Channels o = channels_of<T>(D, row.slice);
    if (idle<T>(o)) return;
    const bool all = whole<T>(o), act = a.s.act != 0;
    const T* x = static_cast<const T*>(a.s.x);
    const T* dy = static_cast<const T*>(a.dy);
    T* dx = static_cast<T*>(a.dx);
    const Weights<W, C> w(a.s, o);
    float dw[W][C], db[C], ahead[W][C];        // ahead: g of the tokens behind this one, the next first
#pragma unroll
    for (int k = 0; k < C; ++k) {
        db[k] = 0.0f;
#pragma unroll
        for (int j = 0; j < W; ++j) dw[j][k] = ahead[j][k] = 0.0f;
    }
    Place p = place_of(bound, bound.at(row.t1 - 1), row.t1 - 1);
    // g of token u by itself.
    const auto alone = [&](int u, float (&xs)[W][C], float (&g)[C]) {
        float c[C];
#pragma unroll
        for (int j = 0; j < W; ++j) input<T, KIND, W>(a.s, p, u - (W - 1) + j, o, xs[j]);
        convolve(w, [&](int j) { return xs[j]; }, c);
        const Raw<T> r = fetch<T, KIND>(dy + u * a.dy_stride, o);
        widen(r[0], r[1], g);
        slope(act, c, g);
    };
#pragma unroll
    for (int j = 0; j + 1 < W; ++j) {          // those behind the run
        const int u = row.t1 + j;
        if (u >= p.end || u >= a.s.tokens) continue;
        float xs[W][C];
        alone(u, xs, ahead[j]);
    }
    // From g: the weights' gradients, and v, the token's input's.
    const auto token = [&](auto xs, const float (&g)[C], float (&v)[C]) {
#pragma unroll
        for (int k = 0; k < C; ++k) {
            db[k] += g[k];
            v[k] = w.w[W - 1][k] * g[k];
#pragma unroll
            for (int j = 0; j < W; ++j) dw[j][k] = __builtin_fmaf(g[k], xs(j)[k], dw[j][k]);
#pragma unroll
            for (int j = 0; j + 1 < W; ++j) v[k] = __builtin_fmaf(w.w[W - 2 - j][k], ahead[j][k], v[k]);
#pragma unroll
            for (int j = W - 2; j > 0; --j) ahead[j][k] = ahead[j - 1][k];
            ahead[0][k] = g[k];
        }
    };
    const int margin = a.dlast ? W - 1 : 0;
    Raw<T> xn[kBack], dn[kBack];               // of the step at hand, then of the one before it
    const auto load = [&](int t) {
        if (t + kBack > row.t1) return;
        const bool here = t >= row.t0;         // else the taps of the run's first tokens
#pragma unroll
        for (int i = kBack - 1; i >= 0; --i) {
            if (!here && i + W <= kBack) continue;
            xn[i] = fetch<T, KIND>(x + (t + i > 0 ? t + i : 0) * a.s.x_stride, o);
            if (here) dn[i] = fetch<T, KIND>(dy + (t + i) * a.dy_stride, o);
        }
    };
    int t = row.t0 + (row.t1 - 1 - row.t0) / kBack * kBack;
    load(t);
    for (; t >= row.t0; t -= kBack) {
        const int top = (t + kBack < row.t1 ? t + kBack : row.t1) - 1;
        if (p.begin > top) p = place_of(bound, bound.at(top), top);
        if (p.begin <= t - (W - 1) && p.end - margin >= t + kBack && t + kBack <= row.t1) {
            if (p.end == t + kBack)
#pragma unroll
                for (int j = 0; j < W; ++j)
#pragma unroll
                    for (int k = 0; k < C; ++k) ahead[j][k] = 0.0f;
            float xs[kBack + W - 1][C];
            Raw<T> dc[kBack];
#pragma unroll
            for (int i = 0; i < kBack; ++i) {
                widen(xn[i][0], xn[i][1], xs[i + W - 1]);
                dc[i] = dn[i];
            }
            load(t - kBack);
#pragma unroll
            for (int i = 0; i + 1 < W; ++i) widen(xn[kBack - (W - 1) + i][0], xn[kBack - (W - 1) + i][1], xs[i]);
#pragma unroll
            for (int i = kBack - 1; i >= 0; --i) {
                float c[C], g[C], v[C];
                convolve(w, [&](int j) { return xs[i + j]; }, c);
                widen(dc[i][0], dc[i][1], g);
                slope(act, c, g);
                token([&](int j) { return xs[i + j]; }, g, v);
                put<T, KIND>(dx + (t + i) * a.dx_stride, o, all, narrow<T>(v));
            }
            continue;
        }
#pragma unroll 1
        for (int u = top; u >= t; --u) {
            p = place_of(bound, bound.at(u), u);
            if (u + 1 == p.end)
#pragma unroll
                for (int j = 0; j < W; ++j)
#pragma unroll
                    for (int k = 0; k < C; ++k) ahead[j][k] = 0.0f;
            float xs[W][C], g[C], v[C];
            alone(u, xs, g);
            token([&](int j) { return xs[j]; }, g, v);
            const int at = u - p.end + (W - 1);
            if (a.dlast && at >= 0 && at < W - 1) {
                float e[C];
                const Raw<T> r = fetch<T, KIND>(static_cast<const T*>(a.dlast) + (static_cast<int64_t>(p.q) * (W - 1) + at) * D, o);
                widen(r[0], r[1], e);
#pragma unroll
                for (int k = 0; k < C; ++k) v[k] += e[k];
            }
            put<T, KIND>(dx + u * a.dx_stride, o, all, narrow<T>(v));
        }
        load(t - kBack);
    }
    float* sums = runs.sums + static_cast<int64_t>(row.run) * (W + 1) * D;
#pragma unroll
    for (int j = 0; j < W; ++j) put_f32(sums + static_cast<int64_t>(j) * D, o, dw[j]);
    put_f32(sums + static_cast<int64_t>(W) * D, o, db);
}

// The runs' sums, a column by four threads.
constexpr int kSumParts = 4, kSumCols = kThreads / kSumParts;

__global__ __launch_bounds__(kThreads) void sum_kernel(const ConvBackArgs a, const Runs runs)
{
    __shared__ float parts[kSumParts][kSumCols];
    const int W = a.s.width, part = threadIdx.x / kSumCols, lane = threadIdx.x % kSumCols;
    const int64_t n = static_cast<int64_t>(W + 1) * a.s.channels;
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * kSumCols; base < n; base += static_cast<int64_t>(gridDim.x) * kSumCols) {
        const int64_t i = base + lane < n ? base + lane : n - 1;
        float sum = 0.0f;
#pragma unroll 8
        for (int r = part; r < runs.count; r += kSumParts) sum += runs.sums[r * n + i];
        parts[part][lane] = sum;
        __syncthreads();
        if (part == 0 && base + lane < n) {
            sum = (parts[0][lane] + parts[1][lane]) + (parts[2][lane] + parts[3][lane]);
            const int64_t j = i / a.s.channels, c = i - j * a.s.channels;
            if (j < W && a.dweight) a.dweight[c * W + j] = sum;
            if (j == W && a.dbias) a.dbias[c] = sum;
        }
        __syncthreads();
    }
}

// ---- launches ----------------------------------------------------------------------

// Tokens of a run: the most that leave the launch `least` rows of 32 lanes.  us backward, with half of kBackwardRows,
// these and twice as many: 8192 x 2048 bfloat16 48, 40, 53; 16384 x 2048 77, 56, 73; 32768 x 512 52, 47, 70.  Forward
// they are within 3% (16384 x 2048 28.3, 28.7, 29.6).
constexpr int kForwardMost = 64, kBackwardMost = 128, kRunLeast = 16;
constexpr int64_t kForwardRows = 8192, kBackwardRows = 4096;
int run_len(int64_t tokens, int64_t slices, int most, int64_t least)
{
    int len = most;
    while (len > kRunLeast && over(tokens, len) * slices < least) len /= 2;
    return len;
}
template <class T> Runs runs_of(const gem_conv& s, int most, int64_t least)
{
    Runs r{};
    r.slices = static_cast<int>(over(s.channels, kSlice<T>));
    r.len = run_len(s.tokens, r.slices, most, least);
    r.count = static_cast<int>(over(s.tokens, r.len));
    return r;
}
Bounds bounds_of(const gem_conv& s) { return {s.offsets, s.offsets ? 0 : s.tokens / s.sequences, s.sequences}; }
dim3 grid_of(const Runs& r) { return dim3(static_cast<unsigned>(over(static_cast<int64_t>(r.count) * r.slices, kRows))); }

template <class T, int KIND, int W> struct Launch {
    static void forward(const ConvArgs& a, hipStream_t stream)
    {
        if (!a.s.offsets && a.s.tokens == a.s.sequences) {
            const int64_t slices = over(a.s.channels, kSlice<T>);
            hipLaunchKernelGGL((step_kernel<T, KIND, W>), loop_grid(over(a.s.tokens * slices, kRows)), dim3(kThreads), 0, stream, a,
                               static_cast<int>(slices));
            return;
        }
        const Runs r = runs_of<T>(a.s, kForwardMost, kForwardRows);
        if (r.count) hipLaunchKernelGGL((forward_kernel<T, KIND, W>), grid_of(r), dim3(kThreads), 0, stream, a, r, bounds_of(a.s));
        if (a.last && W > 1) {
            const int64_t n = static_cast<int64_t>(a.s.sequences) * a.s.channels;
            hipLaunchKernelGGL((last_kernel<T>), loop_grid(over(n, kThreads)), dim3(kThreads), 0, stream, a, bounds_of(a.s));
        }
    }
    static void backward(const ConvBackArgs& a, float* scratch, hipStream_t stream)
    {
        Runs r = runs_of<T>(a.s, kBackwardMost, kBackwardRows);
        r.sums = scratch;
        if (r.count) hipLaunchKernelGGL((backward_kernel<T, KIND, W>), grid_of(r), dim3(kThreads), 0, stream, a, r, bounds_of(a.s));
        if (a.dweight || a.dbias) {
            const int64_t n = static_cast<int64_t>(W + 1) * a.s.channels;
            hipLaunchKernelGGL(sum_kernel, loop_grid(over(n, kSumCols)), dim3(kThreads), 0, stream, a, r);
        }
        if (a.dbefore && W > 1) {
            const int64_t n = static_cast<int64_t>(a.s.sequences) * a.s.channels;
            hipLaunchKernelGGL((before_kernel<T>), loop_grid(over(n, kThreads)), dim3(kThreads), 0, stream, a, bounds_of(a.s));
        }
    }
};

// f(Launch<T, KIND, W>) for the sizes at hand.
template <class T, int KIND, class F> void by_width(int width, F f)
{
    if (width == 1) f(Launch<T, KIND, 1>{});
    else if (width == 2) f(Launch<T, KIND, 2>{});
    else if (width == 3) f(Launch<T, KIND, 3>{});
    else f(Launch<T, KIND, 4>{});
}
template <class T, class F> void by_channels(const gem_conv& s, F f)
{
    if (s.channels < kChan<T>) by_width<T, kFew>(s.width, f);
    else if (s.channels % kChan<T>) by_width<T, kOdd>(s.width, f);
    else by_width<T, kEven>(s.width, f);
}
template <class F> hipError_t launch(const gem_conv& s, bool bf16, F f)
{
    if (bf16) by_channels<uint16_t>(s, f);
    else by_channels<float>(s, f);
    return hipGetLastError();
}
static_assert(GEM_CONV_MAX == 4, "kernels of every width");

}  // namespace

// The most rows of a launch (of the type with the narrower slices).
int64_t conv_rows(int64_t tokens, int64_t channels)
{
    const int64_t slices = over(channels, kSlice<float>);
    return over(tokens, run_len(tokens, slices, kForwardMost, kForwardRows)) * slices;
}

// A run's sums: W + 1 of each channel.
constexpr int64_t kRunBytes = (GEM_CONV_MAX + 1) * static_cast<int64_t>(sizeof(float));

// Enough for these sizes and all smaller ones: runs of the most tokens, or shorter ones, of which
// there are fewer than twice kBackwardRows rows.
int64_t conv_scratch_bytes(int64_t tokens, int64_t channels)
{
    const int64_t longest = over(tokens, kBackwardMost) * channels, shortest = over(tokens, kRunLeast) * channels;
    const int64_t most = 2 * kBackwardRows * kSlice<uint16_t>;
    const int64_t capped = shortest < most ? shortest : most;
    return (longest > capped ? longest : capped) * kRunBytes;
}

hipError_t launch_conv_forward(const ConvArgs& a, bool bf16, hipStream_t stream)
{
    return launch(a.s, bf16, [&](auto l) { l.forward(a, stream); });
}

hipError_t launch_conv_backward(const ConvBackArgs& a, bool bf16, const OpsDevice& d, hipStream_t stream)
{
    return launch(a.s, bf16, [&](auto l) { l.backward(a, static_cast<float*>(d.scan), stream); });
}

}  // namespace gemk
