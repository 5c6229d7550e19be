// gem_ssm.hip -- the selective state space scan and its backward pass, for gfx950.
//
// With u_t = softplus(dt_t + bias), for each channel and each of its states n
//     h_t[n] = exp(u_t A[n]) h_{t-1}[n] + u_t B_t[n] x_t,   y_t = sum_n C_t[n] h_t[n] + D x_t  (times silu(z_t)):
// a chain along the tokens whose decays the data decide.  A step of one state takes six vector
// instructions (its decay's exponent and exponential, which counts twice, what comes in, the new state
// and its part of y), so instructions bound it, not bytes.
//
// A wave has 64 channels of a run of tokens.  Four lanes share four channels, and each has a quarter of
// their states: 16 states a lane in registers, as when a lane had one channel, but sums over states take
// two steps inside the four, sums over channels (of the gradients of B and C, which all channels share)
// begin inside a lane, and what is one value a channel (softplus, gates) is computed by one lane
// each and handed to the four by the lane crossbar.
//
// A run's tokens are one map h -> exp(A sum u) h + h', so runs are joined as in the gated recurrence: the
// maps of all runs, their composition, and the walk again from the state that reaches each run.  Runs
// that begin with a sequence need no maps.  Backward is the same from the last token: e_t = a_t (C_t dy_t +
// e_{t+1}), and forms four states at a time again from the one that forward kept for eight tokens.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "gem_ops.hpp"
#include "gem_ops_device.hpp"
#include "gem_rows_device.hpp"

namespace gemk {
namespace {

constexpr int kWave = 64;
constexpr int kWaves = kThreads / kWave;   // of a block, each with rows of its own
constexpr int kQuad = 4;                   // channels and lanes that belong together

// ---- lanes ---------------------------------------------------------------------------

template <int CTRL> __device__ __forceinline__ float moved(float v)
{
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xF, 0xF, true));
}
// Lane j's value of each four.
template <int J> __device__ __forceinline__ float of_lane(float v) { return moved<J * 0x55>(v); }
__device__ __forceinline__ void spread(float v, float (&out)[kQuad])
{
    out[0] = of_lane<0>(v);
    out[1] = of_lane<1>(v);
    out[2] = of_lane<2>(v);
    out[3] = of_lane<3>(v);
}
// Sums of v[j] over each four lanes, to lane j.
__device__ __forceinline__ float gather(const float (&v)[kQuad])
{
    const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
    const float a = (odd ? v[1] : v[0]) + moved<0xB1>(odd ? v[0] : v[1]);
    const float b = (odd ? v[3] : v[2]) + moved<0xB1>(odd ? v[2] : v[3]);
    return (high ? b : a) + moved<0x4E>(high ? a : b);
}

// ---- values --------------------------------------------------------------------------

// log(1 + exp(v)).  With E = exp(-|v|) it is max(v, 0) + log(1 + E), and log(1 + E) / E on [0, 1] is a
// polynomial interpolated at Chebyshev's points, right to 1.4 units of the last bit however small E is.
__device__ __forceinline__ float softplus(float v)
{
    const float E = __builtin_amdgcn_exp2f(__builtin_fabsf(v) * -kLog2e);
    float p = 0.005253457929939032f;
    p = __builtin_fmaf(p, E, -0.02958850748836994f);
    p = __builtin_fmaf(p, E, 0.07836166769266129f);
    p = __builtin_fmaf(p, E, -0.13674770295619965f);
    p = __builtin_fmaf(p, E, 0.19111430644989014f);
    p = __builtin_fmaf(p, E, -0.24844369292259216f);
    p = __builtin_fmaf(p, E, 0.33319270610809326f);
    p = __builtin_fmaf(p, E, -0.49999502301216125f);
    p = __builtin_fmaf(p, E, 1.0f);
    return (v > 0.0f ? v : 0.0f) + p * E;
}

// Element i of an array whose address is the wave's: a base in scalar registers, 32 bits of offset.
template <class T> __device__ __forceinline__ T* element(T* base, uint32_t i)
{
    return reinterpret_cast<T*>(reinterpret_cast<char*>(const_cast<std::remove_const_t<T>*>(base)) + i * static_cast<uint32_t>(sizeof(T)));
}

// ---- what a lane has --------------------------------------------------------------------

// A row's values of a lane's states, at any address of their own alignment.
template <class T, int S> struct __attribute__((packed, aligned(sizeof(T)))) Short {
    T v[S];
};

// Its own channel `mine` (of which it computes what is one value a channel), and states [n, n + S) of the
// four channels from `first` on.  FULL: there are 4 S states, so that a lane's are whole.
template <int S, bool FULL> struct Lane {
    int mine, first, D, N;
    uint32_t at, n;
    bool in, whole;            // whole: so has every lane of the wave

    // Where the lane stands, as something new: else the addresses of a loop's loads are all formed ahead of
    // it, 64 bits each, and spill.
    __device__ __forceinline__ void here() { asm volatile("" : "+v"(at), "+v"(n), "+v"(first)); }

    __device__ Lane(const gem_ssm& s, int slice)
    {
        const int lane = threadIdx.x % kWave;
        D = s.channels;
        N = s.state;
        mine = slice * kWave + lane;
        in = mine < D;
        whole = slice * kWave + kWave <= D;
        at = in ? mine : D - 1;
        first = slice * kWave + lane / kQuad * kQuad;
        n = lane % kQuad * S;
    }
    // Its states from [channels][N] values, zeros where there are none.
    __device__ __forceinline__ void get(const float* block, float (&h)[kQuad][S]) const
    {
#pragma unroll
        for (int j = 0; j < kQuad; ++j) {
            const bool there = first + j < D;
            const float* row = element(block, static_cast<uint32_t>(there ? first + j : D - 1) * N);
            if constexpr (FULL) {
                using V = float __attribute__((ext_vector_type(S), aligned(4)));
                const V v = *reinterpret_cast<const V*>(row + n);
#pragma unroll
                for (int s = 0; s < S; ++s) h[j][s] = there ? v[s] : 0.0f;
            } else {
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    const bool has = static_cast<int>(n) + s < N;
                    const float v = *element(row, has ? n + s : N - 1);
                    h[j][s] = there && has ? v : 0.0f;
                }
            }
        }
    }
    __device__ __forceinline__ void put(float* block, const float (&h)[kQuad][S]) const
    {
#pragma unroll
        for (int j = 0; j < kQuad; ++j) {
            if (first + j >= D) continue;
            float* row = element(block, static_cast<uint32_t>(first + j) * N);
            if constexpr (FULL) {
                using V = float __attribute__((ext_vector_type(S), aligned(4)));
                V v;
#pragma unroll
                for (int s = 0; s < S; ++s) v[s] = h[j][s];
                *reinterpret_cast<V*>(row + n) = v;
            } else {
#pragma unroll
                for (int s = 0; s < S; ++s)
                    if (static_cast<int>(n) + s < N) row[n + s] = h[j][s];
            }
        }
    }
    __device__ __forceinline__ void get_or_zero(const float* array, int64_t block, float (&h)[kQuad][S]) const
    {
        if (array) {
            get(array + block * D * N, h);
        } else {
#pragma unroll
            for (int j = 0; j < kQuad; ++j)
#pragma unroll
                for (int s = 0; s < S; ++s) h[j][s] = 0.0f;
        }
    }
    // Its states' values of B or C (a row of N) as they are, and as numbers.
    template <class T> __device__ __forceinline__ Short<T, S> shared(const void* array, int64_t stride, int t) const
    {
        const T* row = static_cast<const T*>(array) + t * stride;
        if constexpr (FULL) return *reinterpret_cast<const Short<T, S>*>(element(row, n));
        Short<T, S> r;
#pragma unroll
        for (int s = 0; s < S; ++s) r.v[s] = *element(row, static_cast<int>(n) + s < N ? n + s : N - 1);
        return r;
    }
    template <class T> __device__ __forceinline__ void numbers(const Short<T, S>& r, float (&v)[S]) const
    {
#pragma unroll
        for (int s = 0; s < S; ++s) v[s] = FULL || static_cast<int>(n) + s < N ? load(&r.v[s], 0) : 0.0f;
    }
    // Its channel's value; where it has none, the last channel's.
    template <class T> __device__ __forceinline__ T own(const void* array, int64_t stride, int t) const
    {
        return *element(static_cast<const T*>(array) + t * stride, at);
    }
    template <class T> __device__ __forceinline__ void write(void* array, int64_t stride, int t, float v) const
    {
        if (in) store(element(static_cast<T*>(array) + t * stride, at), 0, v);
    }
    __device__ __forceinline__ float weight(const float* w) const { return w && in ? w[at] : 0.0f; }
};

// ---- runs and sequences --------------------------------------------------------------------

struct Runs {
    int len, count, slices;
    bool whole;                // runs begin and end with sequences: no state passes between them
    bool in_place;             // h_last is h0's memory (ends_kernel)
    float* local;              // [count][D][N]: the state behind a run that nothing reaches
    float* steps;              // [count][D]: the sum of u over the run, -1: what reaches it ends in it
    float* reach;              // [count][D][N]: what reaches each run
    float* shared;             // [slices][tokens][2][NP]: the slices' parts of dB and dC
    float* params;             // [count][D][N], [count][2][D]: the runs' parts of dA, and of dD and the bias's
};
struct Row {
    int run, slice, t0, t1;
};
__device__ __forceinline__ bool row_of(const Runs& r, int tokens, Row& out)
{
    const uint32_t i = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const uint32_t run = i / static_cast<uint32_t>(r.slices);
    if (run >= static_cast<uint32_t>(r.count)) return false;
    out.run = static_cast<int>(run);
    // Blocks go to the eight dies in turn: turned by a block a run, slices visit all of them, and each
    // die's cache has all of its channels at work where rows are a power of two long.
    out.slice = static_cast<int>((i + kWaves * run) % static_cast<uint32_t>(r.slices));
    out.t0 = out.run * r.len;
    out.t1 = tokens - out.t0 > r.len ? out.t0 + r.len : tokens;
    return true;
}

constexpr int kSpan = 4;                   // tokens whose inputs a lane has at a time
static_assert(kStateTokens == 2 * kSpan, "every other span begins where a state is kept");

// A span's tokens: bits of those that are the run's, that begin a sequence, and that end one.  begin and end
// are those of a sequence that some token of the span before belongs to (the last one scanned): where it
// reaches over all of this span, nothing begins or ends here.
struct Window {
    uint32_t valid, starts, ends;
};
__device__ __forceinline__ Window window_of(const Bounds& bound, int w, const Row& row, int& begin, int& end)
{
    const int u0 = w > row.t0 ? w : row.t0, u1 = w + kSpan < row.t1 ? w + kSpan : row.t1;
    Window v{((1u << (u1 - w)) - 1) & ~((1u << (u0 - w)) - 1), 0, 0};
    if (begin < u0 && end > u1) return v;      // inside a sequence
    int q = bound.at(u0);
    begin = bound(q);
    end = bound(q + 1);
    for (int u = u0; u < u1; ++u) {
        if (u >= end && q + 1 < bound.n && bound(q + 1) <= u) {
            while (q + 1 < bound.n && bound(q + 1) <= u) ++q;
            begin = bound(q);
            end = bound(q + 1);
        }
        v.starts |= static_cast<uint32_t>(begin == u) << (u - w);
        v.ends |= static_cast<uint32_t>(end == u + 1) << (u - w);
    }
    return v;
}

// Which of a span's inputs a walk reads.
enum : int { kX = 1, kDt = 2, kZ = 4, kB = 8, kC = 16, kDy = 32 };

// A span's inputs, as they are (from load on, so that they may be on their way through the span before) and
// as numbers.  Tokens that are not the run's have those of its first or last.
template <class T, int S> struct Inputs {
    T x[kSpan], dt[kSpan], z[kSpan], dy[kSpan];
    Short<T, S> b[kSpan], c[kSpan];

    template <int WHAT, class O>
    __device__ __forceinline__ void load(O& o, const gem_ssm& s, const void* dys, int64_t dy_stride, const Row& row, int w)
    {
        o.here();
        // Without a gate x stands for it, unused: a load in a branch is waited for there.
        const void* gates_at = s.z ? s.z : s.x;
        const int64_t gates_stride = s.z ? s.z_stride : s.x_stride;
#pragma unroll
        for (int i = 0; i < kSpan; ++i) {
            int t = w + i < row.t1 ? w + i : row.t1 - 1;
            t = t > row.t0 ? t : row.t0;
            if constexpr (WHAT & kDt) dt[i] = o.template own<T>(s.dt, s.dt_stride, t);
            if constexpr (WHAT & kX) x[i] = o.template own<T>(s.x, s.x_stride, t);
            if constexpr (WHAT & kB) b[i] = o.template shared<T>(s.b, s.b_stride, t);
            if constexpr (WHAT & kC) c[i] = o.template shared<T>(s.c, s.c_stride, t);
            if constexpr (WHAT & kDy) dy[i] = o.template own<T>(dys, dy_stride, t);
            if constexpr (WHAT & kZ) z[i] = o.template own<T>(gates_at, gates_stride, t);
        }
    }
};
template <int S> struct Numbers {
    float x[kSpan], dt[kSpan], z[kSpan], dy[kSpan], B[kSpan][S], C[kSpan][S];

    template <int WHAT, class T, class O> __device__ __forceinline__ void of(const O& o, const Inputs<T, S>& r)
    {
#pragma unroll
        for (int i = 0; i < kSpan; ++i) {
            if constexpr (WHAT & kX) x[i] = load(&r.x[i], 0);
            if constexpr (WHAT & kDt) dt[i] = load(&r.dt[i], 0);
            if constexpr (WHAT & kZ) z[i] = load(&r.z[i], 0);
            if constexpr (WHAT & kDy) dy[i] = load(&r.dy[i], 0);
            if constexpr (WHAT & kB) o.numbers(r.b[i], B[i]);
            if constexpr (WHAT & kC) o.numbers(r.c[i], C[i]);
        }
    }
    // Nothing in lanes without a channel, whatever the last channel holds: u, the gate and all that follows are 0.
    template <int WHAT, class O> __device__ __forceinline__ void only_own(const O& o)
    {
        if (o.whole) return;
#pragma unroll
        for (int i = 0; i < kSpan; ++i) {
            x[i] = o.in ? x[i] : 0.0f;
            dt[i] = o.in ? dt[i] : -kInf;
            if constexpr (WHAT & kDy) dy[i] = o.in ? dy[i] : 0.0f;
            if constexpr (WHAT & kZ) z[i] = o.in ? z[i] : 0.0f;
        }
    }
};

// f(std::true_type) for a span that is all the run's and inside a sequence, which most are: there
// nothing stands in a branch.
template <class F> __device__ __forceinline__ void by_span(const Window& v, F f)
{
    if (v.valid == (1u << kSpan) - 1 && !(v.starts | v.ends)) f(std::true_type{});
    else f(std::false_type{});
}

// ---- forward ---------------------------------------------------------------------------

// OUT: the outputs, from the states that reach the runs; else the runs' maps.  32768 x 2048 x 16 bfloat16 in
// eight sequences: the maps 224 us, which is the time of their vector instructions (105 a token of 64
// channels, 16 of them exponentials), the outputs with the kept states 384 (305 of vector instructions).
template <class T, int S, bool FULL, bool OUT>
__global__ __launch_bounds__(kThreads, OUT ? 3 : 4) void forward_kernel(const SsmArgs a, const Runs runs, const Bounds bound)
{
    Row row;
    if (!row_of(runs, static_cast<int>(a.s.tokens), row)) return;
    Lane<S, FULL> o(a.s, row.slice);
    const int64_t DN = static_cast<int64_t>(o.D) * o.N;
    float A[kQuad][S], h[kQuad][S];
    o.get(a.s.a, A);
#pragma unroll
    for (int j = 0; j < kQuad; ++j)
#pragma unroll
        for (int s = 0; s < S; ++s) A[j][s] *= kLog2e;
    o.get_or_zero(OUT && row.run > 0 && !runs.whole ? runs.reach : nullptr, row.run, h);
    const float bias = o.weight(a.s.dt_bias), skip = o.weight(a.s.d);
    float steps = 0.0f;
    bool cut = false;          // a sequence has begun in the run
    int begin = 0, end = -1;
    constexpr int kWhat = OUT ? kX | kDt | kZ | kB | kC : kX | kDt | kB;
    Inputs<T, S> next;
    next.template load<kWhat>(o, a.s, nullptr, 0, row, row.t0 / kSpan * kSpan);
    for (int w = row.t0 / kSpan * kSpan; w < row.t1; w += kSpan) {
        Numbers<S> k;
        k.template of<kWhat>(o, next);
        if (w + kSpan < row.t1) next.template load<kWhat>(o, a.s, nullptr, 0, row, w + kSpan);
        const Window v = window_of(bound, w, row, begin, end);
        if (OUT && a.states && w % kStateTokens == 0 && (v.valid & 1)) o.put(a.states + static_cast<int64_t>(w / kStateTokens) * DN, h);
        by_span(v, [&](auto inside) {
        constexpr bool kInside = decltype(inside)::value;
#pragma unroll
        for (int i = 0; i < kSpan; ++i) {
            if (!kInside && !(v.valid >> i & 1)) continue;
            if (!kInside && (v.starts >> i & 1)) {
                o.get_or_zero(a.s.h0, bound.at(w + i), h);
                steps = 0.0f;
                cut = true;
            }
            const float u = softplus(k.dt[i] + bias);
            float us[kQuad], ins[kQuad], ys[kQuad];
            spread(u, us);
            spread(u * k.x[i], ins);
            if (!OUT) steps += u;
#pragma unroll
            for (int j = 0; j < kQuad; ++j) {
                ys[j] = 0.0f;
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    h[j][s] = __builtin_fmaf(__builtin_amdgcn_exp2f(us[j] * A[j][s]), h[j][s], ins[j] * k.B[i][s]);
                    if (OUT) ys[j] = __builtin_fmaf(k.C[i][s], h[j][s], ys[j]);
                }
            }
            if (!OUT) continue;
            float y = __builtin_fmaf(skip, k.x[i], gather(ys));
            if (a.s.z) {
                float g, r;
                gates(k.z[i], g, r);
                y *= k.z[i] * g;
            }
            o.template write<T>(a.y, a.y_stride, w + i, y);
            if (!kInside && a.h_last && (v.ends >> i & 1)) {
                // Rows of the sequence's first tokens may still have to read h0.
                if (runs.in_place && !cut) o.put(runs.reach + row.run * DN, h);
                else o.put(a.h_last + bound.at(w + i) * DN, h);
            }
        }
        });
    }
    if (!OUT) {
        o.put(runs.local + row.run * DN, h);
        if (o.in) runs.steps[static_cast<int64_t>(row.run) * o.D + o.mine] = cut ? -1.0f : steps;
    }
}

// One token a sequence: no chain, one launch, a wave for 64 channels of a sequence.  Bytes of the states bound
// it: 64 x 4096 x 16 bfloat16 7.5 us (4.8 TB/s); 8.5 with h0 asked for ahead of the rest.
template <class T, int S, bool FULL>
__global__ __launch_bounds__(kThreads) void step_kernel(const SsmArgs a, int slices)
{
    const int64_t rows = a.s.tokens * slices;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave); i < rows;
         i += static_cast<int64_t>(gridDim.x) * kWaves) {
        const int t = static_cast<int>(i / slices);
        Lane<S, FULL> o(a.s, static_cast<int>(i - static_cast<int64_t>(t) * slices));
        const int64_t DN = static_cast<int64_t>(o.D) * o.N;
        float A[kQuad][S], h[kQuad][S], B[S], C[S];
        const T xr = o.template own<T>(a.s.x, a.s.x_stride, t), dtr = o.template own<T>(a.s.dt, a.s.dt_stride, t);
        const T zr = a.s.z ? o.template own<T>(a.s.z, a.s.z_stride, t) : T{};
        const Short<T, S> br = o.template shared<T>(a.s.b, a.s.b_stride, t), cr = o.template shared<T>(a.s.c, a.s.c_stride, t);
        const float bias = o.weight(a.s.dt_bias), skip = o.weight(a.s.d);
        o.get(a.s.a, A);
        o.get_or_zero(a.s.h0, t, h);
        if (a.states && t % kStateTokens == 0) o.put(a.states + t / kStateTokens * DN, h);
        o.numbers(br, B);
        o.numbers(cr, C);
        const float x = load(&xr, 0), z = load(&zr, 0), u = softplus(load(&dtr, 0) + bias);
        float us[kQuad], ins[kQuad], ys[kQuad];
        spread(u, us);
        spread(u * x, ins);
#pragma unroll
        for (int j = 0; j < kQuad; ++j) {
            ys[j] = 0.0f;
#pragma unroll
            for (int s = 0; s < S; ++s) {
                h[j][s] = __builtin_fmaf(__builtin_amdgcn_exp2f(us[j] * (A[j][s] * kLog2e)), h[j][s], ins[j] * B[s]);
                ys[j] = __builtin_fmaf(C[s], h[j][s], ys[j]);
            }
        }
        if (a.h_last) o.put(a.h_last + t * DN, h);
        float y = __builtin_fmaf(skip, x, gather(ys));
        if (a.s.z) {
            float g, r;
            gates(z, g, r);
            y *= z * g;
        }
        o.template write<T>(a.y, a.y_stride, t, y);
    }
}

// Sequences without tokens, and ends that forward_kernel left in the place of what reached their
// runs: those of sequences that began in an earlier one.
__global__ __launch_bounds__(kThreads) void ends_kernel(const Runs r, const Bounds bound, int64_t DN, int64_t tokens, const float* h0,
                                                        float* h_last)
{
    const int64_t n = bound.n * DN;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int q = static_cast<int>(i / DN);
        const int begin = bound(q), end = bound(q + 1);
        if (end <= begin) {
            if (!r.in_place) h_last[i] = h0 ? h0[i] : 0.0f;
        } else if (r.in_place) {
            const int run = (end - 1) / r.len;
            if (end <= tokens && begin / r.len < run) h_last[i] = r.reach[run * DN + (i - q * DN)];
        }
    }
}

// ---- the states between runs ---------------------------------------------------------------

// Block: CHAINS chains (a channel's states); a thread takes kFold consecutive runs of one, PARTS threads a chain;
// UP in order, else from the last.  32 chains and 16 threads each go through 128 runs a round; with few channels
// runs are many, and 16 chains and 64 threads each go through 512.
constexpr int kFold = 8;

template <bool UP, int CHAINS, int PARTS>
__global__ __launch_bounds__(CHAINS * PARTS) void fold_kernel(const Runs r, const float* A, int D, int N)
{
    __shared__ float sa[PARTS][CHAINS], sb[PARTS][CHAINS];
    const int lane = threadIdx.x % CHAINS, part = threadIdx.x / CHAINS;
    const int64_t DN = static_cast<int64_t>(D) * N, chain = static_cast<int64_t>(blockIdx.x) * CHAINS + lane;
    const bool in = chain < DN;
    const int64_t c = in ? chain : 0;
    const float rate = A[c] * kLog2e;
    float h = 0.0f;            // what reaches the round
    // A map is (a, b); -1 for a: it ignores what reaches it.
    const auto through = [](float a, float b, float h) { return a < 0.0f ? b : __builtin_fmaf(a, h, b); };
    const auto after = [](float& a, float& b, float a0, float b0) {
        b = a < 0.0f ? b : __builtin_fmaf(a, b0, b);
        a = a < 0.0f ? a : a0 < 0.0f ? a0 : a * a0;
    };
    for (int base = 0; base < r.count; base += PARTS * kFold) {
        float a[kFold], b[kFold];
#pragma unroll
        for (int i = 0; i < kFold; ++i) {
            const int at = base + part * kFold + i;            // in the order of the chain
            const int64_t run = at >= r.count ? 0 : UP ? at : r.count - 1 - at;
            a[i] = r.steps[run * D + c / N];
            b[i] = r.local[run * DN + c];
        }
#pragma unroll
        for (int i = 0; i < kFold; ++i) {
            const bool there = base + part * kFold + i < r.count;
            a[i] = !there ? 1.0f : a[i] < 0.0f ? -1.0f : __builtin_amdgcn_exp2f(a[i] * rate);
            b[i] = there ? b[i] : 0.0f;
        }
        float ma = a[0], mb = b[0];
#pragma unroll
        for (int i = 1; i < kFold; ++i) {
            float na = a[i], nb = b[i];
            after(na, nb, ma, mb);
            ma = na;
            mb = nb;
        }
        for (int s = 1; s < PARTS; s *= 2) {              // each round doubles what a part's map covers
            sa[part][lane] = ma;
            sb[part][lane] = mb;
            __syncthreads();
            if (part >= s) after(ma, mb, sa[part - s][lane], sb[part - s][lane]);
            __syncthreads();
        }
        sa[part][lane] = ma;
        sb[part][lane] = mb;
        __syncthreads();
        float now = part ? through(sa[part - 1][lane], sb[part - 1][lane], h) : h;
        h = through(sa[PARTS - 1][lane], sb[PARTS - 1][lane], h);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kFold; ++i) {
            const int at = base + part * kFold + i;
            const int64_t run = UP ? at : r.count - 1 - at;
            if (in && at < r.count) r.reach[run * DN + c] = now;
            now = through(a[i], b[i], now);
        }
    }
}

// ---- backward ------------------------------------------------------------------------------

// The same sizes: 243 us, all of it vector instructions.
template <class T, int S, bool FULL>
__global__ __launch_bounds__(kThreads, 4) void backward_map_kernel(const SsmBackArgs a, const Runs runs, const Bounds bound)
{
    Row row;
    if (!row_of(runs, static_cast<int>(a.s.tokens), row)) return;
    Lane<S, FULL> o(a.s, row.slice);
    float A[kQuad][S], e[kQuad][S];
    o.get(a.s.a, A);
#pragma unroll
    for (int j = 0; j < kQuad; ++j)
#pragma unroll
        for (int s = 0; s < S; ++s) {
            A[j][s] *= kLog2e;
            e[j][s] = 0.0f;
        }
    const float bias = o.weight(a.s.dt_bias);
    float steps = 0.0f;
    bool cut = false;
    int begin = 0, end = -1;
    constexpr int kWhat = kDt | kZ | kDy | kC;
    Inputs<T, S> next;
    next.template load<kWhat>(o, a.s, a.g.dy, a.g.dy_stride, row, (row.t1 - 1) / kSpan * kSpan);
    for (int w = (row.t1 - 1) / kSpan * kSpan; w + kSpan > row.t0; w -= kSpan) {
        Numbers<S> k;
        k.template of<kWhat>(o, next);
        if (w > row.t0) next.template load<kWhat>(o, a.s, a.g.dy, a.g.dy_stride, row, w - kSpan);
        const Window v = window_of(bound, w, row, begin, end);
        by_span(v, [&](auto inside) {
        constexpr bool kInside = decltype(inside)::value;
#pragma unroll
        for (int i = kSpan - 1; i >= 0; --i) {
            if (!kInside && !(v.valid >> i & 1)) continue;
            if (!kInside && (v.ends >> i & 1)) {
                o.get_or_zero(a.g.dh_last, bound.at(w + i), e);
                steps = 0.0f;
                cut = true;
            }
            const float u = softplus(k.dt[i] + bias);
            float d = k.dy[i];
            if (a.s.z) {
                float g, r;
                gates(k.z[i], g, r);
                d *= k.z[i] * g;
            }
            float us[kQuad], ds[kQuad];
            spread(u, us);
            spread(d, ds);
            steps += u;
#pragma unroll
            for (int j = 0; j < kQuad; ++j)
#pragma unroll
                for (int s = 0; s < S; ++s)
                    e[j][s] = __builtin_amdgcn_exp2f(us[j] * A[j][s]) * __builtin_fmaf(k.C[i][s], ds[j], e[j][s]);
        }
        });
    }
    o.put(runs.local + static_cast<int64_t>(row.run) * o.D * o.N, e);
    if (o.in) runs.steps[static_cast<int64_t>(row.run) * o.D + o.mine] = cut ? -1.0f : steps;
}

// The gradients, four tokens at a time from the run's last.  The same sizes: 1190 us, 921 of them vector
// instructions (473 a token of 64 channels).  The rest is waiting with two waves a SIMD: inputs fetched ahead as in
// forward_kernel leave no registers, and spilled ones cost more (the step with its forward pass 4381 us
// instead of 2073).
template <class T, int S, bool FULL>
__global__ __launch_bounds__(kThreads, 2) void backward_kernel(const SsmBackArgs a, const Runs runs, const Bounds bound)
{
    constexpr int NP = kQuad * S;
    // The parts of dB and dC that each sixteen lanes (four channels' worth of fours) have.
    __shared__ float parts[kWaves][kSpan][4][2 * NP];
    Row row;
    if (!row_of(runs, static_cast<int>(a.s.tokens), row)) return;
    Lane<S, FULL> o(a.s, row.slice);
    const int64_t DN = static_cast<int64_t>(o.D) * o.N;
    const int lane = threadIdx.x % kWave;
    float (&mine)[kSpan][4][2 * NP] = parts[threadIdx.x / kWave];
    // A span's states, ahead of each token: with them in registers 200 of those spill.
    using States = float __attribute__((ext_vector_type(S)));
    __shared__ States kept[kWaves][kSpan][kQuad][kWave];
    States (&ahead_of)[kSpan][kQuad][kWave] = kept[threadIdx.x / kWave];
    float A[kQuad][S], e[kQuad][S], dA[kQuad][S];
    o.get(a.s.a, A);
#pragma unroll
    for (int j = 0; j < kQuad; ++j)
#pragma unroll
        for (int s = 0; s < S; ++s) {
            A[j][s] *= kLog2e;
            dA[j][s] = 0.0f;
        }
    o.get_or_zero(row.run + 1 < runs.count && !runs.whole ? runs.reach : nullptr, row.run, e);
    const float bias = o.weight(a.s.dt_bias), skip = o.weight(a.s.d);
    float dskip = 0.0f, dbias = 0.0f;
    int begin = 0, end = -1;
    // The state behind a span's tokens, from the one before.  (Lanes without a channel hold zeros throughout:
    // sums over channels have them too.)
    const auto ahead = [&](int w, float (&h)[kQuad][S]) {
        int from = begin, to = end;
        const Window v = window_of(bound, w, row, from, to);
        by_span(v, [&](auto inside) {
        constexpr bool kInside = decltype(inside)::value;
        Inputs<T, S> r;
        Numbers<S> k;
        r.template load<kX | kDt | kB>(o, a.s, nullptr, 0, row, w);
        k.template of<kX | kDt | kB>(o, r);
        k.template only_own<kX | kDt>(o);
#pragma unroll
        for (int i = 0; i < kSpan; ++i) {
            if (!kInside && !(v.valid >> i & 1)) continue;
            if (!kInside && (v.starts >> i & 1)) o.get_or_zero(a.s.h0, bound.at(w + i), h);
            const float u = softplus(k.dt[i] + bias);
            float us[kQuad], ins[kQuad];
            spread(u, us);
            spread(u * k.x[i], ins);
#pragma unroll
            for (int j = 0; j < kQuad; ++j)
#pragma unroll
                for (int s = 0; s < S; ++s)
                    h[j][s] = __builtin_fmaf(__builtin_amdgcn_exp2f(us[j] * A[j][s]), h[j][s], ins[j] * k.B[i][s]);
        }
        });
    };
    for (int w = (row.t1 - 1) / kSpan * kSpan; w + kSpan > row.t0; w -= kSpan) {
        Window v = window_of(bound, w, row, begin, end);
        // A sequence's tokens, the last sequence's first: a state before a sequence's first token is not the
        // one behind the token ahead of it.
        const auto part = [&](auto inside, uint32_t begun) {
            constexpr bool kInside = decltype(inside)::value;
            o.here();
            constexpr int kWhat = kX | kDt | kZ | kB | kC | kDy;
            Inputs<T, S> r;
            Numbers<S> k;
            float u[kSpan];
            r.template load<kWhat>(o, a.s, a.g.dy, a.g.dy_stride, row, w);
            float h[kQuad][S];
            if (!kInside && begun) {
                o.get_or_zero(nullptr, 0, h);          // its first token takes h0
            } else {
                // The state that was kept, and half of the time the tokens from there to here.
                o.get(a.states + static_cast<int64_t>(w / kStateTokens) * DN, h);
                if (w % kStateTokens) ahead(w - kSpan, h);
            }
            k.template of<kWhat>(o, r);
            k.template only_own<kWhat>(o);
#pragma unroll
            for (int i = 0; i < kSpan; ++i) {
                if (!kInside && !(v.valid >> i & 1)) continue;
                if (!kInside && (v.starts >> i & 1)) o.get_or_zero(a.s.h0, bound.at(w + i), h);
                k.dt[i] += bias;
                u[i] = softplus(k.dt[i]);
                float us[kQuad], ins[kQuad];
                spread(u[i], us);
                spread(u[i] * k.x[i], ins);
#pragma unroll
                for (int j = 0; j < kQuad; ++j) {
                    States v;
#pragma unroll
                    for (int s = 0; s < S; ++s) v[s] = h[j][s];
                    ahead_of[i][j][lane] = v;
#pragma unroll
                    for (int s = 0; s < S; ++s)
                        h[j][s] = __builtin_fmaf(__builtin_amdgcn_exp2f(us[j] * A[j][s]), h[j][s], ins[j] * k.B[i][s]);
                }
            }
#pragma unroll
            for (int i = kSpan - 1; i >= 0; --i) {
                if (!kInside && !(v.valid >> i & 1)) continue;
                if (!kInside && (v.ends >> i & 1)) o.get_or_zero(a.g.dh_last, bound.at(w + i), e);
                float d = k.dy[i], g = 0.0f, rest = 0.0f;
                if (a.s.z) {
                    gates(k.z[i], g, rest);
                    d *= k.z[i] * g;
                }
                // As something new: else the decays of the way there are kept, in registers that are not there.
                asm volatile("" : "+v"(u[i]));
                float us[kQuad], ins[kQuad], ds[kQuad], ys[kQuad], into[kQuad], flow[kQuad], dB[S], dC[S];
                spread(u[i], us);
                spread(u[i] * k.x[i], ins);
                spread(d, ds);
#pragma unroll
                for (int s = 0; s < S; ++s) dB[s] = dC[s] = 0.0f;
#pragma unroll
                for (int j = 0; j < kQuad; ++j) {
                    ys[j] = into[j] = flow[j] = 0.0f;
                    const States before = ahead_of[i][j][lane];
#pragma unroll
                    for (int s = 0; s < S; ++s) {
                        const float now = h[j][s], dh = __builtin_fmaf(k.C[i][s], ds[j], e[j][s]);
                        dC[s] = __builtin_fmaf(ds[j], now, dC[s]);
                        dB[s] = __builtin_fmaf(ins[j], dh, dB[s]);
                        ys[j] = __builtin_fmaf(k.C[i][s], now, ys[j]);
                        into[j] = __builtin_fmaf(dh, k.B[i][s], into[j]);
                        e[j][s] = __builtin_amdgcn_exp2f(us[j] * A[j][s]) * dh;
                        h[j][s] = before[s];
                        const float p = e[j][s] * before[s];
                        flow[j] = __builtin_fmaf(p, A[j][s], flow[j]);
                        dA[j][s] = __builtin_fmaf(p, us[j], dA[j][s]);
                    }
                }
                if (!kInside && a.g.dh0 && (v.starts >> i & 1)) o.put(a.g.dh0 + bound.at(w + i) * DN, e);
                const float in_sum = gather(into), flow_sum = gather(flow) * kLn2;
                float keep, take;
                gates(k.dt[i], keep, take);
                const float ddt = __builtin_fmaf(k.x[i], in_sum, flow_sum) * keep;
                o.template write<T>(a.g.dx, a.g.dx_stride, w + i, __builtin_fmaf(skip, d, u[i] * in_sum));
                o.template write<T>(a.g.ddt, a.g.ddt_stride, w + i, ddt);
                dskip = __builtin_fmaf(d, k.x[i], dskip);
                dbias += ddt;
                if (a.s.z && a.g.dz) {
                    const float y = __builtin_fmaf(skip, k.x[i], gather(ys));
                    o.template write<T>(a.g.dz, a.g.dz_stride, w + i, k.dy[i] * y * __builtin_fmaf(k.z[i] * rest, g, g));
                }
                // Over the sixteen lanes: from the fours next to it, twice.
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    dB[s] += moved<0x124>(dB[s]);
                    dB[s] += moved<0x128>(dB[s]);
                    dC[s] += moved<0x124>(dC[s]);
                    dC[s] += moved<0x128>(dC[s]);
                }
                // Each of the fours stores a state.
                const int f = lane / kQuad % 4;
                float b = dB[0], c = dC[0];
#pragma unroll
                for (int s = 1; s < S; ++s) {
                    b = f == s ? dB[s] : b;
                    c = f == s ? dC[s] : c;
                }
                if (f < S) {
                    mine[i][lane / 16][o.n + f] = b;
                    mine[i][lane / 16][NP + o.n + f] = c;
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            // The wave's sums of the window: [token][2][NP].
            float* shared = runs.shared + (static_cast<int64_t>(row.slice) * a.s.tokens + w) * (2 * NP);
#pragma unroll
            for (int k = 0; k < kSpan * 2 * NP / kWave; ++k) {
                const int i = (k * kWave + lane) / (2 * NP), at = (k * kWave + lane) % (2 * NP);
                if (kInside || (v.valid >> i & 1))
                    shared[k * kWave + lane] = (mine[i][0][at] + mine[i][1][at]) + (mine[i][2][at] + mine[i][3][at]);
            }
            __builtin_amdgcn_wave_barrier();
        };
        if (v.valid == (1u << kSpan) - 1 && !(v.starts | v.ends)) {
            part(std::true_type{}, 0u);
            continue;
        }
        for (uint32_t left = v.valid; left; left &= ~v.valid) {
            const uint32_t begun = left & v.starts;
            v.valid = begun ? left & (~0u << (31 - __builtin_clz(begun))) : left;
            part(std::false_type{}, begun);
        }
    }
    o.put(runs.params + row.run * DN, dA);
    if (o.in) {
        float* p = runs.params + runs.count * DN + static_cast<int64_t>(row.run) * 2 * o.D;
        p[o.mine] = dskip;
        p[o.D + o.mine] = dbias;
    }
}

// dB and dC: the slices' parts added up, four values a thread.
template <class T>
__global__ __launch_bounds__(kThreads) void shared_kernel(const SsmBackArgs a, const Runs r, int NP)
{
    const int each = 2 * NP / 4, N = a.s.state;
    const int64_t n = a.s.tokens * each;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int64_t t = i / each;
        const int k = static_cast<int>(i - t * each) * 4;
        const float4* from = reinterpret_cast<const float4*>(r.shared) + i;
        float v[4] = {};
#pragma unroll 8
        for (int s = 0; s < r.slices; ++s) {
            const float4 p = from[s * n];
            v[0] += p.x;
            v[1] += p.y;
            v[2] += p.z;
            v[3] += p.w;
        }
        T* to = k < NP ? static_cast<T*>(a.g.db) + t * a.g.db_stride + k : static_cast<T*>(a.g.dc) + t * a.g.dc_stride + (k - NP);
#pragma unroll
        for (int s = 0; s < 4; ++s)
            if ((k < NP ? k : k - NP) + s < N) store(to, s, v[s]);
    }
}

// dA, dD and the bias's gradient: the runs' parts added up, a value by four threads.
constexpr int kSumParts = 4, kSumCols = kThreads / kSumParts;

__global__ __launch_bounds__(kThreads) void params_kernel(const SsmBackArgs a, const Runs r)
{
    __shared__ float parts[kSumParts][kSumCols];
    const int part = threadIdx.x / kSumCols, lane = threadIdx.x % kSumCols;
    const int64_t D = a.s.channels, DN = D * a.s.state, n = DN + 2 * D;
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * kSumCols; base < n; base += static_cast<int64_t>(gridDim.x) * kSumCols) {
        const int64_t i = base + lane < n ? base + lane : n - 1;
        const float* from = i < DN ? r.params + i : r.params + r.count * DN + (i - DN);
        const int64_t step = i < DN ? DN : 2 * D;
        float sum = 0.0f;
#pragma unroll 8
        for (int k = part; k < r.count; k += kSumParts) sum += from[k * step];
        parts[part][lane] = sum;
        __syncthreads();
        if (part == 0 && base + lane < n) {
            sum = (parts[0][lane] + parts[1][lane]) + (parts[2][lane] + parts[3][lane]);
            if (i < DN) {
                if (a.g.da) a.g.da[i] = sum;
            } else if (i < DN + D) {
                if (a.g.dd) a.g.dd[i - DN] = sum;
            } else if (a.g.ddt_bias) {
                a.g.ddt_bias[i - DN - D] = sum;
            }
        }
        __syncthreads();
    }
}

// What passes through sequences without tokens.
__global__ __launch_bounds__(kThreads) void empty_kernel(const Bounds bound, bool all, int64_t DN, const float* from, float* to)
{
    const int64_t n = bound.n * DN;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int q = static_cast<int>(i / DN);
        if (all || bound(q + 1) <= bound(q)) to[i] = from ? from[i] : 0.0f;
    }
}

// ---- launches ----------------------------------------------------------------------

// Tokens of a run: the most that leave the launch kRowsLeast waves, four a SIMD, rounded up to where states are kept,
// but no more than kRunMost and no fewer than kRunLeast.  us, by (kRowsLeast, kRunMost): 16384 x 2048 in packed
// sequences forward 346 (2048, 256), 320 (4096, 256), 322 (4096, 128); 32768 x 2048 both directions 2156, 2154, 2122,
// and 2256 (2048, 512).
// Sequences of one length that are shorter are taken whole, as many as that gives; longer ones are where they alone are
// half as many waves.  us forward and in both directions, whole and cut: 64 x 512 tokens x 2048 channels (2048 waves)
// 394, 1681 and 564, 2068; 128 x 256 x 1024 (2048) 196, 853 and 301, 1093; but 32 x 512 x 2048 (1024 waves) 254, 1163
// and 301, 1087.  Past kWholeMost they are cut, which costs forward a third: 64 x 8192 x 2048 6162, 26386 and 8397, 31243.
constexpr int kRunMost = 128, kRunLeast = 16, kWholeMost = 4096;
constexpr int64_t kRowsLeast = 4096;

struct Cut {
    int64_t len;
    bool whole;
};
Cut cut_of(int64_t tokens, int64_t sequences, bool offsets, int64_t channels)
{
    const int64_t slices = over(channels, kWave);
    int64_t len = tokens * slices / kRowsLeast;
    if (!offsets && sequences > 0) {
        const int64_t one = tokens / sequences, most = len < kRunMost ? len : kRunMost;
        if (one <= kRunLeast || one <= most || (one <= kWholeMost && sequences * slices >= kRowsLeast / 2))
            return {one * (most > one ? most / one : 1), true};
    }
    len = over(len, kStateTokens) * kStateTokens;
    return {len < kRunLeast ? kRunLeast : len > kRunMost ? kRunMost : len, false};
}
static_assert(kRunLeast % kStateTokens == 0 && kRunMost % kStateTokens == 0, "runs begin where states are kept");

int padded_states(int64_t state) { return state <= 8 ? 8 : 16; }

// Scratch of a call: floats of the parts in Runs' order.
struct Layout {
    int64_t steps, reach, shared, params, floats;

    Layout(int64_t count, int64_t slices, int64_t tokens, int64_t D, int64_t N, bool back)
    {
        const auto up = [](int64_t n) { return over(n, 64) * 64; };
        steps = up(count * D * N);
        reach = steps + up(count * D);
        shared = reach + up(count * D * N);
        params = shared + (back ? up(slices * tokens * 2 * padded_states(N)) : 0);
        floats = params + (back ? up(count * D * (N + 2)) : 0);
    }
};

Runs runs_of(const gem_ssm& s, bool back, const OpsDevice& d)
{
    const Cut c = cut_of(s.tokens, s.sequences, s.offsets != nullptr, s.channels);
    Runs r{};
    r.slices = static_cast<int>(over(s.channels, kWave));
    r.len = static_cast<int>(c.len);
    r.count = static_cast<int>(over(s.tokens, c.len));
    r.whole = c.whole || r.count == 1;
    const Layout l(r.count, r.slices, s.tokens, s.channels, s.state, back);
    r.local = static_cast<float*>(d.scan);
    r.steps = r.local + l.steps;
    r.reach = r.local + l.reach;
    r.shared = r.local + l.shared;
    r.params = r.local + l.params;
    return r;
}
Bounds bounds_of(const gem_ssm& s) { return {s.offsets, s.offsets ? 0 : s.tokens / s.sequences, s.sequences}; }
dim3 grid_of(const Runs& r) { return dim3(static_cast<unsigned>(over(static_cast<int64_t>(r.count) * r.slices, kWaves))); }

template <bool UP, int CHAINS, int PARTS> void fold_by(const Runs& r, const gem_ssm& s, hipStream_t stream)
{
    const int64_t DN = static_cast<int64_t>(s.channels) * s.state;
    hipLaunchKernelGGL((fold_kernel<UP, CHAINS, PARTS>), dim3(static_cast<unsigned>(over(DN, CHAINS))), dim3(CHAINS * PARTS), 0, stream, r,
                       s.a, s.channels, s.state);
}
// Few chains (blocks of 32 are no more than one a compute unit) in many runs.  A forward call, us, with 32 x 16 and
// with 16 x 64: 131072 tokens of 64 channels 168, 122; 65536 of 128 126, 106; 32768 of 256 107, 100.  Where chains
// are more, 64 threads each are too many: the composition alone of 65537 of 1001 23, 30.
template <bool UP> void fold(const Runs& r, const gem_ssm& s, const OpsDevice& d, hipStream_t stream)
{
    if (static_cast<int64_t>(s.channels) * s.state <= int64_t{32} * d.cus && r.count > 16 * kFold) fold_by<UP, 16, 64>(r, s, stream);
    else fold_by<UP, 32, 16>(r, s, stream);
}

template <class T, int S, bool FULL> struct Launch {
    static void forward(const SsmArgs& a, const OpsDevice& d, hipStream_t stream)
    {
        if (!a.s.offsets && a.s.tokens == a.s.sequences) {
            const int64_t slices = over(a.s.channels, kWave);
            hipLaunchKernelGGL((step_kernel<T, S, FULL>), loop_grid(over(a.s.tokens * slices, kWaves)), dim3(kThreads), 0, stream, a,
                               static_cast<int>(slices));
            return;
        }
        Runs r = runs_of(a.s, false, d);
        const Bounds b = bounds_of(a.s);
        const int64_t DN = static_cast<int64_t>(a.s.channels) * a.s.state, n = a.s.sequences * DN;
        if (!r.whole) {
            hipLaunchKernelGGL((forward_kernel<T, S, FULL, false>), grid_of(r), dim3(kThreads), 0, stream, a, r, b);
            fold<true>(r, a.s, d, stream);
        }
        r.in_place = !r.whole && a.h_last && a.h_last == a.s.h0;
        hipLaunchKernelGGL((forward_kernel<T, S, FULL, true>), grid_of(r), dim3(kThreads), 0, stream, a, r, b);
        if (a.h_last && (r.in_place || (a.s.offsets && a.h_last != a.s.h0)))
            hipLaunchKernelGGL(ends_kernel, loop_grid(over(n, kThreads)), dim3(kThreads), 0, stream, r, b, DN, a.s.tokens, a.s.h0,
                               a.h_last);
    }
    static void backward(const SsmBackArgs& a, const OpsDevice& d, hipStream_t stream)
    {
        const Runs r = runs_of(a.s, true, d);
        const Bounds b = bounds_of(a.s);
        const int64_t DN = static_cast<int64_t>(a.s.channels) * a.s.state, n = a.s.sequences * DN;
        if (!r.whole) {
            hipLaunchKernelGGL((backward_map_kernel<T, S, FULL>), grid_of(r), dim3(kThreads), 0, stream, a, r, b);
            fold<false>(r, a.s, d, stream);
        }
        hipLaunchKernelGGL((backward_kernel<T, S, FULL>), grid_of(r), dim3(kThreads), 0, stream, a, r, b);
        constexpr int NP = kQuad * S;
        hipLaunchKernelGGL((shared_kernel<T>), loop_grid(over(a.s.tokens * (2 * NP / 4), kThreads)), dim3(kThreads), 0, stream, a, r, NP);
        if (a.g.da || a.g.dd || a.g.ddt_bias)
            hipLaunchKernelGGL(params_kernel, loop_grid(over(DN + 2 * a.s.channels, kSumCols)), dim3(kThreads), 0, stream, a, r);
        if (a.g.dh0 && a.s.offsets)
            hipLaunchKernelGGL(empty_kernel, loop_grid(over(n, kThreads)), dim3(kThreads), 0, stream, b, false, DN, a.g.dh_last, a.g.dh0);
    }
};

// f(Launch<T, S, FULL>) for the states at hand: whole vectors of them for the most, 16, and else each by itself, which
// costs (64 x 4096 single tokens of 16 states 7 us, of 8 14; 32768 x 2048 both directions 2058 and 1594).
template <class T, class F> void by_states(int state, F f)
{
    if (state == 16) f(Launch<T, 4, true>{});
    else if (state > 8) f(Launch<T, 4, false>{});
    else f(Launch<T, 2, false>{});
}
template <class F> hipError_t launch(const gem_ssm& s, bool bf16, F f)
{
    if (bf16) by_states<uint16_t>(s.state, f);
    else by_states<float>(s.state, f);
    return hipGetLastError();
}
static_assert(GEM_STATE_MAX == 16, "kernels of all states");

hipError_t pass_all(const gem_ssm& s, const float* from, float* to, hipStream_t stream)
{
    const int64_t DN = static_cast<int64_t>(s.channels) * s.state;
    if (!to || from == to) return hipSuccess;
    hipLaunchKernelGGL(empty_kernel, loop_grid(over(s.sequences * DN, kThreads)), dim3(kThreads), 0, stream, Bounds{nullptr, 0, s.sequences},
                       true, DN, from, to);
    return hipGetLastError();
}

}  // namespace

// Waves of a launch.
int64_t ssm_rows(int64_t tokens, int64_t sequences, bool offsets, int64_t channels)
{
    return tokens == 0 ? 0 : over(tokens, cut_of(tokens, sequences, offsets, channels).len) * over(channels, kWave);
}

int64_t ssm_bytes(int64_t tokens, int64_t sequences, bool offsets, int64_t channels, int64_t state, bool back)
{
    if (tokens == 0) return 0;
    const Cut c = cut_of(tokens, sequences, offsets, channels);
    const int64_t count = over(tokens, c.len);
    // What needs no maps needs no scratch forward.
    if (!back && (c.whole || count == 1)) return 0;
    return Layout(count, over(channels, kWave), tokens, channels, state, back).floats * 4;
}

// Enough for these sizes and all smaller ones, however they are cut.  Runs have at least half of
// kRunMost tokens, or there are at most twice kRowsLeast waves of them and one a slice more: a run that
// is not longer than the tokens that leave kRowsLeast waves has at least half of those, and one sequence
// that is longer has more.
int64_t ssm_scratch_bytes(int64_t tokens, int64_t channels, int64_t state)
{
    if (tokens == 0) return 0;
    const int64_t longest = (over(tokens, kRunMost / 2) + 1) * channels, many = 4 * kRowsLeast * kWave + channels;
    const int64_t most = longest > many ? longest : many;
    const int64_t cells = most < tokens * channels ? most : tokens * channels;     // channels of all runs
    return Layout(1, over(channels, kWave), tokens, cells, state, true).floats * 4;
}

hipError_t launch_ssm_forward(const SsmArgs& a, bool bf16, const OpsDevice& d, hipStream_t stream)
{
    if (a.s.tokens == 0) return pass_all(a.s, a.s.h0, a.h_last, stream);
    return launch(a.s, bf16, [&](auto l) { l.forward(a, d, stream); });
}

hipError_t launch_ssm_backward(const SsmBackArgs& a, bool bf16, const OpsDevice& d, hipStream_t stream)
{
    if (a.s.tokens == 0) {
        const hipError_t e = pass_all(a.s, a.g.dh_last, a.g.dh0, stream);
        if (e != hipSuccess) return e;
        const int64_t n = static_cast<int64_t>(a.s.channels) * (a.s.state + 2);
        if (a.g.da || a.g.dd || a.g.ddt_bias)
            hipLaunchKernelGGL(params_kernel, loop_grid(over(n, kSumCols)), dim3(kThreads), 0, stream, a, Runs{});
        return hipGetLastError();
    }
    return launch(a.s, bf16, [&](auto l) { l.backward(a, d, stream); });
}

}  // namespace gemk
