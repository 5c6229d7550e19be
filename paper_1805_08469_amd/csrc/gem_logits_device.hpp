// gem_logits_device.hpp -- device code shared by the kernels over rows of logits: running
// sums of exponentials, a part of a row, and its stream of vectors.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gem_ops.hpp"
#include "gem_ops_device.hpp"

namespace gemk {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;                 // vectors of a thread in flight, twice
constexpr int kMostWaves = 16;             // of a block

// ---- running sums of exponentials -----------------------------------------------

// 2^d is zero long before this.
constexpr float kLeast = -200.0f;

// Where exponents (x - ref) scale are taken from.  Fused, they are x scale - rc with
// rc = ref scale rounded, which puts them all off by the rounding's error, skew: sums are
// freed of it when they are moved to another reference.  From 2^24 on (a row masked by a
// large value) the error is more than half an octave, and further out it leaves the
// exponent's range: there (wide) the difference comes first.
struct Reference {
    float ref = -kInf, rc = 0.0f;
    bool wide = false;

    __device__ void set(float at, float scale)
    {
        ref = at;
        rc = at * scale;
        wide = !(__builtin_fabsf(rc) < 0x1p24f);
    }
    __device__ float skew(float scale) const
    {
        return wide || ref == -kInf ? 0.0f : __builtin_fmaf(ref, scale, -rc);
    }
    __device__ float exponent(float x, float scale) const
    {
        return wide ? (x - ref) * scale : __builtin_fmaf(x, scale, -rc);
    }
};

// A thread's s = sum 2^d and, with SUM_D, t = sum 2^d d.
struct Run {
    Reference at;
    float limit = -kInf;       // a logit above it moves the reference
    bool wide = false;         // some thread of the wave has a wide one
    float s = 0.0f, t = 0.0f;
};

// Sums moved so that every d grows by d (t with SUM_D).
template <bool SUM_D>
__device__ __forceinline__ void shift_sums(float& s, float& t, float d)
{
    d = __builtin_fmaxf(d, kLeast);
    const float c = __builtin_amdgcn_exp2f(d);
    if constexpr (SUM_D) t = c * __builtin_fmaf(s, d, t);
    s *= c;
}

// Moves the reference where `most` is over the limit: seldom, so the wave's threads are asked
// together.
template <bool SUM_D>
__device__ __forceinline__ void rebase(Run& r, float most, float scale, float reach)
{
    if (__builtin_expect(__ballot(most > r.limit) == 0, 1)) return;
    if (most > r.limit) {
        const Reference from = r.at;
        r.at.set(most, scale);
        r.limit = most + reach;
        if (from.ref > -kInf)  // else nothing is summed but zeros and NaN
            shift_sums<SUM_D>(r.s, r.t, (from.ref - most) * scale + (r.at.skew(scale) - from.skew(scale)));
    }
    r.wide = __ballot(r.at.wide) != 0;
}

template <bool SUM_D, int N>
__device__ __forceinline__ void add(Run& r, const float (&x)[N], float most, float scale, float reach)
{
    rebase<SUM_D>(r, most, scale, reach);
    const auto sum = [&](float d) {
        const float e = __builtin_amdgcn_exp2f(d);
        r.s += e;
        if constexpr (SUM_D) r.t = __builtin_fmaf(e, __builtin_fmaxf(d, kLeast), r.t);
    };
    if (__builtin_expect(!r.wide, 1)) {
#pragma unroll
        for (int i = 0; i < N; ++i) sum(__builtin_fmaf(x[i], scale, -r.at.rc));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) sum(r.at.exponent(x[i], scale));
    }
}

// Scores: a row's (or a part's) sums about the largest of its references; ref is 0 where
// no logit is above -inf, t without SUM_D.
struct Sums {
    float ref, s, t;
};

template <int WAVES, bool SUM_D = true>
__device__ __forceinline__ Sums block_sums(const Run& r, float scale, float (*lds)[4])
{
    const float top = wave_max(r.at.ref);
    float s = r.s, t = r.t;
    if (r.at.ref > -kInf) shift_sums<SUM_D>(s, t, (r.at.ref - top) * scale - r.at.skew(scale));
    s = wave_sum(s);
    if constexpr (SUM_D) t = wave_sum(t);
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
        lds[wave][0] = top;
        lds[wave][1] = s;
        if constexpr (SUM_D) lds[wave][2] = t;
    }
    __syncthreads();
    Sums out{lds[0][0], 0.0f, 0.0f};
#pragma unroll
    for (int w = 1; w < WAVES; ++w) out.ref = __builtin_fmaxf(out.ref, lds[w][0]);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        s = lds[w][1];
        if constexpr (SUM_D) t = lds[w][2];
        if (lds[w][0] > -kInf) shift_sums<SUM_D>(s, t, (lds[w][0] - out.ref) * scale);
        out.s += s;
        if constexpr (SUM_D) out.t += t;
    }
    if (out.ref == -kInf) out.ref = 0.0f;
    return out;
}

template <int WAVES> __device__ __forceinline__ float block_sum(float v, float* lds)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += lds[w];
    return v;
}

template <int WAVES> __device__ __forceinline__ float block_max(float v, float* lds)
{
    v = wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v = __builtin_fmaxf(v, lds[w]);
    return v;
}

// ---- a part of a row ----------------------------------------------------------------

// Elements [begin, begin + n) of a row: up to a vector less one before the first
// aligned address (the head), whole aligned vectors, and a tail.
template <class T> struct Part {
    const T* p;
    int begin, n, head, nvec, tail;

    __device__ Part(const T* row, int vocab, int begin_, int len)
        : p(row + begin_), begin(begin_), n(vocab - begin_ < len ? vocab - begin_ : len)
    {
        const int off = static_cast<int>((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T));
        head = (kVec<T> - off) & (kVec<T> - 1);
        if (head > n) head = n;
        nvec = (n - head) / kVec<T>;
        tail = n - head - nvec * kVec<T>;
    }
    __device__ const u32x4* body() const { return reinterpret_cast<const u32x4*>(p + head); }
    // The element index (from begin) at which the head (of thread 0) or the tail (of
    // thread 1) starts, and its length.
    __device__ int edge_at() const { return threadIdx.x == 0 ? 0 : head + nvec * kVec<T>; }
    __device__ int edge_n() const { return threadIdx.x == 0 ? head : threadIdx.x == 1 ? tail : 0; }
    __device__ void edge(float (&x)[kVec<T>]) const
    {
        const int at = edge_at(), m = edge_n();
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) x[i] = i < m ? load(p, at + i) : -kInf;
    }
};

// The largest that is a number, but NaN after a signalling NaN.  (Written out: for a maximum of
// bits that might be one the compiler quiets them first.)  A sum over the same elements is NaN
// then.
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float m;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
    return m;
}
template <int N> __device__ __forceinline__ float most_of(const float (&x)[N])
{
    float m = max3(x[0], x[1], x[2]);
#pragma unroll
    for (int i = 3; i + 1 < N; i += 2) m = max3(m, x[i], x[i + 1]);
    return max3(m, x[N - 1], x[N - 1]);
}

// The bits of two -inf, or of one.
template <class T> __device__ __forceinline__ uint32_t lowest() { return sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u; }

// Non-temporal: a row's bytes are read once, or again when the caches have long passed them.
__device__ __forceinline__ u32x4 read_once(const u32x4* p) { return __builtin_nontemporal_load(p); }

// f(v, vector) for each vector v of the part by its thread, UNROLL loads ahead.  Every
// thread calls it equally often (f may ask the wave); inside is false past the end, where
// the last vector is given again.
template <int THREADS, int UNROLL, class F>
__device__ __forceinline__ void stream(const u32x4* body, int nvec, F f)
{
    if (nvec == 0) return;
    constexpr int kRound = THREADS * UNROLL;
    const int tid = threadIdx.x, last = nvec - 1;
    u32x4 next[UNROLL];
    const auto load = [&](int base) {
        if (base + kRound <= nvec) {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) next[u] = read_once(body + base + tid + u * THREADS);
        } else {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int v = base + tid + u * THREADS;
                if (base + u * THREADS < nvec) next[u] = read_once(body + (v < last ? v : last));
            }
        }
    };
    load(0);
    int base = 0;
    for (; base + kRound <= nvec; base += kRound) {
        u32x4 cur[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) cur[u] = next[u];
        load(base + kRound);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) f(base + tid + u * THREADS, cur[u], true);
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
        if (base + u * THREADS < nvec) f(base + tid + u * THREADS, next[u], base + tid + u * THREADS < nvec);
}

// ---- what rows are given back ------------------------------------------------------------

__device__ __forceinline__ float log_prob(const LogitArgs& a, float x, float ref, float ls)
{
    return x == -kInf ? x : (x - ref) * a.inv_t - ls * kLn2;
}

// A log probability and an entropy have a side of 0 to be on, which near a single outcome is
// less than their rounding.
__device__ __forceinline__ float at_most_0(float v) { return v > 0.0f ? 0.0f : v; }
__device__ __forceinline__ float at_least_0(float v) { return v < 0.0f ? 0.0f : v; }

// Before a barrier: behind it the block's stores so far are in memory.
__device__ __forceinline__ void stores_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

template <int THREADS, class T>
__device__ __forceinline__ void no_grad(const Part<T>& part, T* grad)
{
    T* out = grad + part.begin;
    const int off = static_cast<int>((reinterpret_cast<uintptr_t>(out) & 15u) / sizeof(T));
    int head = (kVec<T> - off) & (kVec<T> - 1);
    if (head > part.n) head = part.n;
    const int nvec = (part.n - head) / kVec<T>, end = head + nvec * kVec<T>;
    for (int i = threadIdx.x; i < head; i += THREADS) store(out, i, 0.0f);
    for (int i = end + threadIdx.x; i < part.n; i += THREADS) store(out, i, 0.0f);
    for (int v = threadIdx.x; v < nvec; v += THREADS)
        __builtin_nontemporal_store(u32x4{0, 0, 0, 0}, reinterpret_cast<u32x4*>(out + head) + v);
}

}  // namespace
}  // namespace gemk
