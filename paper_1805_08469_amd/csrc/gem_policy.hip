// gem_policy.hip -- the clipped policy loss with its KL term and the gradient of the
// logits, for gfx950.
//
// With lp = z_a - lse of the token a that was taken, ratio = exp(lp - old) and d = ref - lp,
//     loss = -min(ratio A, clip(ratio) A) + kl (e^d - 1 - d),
// a function of lp alone, so the row's gradient is slope (1[v = a] - q_v) with slope = dloss/dlp:
// one sum of exponentials over the row, a few scalars, and the row again.  Bytes of logits bound it;
// with the gradient a row stays in registers between its sum and its gradient.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gem_logits_device.hpp"
#include "gem_ops.hpp"
#include "gem_ops_device.hpp"

namespace gemk {
namespace {

// A row's token, its logit and what came with it; live: the row counts.
struct Taken {
    int token = -1;
    float w = 0.0f, x = -kInf, old = 0.0f, ref = 0.0f, adv = 0.0f;
    bool live = false;
};

template <class T> __device__ __forceinline__ Taken taken_of(const PolicyArgs& a, int64_t r)
{
    Taken t;
    t.token = a.p.action[r];
    t.w = a.weight ? a.weight[r] : 1.0f;
    t.live = t.w != 0.0f && t.token >= 0 && t.token < a.l.vocab;
    if (!t.live) return t;
    t.x = load(static_cast<const T*>(a.l.z) + r * a.l.stride, t.token);
    t.old = a.p.old_logprob[r];
    t.adv = a.p.advantage[r];
    if (a.p.ref_logprob) t.ref = a.p.ref_logprob[r];
    return t;
}

// One value of all lanes, in a scalar register.
__device__ __forceinline__ float of_wave(float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); }
__device__ __forceinline__ float of_lane(float v, int lane)
{
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane));
}
__device__ __forceinline__ Taken of_wave(const Taken& t)
{
    return {static_cast<int>(__builtin_amdgcn_readfirstlane(t.token)), of_wave(t.w), of_wave(t.x), of_wave(t.old), of_wave(t.ref),
            of_wave(t.adv), t.live};
}

// Ahead of a barrier behind which the gradient may be written over the taken logit.
__device__ __forceinline__ void is_read(float x) { asm volatile("" ::"v"(x)); }

// Ratios and the KL term are small differences of logarithms, whose 32 bits would show in them (d = 0.01 of
// lp = -80: the KL term is off by 2^-10).  The differences are formed in 64 bits, and their exponentials and
// series below are in 32 again, off by a few units of the result.  (The library's 64-bit functions spill 70 to
// 89 of a lane's registers in policy_resident_kernel.)

// log s, of a sum's 32 bits: its exponent's part in 64, so that the error is a unit of the mantissa's, which is
// within sqrt(2) of 1.
__device__ __forceinline__ double log_of(float s)
{
    int e = __builtin_amdgcn_frexp_expf(s);
    float m = __builtin_amdgcn_frexp_mantf(s);
    if (m < 0.70710678f) {
        m *= 2.0f;
        e -= 1;
    }
    return e * 0.6931471805599453094 + static_cast<double>(__builtin_log2f(m) * kLn2);
}

// e^d: 2^k of k = d log2(e) rounded, and what rounding left of d and k by the slope.  Below 2^-126 it is 0.
__device__ __forceinline__ float exp_of(double d)
{
    const float hi = static_cast<float>(d), lo = static_cast<float>(d - hi), k = hi * kLog2e;
    constexpr float kRest = static_cast<float>(1.4426950408889634074 - kLog2e);
    float left = __builtin_fmaf(hi, kLog2e, -k);
    left = __builtin_fmaf(hi, kRest, left);
    left = __builtin_fmaf(lo, kLog2e, left) * kLn2;
    const float e = __builtin_amdgcn_exp2f(k);
    return e == kInf || e == 0.0f ? e : __builtin_fmaf(e, left, e);
}

// kl = e^d - 1 - d >= 0 and more = e^d - 1, from d and e = e^d.  Up to |d| = 1, where the differences would lose
// what they are, from the series of the first: up to d^11 / 11!, whose next term is 2^-27 of the sum at 1.
__device__ __forceinline__ void kl_of(double d, float e, float& kl, float& more)
{
    const float hi = static_cast<float>(d);
    if (__builtin_fabsf(hi) < 1.0f) {
        float s = 1.0f / 39916800.0f;
        s = __builtin_fmaf(s, hi, 1.0f / 3628800.0f);
        s = __builtin_fmaf(s, hi, 1.0f / 362880.0f);
        s = __builtin_fmaf(s, hi, 1.0f / 40320.0f);
        s = __builtin_fmaf(s, hi, 1.0f / 5040.0f);
        s = __builtin_fmaf(s, hi, 1.0f / 720.0f);
        s = __builtin_fmaf(s, hi, 1.0f / 120.0f);
        s = __builtin_fmaf(s, hi, 1.0f / 24.0f);
        s = __builtin_fmaf(s, hi, 1.0f / 6.0f);
        s = __builtin_fmaf(s, hi, 0.5f) * hi;
        more = __builtin_fmaf(s, hi, hi);
        kl = __builtin_fmaf(more, static_cast<float>(d - hi), s * hi);      // its slope is e^d - 1
        return;
    }
    more = e - 1.0f;
    kl = e == kInf ? e : static_cast<float>((e - 1.0) - d);
}

struct Terms {
    float loss, lp, ratio, kl, slope;
};

__device__ __forceinline__ Terms terms_of(const PolicyArgs& a, const Taken& k, const Sums& u)
{
    Terms t;
    double lp = k.x == -kInf ? static_cast<double>(k.x) : (static_cast<double>(k.x) - u.ref) * a.per_t - log_of(u.s);
    lp = u.s != u.s ? u.s : lp > 0.0 ? 0.0 : lp;       // near a single outcome its side of 0 is less than its rounding
    t.lp = static_cast<float>(lp);
    // Of both differences at once, lanes in turn.
    const double gap = k.ref - lp;
    const float grown = exp_of(threadIdx.x & 1 ? gap : lp - k.old);
    t.ratio = of_lane(grown, 0);
    const float adv = k.adv;
    const float lo = of_wave(1.0f - a.p.clip_low), hi = of_wave(1.0f + a.p.clip_high);
    const float held = (t.ratio < lo ? lo : t.ratio > hi ? hi : t.ratio) * adv, free = t.ratio * adv;
    const bool clipped = held < free;
    // An advantage of 0 has no part, whatever the ratio, but a row without a log probability has no loss either.
    const bool none = adv == 0.0f && t.lp == t.lp;
    t.loss = none ? 0.0f : -(clipped ? held : free);
    t.slope = none || clipped ? 0.0f : -free;
    t.kl = 0.0f;
    if (a.p.ref_logprob) {
        float more;
        kl_of(gap, of_lane(grown, 1), t.kl, more);
        if (a.p.kl != 0.0f) {
            t.loss = __builtin_fmaf(a.p.kl, t.kl, t.loss);
            t.slope = __builtin_fmaf(-a.p.kl, more, t.slope);
        }
    }
    return t;
}

__device__ __forceinline__ void write_terms(const PolicyArgs& a, int64_t r, const Terms& t)
{
    if (a.out.loss) a.out.loss[r] = t.loss;
    if (a.out.logprob) a.out.logprob[r] = t.lp;
    if (a.out.ratio) a.out.ratio[r] = t.ratio;
    if (a.out.kl) a.out.kl[r] = t.kl;
}

// A row's gradient: c 2^d of every token, and of the taken one f (1 - 2^d / s).
struct Slope {
    Reference at;
    float c, f, inv;

    __device__ Slope(const PolicyArgs& a, const Terms& t, const Sums& u, float w)
    {
        at.set(u.ref, a.l.scale);
        f = of_wave(static_cast<float>(w * a.per_t * t.slope));
        inv = of_wave(u.s == 0.0f ? 0.0f : 1.0f / u.s);
        c = of_wave(-f * inv * __builtin_amdgcn_exp2f(-at.skew(a.l.scale)));
    }
    __device__ float taken(float x, float scale) const
    {
        return f - f * (__builtin_amdgcn_exp2f((x - at.ref) * scale) * inv);
    }
    __device__ float other(float x, float scale) const { return c * __builtin_amdgcn_exp2f(at.exponent(x, scale)); }

    // Vector v of the part; whole: its rows are aligned as the logits'.
    template <class T>
    __device__ __forceinline__ void vector(T* body, uint32_t v, u32x4 raw, bool whole, float scale) const
    {
        float y[kVec<T>];
        unpack(raw, y);
        if (__builtin_expect(!at.wide, 1)) {
#pragma unroll
            for (int i = 0; i < kVec<T>; ++i) y[i] = c * __builtin_amdgcn_exp2f(__builtin_fmaf(y[i], scale, -at.rc));
        } else {
#pragma unroll
            for (int i = 0; i < kVec<T>; ++i) y[i] = c * __builtin_amdgcn_exp2f((y[i] - at.ref) * scale);
        }
        if (whole) {
            __builtin_nontemporal_store(pack(y), reinterpret_cast<u32x4*>(reinterpret_cast<char*>(body) + v * 16u));
        } else {
#pragma unroll
            for (int i = 0; i < kVec<T>; ++i) store(body, static_cast<int64_t>(v) * kVec<T> + i, y[i]);
        }
    }
    template <class T> __device__ __forceinline__ void edges(const Part<T>& part, T* grad, float scale) const
    {
        if (threadIdx.x >= 2) return;
        T* out = grad + part.begin;
        const int from = part.edge_at(), m = part.edge_n();
        for (int i = from; i < from + m; ++i) store(out, i, other(load(part.p, i), scale));
    }
};

// The thread whose store of a part covers its element `at`: it stores the taken token's again,
// behind its own.
template <class T, int THREADS> __device__ __forceinline__ uint32_t owner(const Part<T>& part, int at)
{
    if (at < part.head) return 0;
    const int v = (at - part.head) / kVec<T>;
    return v < part.nvec ? v % THREADS : 1;
}

// A row that does not count, as far as a block is asked for it.
template <int THREADS, class T>
__device__ __forceinline__ void no_row(const PolicyArgs& a, int64_t r, const Part<T>& part, T* grad, bool terms)
{
    if (terms && threadIdx.x == 0) write_terms(a, r, Terms{});
    if (grad) no_grad<THREADS>(part, grad);
}

// What a block does with its part of a row: the sum (left in `sums`, and the taken token's logit in
// `xs`: the gradient may be written over the logits), the rest from those, or both.  37 rows of
// 100003 binary32 take two launches, in parts.
enum : int { kSum = 1, kRest = 2 };

template <class T, int STEP>
__global__ __launch_bounds__(kThreads) void policy_kernel(const PolicyArgs a, int64_t row0, int parts, int len, Sums* sums,
                                                          float* xs)
{
    constexpr int WAVES = kThreads / 64;
    __shared__ float lds[WAVES][4];
    const int blocks = STEP == kRest && !a.grad ? 1 : parts;       // of a row
    const int64_t i = blockIdx.x / blocks, r = row0 + i;
    const int q = blockIdx.x % blocks, tid = threadIdx.x;
    const T* row = static_cast<const T*>(a.l.z) + r * a.l.stride;
    T* grad = a.grad ? static_cast<T*>(a.grad) + r * a.grad_stride : nullptr;
    const Part<T> part(row, a.l.vocab, q * len, len);
    const float scale = a.l.scale;
    Taken t = taken_of<T>(a, r);
    if (!t.live) {
        if (STEP & kRest) no_row<kThreads>(a, r, part, grad, q == 0);
        return;
    }
    if constexpr (!(STEP & kSum)) t.x = xs[i];
    is_read(t.x);
    Run run;
    if constexpr (STEP & kSum) {
        const float reach = 20.0f / scale;
        if (tid < 64) {
            float x[kVec<T>];
            part.edge(x);
            add<false>(run, x, most_of(x), scale, reach);
        }
        stream<kThreads, kUnroll>(part.body(), part.nvec, [&](int, u32x4 raw, bool inside) {
            float x[kVec<T>];
            unpack(inside ? raw : u32x4{lowest<T>(), lowest<T>(), lowest<T>(), lowest<T>()}, x);
            add<false>(run, x, most_of(x), scale, reach);
        });
    } else if (tid < parts) {
        const Sums p = sums[i * parts + tid];
        run.at.ref = p.t;          // -inf: no logit above it
        run.at.wide = true;        // a part's sum has no skew
        run.s = p.s;
    }
    Sums u = block_sums<WAVES, false>(run, scale, lds);
    if constexpr (!(STEP & kRest)) {
        if (tid == 0) {
            // (ref, s, and ref as it is joined)
            u.t = u.s == 0.0f ? -kInf : u.ref;
            sums[blockIdx.x] = u;
            if (q == 0) xs[i] = t.x;
        }
        return;
    }
    const Terms m = terms_of(a, t, u);
    if (q == 0 && tid == 0) write_terms(a, r, m);
    if (!grad) return;
    const Slope g(a, m, u, t.w);
    T* body = grad + part.begin + part.head;
    const bool whole = (reinterpret_cast<uintptr_t>(body) & 15u) == 0;
    g.edges(part, grad, scale);
    stream<kThreads, kUnroll>(part.body(), part.nvec, [&](int v, u32x4 raw, bool inside) {
        if (inside) g.vector(body, v, raw, whole, scale);
    });
    const int at = t.token - part.begin;
    if (at >= 0 && at < part.n && owner<T, kThreads>(part, at) == threadIdx.x) store(grad, t.token, g.taken(t.x, scale));
}

// Loss and gradient with a row's vectors in registers, NV of a thread: what they hold is read
// once (with REST a row has more, which is read twice).  A block goes through rows; as each
// vector of a gradient is stored the next row's takes its place, so that loads and stores go
// on through the sums.  4096 rows of 32768 bfloat16, an eighth without weight: 102 us (5.0 TB/s).
constexpr int kRestUnroll = 2;

template <class T, int THREADS, int NV, bool REST>
__global__ __launch_bounds__(THREADS, 4) void policy_resident_kernel(const PolicyArgs a)
{
    constexpr int WAVES = THREADS / 64, kKept = THREADS * NV;
    __shared__ float lds[2][WAVES][4];     // in turn: a wave may be a row ahead of another's last look
    const uint32_t tid = threadIdx.x;
    const float scale = a.l.scale, reach = of_wave(20.0f / scale);
    const auto part_of = [&](int64_t r) {
        return Part<T>(static_cast<const T*>(a.l.z) + r * a.l.stride, a.l.vocab, 0, a.l.vocab);
    };
    const auto grad_of = [&](int64_t r) { return static_cast<T*>(a.grad) + r * a.grad_stride; };
    Taken taken;
    // The block's next row from r on that counts (or beyond the last).
    const auto next_row = [&](int64_t r) {
        for (; r < a.l.rows; r += gridDim.x) {
            taken = taken_of<T>(a, r);
            if (taken.live) break;
            no_row<THREADS>(a, r, part_of(r), grad_of(r), true);
        }
        return r;
    };
    u32x4 d[NV];
    // The thread's place among a vector's, as something new: places of all vectors, the same
    // for every row, would be kept in registers.
    const auto place = [&]() {
        uint32_t at = tid;
        asm volatile("" : "+v"(at));
        return at;
    };
    // A vector's bits, as something new: else its elements are kept from one pass to the next.
    const auto vector = [&](int u) {
        asm volatile("" : "+v"(d[u]));
        return d[u];
    };
    const auto fetch = [&](const Part<T>& part, int u, uint32_t at) {
        const uint32_t v = u * THREADS + at, last = part.nvec - 1;
        d[u] = read_once(reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(part.body()) + (v < last ? v : last) * 16u));
    };
    int64_t r = next_row(blockIdx.x);
    if (r >= a.l.rows) return;
    {
        const Part<T> part = part_of(r);
#pragma unroll
        for (int u = 0; u < NV; ++u)
            if (u * THREADS < part.nvec) fetch(part, u, tid);
    }
    for (int turn = 0;; turn ^= 1) {
        const Part<T> part = part_of(r);
        T* grad = grad_of(r);
        const Taken now = of_wave(taken);
        float most = -kInf;
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            if (u * THREADS < part.nvec) {
                if ((u + 1) * THREADS > part.nvec) {
                    const bool inside = static_cast<int>(u * THREADS + place()) < part.nvec;
#pragma unroll
                    for (int i = 0; i < 4; ++i) d[u][i] = inside ? d[u][i] : lowest<T>();
                }
                float x[kVec<T>];
                unpack(vector(u), x);
                most = max3(most, most_of(x), most);
            }
            __builtin_amdgcn_sched_barrier(0);         // one vector's elements at a time in registers
        }
        Run run;
        rebase<false>(run, most, scale, reach);
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            if (u * THREADS < part.nvec) {
                float x[kVec<T>];
                unpack(vector(u), x);
                if (__builtin_expect(!run.wide, 1)) {
#pragma unroll
                    for (int i = 0; i < kVec<T>; ++i) run.s += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], scale, -run.at.rc));
                } else {
#pragma unroll
                    for (int i = 0; i < kVec<T>; ++i) run.s += __builtin_amdgcn_exp2f(run.at.exponent(x[i], scale));
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (tid < 64) {
            float x[kVec<T>];
            part.edge(x);
            add<false>(run, x, most_of(x), scale, reach);
        }
        const int more = REST && part.nvec > kKept ? part.nvec - kKept : 0;
        if constexpr (REST)
            stream<THREADS, kRestUnroll>(part.body() + kKept, more, [&](int, u32x4 raw, bool inside) {
                float x[kVec<T>];
                unpack(inside ? raw : u32x4{lowest<T>(), lowest<T>(), lowest<T>(), lowest<T>()}, x);
                add<false>(run, x, most_of(x), scale, reach);
            });
        is_read(now.x);
        Sums sums = block_sums<WAVES, false>(run, scale, lds[turn]);
        sums.ref = of_wave(sums.ref);
        sums.s = of_wave(sums.s);
        const Terms m = terms_of(a, now, sums);
        if (tid == 0) write_terms(a, r, m);
        const Slope g(a, m, sums, now.w);
        T* body = grad + part.head;
        const bool whole = (reinterpret_cast<uintptr_t>(body) & 15u) == 0;
        g.edges(part, grad, scale);
        r = next_row(r + gridDim.x);
        Part<T> next = part;
        if (r < a.l.rows) next = part_of(r);
        else next.nvec = 0;
        if constexpr (REST)
            stream<THREADS, kRestUnroll>(part.body() + kKept, more, [&](int v, u32x4 raw, bool inside) {
                if (inside) g.vector(body + kKept * kVec<T>, v, raw, whole, scale);
            });
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            const uint32_t at = place(), v = u * THREADS + at;
            const u32x4 raw = vector(u);
            if (u * THREADS < next.nvec) fetch(next, u, at);
            if (static_cast<int>(v) < part.nvec) g.vector(body, v, raw, whole, scale);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (owner<T, THREADS>(part, now.token) == tid) store(grad, now.token, g.taken(now.x, scale));
        if (r >= a.l.rows) break;
    }
}

// ---- launches ----------------------------------------------------------------------

template <class T, int THREADS, int NV, bool REST>
void resident(const PolicyArgs& a, const OpsDevice& d, hipStream_t stream)
{
    const int64_t blocks = int64_t{d.cus} * (1024 / THREADS);
    hipLaunchKernelGGL((policy_resident_kernel<T, THREADS, NV, REST>),
                       dim3(static_cast<unsigned>(a.l.rows < blocks ? a.l.rows : blocks)), dim3(THREADS), 0, stream, a);
}

// With rows enough to keep the device busy they stay in registers, in blocks of few threads, so
// that others stream while one sums (the distillation's rule, whose measurements are beside it).
template <class T> bool resident_rows(const PolicyArgs& a, const OpsDevice& d, hipStream_t stream)
{
    const int nvec = a.l.vocab / kVec<T>;
    if (!a.grad || a.l.rows < d.cus) return false;
    if (nvec <= 256 * 8) resident<T, 256, 8, false>(a, d, stream);
    else if (nvec <= 256 * 16) resident<T, 256, 16, false>(a, d, stream);
    else if (nvec <= 512 * 16) resident<T, 512, 16, false>(a, d, stream);
    else if (nvec <= 1024 * 16) resident<T, 512, 16, true>(a, d, stream);
    else return false;
    return true;
}

// Parts of a row where rows are few: as many as give the device three blocks a compute unit, of no
// less than kLeastPart elements, and no more than one wave of threads joins.  Rows of 100003 binary32, us, with two,
// three and six blocks a unit: 37 rows 13.5, 13.3, 14.0; 100 27.7, 26.3, 24.8; 200 49.3, 49.2, 45.9.
constexpr int kLeastPart = 4096, kPartsMax = 64;

template <class T> hipError_t policy(const PolicyArgs& a, const OpsDevice& d, hipStream_t stream)
{
    if (resident_rows<T>(a, d, stream)) return hipGetLastError();
    const int64_t want = (int64_t{3} * d.cus + a.l.rows - 1) / a.l.rows;
    int64_t parts = a.l.vocab / kLeastPart;
    if (parts > want) parts = want;
    if (parts > kPartsMax) parts = kPartsMax;
    if (parts <= 1) {
        hipLaunchKernelGGL((policy_kernel<T, kSum | kRest>), dim3(static_cast<unsigned>(a.l.rows)), dim3(kThreads), 0, stream, a,
                           int64_t{0}, 1, a.l.vocab, nullptr, nullptr);
        return hipGetLastError();
    }
    int len = static_cast<int>((a.l.vocab + parts - 1) / parts);
    len = (len + 63) / 64 * 64;            // parts of aligned rows stay aligned
    parts = (a.l.vocab + len - 1) / len;
    Sums* sums = static_cast<Sums*>(d.scratch);
    const int64_t fit = kFixedScratch / (parts * static_cast<int64_t>(sizeof(Sums)) + 4);
    for (int64_t r = 0; r < a.l.rows; r += fit) {
        const int64_t n = a.l.rows - r < fit ? a.l.rows - r : fit;
        float* xs = reinterpret_cast<float*>(sums + n * parts);
        hipLaunchKernelGGL((policy_kernel<T, kSum>), dim3(static_cast<unsigned>(n * parts)), dim3(kThreads), 0, stream, a, r,
                           static_cast<int>(parts), len, sums, xs);
        // The loss alone is one block's a row.
        const int64_t rest = a.grad ? parts : 1;
        hipLaunchKernelGGL((policy_kernel<T, kRest>), dim3(static_cast<unsigned>(n * rest)), dim3(kThreads), 0, stream, a, r,
                           static_cast<int>(parts), len, sums, xs);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_policy(const PolicyArgs& a, bool bf16, const OpsDevice& d, hipStream_t stream)
{
    return bf16 ? policy<uint16_t>(a, d, stream) : policy<float>(a, d, stream);
}

}  // namespace gemk
