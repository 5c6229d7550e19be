// gem_logits.hip -- scores of rows of logits, and the distillation loss with its
// gradient, for gfx950.  A block takes one row.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gem_ops.hpp"

namespace gemk {
namespace {

constexpr int kThreads = 256;
constexpr float kLn2 = 0.693147180559945309417f;
constexpr float kInf = __builtin_inff();

__device__ __forceinline__ float load(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float load(const uint16_t* p, int64_t i)
{
    return __uint_as_float(static_cast<uint32_t>(p[i]) << 16);
}
__device__ __forceinline__ void store(float* p, int64_t i, float v) { p[i] = v; }
__device__ __forceinline__ void store(uint16_t* p, int64_t i, float v)
{
    const uint32_t b = __float_as_uint(v);
    // nearest even; a NaN keeps a mantissa bit
    p[i] = static_cast<uint16_t>(v != v ? (b >> 16) | 0x40u : (b + 0x7FFFu + ((b >> 16) & 1u)) >> 16);
}

template <class F>
__device__ float block_reduce(float v, float* lds, F f)
{
    __syncthreads();
    lds[threadIdx.x] = v;
    __syncthreads();
    for (int s = kThreads / 2; s > 0; s >>= 1) {
        if (threadIdx.x < s) lds[threadIdx.x] = f(lds[threadIdx.x], lds[threadIdx.x + s]);
        __syncthreads();
    }
    return lds[0];
}

__device__ float add(float a, float b) { return a + b; }
__device__ float most(float a, float b) { return __builtin_fmaxf(a, b); }

// The order of alternatives as an integer's: logits rising, equal ones (the two
// zeros are equal) by falling token.  0 is no alternative.
__device__ __forceinline__ uint64_t rank_key(float v, uint32_t token)
{
    if (!(v > -kInf)) return 0;
    const uint32_t b = __float_as_uint(v == 0.0f ? 0.0f : v);
    const uint32_t o = b & 0x80000000u ? ~b : b | 0x80000000u;
    return (static_cast<uint64_t>(o) << 32) | static_cast<uint32_t>(~token);
}

template <class T>
__global__ __launch_bounds__(kThreads) void score_kernel(const ScoreArgs a)
{
    __shared__ float lds[kThreads];
    __shared__ uint64_t keys[kThreads];
    const int64_t r = blockIdx.x;
    const T* row = static_cast<const T*>(a.l.z) + r * a.l.stride;
    const int V = a.l.vocab;
    float m = -kInf;
    for (int v = threadIdx.x; v < V; v += kThreads) m = __builtin_fmaxf(m, load(row, v));
    m = block_reduce(m, lds, most);
    // Differences are taken before they are scaled: scaled on its own, a logit near the
    // type's lowest value (a mask's) would overflow.
    if (m == -kInf) m = 0.0f;
    float s = 0.0f, t = 0.0f;
    for (int v = threadIdx.x; v < V; v += kThreads) {
        const float d = (load(row, v) - m) * a.l.scale;
        const float e = __builtin_amdgcn_exp2f(d);
        s += e;
        t = __builtin_fmaf(e, __builtin_fmaxf(d, -200.0f), t);
    }
    s = block_reduce(s, lds, add);
    t = block_reduce(t, lds, add);
    const float ls = __builtin_log2f(s);
    if (threadIdx.x == 0) {
        if (a.out.lse) a.out.lse[r] = m * a.l.inv_t + ls * kLn2;
        if (a.out.entropy) a.out.entropy[r] = s == 0.0f ? 0.0f : (ls - t / s) * kLn2;
    }
    for (int i = threadIdx.x; i < a.n_tokens; i += kThreads) {
        const int token = a.tokens[r * a.n_tokens + i];
        float lp = 0.0f;
        if (token >= 0 && token < V) {
            const float x = load(row, token);
            lp = x == -kInf ? x : (x - m) * a.l.inv_t - ls * kLn2;
        }
        a.out.logprob[r * a.n_tokens + i] = lp;
    }
    uint64_t below = ~uint64_t{0};
    for (int i = 0; i < a.top_k; ++i) {
        uint64_t best = 0;
        for (int v = threadIdx.x; v < V; v += kThreads) {
            const uint64_t k = rank_key(load(row, v), v);
            if (k < below && k > best) best = k;
        }
        __syncthreads();
        keys[threadIdx.x] = best;
        __syncthreads();
        for (int h = kThreads / 2; h > 0; h >>= 1) {
            if (threadIdx.x < h && keys[threadIdx.x + h] > keys[threadIdx.x])
                keys[threadIdx.x] = keys[threadIdx.x + h];
            __syncthreads();
        }
        below = keys[0];
        if (threadIdx.x == 0) {
            const int token = below ? static_cast<int>(~static_cast<uint32_t>(below)) : -1;
            if (a.out.top_ids) a.out.top_ids[r * a.top_k + i] = token;
            if (a.out.top_logprob)
                a.out.top_logprob[r * a.top_k + i] =
                    below ? (load(row, token) - m) * a.l.inv_t - ls * kLn2 : -kInf;
        }
    }
}

template <class T>
__global__ __launch_bounds__(kThreads) void distill_kernel(const DistillArgs a)
{
    __shared__ float lds[kThreads];
    __shared__ int ids[GEM_TOP_MAX];
    const int64_t r = blockIdx.x;
    const T* row = static_cast<const T*>(a.l.z) + r * a.l.stride;
    T* grad = a.grad ? static_cast<T*>(a.grad) + r * a.grad_stride : nullptr;
    const int V = a.l.vocab, tid = threadIdx.x;
    const float w = a.weight ? a.weight[r] : 1.0f;
    if (w == 0.0f) {
        if (tid == 0 && a.loss) a.loss[r] = 0.0f;
        if (grad)
            for (int v = tid; v < V; v += kThreads) store(grad, v, 0.0f);
        return;
    }
    int id = -1;
    if (tid < a.k) {
        id = a.ids[r * a.k + tid];
        if (id < 0 || id >= V) id = -1;
        ids[tid] = id;
    }
    __syncthreads();
    if (tid < a.k)
        for (int i = 0; i < tid; ++i)
            if (ids[i] == id) id = -1;
    float m = -kInf;
    for (int v = tid; v < V; v += kThreads) m = __builtin_fmaxf(m, load(row, v));
    m = block_reduce(m, lds, most);
    // Differences are taken before they are scaled: scaled on its own, a logit near the
    // type's lowest value (a mask's) would overflow.
    if (m == -kInf) m = 0.0f;
    float lp = id >= 0 ? a.lp[r * a.k + tid] : -kInf;
    float p, lse_p = 0.0f;
    if (a.tail) {
        p = id >= 0 ? expf(lp) : 0.0f;
    } else {
        const float top = block_reduce(lp, lds, most);
        p = id >= 0 && top > -kInf ? expf(lp - top) : 0.0f;
        const float sum = block_reduce(p, lds, add);
        p = sum > 0.0f ? p / sum : 0.0f;
        lse_p = top + logf(sum);
    }
    const float pt = a.tail ? __builtin_fmaxf(0.0f, 1.0f - block_reduce(p, lds, add)) : 0.0f;
    const float x = id >= 0 ? load(row, id) : 0.0f;
    const float d = (x - m) * a.l.scale;
    float s_all = 0.0f, s_out = 0.0f;
    if (tid < a.k) ids[tid] = id;
    __syncthreads();
    for (int v = tid; v < V; v += kThreads) {
        const float e = __builtin_amdgcn_exp2f((load(row, v) - m) * a.l.scale);
        s_all += e;
        bool listed = false;
        for (int i = 0; i < a.k; ++i) listed |= ids[i] == v;
        if (!listed) s_out += e;
    }
    s_all = block_reduce(s_all, lds, add);
    s_out = block_reduce(s_out, lds, add);
    const float ls = __builtin_log2f(s_all);
    float part = 0.0f;
    if (p > 0.0f) part = p * (lp - lse_p - (x == -kInf ? x : (x - m) * a.l.inv_t - ls * kLn2));
    float loss = block_reduce(part, lds, add);
    if (pt > 0.0f)
        loss += s_out == 0.0f ? kInf : pt * (logf(pt) - (__builtin_log2f(s_out) - ls) * kLn2);
    if (tid == 0 && a.loss) a.loss[r] = loss;
    if (!grad) return;
    const float f = w * a.l.inv_t;
    const float inv = s_all == 0.0f ? 0.0f : 1.0f / s_all;
    const float rest = pt > 0.0f && s_out != 0.0f ? pt / s_out : 0.0f;
    for (int v = tid; v < V; v += kThreads) {
        const float e = __builtin_amdgcn_exp2f((load(row, v) - m) * a.l.scale);
        store(grad, v, f * (e * (inv - rest)));
    }
    __syncthreads();
    if (id >= 0) store(grad, id, f * (__builtin_amdgcn_exp2f(d) * inv - p));
}

}  // namespace

hipError_t launch_scores(const ScoreArgs& a, bool bf16, hipStream_t stream)
{
    const dim3 grid(static_cast<unsigned>(a.l.rows));
    if (bf16) hipLaunchKernelGGL((score_kernel<uint16_t>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((score_kernel<float>), grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_distill(const DistillArgs& a, bool bf16, hipStream_t stream)
{
    const dim3 grid(static_cast<unsigned>(a.l.rows));
    if (bf16) hipLaunchKernelGGL((distill_kernel<uint16_t>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((distill_kernel<float>), grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace gemk
