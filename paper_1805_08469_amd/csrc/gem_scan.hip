// gem_scan.hip -- the gated linear recurrence and its backward pass for gfx950.
// A thread takes one channel of one sequence from its first token to its last.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gem_ops.hpp"

namespace gemk {
namespace {

constexpr int kThreads = 64;
constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float load(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float load(const uint16_t* p, int64_t i)
{
    return __uint_as_float(static_cast<uint32_t>(p[i]) << 16);
}
__device__ __forceinline__ void store(float* p, int64_t i, float v) { p[i] = v; }
__device__ __forceinline__ void store(uint16_t* p, int64_t i, float v)
{
    const uint32_t b = __float_as_uint(v);
    p[i] = static_cast<uint16_t>(v != v ? (b >> 16) | 0x40u : (b + 0x7FFFu + ((b >> 16) & 1u)) >> 16);
}

// a = sigmoid(g) and b = 1 - a, each to full precision whatever its size: with
// E = exp(-|g|) <= 1 the larger is 1 / (1 + E) and the smaller E / (1 + E).
__device__ __forceinline__ void gates(float g, float& a, float& b)
{
    const float E = __builtin_amdgcn_exp2f(__builtin_fabsf(g) * -kLog2e);
    const float big = 1.0f / (1.0f + E);
    const float small = E * big;
    a = g >= 0.0f ? big : small;
    b = g >= 0.0f ? small : big;
}

// Sequence b's tokens, within [0, tokens] whatever the offsets hold.
__device__ __forceinline__ void range(const gem_scan& s, int b, int64_t& lo, int64_t& hi)
{
    if (s.offsets) {
        lo = s.offsets[b];
        hi = s.offsets[b + 1];
    } else {
        const int64_t n = s.tokens / s.sequences;
        lo = b * n;
        hi = lo + n;
    }
    lo = lo < 0 ? 0 : lo > s.tokens ? s.tokens : lo;
    hi = hi < lo ? lo : hi > s.tokens ? s.tokens : hi;
}

template <class T>
__global__ __launch_bounds__(kThreads) void forward_kernel(const ScanArgs a)
{
    const int c = blockIdx.x * kThreads + threadIdx.x, b = blockIdx.y;
    if (c >= a.s.channels) return;
    int64_t lo, hi;
    range(a.s, b, lo, hi);
    const T* x = static_cast<const T*>(a.s.x);
    const T* g = static_cast<const T*>(a.s.gate);
    const int64_t D = a.s.channels;
    float h = a.s.h0 ? a.s.h0[b * D + c] : 0.0f;
    for (int64_t t = lo; t < hi; ++t) {
        if (a.states && t % kScanTile == 0) a.states[t / kScanTile * D + c] = h;
        float k, i;
        gates(load(g, t * a.s.gate_stride + c), k, i);
        h = __builtin_fmaf(k, h, i * load(x, t * a.s.x_stride + c));
        store(static_cast<T*>(a.y), t * a.y_stride + c, h);
    }
    if (a.h_last) a.h_last[b * D + c] = h;
}

template <class T>
__global__ __launch_bounds__(kThreads) void backward_kernel(const ScanBackArgs a)
{
    __shared__ float before[kScanTile][kThreads];
    const int c = blockIdx.x * kThreads + threadIdx.x, b = blockIdx.y;
    if (c >= a.s.channels) return;
    int64_t lo, hi;
    range(a.s, b, lo, hi);
    const T* x = static_cast<const T*>(a.s.x);
    const T* g = static_cast<const T*>(a.s.gate);
    const T* dy = static_cast<const T*>(a.dy);
    const int64_t D = a.s.channels;
    float e = a.dh_last ? a.dh_last[b * D + c] : 0.0f;
    for (int64_t end = hi; end > lo;) {
        int64_t begin = (end - 1) / kScanTile * kScanTile;
        float h;
        if (begin <= lo) {
            begin = lo;
            h = a.s.h0 ? a.s.h0[b * D + c] : 0.0f;
        } else {
            h = a.states[begin / kScanTile * D + c];
        }
        for (int64_t t = begin; t < end; ++t) {
            before[t - begin][threadIdx.x] = h;
            float k, i;
            gates(load(g, t * a.s.gate_stride + c), k, i);
            h = __builtin_fmaf(k, h, i * load(x, t * a.s.x_stride + c));
        }
        for (int64_t t = end - 1; t >= begin; --t) {
            float k, i;
            gates(load(g, t * a.s.gate_stride + c), k, i);
            const float r = load(dy, t * a.dy_stride + c) + e;
            store(static_cast<T*>(a.dx), t * a.dx_stride + c, i * r);
            store(static_cast<T*>(a.dgate), t * a.dgate_stride + c,
                  k * i * (before[t - begin][threadIdx.x] - load(x, t * a.s.x_stride + c)) * r);
            e = k * r;
        }
        end = begin;
    }
    if (a.dh0) a.dh0[b * D + c] = e;
}

}  // namespace

hipError_t launch_scan_forward(const ScanArgs& a, bool bf16, hipStream_t stream)
{
    const dim3 grid((a.s.channels + kThreads - 1) / kThreads, a.s.sequences);
    if (bf16) hipLaunchKernelGGL((forward_kernel<uint16_t>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((forward_kernel<float>), grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_scan_backward(const ScanBackArgs& a, bool bf16, hipStream_t stream)
{
    const dim3 grid((a.s.channels + kThreads - 1) / kThreads, a.s.sequences);
    if (bf16) hipLaunchKernelGGL((backward_kernel<uint16_t>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((backward_kernel<float>), grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace gemk
