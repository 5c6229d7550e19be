// gem_rows_device.hpp -- code shared by the kernels that walk along the tokens of packed
// sequences: a lane's channels, the sequences' bounds, and grids that loop.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gem_ops.hpp"
#include "gem_ops_device.hpp"

namespace gemk {
namespace {

constexpr int kThreads = 256;
constexpr int kLanes = 32;                 // lanes of a row
constexpr int kRows = kThreads / kLanes;   // rows of a block
constexpr int kStep = kStateTokens;        // tokens that a lane loads at a time
// Tokens are counted in ints, and walks look up to three steps past the last one.
static_assert(GEM_TOKENS_MAX <= INT32_MAX - 3 * kStep, "positions of tokens fit an int");

template <class T> constexpr int kChan = 8 / static_cast<int>(sizeof(T));   // channels of a lane
template <class T> constexpr int kSlice = kLanes * kChan<T>;                // and of a row

// ---- elements ----------------------------------------------------------------------

// A lane's channels of a row of the array, at any address of the elements' own alignment.
template <class T> using Raw = uint32_t __attribute__((ext_vector_type(2), aligned(sizeof(T))));

__device__ __forceinline__ void widen(uint32_t lo, uint32_t hi, float (&v)[2])
{
    v[0] = __uint_as_float(lo);
    v[1] = __uint_as_float(hi);
}
__device__ __forceinline__ void widen(uint32_t lo, uint32_t hi, float (&v)[4])
{
    v[0] = __uint_as_float(lo << 16);
    v[1] = __uint_as_float(lo & 0xFFFF0000u);
    v[2] = __uint_as_float(hi << 16);
    v[3] = __uint_as_float(hi & 0xFFFF0000u);
}
template <class T> __device__ __forceinline__ Raw<T> narrow(const float (&v)[kChan<T>])
{
    if constexpr (kChan<T> == 2) return Raw<T>{__float_as_uint(v[0]), __float_as_uint(v[1])};
    else return Raw<T>{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
}

// A lane's channels [c, c + n) of which it stores those in [from, to).  The last slice is
// moved back to be whole, and what it shares with the one before is stored by that one;
// with fewer channels than a slice lanes share them likewise.
struct Channels {
    int c, from, to;
};
template <class T> __device__ __forceinline__ Channels channels_of(int channels, int slice)
{
    const int lane = threadIdx.x % kLanes * kChan<T>;
    if (channels >= kSlice<T>) {
        const int first = slice * kSlice<T>, last = channels - kSlice<T>;
        return {(first < last ? first : last) + lane, first, channels};
    }
    const int last = channels - kChan<T>;
    return {last < 0 ? 0 : lane < last ? lane : last, lane, channels};
}

// Non-temporal, which leaves the Infinity Cache to what is written: rows copied at 6.3 TB/s,
// 5.2 without.  (The maps' pass read for the second one's sake, it took 80 us instead of 53
// for 268 MB and saved the other 8.)
// Channels in all: a multiple of a lane's (a lane that stores any then stores all), not so,
// or fewer than a lane has (the last is repeated).
enum : int { kEven, kOdd, kFew };

template <class T, int KIND>
__device__ __forceinline__ Raw<T> fetch(const T* row, const Channels& o)
{
    if constexpr (KIND != kFew) {
        return __builtin_nontemporal_load(reinterpret_cast<const Raw<T>*>(row + o.c));
    } else {
        Raw<T> r{};
        T* e = reinterpret_cast<T*>(&r);
#pragma unroll
        for (int i = 0; i < kChan<T>; ++i) e[i] = row[i < o.to ? i : o.to - 1];
        return r;
    }
}
template <int N> __device__ __forceinline__ void fetch_f32(const float* row, const Channels& o, float (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = row[o.c + i < o.to ? o.c + i : o.to - 1];
}
template <int N> __device__ __forceinline__ void fetch_or_zero(const float* array, int64_t at, const Channels& o, float (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.0f;
    if (array) fetch_f32(array + at * o.to, o, v);
}

template <class T, int KIND>
__device__ __forceinline__ void put(T* row, const Channels& o, bool whole, const Raw<T>& r)
{
    if (KIND == kEven || whole) {
        *reinterpret_cast<Raw<T>*>(row + o.c) = r;
    } else {
        const T* e = reinterpret_cast<const T*>(&r);
#pragma unroll
        for (int i = 0; i < kChan<T>; ++i)
            if (o.c + i >= o.from && o.c + i < o.to) row[o.c + i] = e[i];
    }
}
// Whether a lane stores none of its channels (it has nothing to do: no lane needs another),
// and whether all of them.
template <class T> __device__ __forceinline__ bool idle(const Channels& o)
{
    return o.c + kChan<T> <= o.from || o.from >= o.to;
}
template <class T> __device__ __forceinline__ bool whole(const Channels& o) { return o.from <= o.c && o.c + kChan<T> <= o.to; }
template <int N> __device__ __forceinline__ void put_f32(float* row, const Channels& o, const float (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (o.c + i >= o.from && o.c + i < o.to) row[o.c + i] = v[i];
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

// ---- sequences ---------------------------------------------------------------------------

// First tokens of sequences; of sequence `sequences` the end.
struct Bounds {
    const int64_t* offsets;
    int64_t len;               // of each sequence, without offsets
    int n;

    __device__ int operator()(int b) const
    {
        const int64_t t = offsets ? offsets[b] : b * len;
        return static_cast<int>(t < 0 ? 0 : t > INT32_MAX ? INT32_MAX : t);
    }

    // The last sequence that begins at or before token t (0 if there is none).
    __device__ int at(int t) const
    {
        if (!offsets) return static_cast<int>(static_cast<uint32_t>(t) / static_cast<uint32_t>(len));
        int lo = 0, hi = n;    // the first that begins later is in (lo, hi]
        while (hi - lo > 1) {
            const int mid = lo + (hi - lo) / 2;
            if (offsets[mid] <= t) lo = mid;
            else hi = mid;
        }
        return lo;
    }
};

// ---- grids -----------------------------------------------------------------------------------

int64_t over(int64_t n, int64_t part) { return (n + part - 1) / part; }

// Blocks of kernels that loop over what is left.
constexpr int64_t kLoopBlocks = int64_t{1} << 20;
dim3 loop_grid(int64_t blocks) { return dim3(static_cast<unsigned>(blocks < kLoopBlocks ? blocks : kLoopBlocks)); }

}  // namespace
}  // namespace gemk
