// gem_logits.hip -- scores of rows of logits, and the distillation loss with its
// gradient, for gfx950.
//
// A row of a large vocabulary is read once: every thread keeps a sum of exponentials
// about a reference of its own, which only moves when a logit lies 20 octaves above
// it (the sums stay far from overflow, and no running maximum is carried from element
// to element).  Bytes of logits bound it, and the vector instructions of an element
// come close: an exponential, two fused multiply-adds, an addition, a conversion and
// half a maximum.
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
// no logit is above -inf.
struct Sums {
    float ref, s, t;
};

template <int WAVES>
__device__ __forceinline__ Sums block_sums(const Run& r, float scale, float (*lds)[4])
{
    const float top = wave_max(r.at.ref);
    float s = r.s, t = r.t;
    if (r.at.ref > -kInf) shift_sums<true>(s, t, (r.at.ref - top) * scale - r.at.skew(scale));
    s = wave_sum(s);
    t = wave_sum(t);
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
        lds[wave][0] = top;
        lds[wave][1] = s;
        lds[wave][2] = t;
    }
    __syncthreads();
    Sums out{lds[0][0], 0.0f, 0.0f};
#pragma unroll
    for (int w = 1; w < WAVES; ++w) out.ref = __builtin_fmaxf(out.ref, lds[w][0]);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        s = lds[w][1];
        t = lds[w][2];
        if (lds[w][0] > -kInf) shift_sums<true>(s, t, (lds[w][0] - out.ref) * scale);
        out.s += s;
        out.t += t;
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

// ---- alternatives ----------------------------------------------------------------

// The order of logits as an integer's (the two zeros are equal); 0 for -inf and NaN,
// which are no alternatives.
__device__ __forceinline__ uint32_t order(float v)
{
    const uint32_t b = __float_as_uint(v + 0.0f);
    const uint32_t o = b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
    return v > -kInf ? o : 0u;
}
__device__ __forceinline__ float ordered(uint32_t o)
{
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
// Larger logits first, of equal ones the lower token.
__device__ __forceinline__ uint64_t rank_key(uint32_t o, uint32_t token)
{
    return o ? (static_cast<uint64_t>(o) << 32) | static_cast<uint32_t>(~token) : 0;
}
__device__ __forceinline__ int key_token(uint64_t key) { return static_cast<int>(~static_cast<uint32_t>(key)); }

// The k largest of a row lie in the k groups of eight whose largest elements rank
// highest (each group ahead of another has an element that ranks ahead of all of the
// other's).  So the pass over the row keeps one key a group in LDS, and only k groups
// are looked at again.  The key of a group is its largest element as it is; of bfloat16 logits
// 16 bits.
constexpr int kGroup = 8;
template <class T> struct GroupKey;
template <> struct GroupKey<uint16_t> {
    using Type = uint16_t;
    static constexpr int kShift = 16;      // bits of an order that a key does not need
    static __device__ Type of(float v) { return static_cast<uint16_t>(__float_as_uint(v) >> 16); }
    static __device__ uint32_t order_of(Type k) { return order(__uint_as_float(static_cast<uint32_t>(k) << 16)) >> 16; }
};
template <> struct GroupKey<float> {
    using Type = float;
    static constexpr int kShift = 0;
    static __device__ Type of(float v) { return v; }
    static __device__ uint32_t order_of(Type k) { return order(k); }
};
// Elements of a part: 32 KiB of group keys.
template <class T> constexpr int kPartMax = (32 << 10) / static_cast<int>(sizeof(typename GroupKey<T>::Type)) * kGroup;

constexpr int kList = 1024;                // GEM_TOP_MAX groups of kGroup
static_assert(kList >= GEM_TOP_MAX * kGroup, "a group's elements fit");

struct TopLds {
    uint64_t list[kList];
    uint64_t sel[GEM_TOP_MAX];
    uint32_t high[kThreads];
    int wave[2][kThreads / 64];
    int count;
};

__device__ __forceinline__ void push(TopLds& l, uint64_t key)
{
    const int at = atomicAdd(&l.count, 1);
    if (at < kList) l.list[at] = key;
}

// The n keys of list in falling order into out, the first k of them.  All keys are
// different, so a key's rank is the number of larger ones.
__device__ __forceinline__ void rank_list(TopLds& l, int n, int k, uint64_t* out)
{
    for (int c = threadIdx.x; c < n; c += kThreads) {
        const uint64_t mine = l.list[c];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += l.list[j] > mine;
        if (rank < k) out[rank] = mine;
    }
}

// A bound below which no key is among the k largest: the list of keys at or above it
// has at least k (or all that are not 0), and at most `fit`.  key(j) gives the j-th of
// this thread's `mine` keys.
template <class F>
__device__ uint64_t bound_of(TopLds& l, int mine, int k, int fit, F key)
{
    uint64_t bound = 0;
    int turn = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const uint64_t trial = bound | (uint64_t{1} << bit);
        int n = 0;
        for (int j = 0; j < mine; ++j) n += key(j) >= trial;
#pragma unroll
        for (int m = 32; m > 0; m >>= 1) n += __shfl_xor(n, m);
        if ((threadIdx.x & 63) == 0) l.wave[turn][threadIdx.x >> 6] = n;
        __syncthreads();
        n = 0;
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) n += l.wave[turn][w];
        turn ^= 1;
        if (n >= k) {
            bound = trial;
            if (n <= fit) break;
        }
    }
    return bound ? bound : 1;
}

// The keys once more, for a part with a NaN: a signalling one may have hidden the numbers beside
// it from max3, and to a comparison all are alike.  Each key is written by the thread that wrote
// it before.
template <class T>
__device__ void key_again(const Part<T>& part, typename GroupKey<T>::Type* keys, int groups, float& high)
{
    constexpr int kLanes = kGroup / kVec<T>;
    const int tid = threadIdx.x;
    const auto most = [](const float (&x)[kVec<T>], float m) {
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) m = x[i] > m ? x[i] : m;
        return m;
    };
    float x[kVec<T>];
    high = -kInf;
    if (tid < 2) {
        part.edge(x);
        high = most(x, high);
        keys[tid == 0 ? 0 : groups - 1] = GroupKey<T>::of(high);
    }
    if (tid % kLanes) return;
    for (int g = tid / kLanes; g < groups - 2; g += kThreads / kLanes) {
        float m = -kInf;
        for (int v = g * kLanes; v < (g + 1) * kLanes && v < part.nvec; ++v) {
            unpack(part.body()[v], x);
            m = most(x, m);
        }
        keys[1 + g] = GroupKey<T>::of(m);
        high = m > high ? m : high;
    }
}

// The part's k largest logits as keys in l.sel (0 where there are fewer).  keys holds
// a key for the head, for each group of the body, and for the tail; high is the
// largest key of this thread's elements, seen the largest that it put there.
template <class T>
__device__ void select_top(TopLds& l, const Part<T>& part, const typename GroupKey<T>::Type* keys, int groups,
                           uint32_t high, uint32_t seen, int k)
{
    constexpr int shift = GroupKey<T>::kShift;
    const int tid = threadIdx.x, lane = tid & 63;
    l.high[tid] = high;
    if (tid == 0) l.count = 0;
    __syncthreads();
    // A first bound: the k-th of the threads' largest elements (16 bits of their keys).
    uint32_t q[kThreads / 64];
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) q[w] = l.high[lane + 64 * w];
    uint32_t low = 0;
#pragma unroll 1
    for (int bit = 31 - shift; bit >= 16 - shift; --bit) {
        const uint32_t trial = low | (1u << bit);
        int n = 0;
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) n += __builtin_popcountll(__ballot(q[w] >= trial));
        if (n >= k) low = trial;
    }
    if (low == 0) low = 1;
    // Each thread looks through the groups that it put there: group g of the body (key
    // 1 + g) begins with the vector of thread g * kLanes % kThreads.
    constexpr int kLanes = kGroup / kVec<T>;
    if (seen >= low && tid % kLanes == 0)
        for (int g = 1 + tid / kLanes; g < groups - 1; g += kThreads / kLanes) {
            const uint32_t o = GroupKey<T>::order_of(keys[g]);
            if (o >= low) push(l, (static_cast<uint64_t>(o) << 32) | static_cast<uint32_t>(~g));
        }
    if (tid < 2) {
        const int g = tid == 0 ? 0 : groups - 1;
        const uint32_t o = GroupKey<T>::order_of(keys[g]);
        if (o >= low) push(l, (static_cast<uint64_t>(o) << 32) | static_cast<uint32_t>(~g));
    }
    __syncthreads();
    int n = l.count;
    if (n > kList) {
        // Many equal groups: a bound that leaves few enough.
        const auto key = [&](int j) {
            const int g = tid + j * kThreads;
            const uint32_t o = GroupKey<T>::order_of(keys[g]);
            return o ? (static_cast<uint64_t>(o) << 32) | static_cast<uint32_t>(~g) : uint64_t{0};
        };
        const int mine = tid < groups ? (groups - tid + kThreads - 1) / kThreads : 0;
        const uint64_t bound = bound_of(l, mine, k, kList, key);
        __syncthreads();
        if (tid == 0) l.count = 0;
        __syncthreads();
        for (int j = 0; j < mine; ++j)
            if (key(j) >= bound) push(l, key(j));
        __syncthreads();
        n = l.count;
    }
    rank_list(l, n, k, l.sel);
    __syncthreads();
    if (tid == 0) l.count = 0;
    const int picked = n < k ? n : k;
    const uint32_t least = picked == k ? static_cast<uint32_t>(l.sel[k - 1] >> 32) : 1u;
    __syncthreads();
    for (int j = tid; j < picked * kGroup; j += kThreads) {
        const int g = static_cast<int>(~static_cast<uint32_t>(l.sel[j / kGroup])), i = j % kGroup;
        const int end = part.head + part.nvec * kVec<T>;
        const int at = g == 0 ? i : g == groups - 1 ? end + i : part.head + (g - 1) * kGroup + i;
        const int stop = g == 0 ? part.head : g == groups - 1 ? part.n : end;
        if (at < stop) {
            const uint32_t o = order(load(part.p, at));
            if ((o >> shift) >= least) push(l, rank_key(o, static_cast<uint32_t>(part.begin + at)));
        }
    }
    __syncthreads();
    n = l.count;
    if (tid < k) l.sel[tid] = 0;
    __syncthreads();
    rank_list(l, n, k, l.sel);
    __syncthreads();
}

// ---- scores -------------------------------------------------------------------------

// What a part of a row leaves for the row's joining block.
struct PartSums {
    float ref, s, t, lref;
};

__device__ __forceinline__ float log_prob(const LogitArgs& a, float x, float ref, float ls)
{
    return x == -kInf ? x : (x - ref) * a.inv_t - ls * kLn2;
}

// A log probability and an entropy have a side of 0 to be on, which near a single outcome is
// less than their rounding.
__device__ __forceinline__ float at_most_0(float v) { return v > 0.0f ? 0.0f : v; }
__device__ __forceinline__ float at_least_0(float v) { return v < 0.0f ? 0.0f : v; }

// A row's outputs from its sums and its alternatives' keys.
template <class T>
__device__ void write_scores(const ScoreArgs& a, int64_t r, const T* row, const Sums& u, const uint64_t* top)
{
    const float ls = __builtin_log2f(u.s);
    if (threadIdx.x == 0) {
        if (a.out.lse) a.out.lse[r] = u.ref * a.l.inv_t + ls * kLn2;
        if (a.out.entropy) a.out.entropy[r] = u.s == 0.0f ? 0.0f : at_least_0((ls - u.t / u.s) * kLn2);
    }
    for (int i = threadIdx.x; i < a.n_tokens; i += kThreads) {
        const int token = a.tokens[r * a.n_tokens + i];
        float lp = 0.0f;
        if (token >= 0 && token < a.l.vocab) lp = at_most_0(log_prob(a.l, load(row, token), u.ref, ls));
        a.out.logprob[r * a.n_tokens + i] = lp;
    }
    for (int i = threadIdx.x; i < a.top_k; i += kThreads) {
        const uint64_t key = top[i];
        if (a.out.top_ids) a.out.top_ids[r * a.top_k + i] = key ? key_token(key) : -1;
        if (a.out.top_logprob)
            a.out.top_logprob[r * a.top_k + i] =
                key ? at_most_0(log_prob(a.l, ordered(static_cast<uint32_t>(key >> 32)), u.ref, ls)) : -kInf;
    }
}

// One part of one row a block.  A whole row is written out; parts leave their sums
// and keys for join_kernel.  Four waves a block leave a compute unit several rows at
// different steps, so that one streams while another selects: 4096 rows of 65536 bfloat16
// with 5 alternatives take 101 us (5.3 TB/s), 2048 of 131072 with 64 125 us.
template <class T, bool TOP>
__global__ __launch_bounds__(kThreads) void score_kernel(const ScoreArgs a, int64_t row0, int parts, int len,
                                                         PartSums* sums, uint64_t* tops)
{
    using Key = typename GroupKey<T>::Type;
    constexpr int shift = GroupKey<T>::kShift;
    extern __shared__ uint32_t dynamic_lds[];
    Key* keys = reinterpret_cast<Key*>(dynamic_lds);
    __shared__ float lds[kThreads / 64][4];
    __shared__ TopLds top;
    const int64_t r = row0 + blockIdx.x / parts;
    const int q = blockIdx.x % parts, tid = threadIdx.x;
    const T* row = static_cast<const T*>(a.l.z) + r * a.l.stride;
    const Part<T> part(row, a.l.vocab, q * len, len);
    const float scale = a.l.scale, reach = 20.0f / scale;
    const int groups = (part.nvec * kVec<T> + kGroup - 1) / kGroup + 2;
    Run run;
    float high = -kInf, seen = -kInf;  // the largest of the thread's elements, and of its groups
    if (tid < 64) {
        float x[kVec<T>];
        part.edge(x);
        const float m = most_of(x);
        add<true>(run, x, m, scale, reach);
        if constexpr (TOP)
            if (tid < 2) {
                high = seen = __builtin_fmaxf(high, m);
                keys[tid == 0 ? 0 : groups - 1] = GroupKey<T>::of(m);
            }
    }
    stream<kThreads, kUnroll>(part.body(), part.nvec, [&](int v, u32x4 raw, bool inside) {
        float x[kVec<T>];
        unpack(inside ? raw : u32x4{lowest<T>(), lowest<T>(), lowest<T>(), lowest<T>()}, x);
        const float m = most_of(x);
        add<true>(run, x, m, scale, reach);
        if constexpr (TOP) {
            high = max3(high, m, m);
            if constexpr (kVec<T> < kGroup) {
                // Two neighbours share a group.
                const float other = __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(m), 0xB1, 0xF, 0xF, true));
                const float both = max3(m, other, other);
                seen = max3(seen, both, both);
                if (inside && (v & 1) == 0) keys[1 + v / 2] = GroupKey<T>::of(both);
            } else if (inside) {
                keys[1 + v] = GroupKey<T>::of(m);
            }
        }
    });
    const Sums u = block_sums<kThreads / 64>(run, scale, lds);
    if constexpr (TOP) {
        if (__builtin_expect(u.s != u.s, 0)) {
            key_again(part, keys, groups, high);
            seen = high;
        }
        select_top(top, part, keys, groups, order(high) >> shift, order(kVec<T> < kGroup ? seen : high) >> shift, a.top_k);
    }
    if (parts == 1) {
        write_scores(a, r, row, u, top.sel);
    } else {
        if (tid == 0) sums[blockIdx.x] = PartSums{u.s == 0.0f ? -kInf : u.ref, u.s, u.t, 0.0f};
        if constexpr (TOP)
            if (tid < a.top_k) tops[static_cast<int64_t>(blockIdx.x) * a.top_k + tid] = top.sel[tid];
    }
}

// A row's parts joined (parts <= kPartsMax).  With few rows only their split keeps the
// device busy: one row of 32768 with 20 alternatives takes 12 us, both launches together.
constexpr int kPartsMax = 64;

template <class T>
__global__ __launch_bounds__(kThreads) void join_kernel(const ScoreArgs a, int64_t row0, int parts,
                                                        const PartSums* sums, const uint64_t* tops)
{
    extern __shared__ uint32_t dynamic_lds[];
    uint64_t* keys = reinterpret_cast<uint64_t*>(dynamic_lds);
    __shared__ float lds[kThreads / 64][4];
    __shared__ TopLds top;
    const int64_t r = row0 + blockIdx.x;
    const int tid = threadIdx.x;
    const T* row = static_cast<const T*>(a.l.z) + r * a.l.stride;
    Run run;
    if (tid < parts) {
        const PartSums p = sums[static_cast<int64_t>(blockIdx.x) * parts + tid];
        run.at.ref = p.ref;    // its sums have no skew
        run.at.wide = true;
        run.s = p.s;
        run.t = p.t;
    }
    const int n = parts * a.top_k;
    for (int j = tid; j < n; j += kThreads) keys[j] = tops[static_cast<int64_t>(blockIdx.x) * n + j];
    if (tid == 0) top.count = 0;
    const Sums u = block_sums<kThreads / 64>(run, a.l.scale, lds);
    if (a.top_k) {
        const int mine = tid < n ? (n - tid + kThreads - 1) / kThreads : 0;
        const auto key = [&](int j) { return keys[tid + j * kThreads]; };
        const uint64_t bound = bound_of(top, mine, a.top_k, kThreads, key);
        for (int j = 0; j < mine; ++j)
            if (key(j) >= bound) push(top, key(j));
        if (tid < a.top_k) top.sel[tid] = 0;
        __syncthreads();
        rank_list(top, top.count, a.top_k, top.sel);
        __syncthreads();
    }
    write_scores(a, r, row, u, top.sel);
}

// ---- distillation ----------------------------------------------------------------

struct DistillLds {
    float sums[kMostWaves][4];
    float red[kMostWaves];
    alignas(16) int ids[GEM_TOP_MAX];
    uint32_t edges[2];         // marks of the head and the tail
};

// Thread i's entry of a row's record as it is given.
struct Entry {
    int id = -1;
    float lp = -kInf;
};

__device__ __forceinline__ Entry entry_of(const DistillArgs& a, int64_t r)
{
    Entry e;
    const int tid = threadIdx.x;
    if (tid < a.k) {
        e.id = a.ids[r * a.k + tid];
        e.lp = a.lp[r * a.k + tid];
        if (e.id < 0 || e.id >= a.l.vocab) e.id = -1;
    }
    return e;
}

// Thread i's token, -1 if an earlier entry has it: of equal ones the first counts.
__device__ __forceinline__ int distinct(const Entry& e, int k, DistillLds& l)
{
    const int tid = threadIdx.x;
    if (tid < GEM_TOP_MAX) l.ids[tid] = e.id;
    __syncthreads();
    if (tid >= k) return -1;
    bool again = false;
    for (int i = 0; i < tid; i += 16) {
        int4 ids[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) ids[j] = reinterpret_cast<const int4*>(l.ids + i)[j];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int at = tid - i - 4 * j;
            again |= (ids[j].x == e.id && at > 0) || (ids[j].y == e.id && at > 1) || (ids[j].z == e.id && at > 2) ||
                     (ids[j].w == e.id && at > 3);
        }
    }
    return again ? -1 : e.id;
}

// Thread i's entry as it counts: its token (-1: none), log probability and probability; the
// row's p_t and mass, the sum of all p and p_t; and the token's logit.  A NaN in a record makes
// its p, the mass and with them loss and gradient NaN.
struct Teacher {
    int id = -1;
    float lp = 0.0f, p = 0.0f, pt = 0.0f, mass = 0.0f, x = -kInf;
};

template <int WAVES>
__device__ __forceinline__ Teacher teacher_of(const DistillArgs& a, const Entry& e, DistillLds& l)
{
    Teacher t;
    t.id = distinct(e, a.k, l);
    const float lp = t.id < 0 ? -kInf : e.lp;
    if (a.tail) {
        t.lp = lp;
        t.p = t.id >= 0 ? expf(lp) : 0.0f;
        const float sum = block_sum<WAVES>(t.p, l.red);
        t.pt = sum > 1.0f ? 0.0f : 1.0f - sum;
        t.mass = sum <= 1.0f ? 1.0f : sum;
    } else {
        const float top = block_max<WAVES>(lp, l.red);
        t.p = lp == -kInf ? 0.0f : expf(lp - top);
        const float sum = block_sum<WAVES>(t.p, l.red);
        t.lp = lp - (top + logf(sum));
        t.p = sum == 0.0f ? 0.0f : t.p / sum;
        t.mass = sum == 0.0f ? 0.0f : sum / sum;
    }
    return t;
}

// Marks a listed token of the part: a bit for its element in the byte of its vector v,
// byte_of(v), or in that of the head or the tail.
template <class T, class F>
__device__ __forceinline__ void mark(const Part<T>& part, uint32_t* marks, DistillLds& l, int id, F byte_of)
{
    const int at = id - part.begin, end = part.head + part.nvec * kVec<T>;
    if (id < 0 || at < 0 || at >= part.n) return;
    if (at < part.head) {
        atomicOr(&l.edges[0], 1u << at);
    } else if (at >= end) {
        atomicOr(&l.edges[1], 1u << (at - end));
    } else {
        const int byte = byte_of((at - part.head) / kVec<T>);
        atomicOr(&marks[byte / 4], 1u << (byte % 4 * 8 + (at - part.head) % kVec<T>));
    }
}
__host__ __device__ constexpr int mark_words(int nvec) { return (nvec + 3) / 4; }

// Without the listed elements.
template <int N> __device__ __forceinline__ void drop(float (&x)[N], uint32_t listed)
{
    if (__builtin_expect(__ballot(listed != 0) == 0, 0)) return;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = listed >> i & 1u ? -kInf : x[i];
}

// The same of a vector's bits.
__device__ __forceinline__ u32x4 drop(u32x4 v, uint32_t listed, float)
{
    if (__builtin_expect(__ballot(listed != 0) == 0, 0)) return v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = listed >> i & 1u ? 0xFF800000u : v[i];
    return v;
}
__device__ __forceinline__ u32x4 drop(u32x4 v, uint32_t listed, uint16_t)
{
    if (__builtin_expect(__ballot(listed != 0) == 0, 0)) return v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = listed >> 2 * i & 1u ? (v[i] & 0xFFFF0000u) | 0xFF80u : v[i];
        v[i] = listed >> (2 * i + 1) & 1u ? (v[i] & 0xFFFFu) | 0xFF800000u : v[i];
    }
    return v;
}

// The head and the tail, without their marked elements.
template <class T>
__device__ __forceinline__ void take_edges(const Part<T>& part, Run& run, const DistillLds& l, float scale, float reach)
{
    if (threadIdx.x >= 64) return;
    float x[kVec<T>];
    part.edge(x);
    drop(x, threadIdx.x < 2 ? l.edges[threadIdx.x] : 0u);
    add<false>(run, x, most_of(x), scale, reach);
}

// With a tail, listed tokens' exponentials are summed apart, about a reference of their own:
// unlisted ones may lie so far below that about a common one they are nothing, and p_t q_v / q_t
// is of q_t's size whatever that is.  An entry's thread has one, about itself.
struct Listed {
    float ref = -kInf, t = 0.0f;
};
template <class T> __device__ __forceinline__ Listed listed_of(const Part<T>& part, const Teacher& t)
{
    Listed l;
    if (t.id >= part.begin && t.id < part.begin + part.n) l.ref = t.x;
    l.t = l.ref == -kInf ? 0.0f : 1.0f;
    return l;
}
__device__ __forceinline__ float moved(float t, float ref, float to, float scale)
{
    return t == 0.0f ? 0.0f : t * __builtin_amdgcn_exp2f((ref - to) * scale);
}

template <int CTRL> __device__ __forceinline__ float other_lane(float v)
{
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xF, 0xF, true));
}
// Two values joined over the wave, step by step together, the steps inside a row of 16 lanes
// without LDS: a small call takes 0.2 to 0.8 us less than with all of them there (2 x 2280 and 1 x
// 8753 binary32).
template <class F> __device__ __forceinline__ void wave_both(float& a, float& b, F f)
{
    const auto step = [&](auto get) {
        const float x = get(a), y = get(b);
        a = f(a, x);
        b = f(b, y);
    };
    step([](float v) { return other_lane<0xB1>(v); });         // its neighbour in a pair
    step([](float v) { return other_lane<0x4E>(v); });         // the other pair of four
    step([](float v) { return other_lane<0x141>(v); });        // the other four of eight
    step([](float v) { return other_lane<0x140>(v); });        // the other eight of sixteen
    step([](float v) { return __shfl_xor(v, 16); });
    step([](float v) { return __shfl_xor(v, 32); });
}

// A row's (or a part's) sums: s of unlisted tokens (without a tail of all) about ref, t of listed
// ones about lref; a reference is -inf where no logit is above it.
template <int WAVES>
__device__ __forceinline__ PartSums block_parts(const Run& r, Listed l, bool tail, float scale, float (*lds)[4])
{
    float top = r.at.ref, ltop = l.ref;
    wave_both(top, ltop, [](float a, float b) { return __builtin_fmaxf(a, b); });
    float s = r.s, none = 0.0f, t = moved(l.t, l.ref, ltop, scale);
    if (r.at.ref > -kInf) shift_sums<false>(s, none, (r.at.ref - top) * scale - r.at.skew(scale));
    wave_both(s, t, [](float a, float b) { return a + b; });
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
        lds[wave][0] = top;
        lds[wave][1] = s;
        lds[wave][2] = t;
        lds[wave][3] = ltop;
    }
    __syncthreads();
    PartSums out{lds[0][0], 0.0f, 0.0f, -kInf};
#pragma unroll
    for (int w = 1; w < WAVES; ++w) out.ref = __builtin_fmaxf(out.ref, lds[w][0]);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        s = lds[w][1];
        if (lds[w][0] > -kInf) shift_sums<false>(s, none, (lds[w][0] - out.ref) * scale);
        out.s += s;
    }
    if (tail) {
        constexpr int kWaves = GEM_TOP_MAX / 64;       // that hold entries
#pragma unroll
        for (int w = 0; w < kWaves; ++w) out.lref = __builtin_fmaxf(out.lref, lds[w][3]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) out.t += moved(lds[w][2], lds[w][3], out.lref, scale);
    }
    return out;
}
static_assert(GEM_TOP_MAX % 64 == 0 && GEM_TOP_MAX <= kThreads, "whole waves hold a row's entries");

// What loss and gradient take of a row's sums: the sum of all about top, log2 of it, and s about
// ref.
struct RowSums {
    float ref, s, top, all, ls;

    __device__ RowSums(const PartSums& p, float scale) : ref(p.ref), s(p.s)
    {
        top = __builtin_fmaxf(p.ref, p.lref);
        if (top == -kInf) top = 0.0f;
        if (ref == -kInf) ref = top;
        all = moved(s, ref, top, scale) + moved(p.t, p.lref, top, scale);
        ls = __builtin_log2f(all);
    }
    // log2 q_t.
    __device__ float rest(float scale) const { return __builtin_log2f(s) + (ref - top) * scale - ls; }
    // No unlisted token can occur: q_t is 0, or below the normal numbers of binary64, which a
    // mask of any value counts as (its gap to the others is no quantity).
    __device__ bool no_rest(float scale) const { return s == 0.0f || rest(scale) < -1022.0f; }
};

// A record of all tokens that can occur leaves its rounding for the tail (log probabilities of
// 32 bits, at most GEM_TOP_MAX of them), which no unlisted token of the student's can answer.
constexpr float kNoTail = 0x1p-16f;
__device__ __forceinline__ void drop_tail(Teacher& t, const RowSums& u, float scale)
{
    if (!(t.pt > 0.0f && t.pt <= kNoTail && u.no_rest(scale))) return;
    t.mass -= t.pt;
    t.pt = 0.0f;
}

// The row's loss, from thread i's entry.
template <int WAVES>
__device__ __forceinline__ float loss_of(const DistillArgs& a, const Teacher& t, const RowSums& u, DistillLds& l)
{
    float part = 0.0f;
    if (t.p != 0.0f) part = t.p * (t.lp - log_prob(a.l, t.x, u.top, u.ls));
    float loss = block_sum<WAVES>(part, l.red);
    if (t.pt > 0.0f) loss += u.no_rest(a.l.scale) ? kInf : t.pt * (logf(t.pt) - u.rest(a.l.scale) * kLn2);
    return loss;
}

// A row's gradient: c 2^d of unlisted tokens, about the reference of theirs, and of a listed one
// f (2^d inv - p) about that of all, with inv the record's mass over the sum of exponentials.  Every
// element is stored as an unlisted token's, and the listed ones again when those stores are
// done (stores_done), which spares the vectors a look at the marks.
struct Grad {
    Reference at;
    float c, f, inv, top;

    __device__ Grad(const DistillArgs& a, const Teacher& t, const RowSums& u, float w) : top(u.top)
    {
        at.set(u.ref, a.l.scale);
        f = w * a.l.inv_t;
        inv = u.all == 0.0f ? 0.0f : t.mass / u.all;
        const float rest = t.pt > 0.0f && !u.no_rest(a.l.scale) ? t.pt / u.s : 0.0f;
        c = f * (moved(inv, u.ref, u.top, a.l.scale) - rest) * __builtin_amdgcn_exp2f(-at.skew(a.l.scale));
    }

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

    template <class T> __device__ __forceinline__ void edges(const LogitArgs& l, const Part<T>& part, T* grad) const
    {
        if (threadIdx.x >= 2) return;
        T* out = grad + part.begin;
        const int from = part.edge_at(), m = part.edge_n();
        for (int i = from; i < from + m; ++i)
            store(out, i, c * __builtin_amdgcn_exp2f(at.exponent(load(part.p, i), l.scale)));
    }

    __device__ float listed(const Teacher& t, float scale) const
    {
        return f * (__builtin_amdgcn_exp2f((t.x - top) * scale) * inv - t.p);
    }
};

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

// What a block does with its part of a row: sums alone (left in part_sums, and the logits of
// the part's listed tokens in part_x, [rows][k]: the gradient may be written over the logits
// while another part's block needs them), the rest from those, or, with one part a row, both.
enum : int { kSums = 1, kRest = 2 };

// The part's sums over unlisted tokens (s); without MARKS over all.
template <class T, bool MARKS>
__device__ __forceinline__ void take_part(const Part<T>& part, Run& run, const uint32_t* marks, const DistillLds& l,
                                          float scale, float reach)
{
    take_edges(part, run, l, scale, reach);
    stream<kThreads, kUnroll>(part.body(), part.nvec, [&](int v, u32x4 raw, bool inside) {
        float x[kVec<T>];
        unpack(inside ? raw : u32x4{lowest<T>(), lowest<T>(), lowest<T>(), lowest<T>()}, x);
        if constexpr (MARKS) drop(x, inside ? reinterpret_cast<const uint8_t*>(marks)[v] : 0u);
        add<false>(run, x, most_of(x), scale, reach);
    });
}

// Bound by the bytes of the logits, and with few rows by its launches: 1024 rows of 50021
// bfloat16, the loss alone, 24 us (3.8 TB/s: all blocks start and end together); 37 rows of
// 100003 binary32 with the gradient 17 us, in parts and two launches.
template <class T, int STEP>
__global__ __launch_bounds__(kThreads) void distill_kernel(const DistillArgs a, int64_t row0, int parts, int len,
                                                           PartSums* part_sums, float* part_x)
{
    constexpr int WAVES = kThreads / 64;
    extern __shared__ uint32_t marks[];
    __shared__ DistillLds l;
    const int blocks = STEP == kRest && !a.grad ? 1 : parts;       // of a row
    const int64_t i = blockIdx.x / blocks, r = row0 + i;
    const int q = blockIdx.x % blocks, tid = threadIdx.x;
    const T* row = static_cast<const T*>(a.l.z) + r * a.l.stride;
    T* grad = a.grad ? static_cast<T*>(a.grad) + r * a.grad_stride : nullptr;
    const Part<T> part(row, a.l.vocab, q * len, len);
    const float w = a.weight ? a.weight[r] : 1.0f, scale = a.l.scale;
    if (w == 0.0f) {
        if (STEP & kRest) {
            if (tid == 0 && q == 0 && a.loss) a.loss[r] = 0.0f;
            if (grad) no_grad<kThreads>(part, grad);
        }
        return;
    }
    const Entry e = entry_of(a, r);
    if (STEP & kSums) {
        if (a.tail)
            for (int j = tid; j < mark_words(part.nvec); j += kThreads) marks[j] = 0;
        if (tid < 2) l.edges[tid] = 0;
    }
    Teacher t;
    if constexpr (STEP & kRest) t = teacher_of<WAVES>(a, e, l);
    else t.id = a.tail ? distinct(e, a.k, l) : e.id;
    if (t.id >= 0) t.x = STEP & kSums ? load(row, t.id) : part_x[i * a.k + tid];
    PartSums sums;
    Run run;
    Listed listed;
    if constexpr (STEP & kSums) {
        const float reach = 20.0f / scale;
        if (a.tail) {
            mark(part, marks, l, t.id, [](int v) { return v; });
            __syncthreads();
            take_part<T, true>(part, run, marks, l, scale, reach);
            listed = listed_of(part, t);
        } else {
            take_part<T, false>(part, run, marks, l, scale, reach);
        }
        sums = block_parts<WAVES>(run, listed, a.tail, scale, l.sums);
        if constexpr (!(STEP & kRest)) {
            if (tid == 0) part_sums[blockIdx.x] = sums;
            if (t.id >= part.begin && t.id < part.begin + part.n) part_x[i * a.k + tid] = t.x;
            return;
        }
    } else {
        if (tid < parts) {
            const PartSums p = part_sums[i * parts + tid];
            run.at.ref = p.ref;    // its sums have no skew
            run.at.wide = true;
            run.s = p.s;
            listed = Listed{p.lref, p.t};
        }
        sums = block_parts<WAVES>(run, listed, a.tail, scale, l.sums);
    }
    const RowSums u(sums, scale);
    drop_tail(t, u, scale);
    const float loss = loss_of<WAVES>(a, t, u, l);     // and every entry's logit is read
    if (a.loss && q == 0 && tid == 0) a.loss[r] = loss;
    if (!grad) return;
    const Grad g(a, t, u, w);
    T* body = grad + part.begin + part.head;
    const bool whole = (reinterpret_cast<uintptr_t>(body) & 15u) == 0;
    g.edges(a.l, part, grad);
    stream<kThreads, kUnroll>(part.body(), part.nvec, [&](int v, u32x4 raw, bool inside) {
        if (inside) g.vector(body, v, raw, whole, scale);
    });
    stores_done();
    __syncthreads();
    if (t.id >= part.begin && t.id < part.begin + part.n) store(grad, t.id, g.listed(t, scale));
}

// Loss and gradient with a row's vectors in registers, NV of a thread: what they hold is read
// once (with REST a row has more, which is read twice).  A block goes through rows; as each
// vector of a gradient is stored the next row's takes its place, so that loads and stores go
// on through the sums, and a row's listed elements are stored behind the next row's.
constexpr int kRestUnroll = 2;

template <class T, int THREADS, int NV, bool REST>
__global__ __launch_bounds__(THREADS, 4) void resident_kernel(const DistillArgs a)
{
    constexpr int WAVES = THREADS / 64, kKept = THREADS * NV;
    extern __shared__ __align__(16) uint32_t marks[];      // a thread's NV bytes, and one of every further vector
    __shared__ DistillLds l;
    const uint32_t tid = threadIdx.x;
    const float scale = a.l.scale, reach = 20.0f / scale;
    const auto part_of = [&](int64_t r) {
        return Part<T>(static_cast<const T*>(a.l.z) + r * a.l.stride, a.l.vocab, 0, a.l.vocab);
    };
    const auto grad_of = [&](int64_t r) { return static_cast<T*>(a.grad) + r * a.grad_stride; };
    const auto byte_of = [](int v) { return !REST || v < kKept ? v % THREADS * NV + v / THREADS : v; };
    float w = 0.0f;
    // The block's next row from r on that has a weight (or beyond the last), which it sets w to;
    // the gradients of those before it are zero.
    const auto next_row = [&](int64_t r) {
        for (; r < a.l.rows; r += gridDim.x) {
            w = a.weight ? a.weight[r] : 1.0f;
            if (w != 0.0f) break;
            if (tid == 0 && a.loss) a.loss[r] = 0.0f;
            no_grad<THREADS>(part_of(r), grad_of(r));
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
    for (uint32_t i = tid; i < static_cast<uint32_t>(mark_words(kKept)); i += THREADS) marks[i] = 0;
    if constexpr (REST)
        for (int i = kKept / 4 + tid; i < mark_words(a.l.vocab / kVec<T>); i += THREADS) marks[i] = 0;
    if (tid < 2) l.edges[tid] = 0;
    Entry e = entry_of(a, r);
    {
        const Part<T> part = part_of(r);
#pragma unroll
        for (int u = 0; u < NV; ++u)
            if (u * THREADS < part.nvec) fetch(part, u, tid);
    }
    __syncthreads();
    int listed_id = -1;        // of the row before
    float listed_value = 0.0f;
    T* listed_grad = nullptr;
    for (;;) {
        const Part<T> part = part_of(r);
        T* grad = grad_of(r);
        if (a.tail) mark(part, marks, l, e.id, byte_of);
        Teacher t = teacher_of<WAVES>(a, e, l);
        if (t.id >= 0) t.x = load(part.p, t.id);
        // Sums, about the largest of the thread's unlisted elements.
        uint32_t words[NV / 4] = {};
        if (a.tail) {
#pragma unroll
            for (int i = 0; i < NV / 4; ++i) {
                words[i] = marks[tid * (NV / 4) + i];
                marks[tid * (NV / 4) + i] = 0;
            }
        }
        float most = -kInf;
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            if (u * THREADS < part.nvec) {
                if ((u + 1) * THREADS > part.nvec) {
                    const bool inside = static_cast<int>(u * THREADS + place()) < part.nvec;
#pragma unroll
                    for (int i = 0; i < 4; ++i) d[u][i] = inside ? d[u][i] : lowest<T>();
                }
                d[u] = drop(d[u], words[u / 4] >> u % 4 * 8 & 0xFFu, T{});
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
        take_edges(part, run, l, scale, reach);
        if (tid < 2) l.edges[tid] = 0;
        const int more = REST && part.nvec > kKept ? part.nvec - kKept : 0;
        if constexpr (REST)
            stream<THREADS, kRestUnroll>(part.body() + kKept, more, [&](int v, u32x4 raw, bool inside) {
                float x[kVec<T>];
                unpack(inside ? raw : u32x4{lowest<T>(), lowest<T>(), lowest<T>(), lowest<T>()}, x);
                uint8_t* byte = reinterpret_cast<uint8_t*>(marks) + kKept + v;
                const uint32_t listed = a.tail && inside ? *byte : 0u;
                if (listed) *byte = 0;
                drop(x, listed);
                add<false>(run, x, most_of(x), scale, reach);
            });
        Listed listed;
        if (a.tail) listed = listed_of(part, t);
        stores_done();
        const RowSums sums(block_parts<WAVES>(run, listed, a.tail, scale, l.sums), scale);
        drop_tail(t, sums, scale);
        if (listed_id >= 0) store(listed_grad, listed_id, listed_value);
        const float loss = loss_of<WAVES>(a, t, sums, l);      // and every entry's logit is read
        if (tid == 0 && a.loss) a.loss[r] = loss;
        const Grad g(a, t, sums, w);
        listed_id = t.id;
        listed_value = g.listed(t, scale);
        listed_grad = grad;
        T* body = grad + part.head;
        const bool whole = (reinterpret_cast<uintptr_t>(body) & 15u) == 0;
        g.edges(a.l, part, grad);
        r = next_row(r + gridDim.x);
        Part<T> next = part;
        if (r < a.l.rows) {
            next = part_of(r);
            e = entry_of(a, r);
        } else {
            next.nvec = 0;
        }
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
        if (r >= a.l.rows) break;
    }
    stores_done();
    __syncthreads();
    if (listed_id >= 0) store(listed_grad, listed_id, listed_value);
}

// ---- launches ----------------------------------------------------------------------

// Parts of a row: at least what the group keys' LDS asks for, and with few rows
// enough blocks for the device, of no less than kLeastPart elements each.
constexpr int kLeastPart = 4096;

struct Split {
    int parts, len;
};

template <class T>
Split split_rows(int64_t rows, int vocab, int cus)
{
    int64_t parts = (vocab + kPartMax<T> - 1) / kPartMax<T>;
    const int64_t want = (int64_t{3} * cus + rows - 1) / rows;
    const int64_t most = vocab / kLeastPart > 1 ? vocab / kLeastPart : 1;
    int64_t more = want < most ? want : most;
    if (more > kPartsMax) more = kPartsMax;
    if (more > parts) parts = more;
    int len = static_cast<int>((vocab + parts - 1) / parts);
    len = (len + 63) / 64 * 64;            // parts of aligned rows stay aligned
    if (len > kPartMax<T>) len = kPartMax<T>;
    return {(vocab + len - 1) / len, len};
}
static_assert(GEM_VOCAB_MAX / kPartMax<float> <= kPartsMax && kPartsMax <= GEM_TOP_MAX,
              "a row's parts are joined by one block, by the threads that hold entries");

template <class T>
hipError_t scores(const ScoreArgs& a, const OpsDevice& d, hipStream_t stream)
{
    const Split s = split_rows<T>(a.l.rows, a.l.vocab, d.cus);
    const size_t key_bytes = (static_cast<size_t>(s.len) / kGroup + 4) * sizeof(typename GroupKey<T>::Type);
    // Rows of one launch: what their parts leave fits the fixed scratch.
    const int64_t left = s.parts * (static_cast<int64_t>(sizeof(PartSums)) + a.top_k * 8);
    int64_t fit = s.parts == 1 ? a.l.rows : kFixedScratch / left;
    PartSums* sums = static_cast<PartSums*>(d.scratch);
    for (int64_t r = 0; r < a.l.rows; r += fit) {
        const int64_t n = a.l.rows - r < fit ? a.l.rows - r : fit;
        uint64_t* tops = reinterpret_cast<uint64_t*>(sums + n * s.parts);
        const dim3 grid(static_cast<unsigned>(n * s.parts));
        if (a.top_k)
            hipLaunchKernelGGL((score_kernel<T, true>), grid, dim3(kThreads), key_bytes, stream, a, r, s.parts, s.len, sums, tops);
        else
            hipLaunchKernelGGL((score_kernel<T, false>), grid, dim3(kThreads), 0, stream, a, r, s.parts, s.len, sums, tops);
        if (s.parts > 1)
            hipLaunchKernelGGL((join_kernel<T>), dim3(static_cast<unsigned>(n)), dim3(kThreads),
                               static_cast<size_t>(s.parts) * a.top_k * 8, stream, a, r, s.parts, sums, tops);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// The gradient with rows in registers.
template <class T, int THREADS, int NV, bool REST>
void resident(const DistillArgs& a, const OpsDevice& d, hipStream_t stream)
{
    const int64_t blocks = int64_t{d.cus} * (1024 / THREADS);
    const int nvec = a.l.vocab / kVec<T> > THREADS * NV ? a.l.vocab / kVec<T> : THREADS * NV;
    hipLaunchKernelGGL((resident_kernel<T, THREADS, NV, REST>), dim3(static_cast<unsigned>(a.l.rows < blocks ? a.l.rows : blocks)),
                       dim3(THREADS), mark_words(nvec) * 4, stream, a);
}

// If there are rows enough to keep the device busy: false where it is not for these sizes.
// Small blocks, as many on a compute unit as its registers hold, stream while others sum:
// 4096 rows of 32768 bfloat16, all with a weight, take 122 us in blocks of 256 threads x 16
// vectors, 137 in 512 x 8, 201 in 1024 x 4; 4096 of 131072 525 us in 512 x 16 with half of a row
// read twice, 562 in 1024 x 8, and 592 in 1024 x 16, which read all of it once.  Rows beyond 1024
// x 16 vectors are read twice as they are split in parts: 1200 of 200000 284 us; 273 here with
// 1024 x 16 kept, by a kernel of its own for 4%.  512 x 16 vectors are more than the registers
// hold: of bfloat16 4 of them spill, and 37 where a row has more.
template <class T> bool resident_grad(const DistillArgs& a, const OpsDevice& d, hipStream_t stream)
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

template <class T>
hipError_t distill(const DistillArgs& a, const OpsDevice& d, hipStream_t stream)
{
    if (resident_grad<T>(a, d, stream)) return hipGetLastError();
    const Split s = split_rows<T>(a.l.rows, a.l.vocab, d.cus);
    const size_t marks = static_cast<size_t>(mark_words(s.len / kVec<T>)) * 4;
    PartSums* sums = static_cast<PartSums*>(d.scratch);
    if (s.parts == 1) {
        hipLaunchKernelGGL((distill_kernel<T, kSums | kRest>), dim3(static_cast<unsigned>(a.l.rows)), dim3(kThreads), marks,
                           stream, a, int64_t{0}, 1, s.len, sums, nullptr);
        return hipGetLastError();
    }
    const int64_t fit = kFixedScratch / (s.parts * static_cast<int64_t>(sizeof(PartSums)) + a.k * 4);
    for (int64_t r = 0; r < a.l.rows; r += fit) {
        const int64_t n = a.l.rows - r < fit ? a.l.rows - r : fit;
        float* x = reinterpret_cast<float*>(sums + n * s.parts);
        const dim3 grid(static_cast<unsigned>(n * s.parts));
        hipLaunchKernelGGL((distill_kernel<T, kSums>), grid, dim3(kThreads), marks, stream, a, r, s.parts, s.len, sums, x);
        // The loss alone is one block's a row.
        const int rest = a.grad ? s.parts : 1;
        hipLaunchKernelGGL((distill_kernel<T, kRest>), dim3(static_cast<unsigned>(n * rest)), dim3(kThreads), marks, stream, a,
                           r, s.parts, s.len, sums, x);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_scores(const ScoreArgs& a, bool bf16, const OpsDevice& d, hipStream_t stream)
{
    return bf16 ? scores<uint16_t>(a, d, stream) : scores<float>(a, d, stream);
}

hipError_t launch_distill(const DistillArgs& a, bool bf16, const OpsDevice& d, hipStream_t stream)
{
    return bf16 ? distill<uint16_t>(a, d, stream) : distill<float>(a, d, stream);
}

}  // namespace gemk
