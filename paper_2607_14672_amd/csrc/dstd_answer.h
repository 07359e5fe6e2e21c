// dstd_answer.h -- device helpers of the kernels that read a network's answer
// row by row: scores as ordered keys, loads of a row, sums over a block.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "dstd_internal.h"

namespace dstd {

using u32 = uint32_t;
using u64 = uint64_t;

// Goodness y of a score: larger is likelier, -inf where the entry is left out.
// cap: what an entry that is not finite counts as (already -+inf where it is
// left out); flip: the sign bit where smaller scores are likelier.
struct ScoreMap {
    float cap;
    u32 flip;
};
__device__ __forceinline__ float goodness(float x, const ScoreMap &m) {
    const float v = isfinite(x) ? x : m.cap;
    return __uint_as_float(__float_as_uint(v) ^ m.flip);
}
// the same for a score that is finite, or whose kind the caller looks at
__device__ __forceinline__ float flipped(float x, const ScoreMap &m) {
    return __uint_as_float(__float_as_uint(x) ^ m.flip);
}
__device__ __forceinline__ float widen1(float x) { return x; }
__device__ __forceinline__ float widen1(uint16_t x) { return bf16_to_f32(x); }

// Order of the goodness as unsigned integers; -0 and +0 are one key. Keys of
// finite values lie above kAbsentKey, the key of -inf.
constexpr u32 kAbsentKey = 0x007fffffu;
__device__ __forceinline__ u32 key_of(float y) {
    const u32 b = __float_as_uint(y + 0.f);
    return b ^ (static_cast<u32>(static_cast<int>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(u32 key) {
    return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xffffffffu));
}
// One number that falls along a row's order: by key, then by index.
__device__ __forceinline__ u64 rank_of(u32 key, int i) {
    return (static_cast<u64>(key) << 32) | static_cast<u32>(~i);
}
__device__ __forceinline__ u32 rank_key(u64 r) { return static_cast<u32>(r >> 32); }
__device__ __forceinline__ int rank_index(u64 r) { return static_cast<int>(~static_cast<u32>(r)); }

// 16 bytes of a row, aligned as its elements are (one access all the same).
template <typename E> struct RowVec;
template <> struct RowVec<float> {
    static constexpr int n = 4;
    using type = float __attribute__((ext_vector_type(4)));
    using any = type __attribute__((aligned(4)));
};
template <> struct RowVec<uint16_t> {
    static constexpr int n = 8;
    using type = uint16_t __attribute__((ext_vector_type(8)));
    using any = type __attribute__((aligned(2)));
};
template <typename E> __device__ __forceinline__ typename RowVec<E>::type load_vec(const E *p) {
    return *reinterpret_cast<const typename RowVec<E>::any *>(p);
}

// f(slot, first index, vector) for the whole vectors of the first n elements of a row, by
// `count` threads, of which this is number `tid`: kAhead a thread on the way at once,
// `slot` the number among these. Returns the index of the first element behind them.
constexpr int kRowAhead = 4;
template <int kAhead, typename E, typename F>
__device__ __forceinline__ int vec_each(const E *p, int n, int tid, int count, F f) {
    using V = RowVec<E>;
    const int nv = n / V::n, whole = nv - nv % (kAhead * count);
    int v = tid;
#pragma unroll 1
    for (; v < whole; v += kAhead * count) {
        typename V::type r[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) r[a] = load_vec<E>(p + static_cast<int64_t>(v + a * count) * V::n);
#pragma unroll
        for (int a = 0; a < kAhead; ++a) f(a, (v + a * count) * V::n, r[a]);
    }
    if (whole < nv) {
        typename V::type r[kAhead] = {};
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
            if (v + a * count < nv) r[a] = load_vec<E>(p + static_cast<int64_t>(v + a * count) * V::n);
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
            if (v + a * count < nv) f(a, (v + a * count) * V::n, r[a]);
    }
    return nv * V::n;
}

// f(index, score) for the first n elements of a row, as vec_each, or (kAhead 0) element by
// element in a loop of few registers, for what rows in earnest do not reach.
template <int kAhead, typename E, typename F>
__device__ __forceinline__ void row_each(const E *p, int n, int tid, int count, F f) {
    int done = 0;
    if constexpr (kAhead > 0)
        done = vec_each<kAhead>(p, n, tid, count, [&](int, int i, typename RowVec<E>::type r) {
#pragma unroll
            for (int k = 0; k < RowVec<E>::n; ++k) f(i + k, widen1(static_cast<E>(r[k])));
        });
#pragma unroll 1
    for (int i = done + tid; i < n; i += count) f(i, widen1(p[i]));
}

// ------------------------------------------------------ sums over a block --
// Every result goes to every thread; `red` holds a u64 per wave and one more.
// The order of each is fixed.
template <int T, typename F> __device__ u64 block_fold(u64 v, u64 *red, F f) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o));
    if (T == kWave) return v;
    __syncthreads();
    if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = v;
    __syncthreads();
    v = red[threadIdx.x % (T / kWave)];
#pragma unroll
    for (int o = T / kWave / 2; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o));
    return v;
}
template <int T> __device__ u64 block_max(u64 v, u64 *red) {
    return block_fold<T>(v, red, [](u64 a, u64 b) { return a > b ? a : b; });
}
template <int T> __device__ u64 block_min(u64 v, u64 *red) {
    return block_fold<T>(v, red, [](u64 a, u64 b) { return a < b ? a : b; });
}
template <int T> __device__ u64 block_add(u64 v, u64 *red) {
    return block_fold<T>(v, red, [](u64 a, u64 b) { return a + b; });
}
// Sum of what lower threads have; the whole in *total.
template <int T> __device__ u64 block_before(u64 v, u64 *red, u64 *total) {
    u64 s = v;
    const int lane = threadIdx.x % kWave;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const u64 up = __shfl_up(s, o);
        if (lane >= o) s += up;
    }
    __syncthreads();
    if (lane == kWave - 1) red[threadIdx.x / kWave] = s;
    __syncthreads();
    // every wave forms the sums over the waves for itself
    constexpr int waves = T / kWave;
    u64 x = red[lane % waves];
#pragma unroll
    for (int o = 1; o < waves; o <<= 1) {
        const u64 up = __shfl_up(x, o);
        if (lane % waves >= o) x += up;
    }
    *total = __shfl(x, waves - 1);
    const int wave = threadIdx.x / kWave;
    const u64 base = __shfl(x, wave > 0 ? wave - 1 : 0);
    return (wave > 0 ? base : 0) + s - v;
}

// A sum of exponentials e^(scale y): the largest y, and the sum relative to it.
// {-inf, 0} is the empty one. Differences of y are taken before they are scaled,
// so a term's relative error is that of its own distance to the largest.
// c2 = scale log2(e).
struct ExpSum {
    float m, s;
};
__device__ __forceinline__ float exp_of(float dy, float c2) { return __builtin_amdgcn_exp2f(dy * c2); }
__device__ __forceinline__ ExpSum exp_join(ExpSum a, ExpSum b, float c2) {
    const float m = fmaxf(a.m, b.m);
    if (!(m > -INFINITY)) return ExpSum{-INFINITY, 0.f};
    return ExpSum{m, a.s * exp_of(a.m - m, c2) + b.s * exp_of(b.m - m, c2)};
}
template <int T> __device__ ExpSum block_exp_sum(ExpSum v, float c2, u64 *red) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1)
        v = exp_join(v, ExpSum{__shfl_xor(v.m, o), __shfl_xor(v.s, o)}, c2);
    if (T == kWave) return v;
    __syncthreads();
    if (threadIdx.x % kWave == 0)
        red[threadIdx.x / kWave] = (static_cast<u64>(__float_as_uint(v.m)) << 32) | __float_as_uint(v.s);
    __syncthreads();
    const u64 x = red[threadIdx.x % (T / kWave)];
    v = ExpSum{__uint_as_float(static_cast<u32>(x >> 32)), __uint_as_float(static_cast<u32>(x))};
#pragma unroll
    for (int o = T / kWave / 2; o > 0; o >>= 1)
        v = exp_join(v, ExpSum{__shfl_xor(v.m, o), __shfl_xor(v.s, o)}, c2);
    return v;
}

}  // namespace dstd
