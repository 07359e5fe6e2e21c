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

// f(first index, vector) for the whole vectors of the first n elements of a row, by `count`
// threads, of which this is number `tid`: kAhead a thread on the way at once. Returns the
// index of the first element behind them.
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
        for (int a = 0; a < kAhead; ++a) f((v + a * count) * V::n, r[a]);
    }
    if (whole < nv) {
        typename V::type r[kAhead] = {};
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
            if (v + a * count < nv) r[a] = load_vec<E>(p + static_cast<int64_t>(v + a * count) * V::n);
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
            if (v + a * count < nv) f((v + a * count) * V::n, r[a]);
    }
    return nv * V::n;
}

// f(index, score) for the first n elements of a row, as vec_each, or (kAhead 0) element by
// element in a loop of few registers, for what rows in earnest do not reach. kTurns: so
// many elements at a time (an f of many registers), 0: as the compiler mixes them.
template <int kAhead, int kTurns = 0, typename E, typename F>
__device__ __forceinline__ void row_each(const E *p, int n, int tid, int count, F f) {
    int done = 0;
    if constexpr (kAhead > 0)
        done = vec_each<kAhead>(p, n, tid, count, [&](int i, typename RowVec<E>::type r) {
#pragma unroll
            for (int k = 0; k < RowVec<E>::n; ++k) {
                f(i + k, widen1(static_cast<E>(r[k])));
                if (kTurns > 0 && k % (kTurns > 0 ? kTurns : 1) == kTurns - 1) __builtin_amdgcn_sched_barrier(0);
            }
        });
#pragma unroll 1
    for (int i = done + tid; i < n; i += count) f(i, widen1(p[i]));
}

// ------------------------------------------------------ sums over a block --
// Lanes exchange by DPP moves (in the vector unit; a shuffle goes through LDS and takes
// some 50 ns more of latency, which is what blocks of one row wait for). A lane without a
// source keeps `none`.
template <int kCtrl, int kRows> __device__ __forceinline__ u32 lane_move(u32 none, u32 v) {
    return static_cast<u32>(__builtin_amdgcn_update_dpp(static_cast<int>(none), static_cast<int>(v), kCtrl, kRows,
                                                        0xf, false));
}
template <int kCtrl, int kRows> __device__ __forceinline__ u64 lane_move(u64 none, u64 v) {
    const u32 lo = lane_move<kCtrl, kRows>(static_cast<u32>(none), static_cast<u32>(v));
    return static_cast<u64>(lane_move<kCtrl, kRows>(static_cast<u32>(none >> 32), static_cast<u32>(v >> 32))) << 32 |
           lo;
}
template <int kCtrl, int kRows> __device__ __forceinline__ float lane_move(float none, float v) {
    return __uint_as_float(lane_move<kCtrl, kRows>(__float_as_uint(none), __float_as_uint(v)));
}
// The value of a lane that is the same for all.
__device__ __forceinline__ u32 lane_value(u32 v, int lane) {
    return static_cast<u32>(__builtin_amdgcn_readlane(static_cast<int>(v), lane));
}
__device__ __forceinline__ u64 lane_value(u64 v, int lane) {
    return static_cast<u64>(lane_value(static_cast<u32>(v >> 32), lane)) << 32 | lane_value(static_cast<u32>(v), lane);
}
__device__ __forceinline__ float lane_value(float v, int lane) {
    return __uint_as_float(lane_value(__float_as_uint(v), lane));
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
template <int kCtrl, int kRows> __device__ __forceinline__ ExpSum lane_move(ExpSum none, ExpSum v) {
    return ExpSum{lane_move<kCtrl, kRows>(none.m, v.m), lane_move<kCtrl, kRows>(none.s, v.s)};
}
__device__ __forceinline__ ExpSum lane_value(ExpSum v, int lane) {
    return ExpSum{lane_value(v.m, lane), lane_value(v.s, lane)};
}

// f over lanes up to and with the own one, of each run of kLanes (a power of two): the
// lanes of a row of 16 by shifts, then row 0's last lane to row 1 and 2's to 3, then
// lane 31 to the upper half.
template <int kLanes, typename V, typename F> __device__ __forceinline__ V wave_upto(V v, V none, F f) {
    if constexpr (kLanes > 1) v = f(v, lane_move<0x111, 0xf>(none, v));
    if constexpr (kLanes > 2) v = f(v, lane_move<0x112, 0xf>(none, v));
    if constexpr (kLanes > 4) v = f(v, lane_move<0x114, 0xf>(none, v));
    if constexpr (kLanes > 8) v = f(v, lane_move<0x118, 0xf>(none, v));
    if constexpr (kLanes > 16) v = f(v, lane_move<0x142, 0xa>(none, v));
    if constexpr (kLanes > 32) v = f(v, lane_move<0x143, 0xc>(none, v));
    return v;
}

// f over all values of a block, to every thread, in a fixed order. `red`: a V for every
// wave. `none`: what leaves a value as it is.
template <int T, typename V, typename F> __device__ __forceinline__ V block_fold(V v, V none, void *red, F f) {
    constexpr int waves = T / kWave;
    v = lane_value(wave_upto<kWave>(v, none, f), kWave - 1);
    if constexpr (waves > 1) {
        V *mem = static_cast<V *>(red);
        __syncthreads();
        if (threadIdx.x % kWave == 0) mem[threadIdx.x / kWave] = v;
        __syncthreads();
        v = lane_value(wave_upto<waves>(mem[threadIdx.x % waves], none, f), waves - 1);
    }
    return v;
}
template <int T> __device__ __forceinline__ u32 block_max(u32 v, void *red) {
    return block_fold<T>(v, 0u, red, [](u32 a, u32 b) { return a > b ? a : b; });
}
template <int T> __device__ __forceinline__ u32 block_min(u32 v, void *red) {
    return block_fold<T>(v, 0xffffffffu, red, [](u32 a, u32 b) { return a < b ? a : b; });
}
template <int T, typename V> __device__ __forceinline__ V block_add(V v, void *red) {
    return block_fold<T>(v, V{0}, red, [](V a, V b) { return a + b; });
}
template <int T> __device__ __forceinline__ ExpSum block_exp_sum(ExpSum v, float c2, void *red) {
    return block_fold<T>(v, ExpSum{-INFINITY, 0.f}, red, [c2](ExpSum a, ExpSum b) { return exp_join(a, b, c2); });
}
// Sum of what lower threads have; the whole in *total.
template <int T, typename V> __device__ __forceinline__ V block_before(V v, void *red, V *total) {
    constexpr int waves = T / kWave;
    auto plus = [](V a, V b) { return a + b; };
    const V s = wave_upto<kWave>(v, V{0}, plus);
    if constexpr (waves == 1) {
        *total = lane_value(s, kWave - 1);
        return s - v;
    } else {
        V *mem = static_cast<V *>(red);
        __syncthreads();
        if (threadIdx.x % kWave == kWave - 1) mem[threadIdx.x / kWave] = s;
        __syncthreads();
        // every wave forms the sums over the waves for itself
        const V x = wave_upto<waves>(mem[threadIdx.x % waves], V{0}, plus);
        *total = lane_value(x, waves - 1);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        return (wave > 0 ? lane_value(x, wave - 1) : V{0}) + s - v;
    }
}

}  // namespace dstd
