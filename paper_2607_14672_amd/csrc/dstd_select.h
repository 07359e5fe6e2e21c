// dstd_select.h -- places in the order of a row of scores and in its sums, found by one
// block: the K-th entry, the prefix of a weight, the index where a sum is reached. Every
// sum is one of integers, so that nothing depends on the order of atomics.
#pragma once
#include <float.h>

#include "dstd_answer.h"
#include "dstd_kernels.h"

namespace dstd {
namespace {

template <int T> constexpr int kBins = T >= 1024 ? 2048 : T >= 256 ? 1024 : 512;  // of a histogram over a row
// entries of a row that are held at once
template <int T> constexpr int kList = kBins<T>;
// vectors a thread on the way in loops with an exponential and a histogram: 64 registers
// a thread hold one (300 x 50021 fp32, top_p 0.95: 106 us with 1, 118 with 4)
template <int T> constexpr int kOrderAhead = T >= 1024 ? 1 : kRowAhead;

template <int T> struct RowShared {
    u64 red[T / kWave + 1];
    u64 list[kList<T>];
    u64 hist[kBins<T>];
    u64 found[2];
    int count, seen;
};

// What is kept of a row: all up to a place in its order.
struct Border {
    u64 last;
    __device__ bool has(u32 key, int i) const { return key > kAbsentKey && rank_of(key, i) >= last; }
    __device__ bool all() const { return last == 0; }
    // the same by goodness and index: y above `at`, or equal with an index up to `upto`
    __device__ float at() const { return all() ? -INFINITY : value_of(rank_key(last)); }
    __device__ int upto() const { return all() ? -1 : rank_index(last); }
};

// Weights of the exponentials in 64-bit integers, the largest 2^shift (shift <= 51): their
// sums do not depend on the order. A weight is off by half a unit, 2^-(shift+1) of the
// largest, and 0 below that; the sum of a row by up to N times as much, 2^-29 of the largest
// at 131072 entries, 2^-24 (a step of a random number) at 2^19, 2^-15 at 2^24, where 64-bit
// floats would lose 2^-29 at most.
struct Mass {
    double top, scale;  // the largest goodness; |scale|
    int shift;
    // how far below the largest weights are 0
    __device__ double span() const { return 0.6931471805599453 * (shift + 1) / scale; }
    __device__ double distance(float y) const { return (top - static_cast<double>(y)) * scale; }
    __device__ double distance(u32 key) const { return distance(value_of(key)); }
    // rint(e^-d 2^shift): d = n ln 2 + r, e^-r by its series to r^11 / 11! (|r| <= ln 2 / 2:
    // 2^-47 relative at the ends; ln 2 is a double, 2^-55 n off), n taken off its exponent.
    // Adding 2^52 leaves the integer in the low bits. From d = 64 on (and for NaN) it is 0.
    static __device__ __forceinline__ u64 fixed_exp(double d, int shift) {
        d = fmin(d, 64.0);
        const double big = 0x1.8p52;
        const double t = fma(d, 1.4426950408889634, big);
        const double n = t - big;
        const double r = fma(n, -0x1.62e42fefa39efp-1, d);
        double p = 1.0 / 39916800;
        p = fma(p, -r, 1.0 / 3628800);
        p = fma(p, -r, 1.0 / 362880);
        p = fma(p, -r, 1.0 / 40320);
        p = fma(p, -r, 1.0 / 5040);
        p = fma(p, -r, 1.0 / 720);
        p = fma(p, -r, 1.0 / 120);
        p = fma(p, -r, 1.0 / 24);
        p = fma(p, -r, 1.0 / 6);
        p = fma(p, -r, 0.5);
        p = fma(p, -r, 1.0);
        p = fma(p, -r, 1.0);
        const int up = (shift - __double2loint(t)) << 20;
        const double v = __hiloint2double(__double2hiint(p) + up, __double2loint(p)) + 0x1p52;
        return __double_as_longlong(v) & 0xfffffffffffffull;
    }
    __device__ u64 of(float y) const { return fixed_exp(distance(y), shift); }
    __device__ u64 operator()(u32 key) const { return fixed_exp(distance(key), shift); }
};
struct One {
    __device__ u64 of(float) const { return 1; }
    __device__ u64 operator()(u32) const { return 1; }
};

// The first n entries of the list in falling order, in place; their high words fall as
// bin(entry), in [0, kBins), rises. Up to 64 are placed by how many are larger. More go to
// their bins' places (counts, and their sums over the bins), and in those by how many of
// the bin are larger; where a bin has too many for that, all by a bitonic network.
template <int T, typename F> __device__ void sort_list(RowShared<T> &sh, int n, F bin) {
    __syncthreads();
    if (n <= kWave) {
        if (threadIdx.x < kWave) {
            const u64 mine = static_cast<int>(threadIdx.x) < n ? sh.list[threadIdx.x] : 0;
            int at = 0;
            for (int k = 0; k < n; ++k) at += sh.list[k] > mine;
            __builtin_amdgcn_wave_barrier();
            if (static_cast<int>(threadIdx.x) < n) sh.list[at] = mine;
        }
        __syncthreads();
        return;
    }
    constexpr int most = 256, share = kList<T> / T, per = kBins<T> / T;
    u32 *count = reinterpret_cast<u32 *>(sh.hist), *first = count + kBins<T>;
    for (int k = threadIdx.x; k < kBins<T>; k += T) count[k] = 0;
    __syncthreads();
    u64 v[share];
    u32 place[share];  // the bin, and how many were there before
    bool over = false;
#pragma unroll
    for (int e = 0; e < share; ++e) {
        const int i = e * T + threadIdx.x;
        if (i >= n) continue;
        v[e] = sh.list[i];
        const u32 at = bin(v[e]), had = atomicAdd(&count[at], 1u);
        over |= had >= most;
        place[e] = at << 16 | had;
    }
    if (!__syncthreads_or(over)) {
        u32 mine = 0, all;
#pragma unroll
        for (int k = 0; k < per; ++k) mine += count[threadIdx.x * per + k];
        u32 at = block_before<T>(mine, sh.red, &all);
#pragma unroll
        for (int k = 0; k < per; ++k) {
            first[threadIdx.x * per + k] = at;
            at += count[threadIdx.x * per + k];
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < share; ++e)
            if (e * T + static_cast<int>(threadIdx.x) < n) sh.list[first[place[e] >> 16] + (place[e] & 0xffff)] = v[e];
        __syncthreads();
#pragma unroll
        for (int e = 0; e < share; ++e) {
            if (e * T + static_cast<int>(threadIdx.x) >= n) continue;
            const u32 lo = first[place[e] >> 16], hi = lo + count[place[e] >> 16];
            u32 to = lo;
            for (u32 k = lo; k < hi; ++k) to += sh.list[k] > v[e];
            place[e] = to;
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < share; ++e)
            if (e * T + static_cast<int>(threadIdx.x) < n) sh.list[place[e]] = v[e];
        __syncthreads();
        return;
    }
    int p = 2 * kWave;
    while (p < n) p *= 2;
    for (int i = n + threadIdx.x; i < p; i += T) sh.list[i] = 0;
#pragma unroll 1
    for (int k = 2; k <= p; k *= 2)
#pragma unroll 1
        for (int j = k / 2; j > 0; j /= 2) {
            __syncthreads();
#pragma unroll 1
            for (int t = threadIdx.x; t < p / 2; t += T) {
                const int i = 2 * t - (t & (j - 1)), o = i + j;
                const u64 x = sh.list[i], y = sh.list[o];
                if ((x < y) == ((i & k) == 0)) {
                    sh.list[i] = y;
                    sh.list[o] = x;
                }
            }
        }
    __syncthreads();
}
// The list in the order of a row: bins of the range of its values.
template <int T> __device__ void sort_by_value(RowShared<T> &sh, int n) {
    float per = 0.f, ymax = 0.f;
    if (n > kWave) {
        u32 hi = 0, lo = 0;  // largest key, largest complement
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += T) {
            hi = max(hi, rank_key(sh.list[i]));
            lo = max(lo, ~rank_key(sh.list[i]));
        }
        ymax = value_of(block_max<T>(hi, sh.red));
        lo = ~block_max<T>(lo, sh.red);
        per = static_cast<float>(kBins<T> / (static_cast<double>(ymax) - static_cast<double>(value_of(lo))));
    }
    sort_list<T>(sh, n, [&](u64 r) {
        return static_cast<u32>(fminf((ymax - value_of(rank_key(r))) * per, kBins<T> - 1.f));
    });
}

// Entries of a row that `want` (goodness, index) holds for, into the list, as many as fit;
// returns how many there are.
template <int T, int kAhead, typename E, typename F>
__device__ int collect(RowShared<T> &sh, const E *row, int n, const ScoreMap &m, F want) {
    __syncthreads();
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    row_each<kAhead>(row, n, threadIdx.x, T, [&](int i, float x) {
        const float y = goodness(x, m);
        if (y > -INFINITY && want(y, i)) {
            const int at = atomicAdd(&sh.count, 1);
            if (at < kList<T>) sh.list[at] = rank_of(key_of(y), i);
        }
    });
    __syncthreads();
    return sh.count;
}

// First index where the sum of weight(score, index) up to it exceeds share times the whole
// sum (returned in *all), -1 where that is 0. The waves sum a part of the row each; the
// part that holds the place is read again.
template <int T, int kAhead, typename E, typename F>
__device__ int by_index(RowShared<T> &sh, const E *row, int n, double share, u64 *all, F weight) {
    constexpr int waves = T / kWave, unit = kWave * RowVec<E>::n;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int part = (n + waves * unit - 1) / (waves * unit) * unit;
    const int lo = min(n, wave * part), hi = min(n, lo + part);
    u64 s = 0;
    row_each<kAhead, 2>(row + lo, hi - lo, lane, kWave,
                [&](int i, float x) { s += weight(x, lo + i); });
    u64 total;
    u64 before = block_before<T>(s, sh.red, &total);
    *all = total;
    if (total == 0) return -1;
    const double target = share * static_cast<double>(total);
    // the part: the first whose end exceeds the target
    const u64 wave_s = block_add<kWave>(s, nullptr);
    before = lane_value(before, 0);
    __syncthreads();
    if (lane == 0 && static_cast<double>(before) <= target && static_cast<double>(before + wave_s) > target) {
        sh.found[0] = before;
        sh.count = wave;
    }
    __syncthreads();
    u64 base = sh.found[0];
    const int first = sh.count * part, last = min(n, first + part);
    // the place: a vector's elements a thread at a time
    constexpr int vn = RowVec<E>::n;
    for (int from = first; from < last; from += T * vn) {
        const int a = from + static_cast<int>(threadIdx.x) * vn;
        u64 w[vn], mine = 0;
        if (a + vn <= last) {
            const auto r = load_vec<E>(row + a);
#pragma unroll
            for (int k = 0; k < vn; ++k) w[k] = weight(widen1(static_cast<E>(r[k])), a + k);
        } else {
#pragma unroll
            for (int k = 0; k < vn; ++k)
                w[k] = a + k < last ? weight(widen1(row[a + k]), a + k) : 0;
        }
#pragma unroll
        for (int k = 0; k < vn; ++k) mine += w[k];
        u64 round;
        u64 at = base + block_before<T>(mine, sh.red, &round);
        base += round;
        if (static_cast<double>(base) <= target) continue;
        __syncthreads();
        if (static_cast<double>(at) <= target && static_cast<double>(at + mine) > target) {
            int k = 0;
#pragma unroll
            for (int q = 0; q < vn; ++q) {
                at += w[q];
                if (static_cast<double>(at) <= target) k = q + 1;
            }
            sh.count = a + k;
        }
        break;
    }
    __syncthreads();
    const int got = sh.count;
    __syncthreads();
    return got;
}

// The place in the row's order, among what is kept, where the sum of the weights
// up to it first reaches `target`, or share times the whole sum if target is 0.
// A histogram over the row's range of values finds the bin with that place, and
// where the bin holds too many for the list, one over the bin's range of keys
// finds a smaller bin, down to a single key; entries of one key go by index.
// ymin, ymax: the range of the finite values of the row; span: how far below ymax
// weights are not 0. The largest weight is not 0.
template <int T, int kAhead, typename E, typename W>
__device__ Border by_order(RowShared<T> &sh, const E *row, int n, const ScoreMap &m, Border kept, float ymin,
                           float ymax, double span, W weight, u64 target_n, double share) {
    u32 lo = 0, hi = 0;   // keys of the bin
    int shift = -1;       // bins of 2^shift keys; -1: bins of the range of values
    const double range = fmin(static_cast<double>(ymax) - static_cast<double>(ymin), span);  // ymin may be -inf
    const float per = static_cast<float>(kBins<T> / range);
    u64 base = 0;
    double target = static_cast<double>(target_n);
    for (;;) {
        auto bin_of = [&](u32 key) {
            if (shift < 0) return static_cast<int>(fminf((ymax - value_of(key)) * per, kBins<T> - 1.f));
            return static_cast<int>((hi - key) >> shift);
        };
        auto in_range = [&](u32 key, int i) { return kept.has(key, i) && (shift < 0 || (key >= lo && key <= hi)); };
        int bin = 0;
        if (shift >= 0 || n > kList<T>) {
            __syncthreads();
            for (int k = threadIdx.x; k < kBins<T>; k += T) sh.hist[k] = 0;
            __syncthreads();
            auto *hist = reinterpret_cast<unsigned long long *>(sh.hist);
            if (shift < 0) {
                const float at = kept.at();
                const int upto = kept.upto();
                row_each<kAhead, 2>(row, n, threadIdx.x, T, [&](int i, float x) {
                    const float y = goodness(x, m);
                    if (!(y > at || (y == at && i <= upto))) return;
                    const u64 w = weight.of(y);
                    if (w) atomicAdd(&hist[static_cast<int>(fminf((ymax - y) * per, kBins<T> - 1.f))], w);
                });
            } else {
                row_each<0>(row, n, threadIdx.x, T, [&](int i, float x) {
                    const u32 key = key_of(goodness(x, m));
                    if (!in_range(key, i)) return;
                    const u64 w = weight(key);
                    if (w) atomicAdd(&hist[static_cast<int>((hi - key) >> shift)], w);
                });
            }
            __syncthreads();
            constexpr int per_thread = kBins<T> / T;
            u64 mine = 0;
#pragma unroll
            for (int k = 0; k < per_thread; ++k) mine += sh.hist[threadIdx.x * per_thread + k];
            u64 all;
            u64 at = base + block_before<T>(mine, sh.red, &all);
            if (target == 0.0) target = share * static_cast<double>(all);
            if (static_cast<double>(at) < target && static_cast<double>(at + mine) >= target)
                for (int k = 0; k < per_thread; ++k) {
                    const u64 next = at + sh.hist[threadIdx.x * per_thread + k];
                    if (static_cast<double>(next) >= target) {
                        sh.found[0] = at;
                        sh.found[1] = threadIdx.x * per_thread + k;
                        break;
                    }
                    at = next;
                }
            __syncthreads();
            base = sh.found[0];
            bin = static_cast<int>(sh.found[1]);
            int count;
            if (shift < 0) {
                const float last = kept.at();
                const int upto = kept.upto();
                count = collect<T, kAhead>(sh, row, n, m, [&](float y, int i) {
                    return static_cast<int>(fminf((ymax - y) * per, kBins<T> - 1.f)) == bin &&
                           (y > last || (y == last && i <= upto));
                });
            } else {
                count = collect<T, 0>(sh, row, n, m, [&](float y, int i) {
                    return in_range(key_of(y), i) && bin_of(key_of(y)) == bin;
                });
            }
            if (count > kList<T>) {
                u32 a = 0xffffffffu, b = 0;
                row_each<0>(row, n, threadIdx.x, T, [&](int i, float x) {
                    const u32 key = key_of(goodness(x, m));
                    if (in_range(key, i) && bin_of(key) == bin) {
                        a = min(a, key);
                        b = max(b, key);
                    }
                });
                lo = block_min<T>(a, sh.red);
                hi = block_max<T>(b, sh.red);
                if (lo == hi) {
                    // entries of one weight: the one that reaches the target
                    const u64 w = weight(lo);
                    u64 k = static_cast<u64>((target - static_cast<double>(base)) / static_cast<double>(w));
                    while (k > 0 && static_cast<double>(base + k * w) >= target) --k;
                    while (static_cast<double>(base + (k + 1) * w) < target) ++k;
                    // k entries of that key lie before it
                    u64 all_ties;
                    const u32 tie = lo;
                    auto is_tie = [&](float x, int i) -> u64 { return key_of(goodness(x, m)) == tie && kept.has(tie, i); };
                    const int i = by_index<T, 0>(sh, row, n, (static_cast<double>(k) + 0.5) / count, &all_ties, is_tie);
                    return Border{rank_of(lo, i)};
                }
                shift = 0;
                while ((static_cast<u64>(hi - lo) >> shift) >= kBins<T>) ++shift;
                continue;
            }
        } else {
            collect<T, kAhead>(sh, row, n, m, [&](float y, int i) { return kept.has(key_of(y), i); });
        }
        // the list in order, and the sums of its weights
        const int count = sh.count;
        sort_by_value<T>(sh, count);
        constexpr int each = kList<T> / T;
        u64 w[each], mine = 0;
#pragma unroll
        for (int k = 0; k < each; ++k) {
            const int i = threadIdx.x * each + k;
            w[k] = i < count ? weight(rank_key(sh.list[i])) : 0;
            mine += w[k];
        }
        u64 all;
        u64 at = base + block_before<T>(mine, sh.red, &all);
        if (target == 0.0) target = share * static_cast<double>(all);
        if (static_cast<double>(at) < target && static_cast<double>(at + mine) >= target)
#pragma unroll
            for (int k = 0; k < each; ++k) {
                if (static_cast<double>(at) < target && static_cast<double>(at + w[k]) >= target)
                    sh.found[0] = sh.list[threadIdx.x * each + k];
                at += w[k];
            }
        __syncthreads();
        const Border b{sh.found[0]};
        __syncthreads();
        return b;
    }
}

// The largest and smallest finite value of a row and how many there are.
struct Extremes {
    float ymin, ymax;
    int count;
};
template <int T, int kAhead, typename E>
__device__ Extremes row_extremes(RowShared<T> &sh, const E *row, int n, const ScoreMap &m) {
    u32 a = 0xffffffffu, b = 0, c = 0;
    row_each<kAhead>(row, n, threadIdx.x, T, [&](int, float x) {
        const u32 key = key_of(goodness(x, m));
        if (key > kAbsentKey) {
            a = min(a, key);
            b = max(b, key);
            ++c;
        }
    });
    const u32 lo = block_min<T>(a, sh.red), hi = block_max<T>(b, sh.red);
    const int count = static_cast<int>(block_add<T>(c, sh.red));
    return Extremes{value_of(lo), value_of(hi), count};
}

// The K first entries of a row; the shortest prefix of what is kept with at least `share`
// of its weight. These and other ways that not every row goes are not inlined: they would
// take registers from the loops that all go through.
template <int T, int kAhead, typename E>
__device__ __attribute__((noinline)) Border pick_count(RowShared<T> &sh, const E *row, int n, ScoreMap m, Extremes ex,
                                                       int K) {
    return by_order<T, kAhead>(sh, row, n, m, Border{0}, ex.ymin, ex.ymax, INFINITY, One{}, K, 0.0);
}
template <int T, int kAhead, typename E>
__device__ __attribute__((noinline)) Border pick_mass(RowShared<T> &sh, const E *row, int n, ScoreMap m, Border kept,
                                                      float ymin, Mass mass, double share) {
    return by_order<T, kAhead>(sh, row, n, m, kept, ymin, static_cast<float>(mass.top), mass.span(), mass, 0, share);
}

// What a draw goes by, and where it is written.
struct DrawArgs {
    double scale, top_p, dmax;  // dmax: -ln min_p, the largest distance that is kept
    int shift, top_k;
    const float *u;
    int32_t *choice;
    float *logp;
};
__device__ __forceinline__ void put_draw(const DrawArgs &a, int64_t b, int i, double distance, u64 all) {
    a.choice[b] = i;
    if (!a.logp) return;
    a.logp[b] = i < 0 ? -INFINITY
                      : static_cast<float>(-distance - log(ldexp(static_cast<double>(all), -a.shift)));
}
inline DrawArgs draw_args(const SampleJob &j) {
    return DrawArgs{j.in.scale, j.top_p, j.min_p > 0.0 ? -log(j.min_p) : INFINITY, j.shift, j.top_k,
                    j.u, j.choice, j.logp};
}
// u outside [0, 1) is drawn in, NaN to 0
__device__ __forceinline__ double share_of(const DrawArgs &a, int64_t b) {
    return fmin(fmax(static_cast<double>(a.u[b]), 0.0), 1.0 - 0x1p-24);
}

}  // namespace
}  // namespace dstd
