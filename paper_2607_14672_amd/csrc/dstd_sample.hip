// dstd_sample.hip -- the largest logits of a row and one class drawn from its
// softmax (gfx950).
//
//   z_i = scale x_i, in the order of falling z, ties by index:
//   top    : the first K, and ln sum e^z of the others
//   sample : w_i = e^(z_i - z_max). Kept are the first top_k, of these the
//            shortest prefix with at least top_p of their sum, of these w_i >=
//            min_p; drawn is the first i, by index, where the sum of the kept
//            w up to i exceeds u times the sum of all kept.
//
// Both order by the score itself, not by its product with the scale.
#include <float.h>
#include <string.h>

#include "dstd_answer.h"
#include "dstd_kernels.h"
#include "dstd_profile.h"

namespace dstd {

namespace {

constexpr int kBins = 2048;  // of a histogram over a row
// Candidates of a row that are held at once, and so the largest top_k that is
// chosen from candidates.
template <int T> constexpr int kList = T >= 1024 ? 2048 : 1024;
constexpr int kMaxPicked = 1024;
constexpr int kGroups = kRowAhead;  // of a thread's share of the row, a maximum each

template <int T> struct RowShared {
    u64 red[T / kWave + 1];
    u64 list[kList<T>];
    u64 hist[kBins];
    u64 found[2];
    int count;
};

// What is kept of a row: all up to a place in its order.
struct Border {
    u64 last;
    __device__ bool has(u32 key, int i) const { return key > kAbsentKey && rank_of(key, i) >= last; }
};

// Weights of the exponentials in 64-bit integers, the largest 2^shift (shift <= 51):
// their sums do not depend on the order, and what is lost of a weight, 2^-(shift+1) of
// the largest, is below what sums in 64-bit floats lose over long rows.
struct Mass {
    double top, scale;  // the largest goodness; |scale|
    int shift;
    __device__ double distance(float y) const { return (top - static_cast<double>(y)) * scale; }
    __device__ double distance(u32 key) const { return distance(value_of(key)); }
    // rint(e^-d 2^shift): d = n ln 2 + r, e^-r by its series to r^12 / 12! (|r| <= ln 2 / 2:
    // 2^-52 relative). Adding 2^52 leaves the integer in the low bits.
    static __device__ __forceinline__ u64 fixed_exp(double d, int shift) {
        const double big = 0x1.8p52;
        const double t = fma(fmin(d, 128.0), 1.4426950408889634, big);
        const double n = t - big;
        const double r = fma(n, -0x1.abc9e3b39803fp-56, fma(n, -0x1.62e42fefa39efp-1, fmin(d, 128.0)));
        double p = 1.0 / 479001600;
        p = fma(p, -r, 1.0 / 39916800);
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
        const double v = ldexp(p, shift - static_cast<int>(__double2loint(t))) + 0x1p52;
        return __double_as_longlong(v) & 0xfffffffffffffull;
    }
    __device__ u64 of(float y) const { return fixed_exp(distance(y), shift); }
    __device__ u64 operator()(u32 key) const { return fixed_exp(distance(key), shift); }
};
struct One {
    __device__ u64 operator()(u32) const { return 1; }
};

// The first n entries of the list in falling order, in place. Few are placed by how
// many are larger, each against all (written back from the histogram's memory); more by
// a bitonic network over the next power of two.
template <int T> __device__ void sort_list(RowShared<T> &sh, int n) {
    __syncthreads();
    if (n <= 128) {
        for (int i = threadIdx.x; i < n; i += T) {
            const u64 mine = sh.list[i];
            int at = 0;
            for (int k = 0; k < n; ++k) at += sh.list[k] > mine;
            sh.hist[at] = mine;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += T) sh.list[i] = sh.hist[i];
        __syncthreads();
        return;
    }
    int p = 256;
    while (p < n) p *= 2;
    for (int i = n + threadIdx.x; i < p; i += T) sh.list[i] = 0;
    for (int k = 2; k <= p; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
            __syncthreads();
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

// Entries of a row that `want` (key, index) holds for, into the list, as many as
// fit; returns how many there are.
template <int T, int kAhead, typename E, typename F>
__device__ int collect(RowShared<T> &sh, const E *row, int n, const ScoreMap &m, F want) {
    __syncthreads();
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    row_each<kAhead>(row, n, threadIdx.x, T, [&](int i, float x) {
        const u32 key = key_of(goodness(x, m));
        if (key > kAbsentKey && want(key, i)) {
            const int at = atomicAdd(&sh.count, 1);
            if (at < kList<T>) sh.list[at] = rank_of(key, i);
        }
    });
    __syncthreads();
    return sh.count;
}

// First index where the sum of weight(key, index) up to it exceeds share times
// the whole sum (returned in *all), -1 where that is 0. The waves sum a part of
// the row each; the part that holds the place is read again.
template <int T, int kAhead, typename E, typename F>
__device__ int by_index(RowShared<T> &sh, const E *row, int n, const ScoreMap &m, double share, u64 *all,
                        F weight) {
    constexpr int waves = T / kWave, unit = kWave * RowVec<E>::n;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int part = (n + waves * unit - 1) / (waves * unit) * unit;
    const int lo = min(n, wave * part), hi = min(n, lo + part);
    u64 s = 0;
    row_each<kAhead>(row + lo, hi - lo, lane, kWave,
                [&](int i, float x) { s += weight(key_of(goodness(x, m)), lo + i); });
    u64 total;
    u64 before = block_before<T>(s, sh.red, &total);
    *all = total;
    if (total == 0) return -1;
    const double target = share * static_cast<double>(total);
    // the part: the first whose end exceeds the target
    const u64 wave_s = block_fold<kWave>(s, nullptr, [](u64 a, u64 b) { return a + b; });
    before = __shfl(before, 0);
    __syncthreads();
    if (lane == 0 && static_cast<double>(before) <= target && static_cast<double>(before + wave_s) > target) {
        sh.found[0] = before;
        sh.count = wave;
    }
    __syncthreads();
    u64 base = sh.found[0];
    const int first = sh.count * part, last = min(n, first + part);
    // the place, T runs of `each` elements in turn
    const int each = (last - first + T - 1) / T;
    const int a = min(last, first + static_cast<int>(threadIdx.x) * each), b = min(last, a + each);
    u64 mine = 0;
    for (int i = a; i < b; ++i) mine += weight(key_of(goodness(widen1(row[i]), m)), i);
    u64 unused;
    base += block_before<T>(mine, sh.red, &unused);
    __syncthreads();
    if (static_cast<double>(base) <= target && static_cast<double>(base + mine) > target)
        for (int i = a; i < b; ++i) {
            base += weight(key_of(goodness(widen1(row[i]), m)), i);
            if (static_cast<double>(base) > target) {
                sh.count = i;
                break;
            }
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
    const double range = fmin(static_cast<double>(ymax) - static_cast<double>(ymin), span);
    const float per = static_cast<float>(kBins / range);
    u64 base = 0;
    double target = static_cast<double>(target_n);
    for (;;) {
        auto bin_of = [&](u32 key) {
            if (shift < 0) return static_cast<int>(fminf((ymax - value_of(key)) * per, kBins - 1.f));
            return static_cast<int>((hi - key) >> shift);
        };
        auto in_range = [&](u32 key, int i) { return kept.has(key, i) && (shift < 0 || (key >= lo && key <= hi)); };
        int bin = 0;
        if (shift >= 0 || n > kList<T>) {
            __syncthreads();
            for (int k = threadIdx.x; k < kBins; k += T) sh.hist[k] = 0;
            __syncthreads();
            row_each<kAhead>(row, n, threadIdx.x, T, [&](int i, float x) {
                const u32 key = key_of(goodness(x, m));
                if (!in_range(key, i)) return;
                const u64 w = weight(key);
                if (w) atomicAdd(reinterpret_cast<unsigned long long *>(&sh.hist[bin_of(key)]), w);
            });
            __syncthreads();
            constexpr int per_thread = kBins / T;
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
            const int count = collect<T, kAhead>(sh, row, n, m, [&](u32 key, int i) {
                return in_range(key, i) && bin_of(key) == bin;
            });
            if (count > kList<T>) {
                u32 a = 0xffffffffu, b = 0;
                row_each<kAhead>(row, n, threadIdx.x, T, [&](int i, float x) {
                    const u32 key = key_of(goodness(x, m));
                    if (in_range(key, i) && bin_of(key) == bin) {
                        a = min(a, key);
                        b = max(b, key);
                    }
                });
                lo = static_cast<u32>(block_min<T>(a, sh.red));
                hi = static_cast<u32>(block_max<T>(b, sh.red));
                if (lo == hi) {
                    // entries of one weight: the one that reaches the target
                    const u64 w = weight(lo);
                    u64 k = static_cast<u64>((target - static_cast<double>(base)) / static_cast<double>(w));
                    while (k > 0 && static_cast<double>(base + k * w) >= target) --k;
                    while (static_cast<double>(base + (k + 1) * w) < target) ++k;
                    // k entries of that key lie before it
                    u64 all_ties;
                    const u32 tie = lo;
                    auto is_tie = [&](u32 key, int i) -> u64 { return key == tie && kept.has(key, i); };
                    const int i = by_index<T, kAhead>(sh, row, n, m, (static_cast<double>(k) + 0.5) / count, &all_ties, is_tie);
                    return Border{rank_of(lo, i)};
                }
                shift = 0;
                while ((static_cast<u64>(hi - lo) >> shift) >= kBins) ++shift;
                continue;
            }
        } else {
            collect<T, kAhead>(sh, row, n, m, [&](u32 key, int i) { return kept.has(key, i); });
        }
        // the list in order, and the sums of its weights
        const int count = sh.count;
        sort_list<T>(sh, count);
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
    const u32 lo = static_cast<u32>(block_min<T>(a, sh.red)), hi = static_cast<u32>(block_max<T>(b, sh.red));
    const int count = static_cast<int>(block_add<T>(c, sh.red));
    return Extremes{value_of(lo), value_of(hi), count};
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
// u outside [0, 1) is drawn in, NaN to 0
__device__ __forceinline__ double share_of(const DrawArgs &a, int64_t b) {
    return fmin(fmax(static_cast<double>(a.u[b]), 0.0), 1.0 - 0x1p-24);
}

// One class of a row by its definition, whatever the values.
template <int T, int kAhead, typename E>
__device__ void sample_row(RowShared<T> &sh, const E *row, int64_t b, int n, const ScoreMap &m, const DrawArgs &a) {
    const Extremes ex = row_extremes<T, kAhead>(sh, row, n, m);
    if (ex.count == 0) {
        if (threadIdx.x == 0) put_draw(a, b, -1, 0.0, 0);
        return;
    }
    const Mass mass{ex.ymax, a.scale, a.shift};
    Border kept{0};
    if (a.top_k > 0 && a.top_k < ex.count)
        kept = by_order<T, kAhead>(sh, row, n, m, kept, ex.ymin, ex.ymax, INFINITY, One{}, a.top_k, 0.0);
    if (a.top_p < 1.0)
        kept = by_order<T, kAhead>(sh, row, n, m, kept, ex.ymin, ex.ymax,
                                   0.6931471805599453 * (a.shift + 1) / a.scale, mass, 0, a.top_p);
    u64 all;
    const int i = by_index<T, kAhead>(sh, row, n, m, share_of(a, b), &all, [&](u32 key, int k) -> u64 {
        return kept.has(key, k) && mass.distance(key) <= a.dmax ? mass(key) : 0;
    });
    if (threadIdx.x == 0) put_draw(a, b, i, mass.distance(key_of(goodness(widen1(row[i]), m))), all);
}

template <int T, typename E>
__global__ __launch_bounds__(T, T >= 1024 ? 8 : 4) void sample_kernel(int n, int64_t ld, const E *__restrict__ x,
                                                                      ScoreMap m, DrawArgs a) {
    __shared__ RowShared<T> sh;
    const int64_t b = blockIdx.x;
    // bf16 rows come here by a cap that no bf16 value equals, or by their size
    sample_row<T, sizeof(E) == 4 ? 1 : 0>(sh, x + b * ld, b, n, m, a);
}

// Candidates for the K first entries of a row's order: all that reach a bound which K
// entries reach at least. The bound is the K-th largest of the groups' largest values, or
// a little less: few others reach it unless the largest lie close together in the row.
// Goodness y without a look at entries that do not count: y < INF is false for these, and
// they are no candidates.
template <int T, typename E>
__device__ float candidate_bound(RowShared<T> &sh, const E *row, int n, const ScoreMap &m, bool caps, int K) {
    float best[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) best[g] = -INFINITY;
    row_groups<E>(row, n, threadIdx.x, T, [&](int g, int, float x) {
        // med3 passes NaN over; +inf gives FLT_MAX, which is looked at below
        const float y = caps ? goodness(x, m) : __uint_as_float(__float_as_uint(x) ^ m.flip);
        best[g] = __builtin_amdgcn_fmed3f(y, best[g], FLT_MAX);
    });
    float lo = INFINITY, hi = -INFINITY;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        if (best[g] > -INFINITY) lo = fminf(lo, best[g]);
        hi = best[g] == best[g] ? fmaxf(hi, best[g]) : FLT_MAX;
    }
    hi = value_of(static_cast<u32>(block_max<T>(key_of(hi), sh.red)));
    lo = value_of(static_cast<u32>(block_min<T>(key_of(lo), sh.red)));
    if (hi >= FLT_MAX || K > kGroups * T) return -FLT_MAX;
    if (!(hi > -INFINITY)) return INFINITY;  // nothing counts
    // bins of the range of the maxima
    const float per = static_cast<float>(kBins / (static_cast<double>(hi) - static_cast<double>(lo)));
    u32 *hist = reinterpret_cast<u32 *>(sh.hist);
    for (int k = threadIdx.x; k < kBins; k += T) hist[k] = 0;
    if (threadIdx.x == 0) sh.count = -1;
    __syncthreads();
    int bin[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        bin[g] = kBins;  // a group without an entry
        if (best[g] > -INFINITY) {
            bin[g] = static_cast<int>(fminf((hi - best[g]) * per, kBins - 1.f));
            atomicAdd(&hist[bin[g]], 1u);
        }
    }
    __syncthreads();
    constexpr int each = kBins / T;
    u64 mine = 0;
#pragma unroll
    for (int k = 0; k < each; ++k) mine += hist[threadIdx.x * each + k];
    u64 all;
    u64 at = block_before<T>(mine, sh.red, &all);
    if (at < static_cast<u64>(K) && at + mine >= static_cast<u64>(K))
        for (int k = 0; k < each; ++k) {
            at += hist[threadIdx.x * each + k];
            if (at >= static_cast<u64>(K)) {
                sh.count = threadIdx.x * each + k;
                break;
            }
        }
    __syncthreads();
    const int last = sh.count;
    float bound = INFINITY;
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
        if (bin[g] <= last) bound = fminf(bound, best[g]);
    bound = value_of(static_cast<u32>(block_min<T>(key_of(bound), sh.red)));
    return last < 0 ? -FLT_MAX : bound;
}

// The K first entries of a row's order and at most a few more, sorted, in the list;
// returns how many there are (fewer than K where the row has fewer). kSum: *others is the
// sum over the entries behind the K-th.
template <int T, bool kSum, typename E>
__device__ int candidates(RowShared<T> &sh, const E *row, int n, const ScoreMap &m, bool caps, int K, float c2,
                          ExpSum *others) {
    float bound = -FLT_MAX;
    if (n > kList<T>) bound = candidate_bound<T>(sh, row, n, m, caps, K);
    if (kSum) *others = ExpSum{-INFINITY, 0.f};
    if (bound == INFINITY) return 0;
    __syncthreads();
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    float sum = 0.f;  // of what is below the bound, relative to it
    row_each<kRowAhead>(row, n, threadIdx.x, T, [&](int i, float x) {
        const float y = caps ? goodness(x, m) : __uint_as_float(__float_as_uint(x) ^ m.flip);
        const float d = y - bound;
        if (d >= 0.f && y < INFINITY) {
            const int at = atomicAdd(&sh.count, 1);
            if (at < kList<T>) sh.list[at] = rank_of(key_of(y), i);
        }
        if (kSum && d < 0.f) sum += exp_of(d, c2);
    });
    __syncthreads();
    int count = sh.count;
    bool listed = bound == -FLT_MAX;  // the sum is that of the list's others alone
    if (count > kList<T>) {
        const Extremes ex = row_extremes<T, 0>(sh, row, n, m);
        const Border kept = by_order<T, 0>(sh, row, n, m, Border{0}, ex.ymin, ex.ymax, INFINITY, One{}, K, 0.0);
        count = collect<T, 0>(sh, row, n, m, [&](u32 key, int i) { return kept.has(key, i); });
        sum = 0.f;
        listed = false;
    }
    sort_list<T>(sh, count);
    if (!kSum || count < K) return count;
    ExpSum s{-INFINITY, 0.f};
    const bool some = __syncthreads_or(sum > 0.f);
    if (some || listed) {
        if (sum > 0.f) s = ExpSum{bound, sum};
        for (int k = K + threadIdx.x; k < count; k += T)
            s = exp_join(s, ExpSum{value_of(rank_key(sh.list[k])), 1.f}, c2);
    } else {
        // all others far below the bound (their sum there is 0), or no bound was found
        const u64 last = sh.list[K - 1];
        row_each<0>(row, n, threadIdx.x, T, [&](int i, float v) {
            const float y = goodness(v, m);
            const u32 key = key_of(y);
            if (key > kAbsentKey && rank_of(key, i) < last) {
                if (y > s.m) {
                    s.s *= exp_of(s.m - y, c2);
                    s.m = y;
                }
                s.s += exp_of(y - s.m, c2);
            }
        });
    }
    *others = block_exp_sum<T>(s, c2, sh.red);
    return count;
}

template <int T, typename E>
__global__ __launch_bounds__(T, T >= 1024 ? 8 : 4) void top_logits_kernel(int n, int64_t ld, const E *__restrict__ x, ScoreMap m,
                                                       bool caps, double scale, float c2, int K,
                                                       int32_t *__restrict__ idx, float *__restrict__ logit,
                                                       float *__restrict__ rest) {
    __shared__ RowShared<T> sh;
    const int64_t b = blockIdx.x;
    const E *row = x + b * ld;
    ExpSum s;
    const int count = candidates<T, true>(sh, row, n, m, caps, K, c2, &s);
    for (int k = threadIdx.x; k < K; k += T) {
        const bool some = k < count;
        const u64 r = some ? sh.list[k] : 0;
        idx[b * K + k] = some ? rank_index(r) : -1;
        logit[b * K + k] = some ? static_cast<float>(static_cast<double>(value_of(rank_key(r))) * scale) : -INFINITY;
    }
    if (threadIdx.x == 0 && rest)
        rest[b] = s.s > 0.f ? static_cast<float>(static_cast<double>(s.m) * scale + log(static_cast<double>(s.s)))
                            : -INFINITY;
}

// One class from the top_k <= kMaxPicked first entries of each row.
template <int T, typename E>
__global__ __launch_bounds__(T, T >= 1024 ? 8 : 4) void sample_picked_kernel(int n, int64_t ld,
                                                                             const E *__restrict__ x, ScoreMap m,
                                                                             bool caps, DrawArgs a) {
    __shared__ RowShared<T> sh;
    const int64_t b = blockIdx.x;
    const E *row = x + b * ld;
    int count = candidates<T, false>(sh, row, n, m, caps, a.top_k, 0.f, nullptr);
    if (count == 0) {
        if (threadIdx.x == 0) put_draw(a, b, -1, 0.0, 0);
        return;
    }
    count = min(count, a.top_k);
    const Mass mass{value_of(rank_key(sh.list[0])), a.scale, a.shift};
    constexpr int each = kMaxPicked / T > 1 ? kMaxPicked / T : 1;
    u64 w[each], mine = 0;
    const int first = threadIdx.x * each;
#pragma unroll
    for (int k = 0; k < each; ++k) {
        w[k] = first + k < count ? mass(rank_key(sh.list[first + k])) : 0;
        mine += w[k];
    }
    u64 all;
    u64 at = block_before<T>(mine, sh.red, &all);
    const double target = a.top_p < 1.0 ? a.top_p * static_cast<double>(all) : INFINITY;
    u64 keeps = 0;
#pragma unroll
    for (int k = 0; k < each; ++k) {
        if (first + k < count && static_cast<double>(at) < target &&
            mass.distance(rank_key(sh.list[first + k])) <= a.dmax)
            ++keeps;
        at += w[k];
    }
    count = static_cast<int>(block_add<T>(keeps, sh.red));
    // what is kept, by index
    u64 back[each];
#pragma unroll
    for (int k = 0; k < each; ++k) {
        const u64 r = first + k < count ? sh.list[first + k] : 0;
        back[k] = (r << 32) | (r >> 32);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < each; ++k)
        if (first + k < count) sh.list[first + k] = back[k];
    sort_list<T>(sh, count);
    mine = 0;
#pragma unroll
    for (int k = 0; k < each; ++k) {
        w[k] = first + k < count ? mass(static_cast<u32>(sh.list[first + k])) : 0;
        mine += w[k];
    }
    at = block_before<T>(mine, sh.red, &all);
    const double goal = share_of(a, b) * static_cast<double>(all);
    if (static_cast<double>(at) <= goal && static_cast<double>(at + mine) > goal)
#pragma unroll
        for (int k = 0; k < each; ++k) {
            if (static_cast<double>(at) <= goal && static_cast<double>(at + w[k]) > goal) {
                const u64 r = sh.list[first + k];
                put_draw(a, b, static_cast<int>(~static_cast<u32>(r >> 32)), mass.distance(static_cast<u32>(r)), all);
            }
            at += w[k];
        }
}

// ---------------------------------------------- rows of few distinct values --
// bf16 scores of a magnitude in [2^-24, 2^8) take 2 * 4095 values, and 0; how often each
// occurs says which are kept and what they weigh, with an exponential a value instead of
// one an entry. Bins fall from the largest value: kHalf - t for the t-th magnitude,
// kHalf for 0, kHalf + t for its negative, and the last for all that is smaller (of
// weight 0, or the row is not drawn from here).
constexpr int kHalf = 4095, kValues = 2 * kHalf + 2, kFirstMag = 0x3381;
constexpr int kNoBin = -1, kOddBin = -2;
struct BinMap {
    u32 flip;  // as of ScoreMap, for 16 bits
    u32 cap;   // bits of what an entry that is not finite counts as; 0x8000 more: left out
};
__device__ __forceinline__ int value_bin(u32 bits, const BinMap &m) {
    const int t = static_cast<int>(bits & 0x7fff) - kFirstMag + 1;
    const int neg = static_cast<int>((bits ^ m.flip) << 16) >> 31;  // 0 or -1
    if (static_cast<u32>(t - 1) < static_cast<u32>(kHalf)) return kHalf + ((t ^ ~neg) - ~neg);
    if ((bits & 0x7fff) >= 0x7f80) {
        if (m.cap > 0xffff) return kNoBin;
        const int tc = static_cast<int>(m.cap & 0x7fff) - kFirstMag + 1;
        const int nc = static_cast<int>((m.cap ^ m.flip) << 16) >> 31;
        return (m.cap & 0x7fff) == 0 ? kHalf : kHalf + ((tc ^ ~nc) - ~nc);
    }
    if ((bits & 0x7fff) == 0) return kHalf;
    return neg && t > kHalf ? kValues - 1 : kOddBin;
}
__device__ __forceinline__ float bin_value(int bin) {
    const int t = bin - kHalf;
    if (t == 0) return 0.f;
    const u32 mag = (t < 0 ? -t : t) + kFirstMag - 1;
    return bf16_to_f32(static_cast<uint16_t>(mag | (t > 0 ? 0x8000u : 0u)));
}

template <int T> struct ValueShared {
    u64 red[T / kWave + 1];
    union {
        RowShared<T> row;
        u64 weight[kValues];
        u32 count[kValues];
    };
    u64 part[T / kWave];
    u32 ties[T / kWave];
    u64 found, tie_weight;
    int tie_bin, tie_keep, at;
};

// f(index, bits) as row_each
template <typename F>
__device__ __forceinline__ void bits_each(const uint16_t *p, int n, int tid, int count, F f) {
    const int nv = n / 8;
#pragma unroll 1
    for (int v0 = tid; v0 < nv; v0 += 2 * count) {
        RowVec<uint16_t>::type r[2] = {};
#pragma unroll
        for (int a = 0; a < 2; ++a)
            if (v0 + a * count < nv) r[a] = load_vec<uint16_t>(p + static_cast<int64_t>(v0 + a * count) * 8);
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            if (v0 + a * count >= nv) break;
#pragma unroll
            for (int k = 0; k < 8; ++k) f((v0 + a * count) * 8 + k, static_cast<u32>(r[a][k]));
        }
    }
    for (int i = nv * 8 + tid; i < n; i += count) f(i, static_cast<u32>(p[i]));
}

template <int T>
__global__ __launch_bounds__(T, T >= 1024 ? 8 : 4) void sample_values_kernel(int n, int64_t ld,
                                                                             const uint16_t *__restrict__ x,
                                                                             ScoreMap m, BinMap bm, DrawArgs a) {
    __shared__ ValueShared<T> sh;
    constexpr int each = kValues / T, waves = T / kWave;
    static_assert(kValues % T == 0, "");
    const int64_t b = blockIdx.x;
    const uint16_t *row = x + b * ld;
    const int tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
    for (int k = tid; k < kValues; k += T) sh.count[k] = 0;
    __syncthreads();
    bool odd = false;
    bits_each(row, n, tid, T, [&](int, u32 bits) {
        const int bin = value_bin(bits, bm);
        if (bin >= 0) atomicAdd(&sh.count[bin], 1u);
        odd |= bin == kOddBin;
    });
    odd = __syncthreads_or(odd);
    // each thread's bins
    u32 count[each];
    u64 first = kValues;
    u64 counted = 0;
#pragma unroll
    for (int k = each - 1; k >= 0; --k) {
        count[k] = sh.count[tid * each + k];
        counted += count[k];
        if (count[k]) first = tid * each + k;
    }
    const u32 below = sh.count[kValues - 1];
    first = block_min<T>(first, sh.red);
    if (first == kValues && !odd) {
        if (tid == 0) put_draw(a, b, -1, 0.0, 0);
        return;
    }
    const Mass mass{bin_value(static_cast<int>(first)), a.scale, a.shift};
    if (odd || (below > 0 && (first == kValues - 1 || mass.of(bin_value(kValues - 2)) != 0))) {
        __syncthreads();
        sample_row<T, 0>(sh.row, row, b, n, m, a);
        return;
    }
    u64 unused, w[each], sum = 0;
    u64 before = block_before<T>(counted, sh.red, &unused);
#pragma unroll
    for (int k = 0; k < each; ++k) {
        u64 keep = count[k];
        if (a.top_k > 0) keep = before >= static_cast<u64>(a.top_k) ? 0 : min(keep, a.top_k - before);
        before += count[k];
        const int bin = tid * each + k;
        w[k] = keep && bin < kValues - 1 ? mass.of(bin_value(bin)) : 0;
        count[k] = static_cast<u32>(keep);
        sum += keep * w[k];
    }
    u64 all;
    u64 at = block_before<T>(sum, sh.red, &all);
    // the counts are in registers: their place takes the weights
    if (tid == 0) {
        sh.tie_bin = -1;
        sh.tie_keep = 0;
        sh.tie_weight = 0;
    }
    __syncthreads();
    u64 in_bin[each];
#pragma unroll
    for (int k = 0; k < each; ++k) in_bin[k] = sh.count[tid * each + k];
    __syncthreads();
    const double target = a.top_p < 1.0 ? a.top_p * static_cast<double>(all) : INFINITY;
    u64 last = 0;
#pragma unroll
    for (int k = 0; k < each; ++k) {
        const int bin = tid * each + k;
        u64 keep = w[k] ? count[k] : 0;
        if (keep) {
            if (static_cast<double>(at) >= target || mass.distance(bin_value(bin)) > a.dmax) {
                keep = 0;
            } else if (static_cast<double>(at + keep * w[k]) >= target) {
                // the fewest that reach the target
                u64 c = static_cast<u64>((target - static_cast<double>(at)) / static_cast<double>(w[k]));
                while (c > 0 && static_cast<double>(at + (c - 1) * w[k]) >= target) --c;
                while (static_cast<double>(at + c * w[k]) < target) ++c;
                at += keep * w[k];
                keep = min(keep, c);
            } else {
                at += keep * w[k];
            }
            if (keep) last = bin;
            if (keep && keep < in_bin[k]) {
                sh.tie_bin = bin;
                sh.tie_keep = static_cast<int>(keep);
                sh.tie_weight = w[k];
                keep = 0;
            }
        }
        sh.weight[bin] = keep ? w[k] : 0;
    }
    last = block_max<T>(last, sh.red);
    const int tie_bin = sh.tie_bin;
    const u64 tie_keep = sh.tie_keep, tie_weight = sh.tie_weight;
    // the kept weights of each wave's part of the row; of the bin that is kept in part, the
    // entries, of which the first tie_keep count
    constexpr int unit = kWave * 8;
    const int part = (n + waves * unit - 1) / (waves * unit) * unit;
    const int lo = min(n, wave * part), hi = min(n, lo + part);
    u64 s = 0, ties = 0;
    auto add = [&](u32 bits) {
        const int bin = value_bin(bits, bm);
        if (static_cast<u32>(bin) <= static_cast<u32>(last)) {
            if (bin == tie_bin) ++ties;
            else s += sh.weight[bin];
        }
    };
    bits_each(row + lo, hi - lo, lane, kWave, [&](int, u32 bits) { add(bits); });
    auto plus = [](u64 p, u64 q) { return p + q; };
    s = block_fold<kWave>(s, nullptr, plus);
    ties = block_fold<kWave>(ties, nullptr, plus);
    if (lane == 0) {
        sh.part[wave] = s;
        sh.ties[wave] = static_cast<u32>(ties);
    }
    __syncthreads();
    u64 t = 0;
    all = 0;
    for (int k = 0; k < waves; ++k) {
        all += sh.part[k] + tie_weight * min<u64>(sh.ties[k], tie_keep - min(t, tie_keep));
        t += sh.ties[k];
    }
    const double goal = share_of(a, b) * static_cast<double>(all);
    u64 base = 0;
    t = 0;
    int from = 0;
    for (; from < waves - 1; ++from) {
        const u64 next = base + sh.part[from] + tie_weight * min<u64>(sh.ties[from], tie_keep - min(t, tie_keep));
        if (static_cast<double>(next) > goal) break;
        base = next;
        t += sh.ties[from];
    }
    // the place in that part, runs of `len` entries a thread
    const int start = from * part, end = min(n, start + part);
    const int len = (end - start + T - 1) / T;
    const int p0 = min(end, start + tid * len), p1 = min(end, p0 + len);
    s = ties = 0;
    for (int i = p0; i < p1; ++i) add(row[i]);
    t += block_before<T>(ties, sh.red, &unused);
    const u64 mine = s + tie_weight * min(ties, tie_keep - min(t, tie_keep));
    base += block_before<T>(mine, sh.red, &unused);
    if (static_cast<double>(base) <= goal && static_cast<double>(base + mine) > goal)
        for (int i = p0; i < p1; ++i) {
            const int bin = value_bin(row[i], bm);
            if (static_cast<u32>(bin) > static_cast<u32>(last)) continue;
            if (bin == tie_bin) base += t++ < tie_keep ? tie_weight : 0;
            else base += sh.weight[bin];
            if (static_cast<double>(base) > goal) {
                put_draw(a, b, i, mass.distance(bin_value(bin)), all);
                break;
            }
        }
}

// Whether a cap is one of the values that have a bin, or is none.
bool cap_has_bin(float cap, u32 *bits) {
    *bits = 0x10000u;
    if (!isfinite(cap)) return true;
    u32 f;
    memcpy(&f, &cap, 4);
    *bits = f >> 16;
    const int t = static_cast<int>(*bits & 0x7fff) - kFirstMag;
    return (f & 0xffff) == 0 && ((*bits & 0x7fff) == 0 || (t >= 0 && t < kHalf));
}

template <typename E>
hipError_t launch_sample_t(const SampleJob &j, hipStream_t st) {
    const int n = static_cast<int>(j.in.N);
    const dim3 grid(static_cast<unsigned>(j.in.B));
    const ScoreMap m{j.in.cap, j.in.flip};
    const DrawArgs a{j.in.scale, j.top_p, j.min_p > 0.0 ? -log(j.min_p) : INFINITY, j.shift, j.top_k,
                     j.u, j.choice, j.logp};
    const E *x = static_cast<const E *>(j.in.x);
    const bool picked = j.top_k > 0 && j.top_k <= kMaxPicked;
    u32 cap;
    if constexpr (sizeof(E) == 2)
        if (!picked && n > 4096 && cap_has_bin(j.in.cap, &cap)) {
            const BinMap bm{j.in.flip >> 16, cap};
            hipLaunchKernelGGL((sample_values_kernel<1024>), grid, dim3(1024), 0, st, n, j.in.ld, x, m, bm, a);
            return hipGetLastError();
        }
#define SAMPLE(T)                                                                                             \
    if (picked)                                                                                               \
        hipLaunchKernelGGL((sample_picked_kernel<T, E>), grid, dim3(T), 0, st, n, j.in.ld, x, m,               \
                           isfinite(j.in.cap), a);                                                            \
    else                                                                                                      \
        hipLaunchKernelGGL((sample_kernel<T, E>), grid, dim3(T), 0, st, n, j.in.ld, x, m, a)
    if (n <= 512) SAMPLE(64);
    else if (n <= 4096) SAMPLE(256);
    else SAMPLE(1024);
#undef SAMPLE
    return hipGetLastError();
}

template <typename E>
hipError_t launch_top_t(const TopJob &j, hipStream_t st) {
    const float c2 = static_cast<float>(j.in.scale * 1.4426950408889634);
#define TOP(T)                                                                                              \
    hipLaunchKernelGGL((top_logits_kernel<T, E>), dim3(static_cast<unsigned>(j.in.B)), dim3(T), 0, st,      \
                       static_cast<int>(j.in.N), j.in.ld, static_cast<const E *>(j.in.x),                   \
                       ScoreMap{j.in.cap, j.in.flip}, isfinite(j.in.cap), j.in.scale, c2, j.K, j.idx,       \
                       j.logit, j.rest)
    if (j.in.N <= 512) TOP(64);
    else if (j.in.N <= 4096) TOP(256);
    else TOP(1024);
#undef TOP
    return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const SampleJob &j, hipStream_t st) {
    if (j.in.B == 0) return hipSuccess;
    ProfScope prof("sample", st);
    return j.in.bf16 ? launch_sample_t<uint16_t>(j, st) : launch_sample_t<float>(j, st);
}

hipError_t launch_top_logits(const TopJob &j, hipStream_t st) {
    if (j.in.B == 0) return hipSuccess;
    ProfScope prof("top_logits", st);
    return j.in.bf16 ? launch_top_t<uint16_t>(j, st) : launch_top_t<float>(j, st);
}

}  // namespace dstd
