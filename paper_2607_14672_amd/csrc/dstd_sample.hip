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

// Weights of the exponentials in 64-bit integers, the largest 2^shift: their sums
// do not depend on the order, and what is lost of a weight, 2^-(shift+1) of the
// largest, is below what sums in 64-bit floats lose over long rows.
struct Mass {
    double top, scale;  // the largest goodness; |scale|
    double one;         // 2^shift
    __device__ double distance(u32 key) const { return (top - static_cast<double>(value_of(key))) * scale; }
    __device__ u64 operator()(u32 key) const {
        const double d = distance(key);
        return d < 64.0 ? static_cast<u64>(rint(exp(-d) * one)) : 0;
    }
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

template <int T, typename E>
__global__ __launch_bounds__(T) void sample_kernel(int n, int64_t ld, const E *__restrict__ x, ScoreMap m,
                                                   double scale, int shift, int top_k, double top_p,
                                                   double min_p, const float *__restrict__ u,
                                                   int32_t *__restrict__ choice, float *__restrict__ logp) {
    __shared__ RowShared<T> sh;
    const int64_t b = blockIdx.x;
    const E *row = x + b * ld;
    const Extremes ex = row_extremes<T, kRowAhead>(sh, row, n, m);
    if (ex.count == 0) {
        if (threadIdx.x == 0) {
            choice[b] = -1;
            if (logp) logp[b] = -INFINITY;
        }
        return;
    }
    const Mass mass{ex.ymax, scale, ldexp(1.0, shift)};
    Border kept{0};
    if (top_k > 0 && top_k < ex.count)
        kept = by_order<T, kRowAhead>(sh, row, n, m, kept, ex.ymin, ex.ymax, INFINITY, One{}, top_k, 0.0);
    if (top_p < 1.0)
        kept = by_order<T, kRowAhead>(sh, row, n, m, kept, ex.ymin, ex.ymax, 0.6931471805599453 * (shift + 1) / scale, mass,
                           0, top_p);
    // u outside [0, 1) is drawn in, NaN to 0
    const double share = fmin(fmax(static_cast<double>(u[b]), 0.0), 1.0 - 0x1p-24);
    u64 all;
    const int i = by_index<T, kRowAhead>(sh, row, n, m, share, &all, [&](u32 key, int k) -> u64 {
        if (!kept.has(key, k)) return 0;
        if (min_p > 0.0 && !(exp(-mass.distance(key)) >= min_p)) return 0;
        return mass(key);
    });
    if (threadIdx.x == 0) {
        choice[b] = i;
        if (logp) {
            const double d = mass.distance(key_of(goodness(widen1(row[i]), m)));
            logp[b] = static_cast<float>(-d - log(static_cast<double>(all) / mass.one));
        }
    }
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
__global__ __launch_bounds__(T, T >= 1024 ? 8 : 4) void sample_picked_kernel(int n, int64_t ld, const E *__restrict__ x, ScoreMap m,
                                                          bool caps, double scale, int shift, int top_k,
                                                          double top_p, double min_p, const float *__restrict__ u,
                                                          int32_t *__restrict__ choice, float *__restrict__ logp) {
    __shared__ RowShared<T> sh;
    const int64_t b = blockIdx.x;
    const E *row = x + b * ld;
    int count = candidates<T, false>(sh, row, n, m, caps, top_k, 0.f, nullptr);
    if (count == 0) {
        if (threadIdx.x == 0) {
            choice[b] = -1;
            if (logp) logp[b] = -INFINITY;
        }
        return;
    }
    count = min(count, top_k);
    const Mass mass{value_of(rank_key(sh.list[0])), scale, ldexp(1.0, shift)};
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
    const double target = top_p < 1.0 ? top_p * static_cast<double>(all) : INFINITY;
    u64 keeps = 0;
#pragma unroll
    for (int k = 0; k < each; ++k) {
        if (first + k < count && static_cast<double>(at) < target &&
            (min_p == 0.0 || exp(-mass.distance(rank_key(sh.list[first + k]))) >= min_p))
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
    const double share = fmin(fmax(static_cast<double>(u[b]), 0.0), 1.0 - 0x1p-24);
    const double goal = share * static_cast<double>(all);
    if (static_cast<double>(at) <= goal && static_cast<double>(at + mine) > goal)
#pragma unroll
        for (int k = 0; k < each; ++k) {
            if (static_cast<double>(at) <= goal && static_cast<double>(at + w[k]) > goal) {
                const u64 r = sh.list[first + k];
                choice[b] = static_cast<int>(~static_cast<u32>(r >> 32));
                if (logp)
                    logp[b] = static_cast<float>(-mass.distance(static_cast<u32>(r)) -
                                                 log(static_cast<double>(all) / mass.one));
            }
            at += w[k];
        }
}

template <typename E>
hipError_t launch_sample_t(const SampleJob &j, hipStream_t st) {
    const bool caps = isfinite(j.in.cap);
#define SAMPLE(T)                                                                                              \
    if (j.top_k > 0 && j.top_k <= kMaxPicked)                                                                  \
        hipLaunchKernelGGL((sample_picked_kernel<T, E>), dim3(static_cast<unsigned>(j.in.B)), dim3(T), 0, st,  \
                           static_cast<int>(j.in.N), j.in.ld, static_cast<const E *>(j.in.x),                  \
                           ScoreMap{j.in.cap, j.in.flip}, caps, j.in.scale, j.shift, j.top_k, j.top_p, j.min_p, \
                           j.u, j.choice, j.logp);                                                             \
    else                                                                                                       \
        hipLaunchKernelGGL((sample_kernel<T, E>), dim3(static_cast<unsigned>(j.in.B)), dim3(T), 0, st,         \
                           static_cast<int>(j.in.N), j.in.ld, static_cast<const E *>(j.in.x),                  \
                           ScoreMap{j.in.cap, j.in.flip}, j.in.scale, j.shift, j.top_k, j.top_p, j.min_p, j.u, \
                           j.choice, j.logp)
    if (j.in.N <= 512) SAMPLE(64);
    else if (j.in.N <= 4096) SAMPLE(256);
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
