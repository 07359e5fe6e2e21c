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

template <int T> constexpr int kBins = T >= 1024 ? 2048 : T >= 256 ? 1024 : 512;  // of a histogram over a row
// Candidates of a row that are held at once, and so the largest top_k that is
// chosen from candidates.
template <int T> constexpr int kList = kBins<T>;
constexpr int kMaxPicked = 1024;
// vectors a thread on the way in loops with an exponential and a histogram: 64 registers
// a thread hold one (300 x 50021 fp32, top_p 0.95: 106 us with 1, 118 with 4)
template <int T> constexpr int kOrderAhead = T >= 1024 ? 1 : kRowAhead;
// groups of a thread's share of the row, a maximum each
template <typename E> constexpr int kGroups = sizeof(E) == 2 ? 2 * kRowAhead : kRowAhead;

template <int T> struct RowShared {
    u64 red[T / kWave + 1];
    u64 list[kList<T>];
    u64 hist[kBins<T>];
    u64 found[2];
    int count, seen;
};

__device__ __forceinline__ float larger(float y, float best) { return y > best ? y : best; }  // not NaN

// What is kept of a row: all up to a place in its order.
struct Border {
    u64 last;
    __device__ bool has(u32 key, int i) const { return key > kAbsentKey && rank_of(key, i) >= last; }
    __device__ bool all() const { return last == 0; }
    // the same by goodness and index: y above `at`, or equal with an index up to `upto`
    __device__ float at() const { return all() ? -INFINITY : value_of(rank_key(last)); }
    __device__ int upto() const { return all() ? -1 : rank_index(last); }
};

// Weights of the exponentials in 64-bit integers, the largest 2^shift (shift <= 51):
// their sums do not depend on the order, and what is lost of a weight, 2^-(shift+1) of
// the largest, is below what sums in 64-bit floats lose over long rows.
struct Mass {
    double top, scale;  // the largest goodness; |scale|
    int shift;
    // how far below the largest weights are 0
    __device__ double span() const { return 0.6931471805599453 * (shift + 1) / scale; }
    __device__ double distance(float y) const { return (top - static_cast<double>(y)) * scale; }
    __device__ double distance(u32 key) const { return distance(value_of(key)); }
    // rint(e^-d 2^shift): d = n ln 2 + r, e^-r by its series to r^12 / 12! (|r| <= ln 2 / 2:
    // 2^-52 relative), n taken off its exponent. Adding 2^52 leaves the integer in the low
    // bits. From d = 64 on (and for NaN) the result is 0.
    static __device__ __forceinline__ u64 fixed_exp(double d, int shift) {
        d = fmin(d, 64.0);
        const double big = 0x1.8p52;
        const double t = fma(d, 1.4426950408889634, big);
        const double n = t - big;
        const double r = fma(n, -0x1.abc9e3b39803fp-56, fma(n, -0x1.62e42fefa39efp-1, d));
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
// u outside [0, 1) is drawn in, NaN to 0
__device__ __forceinline__ double share_of(const DrawArgs &a, int64_t b) {
    return fmin(fmax(static_cast<double>(a.u[b]), 0.0), 1.0 - 0x1p-24);
}

// The draw among what is kept of a row.
template <int T, int kAhead, typename E, typename G>
__device__ __forceinline__ void draw_kept(RowShared<T> &sh, const E *row, int64_t b, int n, const Mass &mass,
                                          const Border &kept, const DrawArgs &a, G good) {
    u64 all;
    int i;
    if (kept.all() && a.dmax == INFINITY) {
        i = by_index<T, kAhead>(sh, row, n, share_of(a, b), &all, [&](float x, int) { return mass.of(good(x)); });
    } else {
        const float at = kept.at();
        const int upto = kept.upto();
        i = by_index<T, kAhead>(sh, row, n, share_of(a, b), &all, [&](float x, int k) -> u64 {
            const float y = good(x);
            return (y > at || (y == at && k <= upto)) && mass.distance(y) <= a.dmax ? mass.of(y) : 0;
        });
    }
    if (threadIdx.x == 0) put_draw(a, b, i, mass.distance(good(widen1(row[i]))), all);
}

// One class of a row by its definition, whatever the values.
template <int T, int kAhead, typename E>
__device__ __attribute__((noinline)) void sample_any_row(RowShared<T> &sh, const E *row, int64_t b, int n, ScoreMap m,
                                                         DrawArgs a) {
    const Extremes ex = row_extremes<T, kAhead>(sh, row, n, m);
    if (ex.count == 0) {
        if (threadIdx.x == 0) put_draw(a, b, -1, 0.0, 0);
        return;
    }
    const Mass mass{ex.ymax, a.scale, a.shift};
    Border kept{0};
    if (a.top_k > 0 && a.top_k < ex.count) kept = pick_count<T, kAhead, E>(sh, row, n, m, ex, a.top_k);
    if (a.top_p < 1.0) kept = pick_mass<T, kAhead, E>(sh, row, n, m, kept, ex.ymin, mass, a.top_p);
    draw_kept<T, kAhead>(sh, row, b, n, mass, kept, a, [&](float x) { return goodness(x, m); });
}

// One class of every row.
// kCount, kMass: with top_k (more than kMaxPicked), with top_p.
template <int T, bool kCount, bool kMass, typename E>
__global__ __launch_bounds__(T, T >= 1024 ? 8 : 4) void sample_kernel(int n, int64_t ld, const E *__restrict__ x,
                                                                      ScoreMap m, DrawArgs a) {
    __shared__ RowShared<T> sh;
    const int64_t b = blockIdx.x;
    const E *row = x + b * ld;
    auto good = [&](float v) { return goodness(v, m); };
    float top = -INFINITY;
    row_each<kRowAhead>(row, n, threadIdx.x, T, [&](int, float v) { top = fmaxf(good(v), top); });
    top = value_of(block_max<T>(key_of(top), sh.red));
    if (!(top > -INFINITY)) {
        if (threadIdx.x == 0) put_draw(a, b, -1, 0.0, 0);
        return;
    }
    const Mass mass{top, a.scale, a.shift};
    Border kept{0};
    if constexpr (kCount) {
        const Extremes ex = row_extremes<T, kRowAhead>(sh, row, n, m);
        if (a.top_k < ex.count)
            kept = by_order<T, kOrderAhead<T>>(sh, row, n, m, kept, ex.ymin, top, INFINITY, One{}, a.top_k, 0.0);
    }
    if constexpr (kMass)
        kept = by_order<T, kOrderAhead<T>>(sh, row, n, m, kept, -INFINITY, top, mass.span(), mass, 0, a.top_p);
    draw_kept<T, kRowAhead>(sh, row, b, n, mass, kept, a, good);
}

// Candidates for the K first entries of a row's order: all that reach a bound which K
// entries reach at least. The bound is the K-th largest of the groups' largest values, or
// a little less: few others reach it unless the largest lie close together in the row.
using i16x2 = int16_t __attribute__((ext_vector_type(2)));
using u32x4 = u32 __attribute__((ext_vector_type(4)));

// bf16 bits as 16-bit integers in the order of the goodness (-0 just below +0; what is
// not finite at the ends), two at a time; flip: 0, or all ones where smaller scores are
// likelier. Its own inverse without flip.
__device__ __forceinline__ i16x2 order16(u32 bits, u32 flip) {
    const i16x2 h = __builtin_bit_cast(i16x2, bits);
    const u32 sign = __builtin_bit_cast(u32, h >> 15);
    return __builtin_bit_cast(i16x2, ((sign & 0x7fff7fffu) ^ bits) ^ flip);
}
__device__ __forceinline__ float order16_value(int16_t k) {
    const u32 bits = static_cast<uint16_t>(k ^ ((k >> 15) & 0x7fff));
    return __uint_as_float(bits << 16);
}

// The largest goodness of each group of a thread. Entries that do not count are not
// looked for: a NaN changes nothing, and where +inf shows up (a NaN too, in 16 bits)
// the bound is given up.
template <int T, bool kCaps, typename E>
__device__ __forceinline__ void group_best(const E *row, int n, const ScoreMap &m, float (&best)[kGroups<E>]) {
    using V = RowVec<E>;
    auto value = [&](float x) { return kCaps ? goodness(x, m) : flipped(x, m); };
    constexpr bool packed = sizeof(E) == 2 && !kCaps;
    const u32 flip = m.flip ? 0xffffffffu : 0;
    i16x2 top[kRowAhead];
#pragma unroll
    for (int g = 0; g < kRowAhead; ++g) top[g] = i16x2{-32768, -32768};
#pragma unroll
    for (int g = 0; g < kGroups<E>; ++g) best[g] = -INFINITY;
    auto take = [&](int g, typename V::type r) {
        if constexpr (packed) {
            const u32x4 w = __builtin_bit_cast(u32x4, r);
#pragma unroll
            for (int k = 0; k < 4; ++k) top[g] = __builtin_elementwise_max(top[g], order16(w[k], flip));
        } else {
#pragma unroll
            for (int k = 0; k < V::n; ++k) best[g] = larger(value(widen1(static_cast<E>(r[k]))), best[g]);
        }
    };
    const int done = vec_each<kRowAhead>(row, n, threadIdx.x, T, [&](int g, int, typename V::type r) { take(g, r); });
    if constexpr (packed) {
#pragma unroll
        for (int g = 0; g < kRowAhead; ++g)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float y = order16_value(top[g][k]);
                best[2 * g + k] = top[g][k] >= 0x7f80 ? INFINITY : y == y ? y : -INFINITY;
            }
    }
    const int i = done + threadIdx.x;
    if (i < n) best[0] = larger(value(widen1(row[i])), best[0]);
}

template <int T, bool kCaps, typename E>
__device__ float candidate_bound(RowShared<T> &sh, const E *row, int n, const ScoreMap &m, int K) {
    constexpr int groups = kGroups<E>;
    float best[groups];
    group_best<T, kCaps>(row, n, m, best);
    float lo = INFINITY, hi = -INFINITY;
#pragma unroll
    for (int g = 0; g < groups; ++g) {
        if (best[g] > -INFINITY) lo = fminf(lo, best[g]);
        hi = fmaxf(hi, best[g]);
    }
    hi = value_of(block_max<T>(key_of(hi), sh.red));
    lo = value_of(block_min<T>(key_of(lo), sh.red));
    if (hi == INFINITY || K > groups * T) return -FLT_MAX;
    if (!(hi > -INFINITY)) return INFINITY;  // nothing counts
    // bins of the range of the maxima
    const float per = static_cast<float>(kBins<T> / (static_cast<double>(hi) - static_cast<double>(lo)));
    u32 *hist = reinterpret_cast<u32 *>(sh.hist);
    for (int k = threadIdx.x; k < kBins<T>; k += T) hist[k] = 0;
    if (threadIdx.x == 0) sh.count = -1;
    __syncthreads();
    int bin[groups];
#pragma unroll
    for (int g = 0; g < groups; ++g) {
        bin[g] = kBins<T>;  // a group without an entry
        if (best[g] > -INFINITY) {
            bin[g] = static_cast<int>(fminf((hi - best[g]) * per, kBins<T> - 1.f));
            atomicAdd(&hist[bin[g]], 1u);
        }
    }
    __syncthreads();
    constexpr int each = kBins<T> / T;
    u32 mine = 0;
#pragma unroll
    for (int k = 0; k < each; ++k) mine += hist[threadIdx.x * each + k];
    u32 all;
    u32 at = block_before<T>(mine, sh.red, &all);
    if (at < static_cast<u32>(K) && at + mine >= static_cast<u32>(K))
        for (int k = 0; k < each; ++k) {
            at += hist[threadIdx.x * each + k];
            if (at >= static_cast<u32>(K)) {
                sh.count = threadIdx.x * each + k;
                break;
            }
        }
    __syncthreads();
    const int last = sh.count;
    float bound = INFINITY;
#pragma unroll
    for (int g = 0; g < groups; ++g)
        if (bin[g] <= last) bound = fminf(bound, best[g]);
    bound = value_of(block_min<T>(key_of(bound), sh.red));
    return last < 0 ? -FLT_MAX : bound;
}

// The K first entries of a row's order and at most a few more, sorted, in the list;
// returns how many there are (fewer than K where the row has fewer). kSum: *others is the
// sum over the entries behind the K-th.
// The K first entries into the list where the candidates are too many for it; and the sum
// over all entries behind a place in the row's order, relative to the largest of them.
template <int T, typename E>
__device__ __attribute__((noinline)) int pick_exactly(RowShared<T> &sh, const E *row, int n, ScoreMap m, int K) {
    const Border kept = pick_count<T, 0, E>(sh, row, n, m, row_extremes<T, 0>(sh, row, n, m), K);
    return collect<T, 0>(sh, row, n, m, [&](float y, int i) { return kept.has(key_of(y), i); });
}
template <int T, typename E>
__device__ __attribute__((noinline)) ExpSum sum_behind(const E *row, int n, ScoreMap m, u64 last, float c2) {
    ExpSum s{-INFINITY, 0.f};
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
    return s;
}

template <int T, bool kSum, bool kCaps, typename E>
__device__ int candidates(RowShared<T> &sh, const E *row, int n, const ScoreMap &m, int K, float c2,
                          ExpSum *others) {
    if (kSum) *others = ExpSum{-INFINITY, 0.f};
    float bound = -FLT_MAX;
    if (n > kList<T>) bound = candidate_bound<T, kCaps>(sh, row, n, m, K);
    if (bound == INFINITY) return 0;
    // the bound among 16-bit keys (the lower of the two zeros)
    const u32 flip16 = m.flip ? 0xffffffffu : 0;
    const int bound16 = bound == 0.f ? -1 : order16(__float_as_uint(bound) >> 16, 0)[0];
    // vectors with a candidate, in the histogram's memory; they are looked through behind
    // the loop, all at once
    constexpr int most = 2 * kBins<T>, vn = RowVec<E>::n;
    u32 *seen = reinterpret_cast<u32 *>(sh.hist);
    __syncthreads();
    if (threadIdx.x == 0) sh.count = sh.seen = 0;
    __syncthreads();
    // what is below the bound is summed relative to it, as 2^(c x - kb); NaN adds 0
    float kb = bound * c2, sum = 0.f;
    const float c = m.flip ? -c2 : c2;
    const bool sums = bound > -FLT_MAX && isfinite(kb);
    if (!sums) kb = 0.f;
    auto term = [&](float x) {
        return __builtin_amdgcn_exp2f(fmaxf(fmaf(x, c, -kb), -1000.f));
    };
    auto capped = [&](float x) { return kCaps && !isfinite(x) ? m.cap : x; };
    auto look = [&](int i) {
        const float x = capped(widen1(row[i])), y = flipped(x, m);
        if (y >= bound && y < INFINITY) {
            const int at = atomicAdd(&sh.count, 1);
            if (at < kList<T>) sh.list[at] = rank_of(key_of(y), i);
        } else if (kSum) {
            sum += y < bound ? term(x) : 0.f;
        }
    };
    const int done = vec_each<kRowAhead>(row, n, threadIdx.x, T, [&](int, int i, typename RowVec<E>::type r) {
        float x[vn];
        bool some;
        if constexpr (sizeof(E) == 2 && !kCaps) {
            const u32x4 w = __builtin_bit_cast(u32x4, r);
            i16x2 top = order16(w[0], flip16);
#pragma unroll
            for (int k = 1; k < 4; ++k) top = __builtin_elementwise_max(top, order16(w[k], flip16));
            some = max(top[0], top[1]) >= bound16;
#pragma unroll
            for (int k = 0; k < vn; ++k) x[k] = widen1(static_cast<E>(r[k]));
        } else {
            float top = -INFINITY;
#pragma unroll
            for (int k = 0; k < vn; ++k) {
                x[k] = capped(widen1(static_cast<E>(r[k])));
                top = larger(flipped(x[k], m), top);
            }
            some = top >= bound;
        }
        if (some) {
            const int at = atomicAdd(&sh.seen, 1);
            if (at < most) seen[at] = i;
        } else if (kSum) {
#pragma unroll
            for (int k = 0; k < vn; ++k) sum += term(x[k]);
        }
    });
    __syncthreads();
    if (sh.seen <= most) {
        for (int k = threadIdx.x; k < sh.seen * vn; k += T) look(seen[k / vn] + k % vn);
    } else {
        sum = 0.f;
#pragma unroll 1
        for (int i = threadIdx.x; i < done; i += T) look(i);
    }
    if (done + static_cast<int>(threadIdx.x) < n) look(done + threadIdx.x);
    __syncthreads();
    int count = sh.count;
    bool listed = bound == -FLT_MAX;  // the sum is that of the list's others alone
    if (count > kList<T>) {
        count = pick_exactly<T, E>(sh, row, n, m, K);
        sum = 0.f;
        listed = false;
    }
    sort_by_value<T>(sh, count);
    if (!kSum || count < K) return count;
    if (!sums) sum = 0.f;
    ExpSum s{-INFINITY, 0.f};
    const bool some = __syncthreads_or(sum > 0.f);
    if (some || listed) {
        // kb was rounded
        if (sum > 0.f) s = ExpSum{bound, sum * __builtin_amdgcn_exp2f(-fmaf(bound, c2, -kb))};
        for (int k = K + threadIdx.x; k < count; k += T)
            s = exp_join(s, ExpSum{value_of(rank_key(sh.list[k])), 1.f}, c2);
    } else {
        // all others far below the bound (their sum there is 0), or no bound was found
        s = sum_behind<T, E>(row, n, m, sh.list[K - 1], c2);
    }
    *others = block_exp_sum<T>(s, c2, sh.red);
    return count;
}

template <int T, bool kCaps, typename E>
__global__ __launch_bounds__(T, T >= 1024 ? 8 : 4) void top_logits_kernel(int n, int64_t ld, const E *__restrict__ x, ScoreMap m,
                                                       double scale, float c2, int K,
                                                       int32_t *__restrict__ idx, float *__restrict__ logit,
                                                       float *__restrict__ rest) {
    __shared__ RowShared<T> sh;
    const int64_t b = blockIdx.x;
    const E *row = x + b * ld;
    ExpSum s;
    const int count = candidates<T, true, kCaps>(sh, row, n, m, K, c2, &s);
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
template <int T, bool kCaps, typename E>
__global__ __launch_bounds__(T, T >= 1024 ? 8 : 4) void sample_picked_kernel(int n, int64_t ld,
                                                                             const E *__restrict__ x, ScoreMap m,
                                                                             DrawArgs a) {
    __shared__ RowShared<T> sh;
    const int64_t b = blockIdx.x;
    const E *row = x + b * ld;
    int count = candidates<T, false, kCaps>(sh, row, n, m, a.top_k, 0.f, nullptr);
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
    u32 keeps = 0;
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
    const float per = static_cast<float>(kBins<T>) / static_cast<float>(n);
    sort_list<T>(sh, count, [&](u64 r) {
        return static_cast<u32>(fminf(static_cast<float>(~static_cast<u32>(r >> 32)) * per, kBins<T> - 1.f));
    });
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
// bf16 scores of a magnitude in [2^-24, 2^8) take 2 * 4096 values: how often each occurs
// says which are kept and what they weigh, with an exponential a value instead of one an
// entry. Zeros are counted apart; the few values nearer to 0 are listed one by one; what is
// larger with a goodness below 0 has to weigh nothing. Other rows are drawn from by their
// definition.
constexpr int kMags = 4096, kFirstMag = 0x3380, kValues = 2 * kMags;
using u16x2 = uint16_t __attribute__((ext_vector_type(2)));

// A value's place among the counters: its magnitude, its sign bit above.
__device__ __forceinline__ u32 slots_of(u32 bits, u16x2 *most) {
    const u16x2 mag = __builtin_bit_cast(u16x2, bits & 0x7fff7fffu) - u16x2{kFirstMag, kFirstMag};
    *most = __builtin_elementwise_max(*most, mag);
    return __builtin_bit_cast(u32, mag) | (bits >> 3 & 0x10001000u);
}

constexpr int kSmall = 16;
template <int T> struct ValueShared {
    u64 red[T / kWave + 1];
    union {
        RowShared<T> row;
        u64 weight[kValues];
        u32 count[kValues];
    };
    u64 part[T / kWave];
    u32 ties[T / kWave];
    u64 tie_weight;
    int tie_slot, tie_keep;
    u32 below, odd;
    // zero and the values nearer to it than 2^-24, falling: places, entries, weights. They
    // have the slots from kValues on.
    u64 small[kSmall], small_weight[kSmall];
    u32 small_count[kSmall];
    int smalls;
    u64 listed[kSmall];
    u32 zeros;
};
constexpr int kNoSlot = -1, kBelow = -2, kOdd = -3, kTiny = -4, kZero = -5;

// The slot of one entry, whatever it is.
struct OneSlot {
    u32 flip, cap;  // as of ScoreMap, in 16 bits; 0x10000: left out
    __device__ int operator()(u32 bits) const {
        if ((bits & 0x7fff) >= 0x7f80) {
            if (cap > 0xffff) return kNoSlot;
            bits = cap;
        }
        const u32 mag = (bits & 0x7fff) - kFirstMag;
        if (mag < static_cast<u32>(kMags)) return static_cast<int>(mag | (bits >> 3 & 0x1000));
        if ((bits & 0x7fff) == 0) return kZero;
        if ((bits & 0x7fff) < kFirstMag) return kTiny;
        return (bits ^ flip) & 0x8000 ? kBelow : kOdd;
    }
};

template <int T>
__global__ __launch_bounds__(T, 8) void sample_values_kernel(int n, int64_t ld, const uint16_t *__restrict__ x,
                                                             ScoreMap m, OneSlot one, DrawArgs a) {
    __shared__ ValueShared<T> sh;
    constexpr int each = kValues / T, waves = T / kWave;
    const int64_t b = blockIdx.x;
    const uint16_t *row = x + b * ld;
    const int tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
    for (int k = tid; k < kValues; k += T) sh.count[k] = 0;
    if (tid == 0) sh.smalls = sh.zeros = sh.below = sh.odd = 0;
    __syncthreads();
    auto count_one = [&](u32 bits, int i) {
        const int slot = one(bits);
        if (slot >= 0) atomicAdd(&sh.count[slot], 1u);
        else if (slot == kZero) atomicAdd(&sh.zeros, 1u);
        else if (slot == kBelow) sh.below = 1;
        else if (slot == kOdd) sh.odd = 1;
        else if (slot == kTiny) {
            const int at = atomicAdd(&sh.smalls, 1);
            if (at < kSmall - 1) sh.listed[at] = rank_of(key_of(goodness(widen1(static_cast<uint16_t>(bits)), m)), i);
        }
    };
    int done = vec_each<kRowAhead>(row, n, tid, T, [&](int, int i, RowVec<uint16_t>::type r) {
        const u32x4 w = __builtin_bit_cast(u32x4, r);
        u16x2 most = {0, 0};
        u32 s[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) s[k] = slots_of(w[k], &most);
        if (max(most[0], most[1]) < kMags) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                atomicAdd(&sh.count[s[k] & 0xffff], 1u);
                atomicAdd(&sh.count[s[k] >> 16], 1u);
            }
        } else {
#pragma unroll 1
            for (int k = 0; k < 4; ++k) {
                const u32 v = k == 0 ? w[0] : k == 1 ? w[1] : k == 2 ? w[2] : w[3];
                count_one(v & 0xffff, i + 2 * k);
                count_one(v >> 16, i + 2 * k + 1);
            }
        }
    });
    if (done + tid < n) count_one(row[done + tid], done + tid);
    __syncthreads();
    // the values in falling order: place p of the first half is magnitude kMags - 1 - p
    // above 0, of the second p - kMags below 0; 0 is taken behind the first half's last
    const u32 above = one.flip ? kMags : 0;
    auto slot_at = [&](int p) -> int {
        return p < kMags ? static_cast<int>(above) + kMags - 1 - p : static_cast<int>(above ^ kMags) + p - kMags;
    };
    auto value_at = [&](int p) {
        const u32 mag = (p < kMags ? kMags - 1 - p : p - kMags) + kFirstMag;
        return __uint_as_float(mag << 16 | (p < kMags ? 0u : 0x80000000u));
    };
    const int tinies = sh.smalls;
    const bool odd = sh.odd || tinies >= kSmall, below = sh.below;
    const int smalls = odd ? 0 : tinies + (sh.zeros > 0 ? 1 : 0);
    if (tid < smalls) {
        const u64 zero = rank_of(key_of(0.f), 0);
        const u64 mine = tid < tinies ? sh.listed[tid] : zero;
        int at = sh.zeros > 0 && zero > mine;
        for (int k = 0; k < tinies; ++k) at += sh.listed[k] > mine;
        sh.small[at] = mine;
        sh.small_count[at] = tid < tinies ? 1 : sh.zeros;
    }
    // the thread of the first half's last values has these behind its own
    const bool has_small = smalls > 0 && tid == kMags / each - 1;
    u32 count[each];
    u32 first = 2 * kValues, counted = 0;
    if (has_small) {
        first = 2 * (tid * each + each) - 1;
        counted = tinies + sh.zeros;
    }
#pragma unroll
    for (int k = each - 1; k >= 0; --k) {
        count[k] = sh.count[slot_at(tid * each + k)];
        if (count[k]) first = 2 * (tid * each + k);
        counted += count[k];
    }
    first = block_min<T>(first, sh.red);
    if (first == 2 * kValues && !odd && !below) {
        if (tid == 0) put_draw(a, b, -1, 0.0, 0);
        return;
    }
    __syncthreads();
    const Mass mass{first % 2 ? value_of(rank_key(sh.small[0])) : value_at(static_cast<int>(first / 2)), a.scale,
                    a.shift};
    if (odd || (below && (first == 2 * kValues || mass.of(value_at(kValues - 1)) != 0))) {
        __syncthreads();
        sample_any_row<T, 0, uint16_t>(sh.row, row, b, n, m, a);
        return;
    }
    // Values in turn, one at a time: nothing but the counts stays in registers, a weight
    // is formed again where it is needed again.
    u64 sum = 0;
    u32 counts;
    u32 before = block_before<T>(counted, sh.red, &counts);
    u32 partly = 0;  // bits of the values of which not all entries are kept
    auto keep_first = [&](u32 have, float value, u32 bit) {
        u32 keep = have;
        if (a.top_k > 0) keep = before >= static_cast<u32>(a.top_k) ? 0 : min(keep, a.top_k - before);
        before += have;
        if (keep < have) partly |= bit;
        if (keep) sum += static_cast<u64>(keep) * mass.of(value);
        return keep;
    };
#pragma unroll
    for (int k = 0; k < each; ++k) {
        __builtin_amdgcn_sched_barrier(0);
        count[k] = keep_first(count[k], value_at(tid * each + k), 1u << k);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (has_small)
        for (int k = 0; k < smalls; ++k)
            sh.small_count[k] = keep_first(sh.small_count[k], value_of(rank_key(sh.small[k])), 256u << k);
    u64 all;
    u64 at = block_before<T>(sum, sh.red, &all);
    // the counts are in registers: their place takes the weights
    if (tid == 0) {
        sh.tie_slot = kNoSlot;
        sh.tie_keep = 0;
        sh.tie_weight = 0;
    }
    __syncthreads();
    const double target = a.top_p < 1.0 ? a.top_p * static_cast<double>(all) : INFINITY;
    u64 tie_at = 0, tie_w = 0;
    u32 tie_keeps = 0;
    int tie = kNoSlot;  // the value of which some entries are kept
    auto weigh = [&](u32 have, float value, u32 bit, int slot) -> u64 {
        if (!have || !(static_cast<double>(at) < target) || mass.distance(value) > a.dmax) return 0;
        const u64 w = mass.of(value), next = at + have * w;
        if (static_cast<double>(next) >= target || (partly & bit)) {
            tie = slot;
            tie_at = at;
            tie_w = w;
            tie_keeps = have;
        }
        at = next;
        return tie == slot ? 0 : w;
    };
#pragma unroll
    for (int k = 0; k < each; ++k) {
        __builtin_amdgcn_sched_barrier(0);
        const int slot = slot_at(tid * each + k);
        sh.weight[slot] = weigh(count[k], value_at(tid * each + k), 1u << k, slot);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (has_small)
        for (int k = 0; k < smalls; ++k)
            sh.small_weight[k] = weigh(sh.small_count[k], value_of(rank_key(sh.small[k])), 256u << k, kValues + k);
    if (tie_w) {
        // the fewest of its entries that reach the target; all of it may be
        u64 keep = tie_keeps;
        if (static_cast<double>(tie_at + keep * tie_w) >= target) {
            u64 c = static_cast<u64>((target - static_cast<double>(tie_at)) / static_cast<double>(tie_w));
            while (c > 0 && static_cast<double>(tie_at + (c - 1) * tie_w) >= target) --c;
            while (static_cast<double>(tie_at + c * tie_w) < target) ++c;
            keep = min(keep, c);
        }
        sh.tie_slot = tie;
        sh.tie_keep = static_cast<int>(keep);
        sh.tie_weight = tie_w;
    }
    __syncthreads();
    const int tie_slot = sh.tie_slot;
    const u64 tie_keep = sh.tie_keep, tie_weight = sh.tie_weight;
    // the kept weights of each wave's part of the row; of the value that is kept in part, the
    // entries, of which the first tie_keep count
    constexpr int unit = kWave * 8;
    const int part = (n + waves * unit - 1) / (waves * unit) * unit;
    const int lo = min(n, wave * part), hi = min(n, lo + part);
    u64 s = 0;
    u32 ties = 0;
    auto slot_of = [&](u32 bits, int i) {
        const int slot = one(bits);
        if (slot != kZero && slot != kTiny) return slot;
        for (int k = 0; k < smalls; ++k)
            if (slot == kZero ? rank_key(sh.small[k]) == key_of(0.f)
                              : rank_index(sh.small[k]) == i && rank_key(sh.small[k]) != key_of(0.f))
                return kValues + k;
        return kNoSlot;
    };
    // the weight of an entry that is kept with all of its value; counts one of the others
    auto weigh_one = [&](u32 bits, int i, u32 &tied) -> u64 {
        const int slot = slot_of(bits, i);
        if (slot < 0) return 0;
        tied += slot == tie_slot;
        return slot < kValues ? sh.weight[slot] : sh.small_weight[slot - kValues];
    };
    done = lo + vec_each<kRowAhead>(row + lo, hi - lo, lane, kWave, [&](int, int i, RowVec<uint16_t>::type r) {
        const u32x4 v = __builtin_bit_cast(u32x4, r);
        u16x2 most = {0, 0};
        u32 p[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) p[k] = slots_of(v[k], &most);
        if (max(most[0], most[1]) < kMags) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int p0 = p[k] & 0xffff, p1 = p[k] >> 16;
                s += sh.weight[p0] + sh.weight[p1];
                ties += p0 == tie_slot;
                ties += p1 == tie_slot;
            }
        } else {
#pragma unroll 1
            for (int k = 0; k < 8; ++k) {
                const u32 q = k < 4 ? (k < 2 ? v[0] : v[1]) : (k < 6 ? v[2] : v[3]);
                s += weigh_one(k % 2 ? q >> 16 : q & 0xffff, lo + i + k, ties);
            }
        }
    });
    if (done + lane < hi) s += weigh_one(row[done + lane], done + lane, ties);
    s = block_add<kWave>(s, nullptr);
    const u32 tied = block_add<kWave>(ties, nullptr);
    if (lane == 0) {
        sh.part[wave] = s;
        sh.ties[wave] = tied;
    }
    __syncthreads();
    // every wave finds the part for itself, a lane for each
    auto plus = [](u64 p, u64 q) { return p + q; };
    const u64 wave_t = sh.ties[lane % waves];
    const u64 t_before = wave_upto<waves>(wave_t, u64{0}, plus) - wave_t;
    const u64 own = sh.part[lane % waves] +
                    tie_weight * (min(t_before + wave_t, tie_keep) - min(t_before, tie_keep));
    const u64 upto = wave_upto<waves>(own, u64{0}, plus);
    all = lane_value(upto, waves - 1);
    const double goal = share_of(a, b) * static_cast<double>(all);
    const int from = __builtin_amdgcn_readfirstlane(
        __ffsll(__ballot(lane < waves && static_cast<double>(upto) > goal)) - 1);
    u64 base = lane_value(upto - own, from), t = lane_value(t_before, from);
    // the place in that part, a vector's entries a thread at a time
    const int start = from * part, end = min(n, start + part);
    for (int p = start; p < end; p += T * 8) {
        const int p0 = p + tid * 8;
        u64 each_w[8], mine = 0;
        u32 tie_bits = 0;
        u32x4 v = {0, 0, 0, 0};
        u16x2 most = {0, 0};
        u32 q[4];
        const int have = min(8, end - p0);
        if (have == 8) v = __builtin_bit_cast(u32x4, load_vec<uint16_t>(row + p0));
#pragma unroll
        for (int k = 0; k < 4; ++k) q[k] = slots_of(v[k], &most);
        if (have == 8 && max(most[0], most[1]) < kMags) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int slot = k % 2 ? q[k / 2] >> 16 : q[k / 2] & 0xffff;
                each_w[k] = sh.weight[slot];
                tie_bits |= static_cast<u32>(slot == tie_slot) << k;
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                u32 tied = 0;
                each_w[k] = k < have ? weigh_one(row[p0 + k], p0 + k, tied) : 0;
                tie_bits |= tied << k;
            }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) mine += each_w[k];
        u32 round_t;
        u64 round, tt = t + block_before<T>(static_cast<u32>(__popc(tie_bits)), sh.red, &round_t);
        mine += tie_weight * (min(tt + __popc(tie_bits), tie_keep) - min(tt, tie_keep));
        u64 g = base + block_before<T>(mine, sh.red, &round);
        if (static_cast<double>(g) <= goal && static_cast<double>(g + mine) > goal) {
            int k = 0;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                if (tie_bits >> q & 1) g += tt++ < tie_keep ? tie_weight : 0;
                else g += each_w[q];
                if (static_cast<double>(g) <= goal) k = q + 1;
            }
            put_draw(a, b, p0 + k, mass.distance(goodness(widen1(row[p0 + k]), m)), all);
        }
        base += round;
        t += round_t;
        if (static_cast<double>(base) > goal) return;
    }
}

// Whether a cap is one of the values that are counted, or is none.
bool cap_has_slot(float cap, u32 *bits) {
    *bits = 0x10000u;
    if (!isfinite(cap)) return true;
    u32 f;
    memcpy(&f, &cap, 4);
    *bits = f >> 16;
    const u32 mag = (*bits & 0x7fff) - kFirstMag;
    return (f & 0xffff) == 0 && mag < static_cast<u32>(kMags);
}

template <int T, typename E>
void launch_sample_rows(dim3 grid, hipStream_t st, int n, int64_t ld, const E *x, ScoreMap m, DrawArgs a) {
    const bool count = a.top_k > 0 && a.top_k < n, mass = a.top_p < 1.0;
#define SAMPLE(...) hipLaunchKernelGGL((__VA_ARGS__), grid, dim3(T), 0, st, n, ld, x, m, a)
    if (a.top_k > 0 && a.top_k <= kMaxPicked) {
        if (isfinite(m.cap)) SAMPLE(sample_picked_kernel<T, true, E>);
        else SAMPLE(sample_picked_kernel<T, false, E>);
    } else if (count && mass) {
        SAMPLE(sample_kernel<T, true, true, E>);
    } else if (count) {
        SAMPLE(sample_kernel<T, true, false, E>);
    } else if (mass) {
        SAMPLE(sample_kernel<T, false, true, E>);
    } else {
        SAMPLE(sample_kernel<T, false, false, E>);
    }
#undef SAMPLE
}

template <typename E>
hipError_t launch_sample_t(const SampleJob &j, hipStream_t st) {
    const int n = static_cast<int>(j.in.N);
    const dim3 grid(static_cast<unsigned>(j.in.B));
    const ScoreMap m{j.in.cap, j.in.flip};
    const DrawArgs a{j.in.scale, j.top_p, j.min_p > 0.0 ? -log(j.min_p) : INFINITY, j.shift, j.top_k,
                     j.u, j.choice, j.logp};
    const E *x = static_cast<const E *>(j.in.x);
    u32 cap;
    if constexpr (sizeof(E) == 2)
        if (!(j.top_k > 0 && j.top_k <= kMaxPicked) && n > 4096 && cap_has_slot(j.in.cap, &cap)) {
            const OneSlot one{j.in.flip >> 16, cap};
            hipLaunchKernelGGL((sample_values_kernel<1024>), grid, dim3(1024), 0, st, n, j.in.ld, x, m, one, a);
            return hipGetLastError();
        }
    if (n <= 512) launch_sample_rows<64, E>(grid, st, n, j.in.ld, x, m, a);
    else if (n <= 4096) launch_sample_rows<256, E>(grid, st, n, j.in.ld, x, m, a);
    else launch_sample_rows<1024, E>(grid, st, n, j.in.ld, x, m, a);
    return hipGetLastError();
}

template <typename E>
hipError_t launch_top_t(const TopJob &j, hipStream_t st) {
    const int n = static_cast<int>(j.in.N);
    const dim3 grid(static_cast<unsigned>(j.in.B));
    const ScoreMap m{j.in.cap, j.in.flip};
    const E *x = static_cast<const E *>(j.in.x);
    const float c2 = static_cast<float>(j.in.scale * 1.4426950408889634);
#define TOP(T)                                                                                                  \
    if (isfinite(j.in.cap))                                                                                     \
        hipLaunchKernelGGL((top_logits_kernel<T, true, E>), grid, dim3(T), 0, st, n, j.in.ld, x, m, j.in.scale, \
                           c2, j.K, j.idx, j.logit, j.rest);                                                    \
    else                                                                                                        \
        hipLaunchKernelGGL((top_logits_kernel<T, false, E>), grid, dim3(T), 0, st, n, j.in.ld, x, m,            \
                           j.in.scale, c2, j.K, j.idx, j.logit, j.rest)
    if (n <= 512) TOP(64);
    else if (n <= 4096) TOP(256);
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
