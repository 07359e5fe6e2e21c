// dstd_top.hip -- the K largest logits of a row, and a class drawn from them (gfx950).
//
//   z_i = scale x_i, in the order of falling z, ties by index: the first K, and
//   ln sum e^z of the others.
//
// Two passes over the row: the largest values of groups of it bound the K-th largest from
// below, then what reaches the bound is listed and what does not is summed. The order is
// that of the scores themselves, not of their products with the scale.
//
// A block a row: 64 threads up to 512 scores (which are all listed), 256 up to kShortRow
// (with K up to 256), 1024 beyond, two of those a CU (64 registers a thread: more loads on
// the way from two blocks than from one of 128). Many long rows are bound by their two passes
// (512 x 131072 bf16: 53 us, 268 MB leave the L2; 6 TB/s would be 44), a few by the issue
// rate of the CU that has one (131072 bf16: 21 us, 35000 operations, one a clock).
#include "dstd_profile.h"
#include "dstd_select.h"

namespace dstd {

namespace {

// Small blocks overlap each other's steps (top 32 of 2000 x 15000 bf16: 31 us with 256
// threads, 52 with 1024; 64 rows: 12.5 with either).
constexpr int kShortRow = 16384;
// groups of a thread's share of the row, a maximum each: by the place in a vector, so that
// short rows have as many as long ones
template <typename E> constexpr int kGroups = RowVec<E>::n;
__device__ __forceinline__ float larger(float y, float best) { return y > best ? y : best; }  // not NaN

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
    i16x2 top[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) top[g] = i16x2{-32768, -32768};
#pragma unroll
    for (int g = 0; g < kGroups<E>; ++g) best[g] = -INFINITY;
    const int done = vec_each<kRowAhead>(row, n, threadIdx.x, T, [&](int, typename V::type r) {
        if constexpr (packed) {
            const u32x4 w = __builtin_bit_cast(u32x4, r);
#pragma unroll
            for (int g = 0; g < 4; ++g) top[g] = __builtin_elementwise_max(top[g], order16(w[g], flip));
        } else {
#pragma unroll
            for (int g = 0; g < V::n; ++g) best[g] = larger(value(widen1(static_cast<E>(r[g]))), best[g]);
        }
    });
    if constexpr (packed) {
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float y = order16_value(top[g][k]);
                best[2 * g + k] = top[g][k] >= 0x7f80 ? INFINITY : y == y ? y : -INFINITY;
            }
    }
    const int i = done + threadIdx.x;
    if (i < n) best[0] = larger(value(widen1(row[i])), best[0]);
}

// Candidates for the K first entries of a row's order are all that reach a bound which K
// entries reach at least: the K-th largest of the groups' largest values, or a little less.
// Few others reach it unless the largest lie close together in the row. (A bound from an
// eighth of the row, the rest read once instead of twice, cost more in candidates than it
// saved: 512 x 131072 bf16, top_k 50: 51 us with it, 48 without.) INFINITY: the row is
// empty; -FLT_MAX: no bound.
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

// The K first entries into the list where the candidates are too many for it; and the sum
// over all entries behind a place in the row's order, relative to the largest of them. Some
// eight and one passes entry by entry, for rows where many entries equal the K-th (fewer than
// K neurons fired, and the silent ones count as a cap) or no bound is found (bf16 rows with
// a NaN, rows with an entry of +inf goodness that does not count): 256 x 4096 spike times of which
// 0.5 % fired, K = 32, 37 us instead of 11, 512 x 65536 without any 463 instead of 48, 512 x 131072
// bf16 all equal 841 and with a NaN a row 400 instead of 56. The sum alone (logits beyond 2^24): 512 x
// 65536 fp32 76 us instead of 47.
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

// The K first entries of a row's order and at most a few more, sorted, in the list;
// returns how many there are (fewer than K where the row has fewer). kSum: *others is the
// sum over the entries behind the K-th.
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
    // what is below the bound is summed relative to it, as 2^(c x - kb); NaN adds 0. The
    // rounding of kb is half a binary order at most
    float kb = bound * c2, sum = 0.f;
    const float c = m.flip ? -c2 : c2;
    const bool sums = bound > -FLT_MAX && fabsf(kb) < 0x1p24f;
    if (!sums) kb = 0.f;
    auto term = [&](float x) {
        return __builtin_amdgcn_exp2f(fmaxf(fmaf(x, c, -kb), -1000.f));
    };
    auto capped = [&](float x) { return kCaps && !isfinite(x) ? m.cap : x; };
    auto look = [&](int i) {
        const float y = flipped(capped(widen1(row[i])), m);
        if (y >= bound && y < INFINITY) {
            const int at = atomicAdd(&sh.count, 1);
            if (at < kList<T>) sh.list[at] = rank_of(key_of(y), i);
        }
    };
    const int done = vec_each<kRowAhead>(row, n, threadIdx.x, T, [&](int i, typename RowVec<E>::type r) {
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
        }
        // (the entries below the bound beside a candidate here all the same: sums keep
        // their order)
        if (kSum && __any(some)) {
#pragma unroll
            for (int k = 0; k < vn; ++k) sum += flipped(x[k], m) < bound ? term(x[k]) : 0.f;
        } else if (kSum) {
#pragma unroll
            for (int k = 0; k < vn; ++k) sum += term(x[k]);
        }
    });
    if (done + static_cast<int>(threadIdx.x) < n) {
        const float x = capped(widen1(row[done + threadIdx.x]));
        look(done + threadIdx.x);
        if (kSum) sum += flipped(x, m) < bound ? term(x) : 0.f;
    }
    __syncthreads();
    if (sh.seen <= most) {
        for (int k = threadIdx.x; k < sh.seen * vn; k += T) look(seen[k / vn] + k % vn);
    } else {
#pragma unroll 1
        for (int i = threadIdx.x; i < done; i += T) look(i);
    }
    __syncthreads();
    int count = sh.count;
    // Whether the others' sum is that of the list and of `sum`: the list holds all others,
    // or one of them that reached the bound, beside which what is 0 in fp32 counts for nothing.
    bool listed = bound == -FLT_MAX || (sums && count > K);
    if (count > kList<T>) {
        count = pick_exactly<T, E>(sh, row, n, m, K);
        sum = 0.f;
        listed = false;
    }
    sort_by_value<T>(sh, count);
    if (!kSum || count < K) return count;
    if (!sums) sum = 0.f;
    ExpSum s{-INFINITY, 0.f};
    // Else terms below 2^-126 are missing: 2^24 of them are 2^-26 of a sum of 2^-76
    const bool some = __syncthreads_or(sum >= 0x1p-76f);
    if (some || listed) {
        // kb was rounded
        if (sum > 0.f) s = ExpSum{bound, sum * __builtin_amdgcn_exp2f(-fmaf(bound, c2, -kb))};
        for (int k = K + threadIdx.x; k < count; k += T)
            s = exp_join(s, ExpSum{value_of(rank_key(sh.list[k])), 1.f}, c2);
    } else {
        // all others lie so far below the bound that terms are lost there, or their sum was
        // not formed (logits beyond 2^24, more candidates than the list holds)
        s = sum_behind<T, E>(row, n, m, sh.list[K - 1], c2);
    }
    *others = block_exp_sum<T>(s, c2, sh.red);
    return count;
}

template <int T, bool kCaps, typename E>
__global__ __launch_bounds__(T, T >= 1024 ? 8 : 4) void top_logits_kernel(int n, int64_t ld,
                                                                          const E *__restrict__ x, ScoreMap m,
                                                                          double scale, float c2, int K,
                                                                          int32_t *__restrict__ idx,
                                                                          float *__restrict__ logit,
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

// One class from the top_k <= kMaxPicked first entries of each row: the candidates in
// order, their weights' sums over the block's threads (top_p, min_p), what is kept once
// more by index, and its sums. 131072 bf16 with top_k 50: 14.4 us, 7 of them the two passes;
// 512 such rows with top_k 1000 64 us, some 15 of them for order and draw.
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

template <int T, typename E> void launch_picked_t(const SampleJob &j, hipStream_t st) {
    const ScoreMap m{j.in.cap, j.in.flip};
    const DrawArgs a = draw_args(j);
    const dim3 grid(static_cast<unsigned>(j.in.B));
    const int n = static_cast<int>(j.in.N);
    const E *x = static_cast<const E *>(j.in.x);
    if (isfinite(j.in.cap))
        hipLaunchKernelGGL((sample_picked_kernel<T, true, E>), grid, dim3(T), 0, st, n, j.in.ld, x, m, a);
    else
        hipLaunchKernelGGL((sample_picked_kernel<T, false, E>), grid, dim3(T), 0, st, n, j.in.ld, x, m, a);
}
template <typename E> void launch_picked(const SampleJob &j, hipStream_t st) {
    if (j.in.N <= 512) launch_picked_t<64, E>(j, st);
    else if (j.in.N <= kShortRow && j.top_k <= 256) launch_picked_t<256, E>(j, st);
    else launch_picked_t<1024, E>(j, st);
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
    else if (n <= kShortRow) TOP(256);
    else TOP(1024);
#undef TOP
    return hipGetLastError();
}

}  // namespace

hipError_t launch_sample_picked(const SampleJob &j, hipStream_t st) {
    if (j.in.bf16) launch_picked<uint16_t>(j, st);
    else launch_picked<float>(j, st);
    return hipGetLastError();
}

hipError_t launch_top_logits(const TopJob &j, hipStream_t st) {
    if (j.in.B == 0) return hipSuccess;
    ProfScope prof("top_logits", st);
    return j.in.bf16 ? launch_top_t<uint16_t>(j, st) : launch_top_t<float>(j, st);
}

}  // namespace dstd
