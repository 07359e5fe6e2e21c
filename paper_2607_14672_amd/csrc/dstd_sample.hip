// dstd_sample.hip -- one class of every row drawn from its softmax (gfx950).
//
//   w_i = e^(z_i - z_max), z = scale x. Kept are the first top_k in the order of falling z
//   (ties by index), of these the shortest prefix with at least top_p of their sum, of
//   these w_i >= min_p; drawn is the first i, by index, where the sum of the kept w up to i
//   exceeds u times the sum of all kept.
//
// A draw turns on sums next to a border, so weights are formed in 64 bits and added as
// integers. Up to kMaxPicked kept entries are drawn from as a list (dstd_top.hip).
#include <string.h>

#include "dstd_profile.h"
#include "dstd_select.h"

namespace dstd {

namespace {

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

// One class of every row, a block each (threads as in dstd_top.hip): the largest score,
// then what top_k and top_p keep, then the draw: two readings of the row, and two or three
// more for each filter. Bound by its fp64 operations, some 30 an entry and reading of
// weights: 300 x 50021 without filters 39 us (the reads alone would take 20), 95 with top_p.
// kCount, kMass: with top_k (more than kMaxPicked), with top_p; a kernel for each, since what
// one of them needs in registers would be taken from the others' loops (with top_p 238 us in
// a kernel of both).
// Two blocks of 1024 threads a CU leave 64 registers a thread, and some of a row's are kept in
// scratch memory: fp32 9 (no filter), 22 (top_p), 12 (top_k), 98 (both), bf16 94 to 135. Against
// one block of 128, 300 x 50021 fp32: 39 and 41 us, 95 and 105, 83 and 97, 159 and 151; 1000 rows 85
// and 96, with top_p 199 and 231. bf16 rows, here only where the cap is no value that is counted
// below, would gain: 50 and 43 us, 125 and 109, 222 and 102, 318 and 186.
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

// ---------------------------------------------- rows of few distinct values --
// bf16 scores of a magnitude in [2^-24, 2^8) take 2 * 4096 values: how often each occurs
// says which are kept and what they weigh, with an exponential a value instead of one an
// entry. Zeros are counted apart; the few values nearer to 0 are listed one by one; what is
// larger with a goodness below 0 has to weigh nothing. Other rows are drawn from by their
// definition.
//
// Two passes, 64 KB of LDS a block (two a CU): the counts (an LDS atomic an entry), then,
// once the weights have taken the counts' place, their sums by parts of the row (a look-up
// an entry). 64 x 131072 with top_p 0.95: 29 us, 8 for the counts, 9 for the values (their
// exponentials twice, which is faster than held in registers: 38), 5 for the look-ups; an
// exponential an entry took 546. 512 rows: 62 us.
constexpr int kMags = 4096, kFirstMag = 0x3380, kValues = 2 * kMags;
using u32x4 = u32 __attribute__((ext_vector_type(4)));
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
    int done = vec_each<kRowAhead>(row, n, tid, T, [&](int i, RowVec<uint16_t>::type r) {
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
    done = lo + vec_each<kRowAhead>(row + lo, hi - lo, lane, kWave, [&](int i, RowVec<uint16_t>::type r) {
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

// kMost: the longest rows that T threads take.
template <int T, int kMost, typename E>
void launch_sample_rows(dim3 grid, hipStream_t st, int n, int64_t ld, const E *x, ScoreMap m, DrawArgs a) {
    const bool mass = a.top_p < 1.0;
#define SAMPLE(kCount, kMass) \
    hipLaunchKernelGGL((sample_kernel<T, kCount, kMass, E>), grid, dim3(T), 0, st, n, ld, x, m, a)
    // a top_k that comes here is more than kMaxPicked, and less than n
    if constexpr (kMost > kMaxPicked) {
        if (a.top_k > 0) {
            if (mass) SAMPLE(true, true);
            else SAMPLE(true, false);
            return;
        }
    }
    if (mass) SAMPLE(false, true);
    else SAMPLE(false, false);
#undef SAMPLE
}

template <typename E>
hipError_t launch_sample_t(const SampleJob &j, hipStream_t st) {
    const int n = static_cast<int>(j.in.N);
    const dim3 grid(static_cast<unsigned>(j.in.B));
    const ScoreMap m{j.in.cap, j.in.flip};
    const DrawArgs a = draw_args(j);
    const E *x = static_cast<const E *>(j.in.x);
    const bool filters = (a.top_k > 0 && a.top_k < n) || a.top_p < 1.0;
    // Counting values pays where a filter needs the order (bf16, top_p 0.9, counted and by
    // definition: 512 x 2500 21 and 26 us, 64 x 5000 14 and 26), else on long rows only (2000
    // x 15000 without filters 84 and 44).
    if constexpr (sizeof(E) == 2) {
        u32 cap;
        if (n > (filters ? 2048 : 16384) && cap_has_slot(j.in.cap, &cap)) {
            const OneSlot one{j.in.flip >> 16, cap};
            hipLaunchKernelGGL((sample_values_kernel<1024>), grid, dim3(1024), 0, st, n, j.in.ld, x, m, one, a);
            return hipGetLastError();
        }
    }
    // Threads a row: small blocks overlap each other's steps, large ones take a long row
    // sooner (fp32, 256 and 1024 threads: 2000 x 9000 34 and 44 us without filters, 78 and 114
    // with top_p; 64 x 15000 with top_p 35 and 25).
    if (n <= 512) launch_sample_rows<64, 512, E>(grid, st, n, j.in.ld, x, m, a);
    else if (n <= (filters ? 8192 : 16384)) launch_sample_rows<256, 16384, E>(grid, st, n, j.in.ld, x, m, a);
    else launch_sample_rows<1024, 1 << 24, E>(grid, st, n, j.in.ld, x, m, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const SampleJob &j, hipStream_t st) {
    if (j.in.B == 0) return hipSuccess;
    ProfScope prof("sample", st);
    if (j.top_k > 0 && j.top_k <= kMaxPicked) return launch_sample_picked(j, st);
    return j.in.bf16 ? launch_sample_t<uint16_t>(j, st) : launch_sample_t<float>(j, st);
}

}  // namespace dstd
