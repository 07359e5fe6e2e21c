// dstd_distill.hip -- distillation from a teacher's top logits (gfx950): the loss
// of a student's spike times t against them, and its gradient.
//
//   z_i = -t_i / tau;  S: the classes that the teacher names
//   p = softmax(logits of S, rest),  R = sum_{i not in S} e^z_i,  Z = R + sum_S e^z_i
//   L = w [ sum_S p_k (ln p_k - ln(e^z_k / Z)) + p_r (ln p_r - ln(R / Z)) ]
//   dL/dz_i = w (e^z_i / Z - p_i) in S,  w e^z_i (1 / Z - p_r / R) elsewhere
//
// R is summed over the others themselves, never as Z less the named classes: it
// keeps its digits where these hold nearly all of Z.
#include "dstd_answer.h"
#include "dstd_kernels.h"
#include "dstd_profile.h"

namespace dstd {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kEach = kKdMaxK / kWave;  // entries of the record a lane

using f32x4 = float __attribute__((ext_vector_type(4)));
using f32x4_any = f32x4 __attribute__((aligned(4)));

// The entries of a row's record as one wave holds them, entry k = lane + 64 j. An
// entry is one if its index is a class and its logit is finite.
template <typename L> struct Entries {
    int at[kEach];  // -1: no entry
    float l[kEach], y[kEach];
    bool fired[kEach];

    __device__ void load(const KdArgs &a, int64_t b, const L *logit, int lane) {
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int k = lane + kWave * j;
            at[j] = -1;
            l[j] = -INFINITY;
            if (k < a.K) {
                const int i = a.idx[b * a.K + k];
                l[j] = widen1(logit[b * a.K + k]);
                if (i >= 0 && i < a.N && isfinite(l[j])) at[j] = i;
            }
        }
        const float *row = a.t + b * a.ld_t;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const float x = at[j] >= 0 ? row[at[j]] : 0.f;
            fired[j] = isfinite(x);
            y[j] = -(fired[j] ? x : a.t_cap);
        }
    }
};

// What a row's gradient goes by: the teacher's logits (p, with the rest), the student's
// over the named classes (zs), and whether the record has an entry.
struct RecordSums {
    ExpSum p, zs;
    float rest;
    int any;
};

// The sums of a record by one wave. first[j]: no earlier entry names the class.
template <typename L>
__device__ RecordSums record_sums(const KdArgs &a, int64_t b, const Entries<L> &e, const bool (&first)[kEach]) {
    RecordSums r;
    r.rest = a.rest ? a.rest[b] : -INFINITY;
    if (!isfinite(r.rest)) r.rest = -INFINITY;
    r.p = ExpSum{r.rest, r.rest > -INFINITY && threadIdx.x % kWave == 0 ? 1.f : 0.f};
    r.zs = ExpSum{-INFINITY, 0.f};
    bool some = false;
#pragma unroll
    for (int j = 0; j < kEach; ++j)
        if (e.at[j] >= 0) {
            some = true;
            r.p = exp_join(r.p, ExpSum{e.l[j], 1.f}, kLog2e);
            if (first[j]) r.zs = exp_join(r.zs, ExpSum{e.y[j], 1.f}, a.c2);
        }
    r.p = block_exp_sum<kWave>(r.p, kLog2e, nullptr);
    r.zs = block_exp_sum<kWave>(r.zs, a.c2, nullptr);
    r.any = __any(some);
    return r;
}

// Which of the entries are the first of their class, where some class is named twice.
template <typename L> __device__ void first_of(const int *list, int K, const Entries<L> &e, bool (&first)[kEach]) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        first[j] = e.at[j] >= 0;
        const int k = threadIdx.x % kWave + kWave * j;
        for (int o = 0; first[j] && o < min(k, K); ++o) first[j] = list[o] != e.at[j];
    }
}

// Factors of a row's gradient, in z: e^((y - r.m) / tau) * other outside S, and
// e^((y - z.m) / tau) * one_z - p in S.
struct RowFactors {
    ExpSum r, z;
    float pr, one_z, other;
    __device__ RowFactors(const RecordSums &s, ExpSum rest, float c2) : r(rest), z(exp_join(rest, s.zs, c2)) {
        pr = s.rest > -INFINITY ? exp_of(s.rest - s.p.m, kLog2e) / s.p.s : 0.f;
        one_z = 1.f / z.s;
        const float qr = r.s * exp_of(r.m - z.m, c2) * one_z;
        other = r.s > 0.f ? (qr - pr) / r.s : 0.f;
    }
};

// The loss of a row, by one wave.
template <typename L>
__device__ void put_loss(const KdArgs &a, int64_t b, const Entries<L> &e, const RecordSums &s, const RowFactors &f) {
    // ln p_k = (l_k - p.m) - ln p.s, ln q_k = (y_k - z.m) / tau - ln z.s: a logarithm added
    // to a large maximum would lose its digits
    const float lp = logf(s.p.s), lz = logf(f.z.s);
    float term = 0.f;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        if (e.at[j] < 0) continue;
        const float p = exp_of(e.l[j] - s.p.m, kLog2e) / s.p.s;
        if (p > 0.f) term += p * (e.l[j] - s.p.m - lp - ((e.y[j] - f.z.m) * a.inv - lz));
    }
    if (threadIdx.x % kWave == 0 && f.pr > 0.f)
        term += f.pr * (s.rest - s.p.m - lp - ((f.r.m - f.z.m) * a.inv + logf(f.r.s) - lz));
    term = block_add<kWave>(term, nullptr);
    if (threadIdx.x % kWave == 0) {
        const float loss = s.any ? term * a.weight : 0.f;
        a.loss[1 + b] = loss;
        if (a.alone) a.loss[0] = loss;  // the total of one row
    }
}

// Gradient of the named classes in [lo, hi), by one wave, behind the others': there 0
// stands, or with accumulate what was there. list: the record's classes.
template <typename L>
__device__ void put_named(const KdArgs &a, int64_t b, const Entries<L> &e, const bool (&first)[kEach],
                          const RecordSums &s, const RowFactors &f, const int *list, const float *logits,
                          bool twice, int lo, int hi) {
    float *grad = a.grad + b * a.ld_g;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = e.at[j];
        if (!first[j] || i < lo || i >= hi || !e.fired[j]) continue;
        float p = exp_of(e.l[j] - s.p.m, kLog2e) / s.p.s;
        if (twice) {
            p = 0.f;
            for (int o = 0; o < a.K; ++o) p += list[o] == i ? exp_of(logits[o] - s.p.m, kLog2e) / s.p.s : 0.f;
        }
        const float g = -a.weight * a.inv * (exp_of(e.y[j] - f.z.m, a.c2) * f.one_z - p);
        grad[i] = a.accumulate ? grad[i] + g : g;
    }
}

// ------------------------------------------------------- one block a row --
// The row stays in registers, V vectors a thread: read once, its exponentials formed
// once, written once, while the first wave does the record. T and V by the row's length,
// blocks as small as hold it, since a CU's blocks overlap each other's steps (2000 x 5000:
// 27 us with 256 threads and 8 vectors, 40 with 512 and 8; 1000 x 20000: 51 with 512 and 16
// in 128 registers, 58 with 1024 and 8). 1024 x 65536: 128 us for the necessary 537 MB (4.2 TB/s); such
// rows fill a CU's registers, so that a block's 11 us of arithmetic are not hidden behind
// another's reads. Read twice by two launches of several blocks a row: 230 us.
template <int T, int V> struct KdShared {
    u32 bits[T * V / 8];
    u64 red[T / kWave + 1];
    int list[kKdMaxK];
    float logit[kKdMaxK];
    RecordSums sums;
    int twice;
};

template <int T, int V, typename L>
__global__ __launch_bounds__(T, V >= 16 ? 4 : 1) void distill_row_kernel(KdArgs a, const L *__restrict__ logit) {
    __shared__ KdShared<T, V> sh;
    const int64_t b = blockIdx.x;
    const int tid = threadIdx.x, lane = tid % kWave, n = a.N;
    const float *row = a.t + b * a.ld_t;
    f32x4 x[V];
    // vector v of the row is v = tid + T j; the last may be cut, what is behind it is taken
    // for silent
    int behind = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int i = (tid + T * j) * 4;
        if (i + 4 <= n) {
            x[j] = *reinterpret_cast<const f32x4_any *>(row + i);
        } else {
            behind += 4 - max(0, n - i);
#pragma unroll
            for (int k = 0; k < 4; ++k) x[j][k] = i + k < n ? row[i + k] : INFINITY;
        }
    }
    for (int k = tid; k < (n + 31) / 32; k += T) sh.bits[k] = 0;
    if (tid == 0) sh.twice = 0;
    Entries<L> e;
    bool first[kEach];
    if (tid < kWave) e.load(a, b, logit, lane);
    __syncthreads();
    if (tid < kWave) {
        bool twice = false;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            first[j] = e.at[j] >= 0;
            if (first[j]) twice |= atomicOr(&sh.bits[e.at[j] / 32], 1u << (e.at[j] % 32)) >> (e.at[j] % 32) & 1;
            sh.list[lane + kWave * j] = e.at[j];
            sh.logit[lane + kWave * j] = e.l[j];
        }
        if (__any(twice)) {
            if (lane == 0) sh.twice = 1;
            __builtin_amdgcn_wave_barrier();  // the list is this wave's own
            first_of(sh.list, a.K, e, first);
        }
        const RecordSums s = record_sums(a, b, e, first);
        if (lane == 0) sh.sums = s;
    }
    __syncthreads();
    // The others' largest y, their exponentials relative to it, which take the places of
    // the times, and their sum. Silent neurons are counted: each adds what t_cap adds, and
    // the 0 in its place is its gradient. So do the named classes' places hold 0.
    int silent = -behind;
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int v = tid + T * j;
        const u32 named = v * 4 < n ? sh.bits[v / 8] >> (v % 8 * 4) & 15u : 0u;
        if (named) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (named >> k & 1) {
                    x[j][k] = INFINITY;
                    --silent;
                }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bool fired = isfinite(x[j][k]);
            silent += !fired;
            x[j][k] = fired ? -x[j][k] : -INFINITY;
            top = fmaxf(top, x[j][k]);
        }
    }
    if (silent > 0) top = fmaxf(top, -a.t_cap);
    top = value_of(block_max<T>(key_of(top), sh.red));
    // 2^(c2 y - kb), off by the rounding of kb, half a binary order at most up to 2^24 (from
    // 2^31 on it may be more than fp32 holds); beyond by the difference itself
    const float ref = top > -INFINITY ? top : 0.f, kb = ref * a.c2;
    const bool fits = fabsf(kb) < 0x1p24f;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[j][k] = __builtin_amdgcn_exp2f(fits ? fmaf(x[j][k], a.c2, -kb) : (x[j][k] - ref) * a.c2);
            sum += x[j][k];
        }
    // what rounding kb took off; 2^-kb is what a silent neuron's term is relative to, too
    const float fix = fits ? __builtin_amdgcn_exp2f(fmaf(ref, -a.c2, kb)) : 1.f;
    if (silent > 0)
        sum += static_cast<float>(silent) *
               __builtin_amdgcn_exp2f(fits ? fmaf(-a.t_cap, a.c2, -kb) : (-a.t_cap - ref) * a.c2);
    sum = block_add<T>(sum, sh.red) * fix;
    const ExpSum r{top, top > -INFINITY ? sum : 0.f};
    const RecordSums s = sh.sums;
    const RowFactors f(s, r, a.c2);
    if (!a.grad) {
        if (tid < kWave) put_loss(a, b, e, s, f);
        return;
    }
    const float w = s.any ? -a.weight * a.inv * f.other * fix : 0.f;
    float *grad = a.grad + b * a.ld_g;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int i = (tid + T * j) * 4;
        const f32x4 g = x[j] * w;
        if (i + 4 <= n) {
            f32x4_any *o = reinterpret_cast<f32x4_any *>(grad + i);
            *o = a.accumulate ? *o + g : g;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + k < n) grad[i + k] = a.accumulate ? grad[i + k] + g[k] : g[k];
        }
    }
    if (tid < kWave) put_loss(a, b, e, s, f);
    __syncthreads();
    if (tid < kWave && s.any) put_named(a, b, e, first, s, f, sh.list, sh.logit, sh.twice != 0, 0, n);
}

// ---------------------------------------------------- several blocks a row --
// For rows that no block's registers hold, and for few rows: 1 x 131072 takes 15 us
// (the host's two launches), 256 x 131072 91 us (its 134 MB read twice, and written).
constexpr int kKdThreads = 256;
constexpr int kKdChunk = 8192;  // classes of a block

// Blocks [0, chunks): the sum over the chunk's classes that the record does not name.
// The last block of a row: the record's sums.
template <typename L>
__global__ __launch_bounds__(kKdThreads) void distill_rest_kernel(KdArgs a, const L *__restrict__ logit) {
    __shared__ u32 bits[kKdChunk / 32];
    __shared__ u64 red[kKdThreads / kWave + 1];
    __shared__ int list[kKdMaxK];
    const int64_t b = blockIdx.y;
    const int chunks = gridDim.x - 1, tid = threadIdx.x;
    float2 *part = a.part + b * kd_row_parts(chunks);
    if (static_cast<int>(blockIdx.x) == chunks) {
        Entries<L> e;
        if (tid < kWave) {
            e.load(a, b, logit, tid);
#pragma unroll
            for (int j = 0; j < kEach; ++j) list[tid + kWave * j] = e.at[j];
        }
        __syncthreads();
        if (tid >= kWave) return;
        bool first[kEach], twice = false;
        first_of(list, a.K, e, first);
#pragma unroll
        for (int j = 0; j < kEach; ++j) twice |= e.at[j] >= 0 && !first[j];
        twice = __any(twice);
        const RecordSums s = record_sums(a, b, e, first);
        if (tid == 0) {
            part[chunks] = make_float2(s.p.m, s.p.s);
            part[chunks + 1] = make_float2(s.zs.m, s.zs.s);
            part[chunks + 2] = make_float2(s.rest, s.any ? (twice ? 2.f : 1.f) : 0.f);
        }
        return;
    }
    const int lo = blockIdx.x * kKdChunk, count = min(kKdChunk, a.N - lo);
    const float *row = a.t + b * a.ld_t + lo;
    for (int k = tid; k < (count + 31) / 32; k += kKdThreads) bits[k] = 0;
    __syncthreads();
    for (int k = tid; k < a.K; k += kKdThreads) {
        const int i = a.idx[b * a.K + k] - lo;
        if (i >= 0 && i < count && isfinite(widen1(logit[b * a.K + k]))) atomicOr(&bits[i / 32], 1u << (i % 32));
    }
    __syncthreads();
    ExpSum s{-INFINITY, 0.f};
    row_each<kRowAhead>(row, count, tid, kKdThreads, [&](int i, float x) {
        if (bits[i / 32] >> (i % 32) & 1) return;
        const float y = -(isfinite(x) ? x : a.t_cap);
        if (y > s.m) {
            s.s *= exp_of(s.m - y, a.c2);
            s.m = y;
        }
        s.s += exp_of(y - s.m, a.c2);
    });
    s = block_exp_sum<kKdThreads>(s, a.c2, red);
    if (tid == 0) part[blockIdx.x] = make_float2(s.m, s.s);
}

template <typename L>
__global__ __launch_bounds__(kKdThreads) void distill_grad_kernel(KdArgs a, const L *__restrict__ logit) {
    __shared__ u64 red[kKdThreads / kWave + 1];
    __shared__ int list[kKdMaxK];
    __shared__ float logits[kKdMaxK];
    const int64_t b = blockIdx.y;
    const int chunks = gridDim.x, tid = threadIdx.x;
    const int lo = blockIdx.x * kKdChunk, count = min(kKdChunk, a.N - lo);
    const float *row = a.t + b * a.ld_t + lo;
    const float2 *part = a.part + b * kd_row_parts(chunks);
    ExpSum r{-INFINITY, 0.f};
    for (int c = tid; c < chunks; c += kKdThreads) r = exp_join(r, ExpSum{part[c].x, part[c].y}, a.c2);
    r = block_exp_sum<kKdThreads>(r, a.c2, red);
    const float2 sp = part[chunks], sz = part[chunks + 1], sr = part[chunks + 2];
    const RecordSums s{ExpSum{sp.x, sp.y}, ExpSum{sz.x, sz.y}, sr.x, sr.y > 0.f};
    const RowFactors f(s, r, a.c2);
    Entries<L> e;
    if (tid < kWave) {
        e.load(a, b, logit, tid);
        if (blockIdx.x == 0) put_loss(a, b, e, s, f);
    }
    if (!a.grad) return;
    float *grad = a.grad + b * a.ld_g + lo;
    const float w = s.any ? -a.weight * a.inv * f.other : 0.f;
    // the named classes among these get their own behind: with accumulate their old
    // value is kept till then
    float old[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) old[j] = 0.f;
    if (tid < kWave && a.accumulate)
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (e.at[j] >= lo && e.at[j] < lo + count) old[j] = grad[e.at[j] - lo];
    __syncthreads();
    row_each<kRowAhead>(row, count, tid, kKdThreads, [&](int i, float x) {
        const float g = isfinite(x) ? exp_of(fminf(-x - f.r.m, 0.f), a.c2) * w : 0.f;
        grad[i] = a.accumulate ? grad[i] + g : g;
    });
    if (tid < kWave)
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            list[tid + kWave * j] = e.at[j];
            logits[tid + kWave * j] = e.l[j];
        }
    __syncthreads();
    if (tid >= kWave) return;
    const bool twice = sr.y > 1.f;
    bool first[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) first[j] = e.at[j] >= 0;
    if (twice) first_of(list, a.K, e, first);
#pragma unroll
    for (int j = 0; j < kEach; ++j)
        if (first[j] && e.at[j] >= lo && e.at[j] < lo + count) grad[e.at[j] - lo] = old[j];
    if (s.any) put_named(a, b, e, first, s, f, list, logits, twice, lo, lo + count);
}

template <int T, int V, typename L> void launch_row(const KdArgs &a, int64_t B, const L *logit, hipStream_t st) {
    hipLaunchKernelGGL((distill_row_kernel<T, V, L>), dim3(static_cast<unsigned>(B)), dim3(T), 0, st, a, logit);
}

// Rows that no block holds, and few of which would leave most CUs idle: 8 x 65536 takes
// 18 us in chunks and 25 in a block each, 77 x 50021 31 and 25, 32 x 16384 20 and 18.
bool in_chunks(int64_t B, int64_t N) { return N > 65536 || (B < 32 && N > 8192); }

template <typename L> void launch_t(const KdArgs &a, int64_t B, const L *logit, hipStream_t st) {
    const int n = a.N;
    if (in_chunks(B, n)) {
        const int chunks = (n + kKdChunk - 1) / kKdChunk;
        hipLaunchKernelGGL((distill_rest_kernel<L>), dim3(chunks + 1, static_cast<unsigned>(B)), dim3(kKdThreads), 0,
                           st, a, logit);
        hipLaunchKernelGGL((distill_grad_kernel<L>), dim3(chunks, static_cast<unsigned>(B)), dim3(kKdThreads), 0, st,
                           a, logit);
    } else if (n <= 256) {
        launch_row<64, 1>(a, B, logit, st);
    } else if (n <= 1024) {
        launch_row<64, 4>(a, B, logit, st);
    } else if (n <= 4096) {
        launch_row<256, 4>(a, B, logit, st);
    } else if (n <= 8192) {
        launch_row<256, 8>(a, B, logit, st);
    } else if (n <= 16384) {
        launch_row<256, 16>(a, B, logit, st);
    } else if (n <= 32768) {
        launch_row<512, 16>(a, B, logit, st);
    } else {
        launch_row<1024, 16>(a, B, logit, st);
    }
}

}  // namespace

int64_t distill_parts(int64_t B, int64_t N) {
    return in_chunks(B, N) ? kd_row_parts((N + kKdChunk - 1) / kKdChunk) : 0;
}

hipError_t launch_distill(const KdArgs &args, int64_t B, const void *logit, bool bf16, hipStream_t st) {
    ProfScope prof("distill", st);
    KdArgs a = args;
    a.alone = B == 1;  // a launch less: 10.2 us a call instead of 13.2
    if (B > 0) {
        if (bf16) launch_t(a, B, static_cast<const uint16_t *>(logit), st);
        else launch_t(a, B, static_cast<const float *>(logit), st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return a.alone ? hipSuccess : launch_loss_total(B, a.loss, st);
}

}  // namespace dstd
