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

constexpr int kKdThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kKdChunk = 8192;  // classes of a block

// Bits of the classes [lo, lo + count) that a row's record names. An entry is one
// if its index is a class and its logit is finite.
template <typename L>
__device__ __forceinline__ bool named(const int32_t *idx, const L *logit, int k, int N, int *i, float *l) {
    *i = idx[k];
    *l = widen1(logit[k]);
    return *i >= 0 && *i < N && isfinite(*l);
}

template <typename L>
__device__ void mark(u32 *bits, int lo, int count, const int32_t *idx, const L *logit, int K, int N) {
    for (int k = threadIdx.x; k < (count + 31) / 32; k += kKdThreads) bits[k] = 0;
    __syncthreads();
    for (int k = threadIdx.x; k < K; k += kKdThreads) {
        int i;
        float l;
        if (named(idx, logit, k, N, &i, &l) && i >= lo && i < lo + count)
            atomicOr(&bits[(i - lo) / 32], 1u << ((i - lo) % 32));
    }
    __syncthreads();
}
__device__ __forceinline__ bool marked(const u32 *bits, int i) { return bits[i / 32] >> (i % 32) & 1; }

// part[b][chunk]: the sum over the chunk's classes that the record does not name
template <typename L>
__global__ __launch_bounds__(kKdThreads) void distill_rest_kernel(KdArgs a, const L *__restrict__ logit) {
    __shared__ u32 bits[kKdChunk / 32];
    __shared__ u64 red[kKdThreads / kWave + 1];
    const int64_t b = blockIdx.y;
    const int lo = blockIdx.x * kKdChunk, count = min(kKdChunk, a.N - lo);
    const float *row = a.t + b * a.ld_t + lo;
    mark(bits, lo, count, a.idx + b * a.K, logit + b * a.K, a.K, a.N);
    ExpSum s{-INFINITY, 0.f};
    row_each<kRowAhead>(row, count, threadIdx.x, kKdThreads, [&](int i, float x) {
        if (marked(bits, i)) return;
        const float y = -(isfinite(x) ? x : a.t_cap);
        if (y > s.m) {
            s.s *= exp_of(s.m - y, a.c2);
            s.m = y;
        }
        s.s += exp_of(y - s.m, a.c2);
    });
    s = block_exp_sum<kKdThreads>(s, a.c2, red);
    if (threadIdx.x == 0) a.part[b * gridDim.x + blockIdx.x] = make_float2(s.m, s.s);
}

template <typename L>
__global__ __launch_bounds__(kKdThreads) void distill_grad_kernel(KdArgs a, const L *__restrict__ logit_of) {
    __shared__ u32 bits[kKdChunk / 32];
    __shared__ u64 red[kKdThreads / kWave + 1];
    __shared__ int at[kKdMaxK];
    __shared__ float prob[kKdMaxK];
    const int64_t b = blockIdx.y;
    const int lo = blockIdx.x * kKdChunk, count = min(kKdChunk, a.N - lo);
    const float *row = a.t + b * a.ld_t;
    const int32_t *idx = a.idx + b * a.K;
    const L *logit = logit_of + b * a.K;
    mark(bits, lo, count, idx, logit, a.K, a.N);
    // the teacher
    float rest = a.rest ? a.rest[b] : -INFINITY;
    if (!isfinite(rest)) rest = -INFINITY;
    ExpSum p{rest, rest > -INFINITY && threadIdx.x == 0 ? 1.f : 0.f};
    u64 some = 0;
    for (int k = threadIdx.x; k < a.K; k += kKdThreads) {
        int i;
        float l;
        const bool is = named(idx, logit, k, a.N, &i, &l);
        at[k] = is ? i : -1;
        if (is) {
            p = exp_join(p, ExpSum{l, 1.f}, kLog2e);
            some = 1;
        }
    }
    p = block_exp_sum<kKdThreads>(p, kLog2e, red);
    const bool any = block_max<kKdThreads>(some, red) != 0;
    // the student
    ExpSum r{-INFINITY, 0.f};
    for (int c = threadIdx.x; c < static_cast<int>(gridDim.x); c += kKdThreads) {
        const float2 v = a.part[b * gridDim.x + c];
        r = exp_join(r, ExpSum{v.x, v.y}, a.c2);
    }
    r = block_exp_sum<kKdThreads>(r, a.c2, red);
    ExpSum z = threadIdx.x == 0 ? r : ExpSum{-INFINITY, 0.f};
    for (int k = threadIdx.x; k < a.K; k += kKdThreads) {
        const int i = at[k];
        if (i < 0) continue;
        const float l = widen1(logit[k]);
        prob[k] = exp_of(l - p.m, kLog2e) / p.s;
        bool first = true;
        for (int o = 0; o < k; ++o) first = first && at[o] != i;
        const float x = row[i];
        if (first) z = exp_join(z, ExpSum{-(isfinite(x) ? x : a.t_cap), 1.f}, a.c2);
    }
    z = block_exp_sum<kKdThreads>(z, a.c2, red);
    const float logp0 = p.m + logf(p.s);
    const float pr = rest > -INFINITY ? exp_of(rest - p.m, kLog2e) / p.s : 0.f;
    if (blockIdx.x == 0) {
        // ln q_k = (y_k - z.m) / tau - ln z.s
        float term = 0.f;
        const float lz = logf(z.s);
        for (int k = threadIdx.x; k < a.K; k += kKdThreads) {
            if (at[k] < 0 || !(prob[k] > 0.f)) continue;
            const float x = row[at[k]];
            const float lq = (-(isfinite(x) ? x : a.t_cap) - z.m) * a.inv - lz;
            term += prob[k] * (widen1(logit[k]) - logp0 - lq);
        }
        if (threadIdx.x == 0 && pr > 0.f) term += pr * (rest - logp0 - ((r.m - z.m) * a.inv + logf(r.s) - lz));
#pragma unroll
        for (int o = kWave / 2; o > 0; o >>= 1) term += __shfl_xor(term, o);
        float *fred = reinterpret_cast<float *>(red);
        __syncthreads();
        if (threadIdx.x % kWave == 0) fred[threadIdx.x / kWave] = term;
        __syncthreads();
        term = 0.f;
        for (int k = 0; k < kKdThreads / kWave; ++k) term += fred[k];
        if (threadIdx.x == 0) a.loss[1 + b] = any ? term * a.weight : 0.f;
    }
    if (!a.grad) return;
    float *grad = a.grad + b * a.ld_g;
    const float w = -a.weight * a.inv;
    // e^z / Z = e^(z - z.m) / z.s; others: times 1 - p_r Z / R = (q_r - p_r) / q_r
    const float one_z = 1.f / z.s;
    const float qr = r.s * exp_of(r.m - z.m, a.c2) * one_z;
    const float other = r.s > 0.f ? (qr - pr) / r.s : 0.f;
    __syncthreads();
    row_each<kRowAhead>(row + lo, count, threadIdx.x, kKdThreads, [&](int i, float x) {
        float g = 0.f;
        if (isfinite(x) && any) {
            if (!marked(bits, i)) {
                g = exp_of(-x - r.m, a.c2) * other;
            } else {
                float pk = 0.f;
                for (int k = 0; k < a.K; ++k) pk += at[k] == lo + i ? prob[k] : 0.f;
                g = exp_of(-x - z.m, a.c2) * one_z - pk;
            }
            g *= w;
        }
        float *o = grad + lo + i;
        if (a.accumulate) g += *o;
        *o = g;
    });
}

template <typename L> void launch_t(const KdArgs &a, const L *logit, dim3 grid, hipStream_t st) {
    hipLaunchKernelGGL((distill_rest_kernel<L>), grid, dim3(kKdThreads), 0, st, a, logit);
    hipLaunchKernelGGL((distill_grad_kernel<L>), grid, dim3(kKdThreads), 0, st, a, logit);
}

}  // namespace

int64_t distill_parts(int64_t N) { return (N + kKdChunk - 1) / kKdChunk; }

hipError_t launch_distill(const KdArgs &a, int64_t B, const void *logit, bool bf16, hipStream_t st) {
    ProfScope prof("distill", st);
    if (B > 0) {
        const dim3 grid(static_cast<unsigned>(distill_parts(a.N)), static_cast<unsigned>(B));
        if (bf16) launch_t(a, static_cast<const uint16_t *>(logit), grid, st);
        else launch_t(a, static_cast<const float *>(logit), grid, st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return launch_loss_total(B, a.loss, st);
}

}  // namespace dstd
