// dstd_optim.hip -- what follows the gradients in a training step (gfx950):
// the global norm over a list of gradient tensors, clipping by it, and the
// AdamW update.
//
//   S = sum over all tensors of g^2,  norm = sqrt(S)
//   c = max_norm / norm where norm > max_norm, else 1
//   clip : out = c g
//   AdamW: m = b1 m + (1 - b1) c g,  v = b2 v + (1 - b2) (c g)^2,
//          w -= lr (m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps) + decay w)
//
// All three stream their arrays once and are bound by HBM. A list's tensors
// are cut into chunks of kOptChunk elements; a table in device memory gives
// each chunk its tensor, so that one launch covers any number of tensors of
// any sizes. The norm needs every gradient before the first is scaled: one
// launch sums the squares of a fixed set of chunks per block (partials), and
// the launch that follows adds the partials again in every block, in a fixed
// order, rather than in a launch of its own.
#include "dstd_internal.h"
#include "dstd_kernels.h"
#include "dstd_profile.h"

namespace dstd {

namespace {

constexpr int kOptThreads = 256;
constexpr int kOptGroups = static_cast<int>(kOptChunk) / (kOptThreads * 4);  // of 4 elements per thread

using f32x4 = float __attribute__((ext_vector_type(4)));
using u16x4 = uint16_t __attribute__((ext_vector_type(4)));
using bf16x4 = __bf16 __attribute__((ext_vector_type(4)));
// Tensors start anywhere: vectors are only as aligned as their elements (one
// 16- or 8-byte access all the same). Pointers that come out of a table are
// said to be global ones, or every access would be a flat one.
#define DSTD_GLOBAL __attribute__((address_space(1)))
using gf32 = DSTD_GLOBAL float;
using gu16 = DSTD_GLOBAL uint16_t;
using f32x4_any = f32x4 __attribute__((aligned(4)));
using u16x4_any = u16x4 __attribute__((aligned(2)));

__device__ __forceinline__ f32x4 widen(u16x4 h) {
    f32x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = bf16_to_f32(h[k]);
    return r;
}

// Four elements at p as fp32, or the first `left` of them and zeros.
__device__ __forceinline__ f32x4 load4(const gf32 *p, bool full, int left) {
    if (full) return *reinterpret_cast<const DSTD_GLOBAL f32x4_any *>(p);
    f32x4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (k < left) r[k] = p[k];
    return r;
}
__device__ __forceinline__ f32x4 load4(const gu16 *p, bool full, int left) {
    if (full) return widen(*reinterpret_cast<const DSTD_GLOBAL u16x4_any *>(p));
    u16x4 h = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (k < left) h[k] = p[k];
    return widen(h);
}

__device__ __forceinline__ void store4(gf32 *p, f32x4 v, bool full, int left) {
    if (full) {
        *reinterpret_cast<DSTD_GLOBAL f32x4_any *>(p) = v;
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (k < left) p[k] = v[k];
}
// rounded once, to nearest even
__device__ __forceinline__ void store4(gu16 *p, f32x4 v, bool full, int left) {
    const u16x4 h = __builtin_bit_cast(u16x4, __builtin_convertvector(v, bf16x4));
    if (full) {
        *reinterpret_cast<DSTD_GLOBAL u16x4_any *>(p) = h;
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (k < left) p[k] = h[k];
}

__device__ __forceinline__ gf32 *f32_at(void *p, int64_t start) { return (gf32 *)p + start; }
__device__ __forceinline__ gu16 *u16_at(void *p, int64_t start) { return (gu16 *)p + start; }

// Sum over the block, in a fixed order, to every thread. sh: one double per wave.
__device__ double block_sum(double v, double *sh) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if (threadIdx.x % kWave == 0) sh[threadIdx.x / kWave] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < kOptThreads / kWave; ++k) s += sh[k];
    return s;
}

// Squares are formed and added in 64 bits: the square of an fp32 value is
// exact there and neither overflows nor underflows.
template <typename T>
__device__ __forceinline__ double chunk_squares(const T *g, int count) {
    double s = 0.0;
    f32x4 x[kOptGroups];
#pragma unroll
    for (int i = 0; i < kOptGroups; ++i) {
        const int e = (i * kOptThreads + threadIdx.x) * 4;
        x[i] = (e < count) ? load4(g + e, e + 4 <= count, count - e) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int i = 0; i < kOptGroups; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) s = fma(static_cast<double>(x[i][k]), static_cast<double>(x[i][k]), s);
    return s;
}

// Blocks: part[block] = the squares of chunks block, block + gridDim.x, ...
// Block 0 also takes the step number of an AdamW step and its corrections
// 1 / (1 - beta^t): the update writes the number, so its other blocks must
// not read it.
__global__ __launch_bounds__(kOptThreads) void grad_squares_kernel(
    const OptTensor *__restrict__ ten, const OptChunk *__restrict__ chunks, int n_chunks,
    double *__restrict__ part, const int64_t *step, double beta1, double beta2,
    OptStep *__restrict__ at) {
    __shared__ double sh[kOptThreads / kWave];
    double s = 0.0;
    for (int k = blockIdx.x; k < n_chunks; k += gridDim.x) {
        const OptChunk c = chunks[k];
        const OptTensor &t = ten[c.tensor];
        if (t.types & kOptGradBf16)
            s += chunk_squares(u16_at(t.g, c.start), c.count);
        else
            s += chunk_squares(f32_at(t.g, c.start), c.count);
    }
    s = block_sum(s, sh);
    if (threadIdx.x == 0) {
        part[blockIdx.x] = s;
        if (step && blockIdx.x == 0) {
            const int64_t t = *step + 1;
            at->t = t;
            at->inv_c1 = static_cast<float>(1.0 / (1.0 - pow(beta1, static_cast<double>(t))));
            at->inv_c2 = static_cast<float>(1.0 / (1.0 - pow(beta2, static_cast<double>(t))));
        }
    }
}

// The norm and its clipping factor, in every thread of the block: from the
// partials, or as given. A norm that is not finite clips nothing (factor 1).
struct NormFactor {
    float norm, c;
    bool finite;
};
__device__ NormFactor norm_factor(const OptNorm &nm, double *sh) {
    double n = 0.0;
    if (nm.n_part >= 0) {
        double s = 0.0;
        for (int k = threadIdx.x; k < nm.n_part; k += kOptThreads) s += nm.part[k];
        n = sqrt(block_sum(s, sh));
    } else if (nm.norm) {
        n = static_cast<double>(*nm.norm);
    }
    NormFactor r;
    r.norm = static_cast<float>(n);
    r.finite = isfinite(r.norm);
    r.c = (r.finite && n > nm.max_norm) ? static_cast<float>(nm.max_norm / n) : 1.f;
    return r;
}

__global__ __launch_bounds__(kOptThreads) void grad_norm_kernel(OptNorm nm) {
    __shared__ double sh[kOptThreads / kWave];
    const NormFactor f = norm_factor(nm, sh);
    if (threadIdx.x == 0) *nm.norm = f.norm;
}

template <typename TI, typename TO>
__device__ __forceinline__ void scale_chunk(const TI *g, TO *out, int count, float c) {
    f32x4 x[kOptGroups];
#pragma unroll
    for (int i = 0; i < kOptGroups; ++i) {
        const int e = (i * kOptThreads + threadIdx.x) * 4;
        if (e < count) x[i] = load4(g + e, e + 4 <= count, count - e);
    }
#pragma unroll
    for (int i = 0; i < kOptGroups; ++i) {
        const int e = (i * kOptThreads + threadIdx.x) * 4;
        if (e < count) store4(out + e, x[i] * c, e + 4 <= count, count - e);
    }
}

__global__ __launch_bounds__(kOptThreads) void grad_clip_kernel(
    const OptTensor *__restrict__ ten, const OptChunk *__restrict__ chunks, int n_chunks,
    OptNorm nm) {
    __shared__ double sh[kOptThreads / kWave];
    const NormFactor f = norm_factor(nm, sh);
    if (nm.n_part >= 0 && nm.norm && blockIdx.x == 0 && threadIdx.x == 0) *nm.norm = f.norm;
    for (int k = blockIdx.x; k < n_chunks; k += gridDim.x) {
        const OptChunk ch = chunks[k];
        const OptTensor &t = ten[ch.tensor];
        if (f.c == 1.f && t.g == t.out) continue;  // in place, nothing to clip
        const bool gb = t.types & kOptGradBf16, ob = t.types & kOptOutBf16;
        gu16 *gh = u16_at(t.g, ch.start), *oh = u16_at(t.out, ch.start);
        gf32 *gf = f32_at(t.g, ch.start), *of = f32_at(t.out, ch.start);
        if (gb && ob) scale_chunk(gh, oh, ch.count, f.c);
        else if (gb) scale_chunk(gh, of, ch.count, f.c);
        else if (ob) scale_chunk(gf, oh, ch.count, f.c);
        else scale_chunk(gf, of, ch.count, f.c);
    }
}

// One chunk's update in fp32. WM: 0 = fp32 weights, 1 = bf16 weights (the
// update is added to the widened weight and rounded once), 2 = bf16 weights
// with an fp32 copy, which the update works on.
struct StepConst {
    float c, b1, b2, a1, a2, inv_c1, inv_c2, eps, lr, decay;
};
template <typename GT, int WM>
__device__ __forceinline__ void adamw_chunk(const OptTensor &t, int64_t start, int count,
                                            const StepConst &q) {
    const GT *g = (const GT *)t.g + start;
    gf32 *wf = f32_at(WM == 2 ? t.w32 : t.w, start), *m = f32_at(t.m, start), *v = f32_at(t.v, start);
    gu16 *wh = u16_at(t.w, start);
#pragma unroll
    for (int i = 0; i < kOptGroups; ++i) {
        const int e = (i * kOptThreads + threadIdx.x) * 4;
        if (e >= count) continue;
        const bool full = e + 4 <= count;
        const int left = count - e;
        f32x4 gx = load4(g + e, full, left);
        f32x4 wx = (WM == 1) ? load4(wh + e, full, left) : load4(wf + e, full, left);
        f32x4 mx = load4(m + e, full, left);
        f32x4 vx = load4(v + e, full, left);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float gk = gx[k] * q.c;
            const float mk = fmaf(q.b1, mx[k], q.a1 * gk);
            const float vk = fmaf(q.b2, vx[k], q.a2 * gk * gk);
            const float u = (mk * q.inv_c1) / (sqrtf(vk * q.inv_c2) + q.eps);
            mx[k] = mk;
            vx[k] = vk;
            wx[k] = wx[k] - q.lr * fmaf(q.decay, wx[k], u);
        }
        store4(m + e, mx, full, left);
        store4(v + e, vx, full, left);
        if (WM != 1) store4(wf + e, wx, full, left);
        if (WM != 0) store4(wh + e, wx, full, left);
    }
}

__global__ __launch_bounds__(kOptThreads) void adamw_kernel(
    const OptTensor *__restrict__ ten, const OptChunk *__restrict__ chunks, int n_chunks,
    OptNorm nm, OptAdamW hp, const float *__restrict__ lr, const OptStep *__restrict__ at,
    int64_t *step) {
    __shared__ double sh[kOptThreads / kWave];
    const NormFactor f = norm_factor(nm, sh);
    const bool first = blockIdx.x == 0 && threadIdx.x == 0;
    if (nm.n_part >= 0 && nm.norm && first) *nm.norm = f.norm;
    if (!f.finite) return;  // the step is skipped
    if (first) *step = at->t;
    StepConst q{f.c, hp.b1, hp.b2, hp.a1, hp.a2, at->inv_c1, at->inv_c2, hp.eps, 0.f, 0.f};
    const float rate = lr ? *lr : hp.lr;
    for (int k = blockIdx.x; k < n_chunks; k += gridDim.x) {
        const OptChunk ch = chunks[k];
        const OptTensor &t = ten[ch.tensor];
        q.lr = rate * t.lr_scale;
        q.decay = hp.decay * t.decay_scale;
        const int wm = (t.types & kOptWeightBf16) ? (t.w32 ? 2 : 1) : 0;
        if (t.types & kOptGradBf16) {
            if (wm == 0) adamw_chunk<gu16, 0>(t, ch.start, ch.count, q);
            else if (wm == 1) adamw_chunk<gu16, 1>(t, ch.start, ch.count, q);
            else adamw_chunk<gu16, 2>(t, ch.start, ch.count, q);
        } else {
            if (wm == 0) adamw_chunk<gf32, 0>(t, ch.start, ch.count, q);
            else if (wm == 1) adamw_chunk<gf32, 1>(t, ch.start, ch.count, q);
            else adamw_chunk<gf32, 2>(t, ch.start, ch.count, q);
        }
    }
}

// Writes a batch of a list's tensors, which come as kernel arguments (no host
// memory to keep alive, and capturable), and their chunks: one block a tensor.
__global__ __launch_bounds__(kOptThreads) void tensor_list_kernel(OptBatch b, OptTensor *ten,
                                                                  OptChunk *chunks) {
    const int k = blockIdx.x;
    if (threadIdx.x == 0) ten[b.first + k] = b.ten[k];
    const int64_t n = b.n[k], nc = (n + kOptChunk - 1) / kOptChunk;
    for (int64_t c = threadIdx.x; c < nc; c += kOptThreads) {
        const int64_t start = c * kOptChunk;
        const int64_t left = n - start;
        chunks[b.chunk0[k] + c] =
            OptChunk{b.first + k, static_cast<int>(left < kOptChunk ? left : kOptChunk), start};
    }
}

int opt_blocks(int n_chunks, int most) { return n_chunks < 1 ? 1 : n_chunks < most ? n_chunks : most; }

hipError_t launch_squares(const OptList &L, const OptNorm &nm, const int64_t *step, double beta1,
                          double beta2, OptStep *at, hipStream_t st) {
    const bool sums = nm.n_part >= 0;
    ProfScope prof(sums ? "grad_squares" : "adamw_count", st);
    hipLaunchKernelGGL(grad_squares_kernel, dim3(sums ? nm.n_part : 1), dim3(kOptThreads), 0, st,
                       L.ten, L.chunks, sums ? L.n_chunks : 0, nm.part, step, beta1, beta2, at);
    return hipGetLastError();
}

}  // namespace

int opt_norm_blocks(int n_chunks) { return opt_blocks(n_chunks, kOptMaxPart); }

hipError_t launch_tensor_list(const OptBatch &b, int count, OptTensor *ten, OptChunk *chunks,
                              hipStream_t st) {
    ProfScope prof("tensor_list", st);
    hipLaunchKernelGGL(tensor_list_kernel, dim3(static_cast<unsigned>(count)), dim3(kOptThreads), 0,
                       st, b, ten, chunks);
    return hipGetLastError();
}

hipError_t launch_grad_norm(const OptList &L, const OptNorm &nm, hipStream_t st) {
    hipError_t e = launch_squares(L, nm, nullptr, 0.0, 0.0, nullptr, st);
    if (e != hipSuccess) return e;
    ProfScope prof("grad_norm", st);
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(kOptThreads), 0, st, nm);
    return hipGetLastError();
}

hipError_t launch_grad_clip(const OptList &L, const OptNorm &nm, hipStream_t st) {
    if (nm.n_part >= 0) {
        hipError_t e = launch_squares(L, nm, nullptr, 0.0, 0.0, nullptr, st);
        if (e != hipSuccess) return e;
    }
    ProfScope prof("grad_clip", st);
    hipLaunchKernelGGL(grad_clip_kernel, dim3(opt_blocks(L.n_chunks, 2048)), dim3(kOptThreads), 0,
                       st, L.ten, L.chunks, L.n_chunks, nm);
    return hipGetLastError();
}

hipError_t launch_adamw(const OptList &L, const OptNorm &nm, const OptAdamW &hp, const float *lr,
                        int64_t *step, OptStep *at, hipStream_t st) {
    hipError_t e = launch_squares(L, nm, step, hp.beta1, hp.beta2, at, st);
    if (e != hipSuccess) return e;
    ProfScope prof("adamw", st);
    hipLaunchKernelGGL(adamw_kernel, dim3(opt_blocks(L.n_chunks, 2048)), dim3(kOptThreads), 0, st,
                       L.ten, L.chunks, L.n_chunks, nm, hp, lr, at, step);
    return hipGetLastError();
}

}  // namespace dstd
