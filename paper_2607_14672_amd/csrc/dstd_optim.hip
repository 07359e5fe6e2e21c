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
// All three stream their arrays once and are bound by HBM: norm of 201 M fp32
// gradients 122 us (6.6 TB/s), clip of 67 M bf16 gradients into fp32 84 us,
// clipped step of 201 M fp32 weights 1030 us (6.0 TB/s with the gradients
// counted twice; the update alone 6.2, as a streamed copy by the same code).
//
// A list's tensors are cut into chunks of kOptChunk elements; a table of the
// chunks in device memory lets one launch cover any number of tensors of any
// sizes. The norm needs every gradient before the first is scaled: one launch
// sums the squares of a fixed set of chunks per block (partials), and the
// launch that follows adds the partials again in every block, in a fixed
// order. A thread's first partial is read while the block's chunk is on its
// way; the others (four a thread at most in a clip, two in a step), the step's
// constants and the learning rate are read one after the other behind it, which
// is what launches of a few us wait for (grad_norm_kernel, which does nothing
// else: 1.7 us for 106 partials, 4.4 for 1024). A launch of its own for the
// partials gains nothing (201 M weights: 1075 us with it, 1065 without, at that
// step).
#include <float.h>

#include "dstd_internal.h"
#include "dstd_kernels.h"
#include "dstd_profile.h"

namespace dstd {

namespace {

// Threads of a block, and so 4-element vectors of a chunk per thread. The
// update has up to seven arrays on the way: with fewer vectors of each per
// thread its registers leave more waves (clipped step of 201 M weights 1057 us
// with 256 threads, 1030 with 512, 1034 with 1024; of 2.4 M 17.8, 16.8 and
// 18.9). The norm of 201 M gradients takes 122 us with 256 threads, 124 with 512.
constexpr int kOptThreads = 256;
constexpr int kOptBlocks = 2048;  // of kOptThreads: all waves that 256 CUs hold
constexpr int kStepThreads = 512;
// Lists of up to so many chunks take one launch of one block: a pass is then
// bound by what the host spends on a launch (3.6 us), and two launches cost
// 7.6 us (an AdamW step 8.5) whatever such a list holds. One block takes 4.1 us
// for the norm of 1 chunk, 6.3 for 20 (one round of reads) and 8.4 for 24;
// clipping 4.3 us for 1, 7.2 for 8, 8.0 for 10; a step 6.1 us for 1, 8.1 for 3,
// 9.4 for 4.
constexpr int kSoloThreads = 1024;
constexpr int kSoloNormChunks = 20, kSoloClipChunks = 8, kSoloStepChunks = 3;
template <int kThreads> constexpr int kVecs = static_cast<int>(kOptChunk) / (kThreads * 4);
constexpr int kOptGroups = kVecs<kOptThreads>;

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
__device__ __forceinline__ f32x4 widen(f32x4 v) { return v; }
template <typename T> struct Vec4;  // four elements of a type
template <> struct Vec4<gf32> { using type = f32x4; using any = DSTD_GLOBAL f32x4_any; };
template <> struct Vec4<gu16> { using type = u16x4; using any = DSTD_GLOBAL u16x4_any; };

// Four elements at p. NT: marked as an access that nothing repeats soon.
template <bool NT, typename T>
__device__ __forceinline__ typename Vec4<T>::type load4(const T *p) {
    using V = const typename Vec4<T>::any;
    return NT ? __builtin_nontemporal_load((V *)p) : *(V *)p;
}
template <bool NT> __device__ __forceinline__ void store4(gf32 *p, f32x4 v) {
    if (NT) __builtin_nontemporal_store(v, (DSTD_GLOBAL f32x4_any *)p);
    else *(DSTD_GLOBAL f32x4_any *)p = v;
}
// rounded once, to nearest even
template <bool NT> __device__ __forceinline__ void store4(gu16 *p, f32x4 v) {
    const u16x4 h = __builtin_bit_cast(u16x4, __builtin_convertvector(v, bf16x4));
    if (NT) __builtin_nontemporal_store(h, (DSTD_GLOBAL u16x4_any *)p);
    else *(DSTD_GLOBAL u16x4_any *)p = h;
}
__device__ __forceinline__ float load1(const gf32 *p) { return *p; }
__device__ __forceinline__ float load1(const gu16 *p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void store1(gf32 *p, float v) { *p = v; }
__device__ __forceinline__ void store1(gu16 *p, float v) {
    *p = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
}

// Sum over the block, in a fixed order, to every thread. sh: one double per wave.
template <int kThreads> __device__ double block_sum(double v, double *sh) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if (threadIdx.x % kWave == 0) sh[threadIdx.x / kWave] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < kThreads / kWave; ++k) s += sh[k];
    return s;
}

// Squares are formed and added in 64 bits: the square of an fp32 value is
// exact there and neither overflows nor underflows.
__device__ __forceinline__ double add_square(double s, float x) {
    const double y = x;
    return fma(y, y, s);
}

// A chunk's elements: n4 vectors of four from its first whole line on, and at
// most kOptAlign + 2 single ones before and behind them, the one of thread tid
// at `one`, if it is below `count`.
struct Span {
    int lead, n4, one, count;
};
__device__ __forceinline__ Span span_of(int count, int lead, int tid) {
    Span p;
    p.lead = lead;
    p.n4 = (count - lead) / 4;
    p.one = tid < lead ? tid : p.n4 * 4 + tid;
    p.count = count;
    return p;
}

// A thread's vectors of four elements of a gradient chunk, zeros past the last
// whole one. As read: they are widened where they are used, for a conversion
// next to the loads would wait for them before the next chunk's are issued.
template <typename T> struct Share {
    typename Vec4<T>::type x[kOptGroups];
};
template <bool NT, typename T>
__device__ __forceinline__ void read_share(Share<T> &r, const T *g, const Span &p, int tid) {
#pragma unroll
    for (int i = 0; i < kOptGroups; ++i) {
        r.x[i] = typename Vec4<T>::type{0, 0, 0, 0};
        if (i * kOptThreads + tid < p.n4)
            r.x[i] = load4<NT>(g + p.lead + (i * kOptThreads + tid) * 4);
    }
}
template <typename T> __device__ __forceinline__ double add_share(double s, const Share<T> &r) {
#pragma unroll
    for (int i = 0; i < kOptGroups; ++i) {
        const f32x4 y = widen(r.x[i]);
#pragma unroll
        for (int k = 0; k < 4; ++k) s = add_square(s, y[k]);
    }
    return s;
}
// the single elements
template <typename T>
__device__ __forceinline__ double add_rest(double s, const T *g, const Span &p) {
    if (p.n4 * 4 < p.count && p.one < p.count) s = add_square(s, load1(g + p.one));
    return s;
}

// The gradient of a chunk, if it is of type T; count 0 else and past the end.
template <typename T> struct ChunkAt {
    const T *g;
    int count, lead;
};
template <typename T>
__device__ __forceinline__ ChunkAt<T> chunk_at(const OptChunk *chunks, int64_t k, int64_t end) {
    constexpr uint32_t type = sizeof(T) == 2 ? kOptGradBf16 : 0;
    ChunkAt<T> a{nullptr, 0, 0};
    if (k < end) {
        const OptChunk &c = chunks[k];
        a.g = (const T *)c.g;
        if ((c.types & kOptGradBf16) == type) {
            a.count = c.count;
            a.lead = c.lead;
        }
    }
    return a;
}

// The squares of the chunks first, first + by, ... of type T in [lo, end), by
// the kOptThreads threads `tid`: kAtOnce of them at a time, the places of the
// next looked up while these are read.
template <int kAtOnce, bool NT, typename T>
__device__ double range_squares(const OptChunk *chunks, int64_t lo, int64_t end, int first, int by,
                                int tid) {
    double s = 0.0;
    ChunkAt<T> a[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j)
        a[j] = chunk_at<T>(chunks, lo + first + static_cast<int64_t>(j) * by, end);
    for (int64_t k = lo + first; k < end; k += static_cast<int64_t>(kAtOnce) * by) {
        Share<T> r[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
            read_share<NT>(r[j], a[j].g, span_of(a[j].count, a[j].lead, tid), tid);
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
            s = add_rest(s, a[j].g, span_of(a[j].count, a[j].lead, tid));
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
            a[j] = chunk_at<T>(chunks, k + static_cast<int64_t>(kAtOnce + j) * by, end);
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) s = add_share(s, r[j]);
    }
    return s;
}

__device__ OptStep step_at(const int64_t *step, double beta1, double beta2) {
    OptStep r;
    r.t = *step + 1;
    r.inv_c1 = static_cast<float>(1.0 / (1.0 - pow(beta1, static_cast<double>(r.t))));
    r.inv_c2 = static_cast<float>(1.0 / (1.0 - pow(beta2, static_cast<double>(r.t))));
    return r;
}

// Blocks: part[block] = the squares of every gridDim.x-th chunk. The first
// n_stream chunks are read without being kept in the caches, so that the last
// ones, which the launch that scales the gradients reads first, are still
// there.
// Block 0 also takes the step number of an AdamW step and its corrections
// 1 / (1 - beta^t): the update writes the number, so its other blocks must
// not read it.
__global__ __launch_bounds__(kOptThreads) void grad_squares_kernel(
    const OptChunk *__restrict__ chunks, int n_chunks, int n_stream, uint32_t types,
    double *__restrict__ part, const int64_t *step, double beta1, double beta2,
    OptStep *__restrict__ at) {
    __shared__ double sh[kOptThreads / kWave];
    double s = 0.0;
    const int b = blockIdx.x, by = gridDim.x, tid = threadIdx.x;
    // 32 registers of gradients on the way
    if (types & kOptListF32) {
        s += range_squares<2, true, gf32>(chunks, 0, n_stream, b, by, tid);
        s += range_squares<2, false, gf32>(chunks, n_stream, n_chunks, b, by, tid);
    }
    if (types & kOptListBf16) {
        s += range_squares<4, true, gu16>(chunks, 0, n_stream, b, by, tid);
        s += range_squares<4, false, gu16>(chunks, n_stream, n_chunks, b, by, tid);
    }
    s = block_sum<kOptThreads>(s, sh);
    if (threadIdx.x == 0) {
        part[blockIdx.x] = s;
        if (step && blockIdx.x == 0) *at = step_at(step, beta1, beta2);
    }
}

// The norm and its clipping factor, in every thread of the block: from the
// partials, or as given. A norm that is not finite clips nothing (factor 1).
// The norm of finite gradients is finite in 64 bits; where it leaves fp32 it
// counts as finite if max_norm is a bound in fp32, which it is then clipped to.
// The factor is c c2: max_norm / norm and 1, or where that is no normal fp32
// number, 2^126 times it and 2^-126. So it keeps its 24 bits (down to 2^-252),
// which gradients of 1e35 clipped to a norm of 1e-3 would lose to a factor of
// 4e-41; x c cannot overflow, and the product with c2 is exact or the one
// rounding of a subnormal result.
struct NormFactor {
    float norm, c, c2;
    bool finite;
    __device__ bool one() const { return c == 1.f && c2 == 1.f; }
};
__device__ __forceinline__ float scaled(float x, const NormFactor &f) { return x * f.c * f.c2; }
__device__ NormFactor factor_of(double n, double max_norm) {
    NormFactor r;
    r.norm = static_cast<float>(n);
    r.finite = isfinite(r.norm);
    // what is rare goes by branches that are the same in every lane
    if (__builtin_amdgcn_readfirstlane(!r.finite))
        r.finite = isfinite(n) && max_norm <= FLT_MAX;
    r.c = (r.finite && n > max_norm) ? static_cast<float>(max_norm / n) : 1.f;
    r.c2 = 1.f;
    if (__builtin_amdgcn_readfirstlane(r.c < 0x1p-126f)) {
        r.c = static_cast<float>(max_norm / n * 0x1p126);
        r.c2 = 0x1p-126f;
    }
    return r;
}
template <int kThreads> __device__ NormFactor norm_factor(const OptNorm &nm, double *sh) {
    double n = 0.0;
    if (nm.n_part >= 0) {
        double s = 0.0;
        for (int k = threadIdx.x; k < nm.n_part; k += kThreads) s += nm.part[k];
        n = sqrt(block_sum<kThreads>(s, sh));
    } else if (nm.norm) {
        n = static_cast<double>(*nm.norm);
    }
    return factor_of(n, nm.max_norm);
}

__global__ __launch_bounds__(kOptThreads) void grad_norm_kernel(OptNorm nm) {
    __shared__ double sh[kOptThreads / kWave];
    const NormFactor f = norm_factor<kOptThreads>(nm, sh);
    if (threadIdx.x == 0) *nm.norm = f.norm;
}

// One chunk by kOptThreads threads. The factor is asked for once the chunk's
// reads are on their way.
template <bool NT, typename TI, typename TO, typename F>
__device__ __forceinline__ void clip_values(const TI *g, TO *out, const Span &p, int tid,
                                            const F &factor) {
    typename Vec4<TI>::type x[kOptGroups];
#pragma unroll
    for (int i = 0; i < kOptGroups; ++i)
        if (i * kOptThreads + tid < p.n4) x[i] = load4<NT>(g + p.lead + (i * kOptThreads + tid) * 4);
    const float x1 = p.one < p.count ? load1(g + p.one) : 0.f;
    const NormFactor f = factor();
#pragma unroll
    for (int i = 0; i < kOptGroups; ++i)
        if (i * kOptThreads + tid < p.n4)
            store4<NT>(out + p.lead + (i * kOptThreads + tid) * 4, widen(x[i]) * f.c * f.c2);
    if (p.one < p.count) store1(out + p.one, scaled(x1, f));
}

template <bool NT, typename F>
__device__ __forceinline__ void clip_chunk(const OptChunk &t, int tid, const F &factor) {
    if (t.g == t.out && factor().one()) return;  // in place, nothing to clip
    const bool gb = t.types & kOptGradBf16, ob = t.types & kOptOutBf16;
    gu16 *gh = (gu16 *)t.g, *oh = (gu16 *)t.out;
    gf32 *gf = (gf32 *)t.g, *of = (gf32 *)t.out;
    const Span p = span_of(t.count, t.lead, tid);
    if (gb && ob) clip_values<NT>(gh, oh, p, tid, factor);
    else if (gb) clip_values<NT>(gh, of, p, tid, factor);
    else if (ob) clip_values<NT>(gf, oh, p, tid, factor);
    else clip_values<NT>(gf, of, p, tid, factor);
}

// From the last chunk to the first: the norm's launch has read the last ones
// most recently. One chunk a block; a list that is clipped in place has fewer
// blocks, which ask for the factor first and end where there is nothing to
// clip, as in most steps (201 M gradients: 120 us with the norm; 156 where a
// block for each chunk adds the partials to find that out; 379 and 387 where
// they are clipped).
template <bool NT, bool kInPlace>
__global__ __launch_bounds__(kOptThreads) void grad_clip_kernel(
    const OptChunk *__restrict__ chunks, int n_chunks, OptNorm nm) {
    __shared__ double sh[kOptThreads / kWave];
    const auto factor = [&] { return norm_factor<kOptThreads>(nm, sh); };
    const bool write_norm = nm.n_part >= 0 && nm.norm && blockIdx.x == 0;
    int k = n_chunks - 1 - static_cast<int>(blockIdx.x);
    if (kInPlace) {
        const NormFactor f = factor();
        if (write_norm && threadIdx.x == 0) *nm.norm = f.norm;
        if (f.one()) return;
        for (; k >= 0; k -= gridDim.x) clip_chunk<NT>(chunks[k], threadIdx.x, [&] { return f; });
        return;
    }
    if (write_norm) {
        const NormFactor f = factor();
        if (threadIdx.x == 0) *nm.norm = f.norm;
    }
    clip_chunk<NT>(chunks[k], threadIdx.x, factor);
}

// One chunk's update in fp32. WM: 0 = fp32 weights, 1 = bf16 weights (the
// update is added to the widened weight and rounded once), 2 = bf16 weights
// with an fp32 copy, which the update works on.
struct StepConst {
    NormFactor f;
    float b1, b1_lo, b2, b2_lo, a1, a2, inv_c1, inv_c2, eps, lr, decay;
};
// A moment settles where what it loses in a step is what it takes in, so beta
// and 1 - beta have to add to 1: with beta rounded to fp32 (off by up to 2^-25)
// the second moment settled 1.3e-5 off for beta2 = 0.999 and 1.4e-3 off for
// 0.99999. So beta comes in two parts. The low one is above zero, for an
// overflowed v (inf) has to stay one and not become inf - inf.
__device__ __forceinline__ void adamw_one(const StepConst &q, float g, float &w, float &m, float &v) {
    g = scaled(g, q.f);
    m = fmaf(q.b1, m, fmaf(q.a1, g, q.b1_lo * m));
    v = fmaf(q.b2, v, fmaf(q.a2 * g, g, q.b2_lo * v));
    const float u = (m * q.inv_c1) / (sqrtf(v * q.inv_c2) + q.eps);
    w -= q.lr * fmaf(q.decay, w, u);
}
// What a step's chunks wait for.
struct StepIn {
    NormFactor f;
    OptStep at;
};
struct StepArgs {
    OptNorm nm;
    OptAdamW hp;
    const float *lr;
    OptStep *at;
    int64_t *step;
};
// One chunk by kThreads threads. `in` is asked for once the chunk's reads are
// on their way.
template <int kThreads, bool NT, bool NTG, typename GT, int WM, typename F>
__device__ __forceinline__ void adamw_values(const OptChunk &t, const Span &p, const StepArgs &a,
                                             int tid, const F &in) {
    const GT *g = (const GT *)t.g;
    gf32 *wf = (gf32 *)(WM == 2 ? t.w32 : t.w), *m = (gf32 *)t.m, *v = (gf32 *)t.v;
    gu16 *wh = (gu16 *)t.w;
    typename Vec4<GT>::type gx[kVecs<kThreads>];
    f32x4 wx[kVecs<kThreads>], mx[kVecs<kThreads>], vx[kVecs<kThreads>];
    u16x4 hx[kVecs<kThreads>];
#pragma unroll
    for (int i = 0; i < kVecs<kThreads>; ++i) {
        if (i * kThreads + tid >= p.n4) continue;
        const int e = p.lead + (i * kThreads + tid) * 4;
        gx[i] = load4<NTG>(g + e);
        if (WM == 1) hx[i] = load4<NT>(wh + e);
        else wx[i] = load4<NT>(wf + e);
        mx[i] = load4<NT>(m + e);
        vx[i] = load4<NT>(v + e);
    }
    float g1 = 0.f, w1 = 0.f, m1 = 0.f, v1 = 0.f;  // of the single element
    if (p.one < p.count) {
        g1 = load1(g + p.one);
        w1 = (WM == 1) ? load1(wh + p.one) : wf[p.one];
        m1 = m[p.one];
        v1 = v[p.one];
    }
    const StepIn si = in();
    if (!si.f.finite) return;  // the step is skipped
    const float rate = a.lr ? *a.lr : a.hp.lr;
    const StepConst q{si.f, a.hp.b1, a.hp.b1_lo, a.hp.b2, a.hp.b2_lo, a.hp.a1, a.hp.a2, si.at.inv_c1,
                      si.at.inv_c2, a.hp.eps, rate * t.lr_scale, a.hp.decay * t.decay_scale};
#pragma unroll
    for (int i = 0; i < kVecs<kThreads>; ++i) {
        if (i * kThreads + tid >= p.n4) continue;
        const int e = p.lead + (i * kThreads + tid) * 4;
        const f32x4 g4 = widen(gx[i]);
        if (WM == 1) wx[i] = widen(hx[i]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float wk = wx[i][k], mk = mx[i][k], vk = vx[i][k];
            adamw_one(q, g4[k], wk, mk, vk);
            wx[i][k] = wk;
            mx[i][k] = mk;
            vx[i][k] = vk;
        }
        store4<NT>(m + e, mx[i]);
        store4<NT>(v + e, vx[i]);
        if (WM != 1) store4<NT>(wf + e, wx[i]);
        if (WM != 0) store4<NT>(wh + e, wx[i]);
    }
    if (p.one < p.count) {
        adamw_one(q, g1, w1, m1, v1);
        m[p.one] = m1;
        v[p.one] = v1;
        if (WM != 1) wf[p.one] = w1;
        if (WM != 0) store1(wh + p.one, w1);
    }
}

template <int kThreads, bool NT, bool NTG, typename F>
__device__ __forceinline__ void adamw_chunk(const OptChunk &t, const StepArgs &a, int tid,
                                            const F &in) {
    const int wm = (t.types & kOptWeightBf16) ? (t.w32 ? 2 : 1) : 0;
    const Span p = span_of(t.count, t.lead, tid);
    if (t.types & kOptGradBf16) {
        if (wm == 0) adamw_values<kThreads, NT, NTG, gu16, 0>(t, p, a, tid, in);
        else if (wm == 1) adamw_values<kThreads, NT, NTG, gu16, 1>(t, p, a, tid, in);
        else adamw_values<kThreads, NT, NTG, gu16, 2>(t, p, a, tid, in);
    } else {
        if (wm == 0) adamw_values<kThreads, NT, NTG, gf32, 0>(t, p, a, tid, in);
        else if (wm == 1) adamw_values<kThreads, NT, NTG, gf32, 1>(t, p, a, tid, in);
        else adamw_values<kThreads, NT, NTG, gf32, 2>(t, p, a, tid, in);
    }
}

// One chunk a block, from the last to the first, as grad_clip_kernel.
template <bool NT, bool NTG>
__global__ __launch_bounds__(kStepThreads) void adamw_kernel(const OptChunk *__restrict__ chunks,
                                                             int n_chunks, StepArgs a) {
    __shared__ double sh[kStepThreads / kWave];
    const auto in = [&] { return StepIn{norm_factor<kStepThreads>(a.nm, sh), *a.at}; };
    if (blockIdx.x == 0) {
        const StepIn si = in();
        if (threadIdx.x == 0) {
            if (a.nm.n_part >= 0 && a.nm.norm) *a.nm.norm = si.f.norm;
            if (si.f.finite) *a.step = si.at.t;
        }
    }
    adamw_chunk<kStepThreads, NT, NTG>(chunks[n_chunks - 1 - static_cast<int>(blockIdx.x)], a,
                                       threadIdx.x, in);
}

// A small list in one launch of one block, four teams of kOptThreads that
// share its chunks: the squares, the norm, and then what is done with it.
enum SoloOp { kSoloNorm, kSoloClip, kSoloStep };
constexpr int kSoloChunks[] = {kSoloNormChunks, kSoloClipChunks, kSoloStepChunks};
template <SoloOp kOp>
__global__ __launch_bounds__(kSoloThreads) void solo_kernel(const OptChunk *__restrict__ chunks,
                                                            int n_chunks, uint32_t types, StepArgs a) {
    constexpr int kTeams = kSoloThreads / kOptThreads;
    __shared__ double sh[kSoloThreads / kWave];
    __shared__ OptStep at;
    const int team = __builtin_amdgcn_readfirstlane(threadIdx.x / kOptThreads);
    const int tid = threadIdx.x % kOptThreads;
    // by the one thread that also writes the step number, off the first wave
    const bool last = threadIdx.x == kSoloThreads - 1;
    if (kOp == kSoloStep && last) at = step_at(a.step, a.hp.beta1, a.hp.beta2);
    double n = 0.0;
    if (a.nm.n_part >= 0) {
        double s = 0.0;
        constexpr int kAtOnce = (kSoloChunks[kOp] + kTeams - 1) / kTeams;  // one round of reads
        if (types & kOptListF32)
            s += range_squares<kAtOnce, false, gf32>(chunks, 0, n_chunks, team, kTeams, tid);
        if (types & kOptListBf16)
            s += range_squares<kAtOnce, false, gu16>(chunks, 0, n_chunks, team, kTeams, tid);
        n = sqrt(block_sum<kSoloThreads>(s, sh));
    } else if (a.nm.norm) {
        n = static_cast<double>(*a.nm.norm);
    }
    __syncthreads();  // every gradient is read, and `at` written
    const NormFactor f = factor_of(n, a.nm.max_norm);
    if (a.nm.n_part >= 0 && a.nm.norm && threadIdx.x == 0) *a.nm.norm = f.norm;
    if (kOp == kSoloStep && last && f.finite) *a.step = at.t;
    if (kOp == kSoloClip)
        for (int k = team; k < n_chunks; k += kTeams)
            clip_chunk<false>(chunks[k], tid, [&] { return f; });
    if (kOp == kSoloStep)
        for (int k = team; k < n_chunks; k += kTeams)
            adamw_chunk<kOptThreads, false, false>(chunks[k], a, tid, [&] { return StepIn{f, at}; });
}

// Writes the chunks of a batch of a list's tensors, which come as kernel
// arguments (no host memory to keep alive, and capturable): one block a tensor.
__global__ __launch_bounds__(kOptThreads) void tensor_list_kernel(OptBatch b, OptChunk *chunks) {
    const OptChunk t = b.ten[blockIdx.x];
    const int64_t n = b.n[blockIdx.x], phase = t.lead, nc = opt_chunks(n, phase);
    const auto at = [](void *p, int64_t start, uint32_t bf16) {
        return static_cast<void *>(static_cast<char *>(p) + start * (bf16 ? 2 : 4));
    };
    for (int64_t c = threadIdx.x; c < nc; c += kOptThreads) {
        const int64_t start = max<int64_t>(c * kOptChunk - phase, 0);
        const int64_t count = min((c + 1) * kOptChunk - phase, n) - start;
        const int64_t lead = (c == 0 && phase > 0) ? min<int64_t>(kOptAlign - phase, count) : 0;
        OptChunk r = t;
        r.g = at(t.g, start, t.types & kOptGradBf16);
        r.out = at(t.out, start, t.types & kOptOutBf16);
        if (t.w) r.w = at(t.w, start, t.types & kOptWeightBf16);
        if (t.w32) r.w32 = t.w32 + start;
        if (t.m) r.m = t.m + start;
        if (t.v) r.v = t.v + start;
        r.count = static_cast<uint16_t>(count);
        r.lead = static_cast<uint16_t>(lead);
        chunks[b.chunk0[blockIdx.x] + c] = r;
    }
}

// Which accesses are marked non-temporal, for a last cache level of 256 MB.
// Gradients of up to kOptCached bytes, or the last so many, stay there from the
// norm's launch to the one that scales them (201 M weights: a clipped step takes
// 1030 us with 240 MB, 1038 with 200, 1045 with 160 and 1071 if no read of the
// gradients is marked; with no access marked at all 1220, and 17 M bf16 weights
// with fp32 copies 100 instead of 81).
// What a step or a clip writes stays there for the next one only if the list
// leaves room for all that runs between: lists beyond kOptKept bytes are
// streamed (three lists in turn, 4 / 6 / 8 M weights of 16 bytes each: 22 / 36 /
// 50 us kept, 25 / 36 / 44 streamed; one list alone 22 / 32 / 40 kept, 24 / 35 /
// 43 streamed).
constexpr int64_t kOptCached = 240 << 20;
constexpr int64_t kOptKept = 96 << 20;

// `scaled`: a launch that reads the gradients again follows
hipError_t launch_squares(const OptList &L, const OptNorm &nm, bool scaled, const int64_t *step,
                          double beta1, double beta2, OptStep *at, hipStream_t st) {
    const bool sums = nm.n_part >= 0;
    int n_stream = 0;
    if (L.g_bytes > kOptCached) {
        const double kept = static_cast<double>(L.n_chunks) * kOptCached / L.g_bytes;
        n_stream = L.n_chunks - (scaled ? static_cast<int>(kept) : 0);
    }
    ProfScope prof(sums ? "grad_squares" : "adamw_count", st);
    hipLaunchKernelGGL(grad_squares_kernel, dim3(sums ? nm.n_part : 1), dim3(kOptThreads), 0, st,
                       L.chunks, sums ? L.n_chunks : 0, n_stream, sums ? L.g_types : 0u, nm.part,
                       step, beta1, beta2, at);
    return hipGetLastError();
}

}  // namespace

int opt_norm_blocks(int n_chunks) { return n_chunks < kOptMaxPart ? n_chunks : kOptMaxPart; }

hipError_t launch_tensor_list(const OptBatch &b, int count, OptChunk *chunks, hipStream_t st) {
    ProfScope prof("tensor_list", st);
    hipLaunchKernelGGL(tensor_list_kernel, dim3(static_cast<unsigned>(count)), dim3(kOptThreads), 0,
                       st, b, chunks);
    return hipGetLastError();
}

hipError_t launch_grad_norm(const OptList &L, const OptNorm &nm, hipStream_t st) {
    if (L.n_chunks <= kSoloNormChunks) {
        ProfScope prof("grad_norm", st);
        hipLaunchKernelGGL(solo_kernel<kSoloNorm>, dim3(1), dim3(kSoloThreads), 0, st, L.chunks,
                           L.n_chunks, L.g_types, StepArgs{nm, {}, nullptr, nullptr, nullptr});
        return hipGetLastError();
    }
    hipError_t e = launch_squares(L, nm, false, nullptr, 0.0, 0.0, nullptr, st);
    if (e != hipSuccess) return e;
    ProfScope prof("grad_norm", st);
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(kOptThreads), 0, st, nm);
    return hipGetLastError();
}

hipError_t launch_grad_clip(const OptList &L, const OptNorm &nm, hipStream_t st) {
    if (L.n_chunks <= kSoloClipChunks) {
        ProfScope prof("grad_clip", st);
        hipLaunchKernelGGL(solo_kernel<kSoloClip>, dim3(1), dim3(kSoloThreads), 0, st, L.chunks,
                           L.n_chunks, L.g_types, StepArgs{nm, {}, nullptr, nullptr, nullptr});
        return hipGetLastError();
    }
    if (nm.n_part >= 0) {
        hipError_t e = launch_squares(L, nm, true, nullptr, 0.0, 0.0, nullptr, st);
        if (e != hipSuccess) return e;
    }
    ProfScope prof("grad_clip", st);
    const bool nt = L.g_bytes + L.out_bytes > kOptKept, in_place = L.out_bytes == 0;
    const auto kernel = in_place ? (nt ? grad_clip_kernel<true, true> : grad_clip_kernel<false, true>)
                                 : (nt ? grad_clip_kernel<true, false> : grad_clip_kernel<false, false>);
    const int blocks = in_place && L.n_chunks > kOptBlocks ? kOptBlocks : L.n_chunks;
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(kOptThreads), 0, st, L.chunks,
                       L.n_chunks, nm);
    return hipGetLastError();
}

hipError_t launch_adamw(const OptList &L, const OptNorm &nm, const OptAdamW &hp, const float *lr,
                        int64_t *step, OptStep *at, hipStream_t st) {
    if (L.n_chunks <= kSoloStepChunks) {
        ProfScope prof("adamw", st);
        hipLaunchKernelGGL(solo_kernel<kSoloStep>, dim3(1), dim3(kSoloThreads), 0, st, L.chunks,
                           L.n_chunks, L.g_types, StepArgs{nm, hp, lr, at, step});
        return hipGetLastError();
    }
    hipError_t e = launch_squares(L, nm, true, step, hp.beta1, hp.beta2, at, st);
    if (e != hipSuccess) return e;
    ProfScope prof("adamw", st);
    const auto kernel = L.g_bytes > kOptCached             ? adamw_kernel<true, true>
                        : L.g_bytes + L.w_bytes > kOptKept ? adamw_kernel<true, false>
                                                             : adamw_kernel<false, false>;
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(L.n_chunks)), dim3(kStepThreads), 0, st,
                       L.chunks, L.n_chunks, StepArgs{nm, hp, lr, at, step});
    return hipGetLastError();
}

}  // namespace dstd
