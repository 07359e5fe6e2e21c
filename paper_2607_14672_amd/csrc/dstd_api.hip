// dstd_api.hip -- C ABI of the DSTD-LIF library: argument validation (host
// only, before anything is enqueued), layer constants, workspace layout and
// kernel dispatch. The contract of every entry point is documented in
// include/dstd_lif.h.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <exception>
#include <mutex>
#include <vector>

#include "../../include/dstd_lif.h"
#include "dstd_internal.h"
#include "dstd_kernels.h"

using dstd::LifConst;

namespace {

thread_local char g_err[512] = "";

dstd_status fail(dstd_status s, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
    return s;
}

constexpr size_t kAlign = 256;
size_t align_up(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

// Host validation of the layer parameters (no device access).
dstd_status check_params(const dstd_lif_params *p, int32_t allowed_flags = 0) {
    if (!p) return fail(DSTD_ERR_NULL, "params is NULL");
    // each time constant is > 0, finite or +inf (the closed-form rows)
    if (!(p->tau_m > 0.f) || !(p->tau_s > 0.f))
        return fail(DSTD_ERR_PARAM, "time constants must be > 0 or +inf (tau_m=%g tau_s=%g)",
                    (double)p->tau_m, (double)p->tau_s);
    if (isfinite(p->tau_m) && isfinite(p->tau_s) && p->tau_m != p->tau_s) {
        double tmax = std::max((double)p->tau_m, (double)p->tau_s);
        if (fabs((double)p->tau_m - (double)p->tau_s) <= 1e-3 * tmax)
            return fail(DSTD_ERR_UNSUPPORTED,
                        "tau_m and tau_s differ by less than 1e-3 relative without being equal: "
                        "use equal constants (the (tau, tau) row) or separate them further");
    }
    if (!(isfinite(p->threshold) && p->threshold > 0.f))
        return fail(DSTD_ERR_PARAM, "threshold must be finite and > 0");
    if (p->M < 1) return fail(DSTD_ERR_PARAM, "M must be >= 1 (got %d)", p->M);
    if (p->M > DSTD_MAX_M)
        return fail(DSTD_ERR_UNSUPPORTED, "M = %d exceeds DSTD_MAX_M = %d", p->M, DSTD_MAX_M);
    if (!(isfinite(p->dt) && p->dt > 0.f)) return fail(DSTD_ERR_PARAM, "dt must be finite and > 0");
    if (!isfinite(p->t0)) return fail(DSTD_ERR_PARAM, "t0 must be finite");
    double TM = (double)p->t0 + (double)p->M * (double)p->dt;
    if (isnan(p->t_max) || !((double)p->t_max > TM))
        return fail(DSTD_ERR_PARAM, "t_max must be > T_M = t0 + M*dt (got %g, T_M = %g)",
                    (double)p->t_max, TM);
    if ((p->flags & ~allowed_flags) != 0) {
        const int32_t extra = p->flags & ~allowed_flags;
        if (extra & (DSTD_FLAG_CONTRACT_SPARSE | DSTD_FLAG_CONTRACT_MFMA))
            return fail(DSTD_ERR_UNSUPPORTED, "the contraction flags apply to dense layers only");
        if (extra & DSTD_FLAG_CONV_KEEP)
            return fail(DSTD_ERR_UNSUPPORTED, "DSTD_FLAG_CONV_KEEP applies to the conv forward only");
        if (extra & DSTD_FLAG_CONV_REUSE)
            return fail(DSTD_ERR_UNSUPPORTED, "DSTD_FLAG_CONV_REUSE applies to the conv backward only");
        return fail(DSTD_ERR_PARAM, "unknown flags 0x%x", (unsigned)p->flags);
    }
    if ((p->flags & DSTD_FLAG_CONTRACT_SPARSE) && (p->flags & DSTD_FLAG_CONTRACT_MFMA))
        return fail(DSTD_ERR_PARAM, "DSTD_FLAG_CONTRACT_SPARSE and _MFMA exclude each other");
    return DSTD_OK;
}

constexpr int32_t kDenseFlags = DSTD_FLAG_CONTRACT_SPARSE | DSTD_FLAG_CONTRACT_MFMA;

// The dense forward's contraction: the event-sparse VALU kernels, or the
// dense bf16 MFMA product of the event matrix and W (bf16 weights only). The
// automatic choice is by shape, from measured times on MI355X (the dense
// product does (M+1)/2 times the method's work, so it wins only for small M
// on large layers).
bool mfma_shape_auto(int M, int64_t B, int64_t N_in, int64_t N_out) {
    return M <= dstd::kMfmaAutoMaxM && N_out >= 1024 && N_in >= 1024 && B * N_out >= (int64_t)1 << 18;
}

// could this call take the MFMA path (the workspace query does not know the
// weight type, so it reserves room whenever it could)
bool mfma_possible(const dstd_lif_params *p, int64_t B, int64_t N_in, int64_t N_out) {
    if (p->flags & DSTD_FLAG_CONTRACT_SPARSE) return false;
    if (p->flags & DSTD_FLAG_CONTRACT_MFMA) return true;
    return mfma_shape_auto(p->M, B, N_in, N_out);
}

size_t mfma_ws_events(int64_t B, int64_t N_in) { return align_up((size_t)(B * N_in) * 16); }
size_t mfma_ws_bytes(int M, int64_t B, int64_t N_in, int64_t N_out) {
    if (B * N_out == 0) return 0;
    return mfma_ws_events(B, N_in) + align_up((size_t)B * (size_t)(M + 1) * (size_t)N_out * sizeof(float));
}

// Row of Table "tab:kernel" for the canonical pair tv >= ti (tv may be inf).
int kind_of(double tv, double ti) {
    if (isinf(ti)) return dstd::kInfInf;
    if (isinf(tv)) return dstd::kInfTau;
    if (tv == ti) return dstd::kEqual;
    return dstd::kGeneral;
}

// K(u), u >= 0 (u may be +inf for the (inf, tau) row's limit)
double kern_d(int kind, double tv, double ti, double u) {
    switch (kind) {
        case dstd::kEqual: return u * exp(-u / ti);
        case dstd::kInfTau: return -ti * expm1(-u / ti);
        case dstd::kInfInf: return u;
        default: {
            double c = tv * ti / (tv - ti), kap = 1.0 / ti - 1.0 / tv;
            return -c * exp(-u / tv) * expm1(-kap * u);
        }
    }
}

LifConst make_const(const dstd_lif_params *p) {
    double tv = std::max((double)p->tau_m, (double)p->tau_s);
    double ti = std::min((double)p->tau_m, (double)p->tau_s);
    const int kind = kind_of(tv, ti);
    double dt = p->dt;
    // K's maximum on [0, len] sits at min(len, peak): the general row peaks
    // at ln(tv/ti)/kappa, (tau, tau) at tau; the other rows increase
    double kap = (kind == dstd::kGeneral) ? 1.0 / ti - 1.0 / tv : 0.0;
    double upk = (kind == dstd::kGeneral) ? log(tv / ti) / kap
                 : (kind == dstd::kEqual) ? ti : INFINITY;
    double TM = (double)p->t0 + (double)p->M * dt;
    double last = isinf(p->t_max) ? INFINITY : (double)p->t_max - TM;
    LifConst C{};
    C.kind = kind;
    C.tv = (float)tv;
    C.ti = (float)ti;
    C.inv_tv = (float)(1.0 / tv);  // 0 for an infinite constant
    C.inv_ti = (float)(1.0 / ti);
    C.c = (kind == dstd::kGeneral) ? (float)(tv * ti / (tv - ti)) : 0.f;
    C.kappa = (float)kap;
    C.alpha = (float)exp(-dt / tv);
    C.beta = (float)exp(-dt / ti);
    C.k_dt = (float)kern_d(kind, tv, ti, dt);
    C.inv_em1 = (kind == dstd::kGeneral) ? (float)(1.0 / expm1(-kap * dt)) : 0.f;
    C.kmax_dt_d = kern_d(kind, tv, ti, std::min(dt, upk));
    C.kmax_last_d = kern_d(kind, tv, ti, std::min(last, upk));
    C.theta_lo_d = (double)p->threshold / 1.0001;
    C.kpeak_d = kern_d(kind, tv, ti, std::min((double)p->M * dt + last, upk));
    // max |K''| on [0, dt]: general row c |e^{-u/tv}/tv^2 - e^{-u/ti}/ti^2|
    // <= c / ti^2; (tau, tau) e^{-u/tau} |u/tau^2 - 2/tau| <= 2/tau + dt/tau^2;
    // (inf, tau) e^{-u/tau}/tau <= 1/tau; (inf, inf) 0
    const double kpp = (kind == dstd::kGeneral) ? tv / (ti * (tv - ti))
                       : (kind == dstd::kEqual) ? 2.0 / ti + dt / (ti * ti)
                       : (kind == dstd::kInfTau) ? 1.0 / ti : 0.0;
    C.curv_v_d = dt * dt / 8.0 * (isinf(tv) ? 0.0 : 1.0 / (tv * tv));
    C.curv_i_d = dt * dt / 8.0 * kpp;
    C.twice = (kind == dstd::kGeneral && tv == 2.0 * ti) ? 1 : 0;
    C.inv_dt = (float)(1.0 / dt);
    C.e_mdt = (float)exp(-dt / ti);
    C.inv_D = (kind == dstd::kInfTau) ? (float)(-1.0 / expm1(-dt / ti)) : 0.f;
    C.theta = p->threshold;
    C.t0 = p->t0;
    C.dt = p->dt;
    C.last_len = (float)last;
    C.slope_floor = 1e-12f * p->threshold;
    C.M = p->M;
    C.alpha_d = exp(-dt / tv);
    C.beta_d = exp(-dt / ti);
    C.k_dt_d = kern_d(kind, tv, ti, dt);
    C.r_lo_dt = (float)exp(-kap * dt);
    C.r_lo_last = isinf(last) ? 0.f : (float)exp(-kap * last);
    return C;
}

dstd_status check_dims(int64_t B, int64_t N_in, int64_t N_out) {
    if (B < 0 || N_in < 0 || N_out < 0)
        return fail(DSTD_ERR_SHAPE, "sizes must be >= 0 (B=%lld N_in=%lld N_out=%lld)",
                    (long long)B, (long long)N_in, (long long)N_out);
    const int64_t lim = (int64_t)1 << 24;
    if (N_in >= lim || N_out >= lim)
        return fail(DSTD_ERR_SHAPE, "N_in and N_out must be < 2^24");
    if (B > 65535)
        return fail(DSTD_ERR_SHAPE, "B = %lld exceeds the supported batch (65535)", (long long)B);
    if (N_in * N_out * 4 >= ((int64_t)1 << 31))
        return fail(DSTD_ERR_SHAPE, "N_in * N_out = %lld exceeds 2^29 weights",
                    (long long)(N_in * N_out));
    return DSTD_OK;
}

struct DenseWs {
    size_t ev, tri, P, part, dq, wt, sj, sr, sL, sR, nvalid, rs, total;
    int64_t sstride;
    int n_buf;
};

DenseWs dense_ws_layout(int M, int64_t B, int64_t N_in, int64_t N_out, bool backward) {
    DenseWs w{};
    size_t off = 0;
    size_t n = (size_t)(B * N_in);
    if (backward) {
        // events, gradient triples, dt_in buffers, dead-neuron terms, dW partials
        w.ev = off; off += align_up(n * 5 * sizeof(float));
        w.tri = off; off += align_up((size_t)B * (size_t)N_out * 3 * sizeof(float));
        w.n_buf = (int)dstd::back_buf_cap(B, N_in, 1, N_out);
        w.P = off; off += align_up(n * (size_t)w.n_buf * sizeof(float));
        w.dq = off; off += align_up((size_t)N_out * sizeof(float));
        const size_t cap = (size_t)dstd::back_split_cap(B, N_in, N_out);
        w.part = off; off += align_up((cap > 1 ? cap : 0) * (size_t)N_out * (size_t)N_in * sizeof(float));
        // and the forward's, so that one buffer serves both and a larger layer
        // (more intervals too) never takes a smaller one
        w.total = off + dense_ws_layout(M, B, N_in, N_out, false).total;
        return w;
    }
    if (B * N_out == 0) return w;  // the forward enqueues nothing
    // transposed weights (room for fp32) and the row-sorted event records of
    // every sample
    w.wt = off; off += align_up((size_t)N_in * (size_t)N_out * sizeof(float));
    // sorted event lists: per sample N_in records; the last sample's list
    // is padded so batched reads past its end stay in the allocation
    w.sstride = N_in;
    size_t ns = n + dstd::kSortPad;
    w.sj = off; off += align_up(ns * sizeof(int));
    w.sr = off; off += align_up(ns * sizeof(int));
    w.sL = off; off += align_up(ns * sizeof(float));
    w.sR = off; off += align_up(ns * sizeof(float));
    w.nvalid = off; off += align_up((size_t)B * sizeof(int));
    w.rs = off; off += align_up((size_t)B * (M + 4) * sizeof(int));
    w.total = off;
    return w;
}

dstd_status check_ws(void *ws, size_t ws_bytes, size_t need) {
    if (need == 0) return DSTD_OK;
    if (!ws) return fail(DSTD_ERR_NULL, "workspace is NULL (%zu bytes needed)", need);
    if (((uintptr_t)ws) % kAlign != 0) return fail(DSTD_ERR_WORKSPACE, "workspace must be 256-byte aligned");
    if (ws_bytes < need)
        return fail(DSTD_ERR_WORKSPACE, "workspace too small: %zu < %zu bytes", ws_bytes, need);
    return DSTD_OK;
}

dstd_status hip_status(hipError_t e, const char *what) {
    if (e == hipSuccess) return DSTD_OK;
    return fail(DSTD_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

template <typename T> T *at(void *ws, size_t off) {
    return reinterpret_cast<T *>(static_cast<char *>(ws) + off);
}


// Host validation of a conv layer; fills the derived geometry.
dstd_status check_conv(const dstd_conv_shape *cs, int64_t B, int M, dstd::ConvGeom *g) {
    if (!cs) return fail(DSTD_ERR_NULL, "conv shape is NULL");
    if (B < 0) return fail(DSTD_ERR_SHAPE, "B must be >= 0");
    if (cs->C_in < 1 || cs->H < 1 || cs->W < 1 || cs->C_out < 1)
        return fail(DSTD_ERR_SHAPE, "C_in, H, W and C_out must be >= 1");
    if (cs->C_in > (1 << 20) || cs->C_out > (1 << 20))
        return fail(DSTD_ERR_SHAPE, "C_in and C_out must be <= 2^20");
    if (cs->KH < 1 || cs->KW < 1 || cs->KH > dstd::kConvMaxK || cs->KW > dstd::kConvMaxK)
        return fail(DSTD_ERR_UNSUPPORTED, "kernel size %dx%d: 1..%d supported", cs->KH, cs->KW,
                    dstd::kConvMaxK);
    if (cs->stride < 1 || cs->pad < 0 || cs->pad >= std::max(cs->KH, cs->KW) + 1)
        return fail(DSTD_ERR_SHAPE, "need stride >= 1 and 0 <= pad <= max(KH, KW)");
    if (cs->pool_in != 0 && cs->pool_in != 1 && cs->pool_in != 2)
        return fail(DSTD_ERR_PARAM, "pool_in must be 0, 1 or 2 (got %d)", cs->pool_in);
    if (cs->pool_in == 2 && (cs->H % 2 != 0 || cs->W % 2 != 0))
        return fail(DSTD_ERR_SHAPE, "2x2 event pooling needs even H and W (got %dx%d)", cs->H, cs->W);
    dstd::ConvGeom &G = *g;
    G.C_in = cs->C_in; G.H = cs->H; G.W = cs->W; G.C_out = cs->C_out;
    G.KH = cs->KH; G.KW = cs->KW; G.stride = cs->stride; G.pad = cs->pad; G.pool = cs->pool_in;
    if (G.pool == 2) { G.Hp = G.H / 2; G.Wp = G.W / 2; G.P = 4; }
    else if (G.pool == 0) { G.Hp = 1; G.Wp = 1; G.P = G.H * G.W; }
    else { G.Hp = G.H; G.Wp = G.W; G.P = 1; }
    const int64_t ho = ((int64_t)G.Hp + 2 * G.pad - G.KH) / G.stride + 1;
    const int64_t wo = ((int64_t)G.Wp + 2 * G.pad - G.KW) / G.stride + 1;
    if ((int64_t)G.Hp + 2 * G.pad < G.KH || (int64_t)G.Wp + 2 * G.pad < G.KW || ho < 1 || wo < 1)
        return fail(DSTD_ERR_SHAPE, "kernel larger than the padded input map");
    G.Ho = (int)ho; G.Wo = (int)wo;
    const int64_t pc = (int64_t)G.P * G.C_in;
    const int64_t lim = (int64_t)1 << 30;
    const int64_t nw = (int64_t)G.KH * G.KW * G.C_in * G.C_out;
    if (pc * G.Wp >= lim || (int64_t)G.C_in * G.H * G.W >= lim || nw * 4 >= lim ||
        (int64_t)G.C_out * G.Ho * G.Wo >= lim)
        return fail(DSTD_ERR_SHAPE, "conv layer too large (per-sample sizes must stay below 2^30)");
    if (B * G.Hp >= ((int64_t)1 << 31) || B * G.Ho * G.Wo >= ((int64_t)1 << 31))
        return fail(DSTD_ERR_SHAPE, "batch too large for this map size");
    if ((int64_t)(M + 3) * G.Wp + 256 > 16384)
        return fail(DSTD_ERR_UNSUPPORTED, "(M + 3) * W_p = %lld exceeds the cell-row sort's LDS "
                    "table (16128 buckets)", (long long)(M + 3) * G.Wp);
    G.PC = (int)pc;
    G.inv_P = (float)(1.0 / G.P);
    G.dv_pch = dstd::fast_div((uint32_t)(G.Wp * G.P));
    G.dv_w = dstd::fast_div((uint32_t)G.W);
    G.dv_cin = dstd::fast_div((uint32_t)G.C_in);
    G.dv_p = dstd::fast_div((uint32_t)G.P);
    G.dv_kw = dstd::fast_div((uint32_t)G.KW);
    G.dv_pc = dstd::fast_div((uint32_t)G.PC);
    return DSTD_OK;
}

struct ConvWs {
    size_t wt, key, L, R, off;                        // both passes
    size_t P, ev, crlive, tri, rend, part, zlive, dq;  // backward
    size_t total;
};

ConvWs conv_ws_layout(int M, const dstd::ConvGeom &g, int64_t B, bool backward) {
    ConvWs w{};
    size_t off = 0;
    const size_t n = (size_t)B * g.Hp * g.Wp * g.PC;  // inputs (cell-major)
    const size_t nw = (size_t)g.KH * g.KW * g.C_in * g.C_out;
    const size_t nout = (size_t)B * g.Ho * g.Wo * g.C_out;
    const int R = M + 3;
    if (B == 0 && !backward) return w;
    // weights / P and the records sorted per cell row; batched reads may run
    // past the last record by up to kSortPad slots
    w.wt = off; off += align_up(nw * sizeof(float));
    const size_t nr = n + dstd::kSortPad;
    w.key = off; off += align_up(nr * sizeof(int));
    w.L = off; off += align_up(nr * sizeof(float));
    w.R = off; off += align_up(nr * sizeof(float));
    w.off = off; off += align_up((size_t)B * g.Hp * (size_t)dstd::conv_off_stride(R, g) * sizeof(int));
    if (backward) {
        const dstd::ConvBackPlan dp = dstd::plan_conv_back(g, B, M, true, true);
        w.ev = off; off += align_up(n * 5 * sizeof(float));
        w.P = off; off += align_up(n * (size_t)(g.KH * dp.kg * dp.tiles_dt) * sizeof(float));
        w.crlive = off; off += align_up((size_t)B * g.Hp * sizeof(int));
        w.tri = off; off += align_up(3 * nout * sizeof(float));
        w.rend = off; off += align_up((size_t)B * g.Ho * g.Wo * sizeof(int));
        w.dq = off; off += align_up((size_t)g.C_out * sizeof(float));  // dead-neuron term per channel
        w.part = off; off += align_up((size_t)dp.nsplit * nw * sizeof(float));
        w.zlive = off; off += align_up((size_t)dp.nsplit * sizeof(int));
    }
    w.total = off;
    return w;
}

dstd::CellEv cell_events(void *ws, const ConvWs &L) {
    return dstd::CellEv{at<float>(ws, L.ev), at<int>(ws, L.crlive)};
}

// Synfire terms of a backward call (NULL: off).
dstd_status check_synfire(const dstd_synfire_params *sp) {
    if (!sp) return DSTD_OK;
    const float g[3] = {sp->gamma_head, sp->gamma_tail, sp->gamma_q};
    for (float v : g)
        if (!(isfinite(v) && v >= 0.f))
            return fail(DSTD_ERR_PARAM, "synfire gammas must be finite and >= 0");
    if (!isfinite(sp->t_head) || !isfinite(sp->t_tail))
        return fail(DSTD_ERR_PARAM, "synfire t_head and t_tail must be finite");
    if (!(isfinite(sp->scale) && sp->scale > 0.f))
        return fail(DSTD_ERR_PARAM, "synfire scale must be finite and > 0");
    return DSTD_OK;
}

dstd::Synfire make_synfire(const dstd_synfire_params *sp, float *dq) {
    dstd::Synfire f{};
    if (!sp) return f;
    f.on = 1;
    f.gh = sp->gamma_head;
    f.gt = sp->gamma_tail;
    f.th = sp->t_head;
    f.tt = sp->t_tail;
    f.gq = sp->gamma_q;
    f.scale = sp->scale;
    f.dq = dq;
    return f;
}

dstd_status dense_backward(const dstd_lif_params *p, const dstd_synfire_params *sp, int64_t B,
                           int64_t N_in, int64_t N_out, const float *t_in, const void *W,
                           dstd_dtype w_dtype, const float *t_out, const float *slope,
                           const int32_t *q_idx, const float *grad_t_out, float *grad_W,
                           float *grad_t_in, void *ws, size_t ws_bytes, void *stream);
dstd_status conv_backward(const dstd_lif_params *p, const dstd_synfire_params *sp,
                          const dstd_conv_shape *cs, int64_t B, const float *t_in, const void *W,
                          dstd_dtype w_dtype, const float *t_out, const float *slope,
                          const int32_t *q_idx, const float *grad_t_out, float *grad_W,
                          float *grad_t_in, void *ws, size_t ws_bytes, void *stream);

}  // namespace

extern "C" {

const char *dstd_status_string(dstd_status s) {
    switch (s) {
        case DSTD_OK: return "ok";
        case DSTD_ERR_NULL: return "null pointer";
        case DSTD_ERR_SHAPE: return "invalid shape";
        case DSTD_ERR_PARAM: return "invalid parameter";
        case DSTD_ERR_UNSUPPORTED: return "unsupported";
        case DSTD_ERR_WORKSPACE: return "workspace too small or misaligned";
        case DSTD_ERR_HIP: return "HIP error";
    }
    return "unknown status";
}

const char *dstd_last_error(void) { return g_err; }

int32_t dstd_version(void) { return 102; }

size_t dstd_lif_forward_workspace_size(const dstd_lif_params *p, int64_t B, int64_t N_in,
                                       int64_t N_out) {
    if (check_params(p, kDenseFlags) != DSTD_OK || check_dims(B, N_in, N_out) != DSTD_OK) return 0;
    size_t need = (p->flags & DSTD_FLAG_CONTRACT_MFMA) ? 0 : dense_ws_layout(p->M, B, N_in, N_out, false).total;
    if (mfma_possible(p, B, N_in, N_out)) need = std::max(need, mfma_ws_bytes(p->M, B, N_in, N_out));
    return need;
}

size_t dstd_lif_backward_workspace_size(const dstd_lif_params *p, int64_t B, int64_t N_in,
                                        int64_t N_out) {
    if (check_params(p, kDenseFlags) != DSTD_OK || check_dims(B, N_in, N_out) != DSTD_OK) return 0;
    return dense_ws_layout(p->M, B, N_in, N_out, true).total;
}

dstd_status dstd_lif_forward(const dstd_lif_params *p, int64_t B, int64_t N_in, int64_t N_out,
                             const float *t_in, const void *W, dstd_dtype w_dtype, float *t_out,
                             float *slope, int32_t *q_idx, void *ws, size_t ws_bytes,
                             void *stream) {
    dstd_status s = check_params(p, kDenseFlags);
    if (s != DSTD_OK) return s;
    if ((s = check_dims(B, N_in, N_out)) != DSTD_OK) return s;
    if (w_dtype != DSTD_F32 && w_dtype != DSTD_BF16)
        return fail(DSTD_ERR_PARAM, "unknown weight dtype %d", (int)w_dtype);
    if ((p->flags & DSTD_FLAG_CONTRACT_MFMA) && w_dtype != DSTD_BF16)
        return fail(DSTD_ERR_UNSUPPORTED, "the MFMA contraction takes bf16 weights");
    if (B * N_out > 0 && (!t_out || !slope || !q_idx))
        return fail(DSTD_ERR_NULL, "t_out, slope and q_idx are required");
    if (B * N_in > 0 && !t_in) return fail(DSTD_ERR_NULL, "t_in is NULL");
    if (N_in * N_out > 0 && !W) return fail(DSTD_ERR_NULL, "W is NULL");
    const bool mfma = w_dtype == DSTD_BF16 && mfma_possible(p, B, N_in, N_out);
    if (mfma) {
        if ((s = check_ws(ws, ws_bytes, mfma_ws_bytes(p->M, B, N_in, N_out))) != DSTD_OK) return s;
        if (B * N_out == 0) return DSTD_OK;
        LifConst C = make_const(p);
        hipError_t e = dstd::launch_forward_mfma(
            C, B, N_in, N_out, static_cast<const uint16_t *>(W), ws,
            at<float>(ws, mfma_ws_events(B, N_in)), t_in, t_out, slope, q_idx,
            static_cast<hipStream_t>(stream));
        return hip_status(e, "forward (MFMA) launch");
    }
    DenseWs L = dense_ws_layout(p->M, B, N_in, N_out, false);
    if ((s = check_ws(ws, ws_bytes, L.total)) != DSTD_OK) return s;
    if (B * N_out == 0) return DSTD_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    LifConst C = make_const(p);
    dstd::SortedEv srt{at<int>(ws, L.sj), at<int>(ws, L.sr), at<float>(ws, L.sL),
                       at<float>(ws, L.sR), L.sstride, at<int>(ws, L.rs)};
    hipError_t e = dstd::launch_forward(C, B, N_in, N_out, W, w_dtype == DSTD_BF16, at<void>(ws, L.wt),
                                        srt, at<int>(ws, L.nvalid), t_in, t_out, slope, q_idx, st);
    return hip_status(e, "forward launch");
}

}  // extern "C"

// Scratch of the allocation-free forward: one array per GPU, reserved when the
// library's code object is loaded there and kept until the process ends. In
// host code `scratch` only names the symbol; its device address comes from
// hipGetSymbolAddress, once per device, with that device current.
static __device__ __align__(256) unsigned char scratch[DSTD_NOALLOC_SCRATCH_BYTES];

namespace {

constexpr int kMaxDevices = 64;
void *g_scratch_ptr[kMaxDevices] = {};
std::mutex g_scratch_mu;

dstd_status scratch_for_current_device(void **out) {
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return fail(DSTD_ERR_HIP, "hipGetDevice: %s", hipGetErrorString(e));
    if (dev < 0 || dev >= kMaxDevices)
        return fail(DSTD_ERR_UNSUPPORTED, "device index %d beyond %d", dev, kMaxDevices);
    std::lock_guard<std::mutex> lock(g_scratch_mu);
    if (!g_scratch_ptr[dev]) {
        void *ptr = nullptr;
        e = hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch));
        if (e != hipSuccess || !ptr)
            return fail(DSTD_ERR_HIP, "hipGetSymbolAddress(scratch) on device %d: %s", dev,
                        hipGetErrorString(e));
        g_scratch_ptr[dev] = ptr;
    }
    *out = g_scratch_ptr[dev];
    return DSTD_OK;
}

}  // namespace

extern "C" {

dstd_status dstd_lif_forward_noalloc(const dstd_lif_params *p, int64_t B, int64_t N_in,
                                     int64_t N_out, const float *t_in, const void *W,
                                     dstd_dtype w_dtype, float *t_out, float *slope,
                                     int32_t *q_idx, void *stream) {
    // host validation first: nothing touches the device before the sizes pass
    dstd_status s = check_params(p, kDenseFlags);
    if (s != DSTD_OK) return s;
    if ((s = check_dims(B, N_in, N_out)) != DSTD_OK) return s;
    const size_t need = dstd_lif_forward_workspace_size(p, B, N_in, N_out);
    if (need > (size_t)DSTD_NOALLOC_SCRATCH_BYTES)
        return fail(DSTD_ERR_WORKSPACE,
                    "layer needs %zu bytes of scratch; the allocation-free forward holds %zu "
                    "(use dstd_lif_forward with a caller workspace)",
                    need, (size_t)DSTD_NOALLOC_SCRATCH_BYTES);
    void *ws = nullptr;
    if (need > 0 && (s = scratch_for_current_device(&ws)) != DSTD_OK) return s;
    // the forward's kernels write every scratch word they read: nothing to clear
    return dstd_lif_forward(p, B, N_in, N_out, t_in, W, w_dtype, t_out, slope, q_idx, ws,
                            need > 0 ? (size_t)DSTD_NOALLOC_SCRATCH_BYTES : 0, stream);
}

dstd_status dstd_lif_backward(const dstd_lif_params *p, int64_t B, int64_t N_in, int64_t N_out,
                              const float *t_in, const void *W, dstd_dtype w_dtype,
                              const float *t_out, const float *slope, const int32_t *q_idx,
                              const float *grad_t_out, float *grad_W, float *grad_t_in, void *ws,
                              size_t ws_bytes, void *stream) {
    return dense_backward(p, nullptr, B, N_in, N_out, t_in, W, w_dtype, t_out, slope, q_idx,
                          grad_t_out, grad_W, grad_t_in, ws, ws_bytes, stream);
}

dstd_status dstd_lif_backward_synfire(const dstd_lif_params *p, const dstd_synfire_params *sp,
                                      int64_t B, int64_t N_in, int64_t N_out, const float *t_in,
                                      const void *W, dstd_dtype w_dtype, const float *t_out,
                                      const float *slope, const int32_t *q_idx,
                                      const float *grad_t_out, float *grad_W, float *grad_t_in,
                                      void *ws, size_t ws_bytes, void *stream) {
    return dense_backward(p, sp, B, N_in, N_out, t_in, W, w_dtype, t_out, slope, q_idx,
                          grad_t_out, grad_W, grad_t_in, ws, ws_bytes, stream);
}

}  // extern "C"

namespace {

dstd_status dense_backward(const dstd_lif_params *p, const dstd_synfire_params *sp, int64_t B,
                           int64_t N_in, int64_t N_out, const float *t_in, const void *W,
                           dstd_dtype w_dtype, const float *t_out, const float *slope,
                           const int32_t *q_idx, const float *grad_t_out, float *grad_W,
                           float *grad_t_in, void *ws, size_t ws_bytes, void *stream) {
    // the contraction flags select the forward's kernels; the backward takes them as given
    dstd_status s = check_params(p, kDenseFlags);
    if (s != DSTD_OK) return s;
    if ((s = check_synfire(sp)) != DSTD_OK) return s;
    if ((s = check_dims(B, N_in, N_out)) != DSTD_OK) return s;
    if (w_dtype != DSTD_F32 && w_dtype != DSTD_BF16)
        return fail(DSTD_ERR_PARAM, "unknown weight dtype %d", (int)w_dtype);
    if (B * N_out > 0 && (!t_out || !slope || !q_idx || !grad_t_out))
        return fail(DSTD_ERR_NULL, "t_out, slope, q_idx and grad_t_out are required");
    if (B * N_in > 0 && !t_in) return fail(DSTD_ERR_NULL, "t_in is NULL");
    if (grad_t_in && N_in * N_out > 0 && !W) return fail(DSTD_ERR_NULL, "W is NULL");
    DenseWs L = dense_ws_layout(p->M, B, N_in, N_out, true);
    if ((s = check_ws(ws, ws_bytes, L.total)) != DSTD_OK) return s;
    hipStream_t st = static_cast<hipStream_t>(stream);
    hipError_t e;
    // Empty sizes need no special case: with B == 0 the contraction writes zeros
    // to dW, and without neurons to dt_in (no memset is used, so the call stays
    // safe to capture in a graph).
    LifConst C = make_const(p);
    dstd::DenseBwdWs bw;
    bw.ev = at<float>(ws, L.ev);
    bw.tri = at<float>(ws, L.tri);
    bw.P = at<float>(ws, L.P);
    bw.n_buf = L.n_buf;
    bw.part = at<float>(ws, L.part);
    e = dstd::launch_backward(C, B, N_in, N_out, W, w_dtype == DSTD_BF16, t_in, t_out, slope,
                              q_idx, grad_t_out, bw, grad_W, grad_t_in,
                              make_synfire(sp, at<float>(ws, L.dq)), st);
    return hip_status(e, "backward launch");
}

}  // namespace

extern "C" {

dstd_status dstd_softmax_ce_grad(int64_t B, int64_t N, const float *t_out, const int32_t *labels,
                                 float tau_soft, float t_cap, float *grad_t, float *loss,
                                 void *stream) {
    if (B < 0 || B > 65535 || N < 1 || N >= (1 << 24))
        return fail(DSTD_ERR_SHAPE, "need 0 <= B <= 65535 and 1 <= N < 2^24");
    if (!(isfinite(tau_soft) && tau_soft > 0.f)) return fail(DSTD_ERR_PARAM, "tau_soft must be > 0");
    if (!isfinite(t_cap)) return fail(DSTD_ERR_PARAM, "t_cap must be finite");
    if (!loss || (B > 0 && (!t_out || !labels || !grad_t)))
        return fail(DSTD_ERR_NULL, "t_out, labels, grad_t and loss are required");
    hipError_t e = dstd::launch_softmax_ce(B, N, t_out, labels, tau_soft, t_cap, grad_t, loss,
                                           static_cast<hipStream_t>(stream));
    return hip_status(e, "softmax_ce launch");
}

dstd_status dstd_mse_grad(int64_t B, int64_t N, const float *t_out, const float *target,
                          float *grad_t, float *loss, void *stream) {
    if (B < 0 || B > 65535 || N < 1 || N >= (1 << 24))
        return fail(DSTD_ERR_SHAPE, "need 0 <= B <= 65535 and 1 <= N < 2^24");
    if (!loss || (B > 0 && (!t_out || !target || !grad_t)))
        return fail(DSTD_ERR_NULL, "t_out, target, grad_t and loss are required");
    hipError_t e = dstd::launch_mse(B, N, t_out, target, grad_t, loss,
                                    static_cast<hipStream_t>(stream));
    return hip_status(e, "mse launch");
}

size_t dstd_lif_conv_forward_workspace_size(const dstd_lif_params *p, const dstd_conv_shape *cs,
                                            int64_t B) {
    dstd::ConvGeom g;
    if (check_params(p, DSTD_FLAG_CONV_KEEP) != DSTD_OK || check_conv(cs, B, p->M, &g) != DSTD_OK)
        return 0;
    // a forward that keeps its sort for the backward needs the backward's size
    return conv_ws_layout(p->M, g, B, (p->flags & DSTD_FLAG_CONV_KEEP) != 0).total;
}

size_t dstd_lif_conv_backward_workspace_size(const dstd_lif_params *p, const dstd_conv_shape *cs,
                                             int64_t B) {
    dstd::ConvGeom g;
    if (check_params(p, DSTD_FLAG_CONV_REUSE) != DSTD_OK || check_conv(cs, B, p->M, &g) != DSTD_OK)
        return 0;
    return conv_ws_layout(p->M, g, B, true).total;
}

dstd_status dstd_lif_conv_forward(const dstd_lif_params *p, const dstd_conv_shape *cs, int64_t B,
                                  const float *t_in, const void *W, dstd_dtype w_dtype,
                                  float *t_out, float *slope, int32_t *q_idx, void *ws,
                                  size_t ws_bytes, void *stream) {
    dstd_status s = check_params(p, DSTD_FLAG_CONV_KEEP);
    if (s != DSTD_OK) return s;
    dstd::ConvGeom g;
    if ((s = check_conv(cs, B, p->M, &g)) != DSTD_OK) return s;
    if (w_dtype != DSTD_F32 && w_dtype != DSTD_BF16)
        return fail(DSTD_ERR_PARAM, "unknown weight dtype %d", (int)w_dtype);
    if (B > 0 && (!t_in || !W || !t_out || !slope || !q_idx))
        return fail(DSTD_ERR_NULL, "t_in, W, t_out, slope and q_idx are required");
    // keeping the sort for the backward needs the backward's workspace
    const bool keep = (p->flags & DSTD_FLAG_CONV_KEEP) != 0;
    ConvWs L = conv_ws_layout(p->M, g, B, keep);
    if ((s = check_ws(ws, ws_bytes, L.total)) != DSTD_OK) return s;
    if (B == 0) return DSTD_OK;
    LifConst C = make_const(p);
    dstd::ConvSorted srt{at<int>(ws, L.key), at<float>(ws, L.L), at<float>(ws, L.R),
                         at<int>(ws, L.off)};
    dstd::CellEv ev{};
    if (keep) ev = cell_events(ws, L);
    hipError_t e = dstd::launch_conv_forward(C, g, B, W, w_dtype == DSTD_BF16, at<float>(ws, L.wt),
                                             srt, ev, t_in, t_out, slope, q_idx,
                                             static_cast<hipStream_t>(stream));
    return hip_status(e, "conv forward launch");
}

dstd_status dstd_lif_conv_backward(const dstd_lif_params *p, const dstd_conv_shape *cs, int64_t B,
                                   const float *t_in, const void *W, dstd_dtype w_dtype,
                                   const float *t_out, const float *slope, const int32_t *q_idx,
                                   const float *grad_t_out, float *grad_W, float *grad_t_in,
                                   void *ws, size_t ws_bytes, void *stream) {
    return conv_backward(p, nullptr, cs, B, t_in, W, w_dtype, t_out, slope, q_idx, grad_t_out,
                         grad_W, grad_t_in, ws, ws_bytes, stream);
}

dstd_status dstd_lif_conv_backward_synfire(const dstd_lif_params *p, const dstd_synfire_params *sp,
                                           const dstd_conv_shape *cs, int64_t B,
                                           const float *t_in, const void *W, dstd_dtype w_dtype,
                                           const float *t_out, const float *slope,
                                           const int32_t *q_idx, const float *grad_t_out,
                                           float *grad_W, float *grad_t_in, void *ws,
                                           size_t ws_bytes, void *stream) {
    return conv_backward(p, sp, cs, B, t_in, W, w_dtype, t_out, slope, q_idx, grad_t_out,
                         grad_W, grad_t_in, ws, ws_bytes, stream);
}

size_t dstd_synfire_penalty_workspace_size(int64_t B, int64_t rows, int64_t spatial) {
    if (B < 0 || rows < 0 || spatial < 0) return 0;
    const int64_t n_tb = dstd::synfire_value_blocks(B * rows * spatial);
    return align_up((size_t)(rows + n_tb) * sizeof(float));
}

dstd_status dstd_synfire_penalty(const dstd_synfire_params *sp, int64_t B, int64_t rows,
                                 int64_t spatial, int64_t row_len, const float *t_out,
                                 const void *W, dstd_dtype w_dtype, float *value, void *ws,
                                 size_t ws_bytes, void *stream) {
    if (!sp || !value) return fail(DSTD_ERR_NULL, "synfire parameters and value are required");
    dstd_status s = check_synfire(sp);
    if (s != DSTD_OK) return s;
    if (B < 0 || rows < 0 || spatial < 0 || row_len < 0)
        return fail(DSTD_ERR_SHAPE, "sizes must be >= 0");
    const int64_t lim = (int64_t)1 << 31;
    if (B > 0 && rows > 0 && spatial > 0 && B * rows * spatial >= lim)
        return fail(DSTD_ERR_SHAPE, "B * rows * spatial must be < 2^31");
    if (rows > 0 && row_len > 0 && rows * row_len >= lim)
        return fail(DSTD_ERR_SHAPE, "rows * row_len must be < 2^31");
    if (w_dtype != DSTD_F32 && w_dtype != DSTD_BF16)
        return fail(DSTD_ERR_PARAM, "unknown weight dtype %d", (int)w_dtype);
    if (B * rows * spatial > 0 && !t_out) return fail(DSTD_ERR_NULL, "t_out is NULL");
    if (rows * row_len > 0 && !W) return fail(DSTD_ERR_NULL, "W is NULL");
    if ((s = check_ws(ws, ws_bytes, dstd_synfire_penalty_workspace_size(B, rows, spatial))) != DSTD_OK)
        return s;
    hipError_t e = dstd::launch_synfire_value(make_synfire(sp, nullptr), B, rows, spatial, row_len,
                                              t_out, W, w_dtype == DSTD_BF16,
                                              static_cast<float *>(ws), value,
                                              static_cast<hipStream_t>(stream));
    return hip_status(e, "synfire value launch");
}

}  // extern "C"

namespace {

dstd_status conv_backward(const dstd_lif_params *p, const dstd_synfire_params *sp,
                          const dstd_conv_shape *cs, int64_t B, const float *t_in, const void *W,
                          dstd_dtype w_dtype, const float *t_out, const float *slope,
                          const int32_t *q_idx, const float *grad_t_out, float *grad_W,
                          float *grad_t_in, void *ws, size_t ws_bytes, void *stream) {
    dstd_status s = check_params(p, DSTD_FLAG_CONV_REUSE);
    if (s != DSTD_OK) return s;
    if ((s = check_synfire(sp)) != DSTD_OK) return s;
    dstd::ConvGeom g;
    if ((s = check_conv(cs, B, p->M, &g)) != DSTD_OK) return s;
    if (w_dtype != DSTD_F32 && w_dtype != DSTD_BF16)
        return fail(DSTD_ERR_PARAM, "unknown weight dtype %d", (int)w_dtype);
    if (B > 0 && (!t_in || !t_out || !slope || !q_idx || !grad_t_out))
        return fail(DSTD_ERR_NULL, "t_in, t_out, slope, q_idx and grad_t_out are required");
    if (grad_t_in && B > 0 && !W) return fail(DSTD_ERR_NULL, "W is NULL");
    if (grad_t_in && g.C_out > dstd::kConvMaxCoutDt)
        return fail(DSTD_ERR_UNSUPPORTED, "grad_t_in of a conv layer needs C_out <= %d",
                    dstd::kConvMaxCoutDt);
    ConvWs L = conv_ws_layout(p->M, g, B, true);
    if ((s = check_ws(ws, ws_bytes, L.total)) != DSTD_OK) return s;
    LifConst C = make_const(p);
    dstd::ConvBwdWs bw;
    bw.ev = cell_events(ws, L);
    bw.tri = at<float>(ws, L.tri);
    bw.rend = at<int>(ws, L.rend);
    bw.P = at<float>(ws, L.P);
    bw.part = at<float>(ws, L.part);
    bw.zlive = at<int>(ws, L.zlive);
    bw.wt = at<float>(ws, L.wt);
    const bool reuse = (p->flags & DSTD_FLAG_CONV_REUSE) != 0;
    // With B == 0 the dW kernel still runs (one empty split) and writes zeros.
    hipError_t e = dstd::launch_conv_backward(C, g, B, W, w_dtype == DSTD_BF16, t_in, t_out, slope,
                                              q_idx, grad_t_out, bw, grad_W, grad_t_in,
                                              make_synfire(sp, at<float>(ws, L.dq)), reuse,
                                              static_cast<hipStream_t>(stream));
    return hip_status(e, "conv backward launch");
}

}  // namespace

// ------------------------------------------------------------------ exact --
namespace {

// The exact path uses tau_m, tau_s, threshold, t_max and flags; the grid
// fields (M, t0, dt) do not apply and are not read.
dstd_status check_exact(const dstd_lif_params *p, int64_t B, int64_t N_in, int64_t N_out,
                        dstd_lif_params *q) {
    if (!p) return fail(DSTD_ERR_NULL, "params is NULL");
    *q = *p;
    q->M = 1;
    q->t0 = 0.f;
    q->dt = 1.f;
    q->t_max = INFINITY;
    dstd_status s = check_params(q);
    if (s != DSTD_OK) return s;
    if (isnan(p->t_max)) return fail(DSTD_ERR_PARAM, "t_max must not be NaN");
    if ((s = check_dims(B, N_in, N_out)) != DSTD_OK) return s;
    if (N_in > dstd::kExactMaxIn)
        return fail(DSTD_ERR_UNSUPPORTED, "the exact path sorts at most %d inputs per sample (N_in = %lld)",
                    dstd::kExactMaxIn, (long long)N_in);
    return DSTD_OK;
}

struct ExactWs {
    size_t wt, j, t, len, r_lo, alpha, beta, kl, kmax, n, P, PT, total;
};

ExactWs exact_ws_layout(int64_t B, int64_t N_in, int64_t N_out, bool backward) {
    ExactWs w{};
    size_t off = 0;
    if (backward) {
        w.P = off; off += align_up((size_t)B * (size_t)N_out * 4 * sizeof(float));
        w.PT = off; off += align_up((size_t)B * (size_t)N_out * 4 * sizeof(float));
    } else if (B * N_out > 0) {
        const size_t ns = (size_t)(B * N_in) + dstd::kExactPad;
        w.wt = off; off += align_up((size_t)N_in * (size_t)N_out * sizeof(float));
        w.j = off; off += align_up(ns * sizeof(int));
        w.t = off; off += align_up(ns * sizeof(float));
        w.len = off; off += align_up(ns * sizeof(float));
        w.r_lo = off; off += align_up(ns * sizeof(float));
        w.alpha = off; off += align_up(ns * sizeof(double));
        w.beta = off; off += align_up(ns * sizeof(double));
        w.kl = off; off += align_up(ns * sizeof(double));
        w.kmax = off; off += align_up(ns * sizeof(float));
        w.n = off; off += align_up((size_t)B * sizeof(int));
    }
    w.total = off;
    return w;
}

}  // namespace

extern "C" {

size_t dstd_exact_forward_workspace_size(const dstd_lif_params *p, int64_t B, int64_t N_in,
                                         int64_t N_out) {
    dstd_lif_params q;
    if (check_exact(p, B, N_in, N_out, &q) != DSTD_OK) return 0;
    return exact_ws_layout(B, N_in, N_out, false).total;
}

size_t dstd_exact_backward_workspace_size(const dstd_lif_params *p, int64_t B, int64_t N_in,
                                          int64_t N_out) {
    dstd_lif_params q;
    if (check_exact(p, B, N_in, N_out, &q) != DSTD_OK) return 0;
    return exact_ws_layout(B, N_in, N_out, true).total;
}

dstd_status dstd_exact_forward(const dstd_lif_params *p, int64_t B, int64_t N_in, int64_t N_out,
                               const float *t_in, const void *W, dstd_dtype w_dtype, float *t_out,
                               float *slope, int32_t *k_idx, void *ws, size_t ws_bytes,
                               void *stream) {
    dstd_lif_params q;
    dstd_status s = check_exact(p, B, N_in, N_out, &q);
    if (s != DSTD_OK) return s;
    if (w_dtype != DSTD_F32 && w_dtype != DSTD_BF16)
        return fail(DSTD_ERR_PARAM, "unknown weight dtype %d", (int)w_dtype);
    if (B * N_out > 0 && (!t_out || !slope || !k_idx))
        return fail(DSTD_ERR_NULL, "t_out, slope and k_idx are required");
    if (B * N_in > 0 && !t_in) return fail(DSTD_ERR_NULL, "t_in is NULL");
    if (N_in * N_out > 0 && !W) return fail(DSTD_ERR_NULL, "W is NULL");
    ExactWs L = exact_ws_layout(B, N_in, N_out, false);
    if ((s = check_ws(ws, ws_bytes, L.total)) != DSTD_OK) return s;
    if (B * N_out == 0) return DSTD_OK;
    LifConst C = make_const(&q);
    dstd::ExactRecs rec{at<int>(ws, L.j), at<float>(ws, L.t), at<float>(ws, L.len),
                        at<float>(ws, L.r_lo), at<float>(ws, L.kmax), at<double>(ws, L.alpha),
                        at<double>(ws, L.beta), at<double>(ws, L.kl), at<int>(ws, L.n), N_in};
    hipError_t e = dstd::launch_exact_forward(C, B, N_in, N_out, W, w_dtype == DSTD_BF16,
                                              at<void>(ws, L.wt), rec, t_in, p->t_max, t_out,
                                              slope, k_idx, static_cast<hipStream_t>(stream));
    return hip_status(e, "exact forward launch");
}

dstd_status dstd_exact_backward(const dstd_lif_params *p, int64_t B, int64_t N_in, int64_t N_out,
                                const float *t_in, const void *W, dstd_dtype w_dtype,
                                const float *t_out, const float *slope, const int32_t *k_idx,
                                const float *grad_t_out, float *grad_W, float *grad_t_in,
                                void *ws, size_t ws_bytes, void *stream) {
    dstd_lif_params q;
    dstd_status s = check_exact(p, B, N_in, N_out, &q);
    if (s != DSTD_OK) return s;
    if (w_dtype != DSTD_F32 && w_dtype != DSTD_BF16)
        return fail(DSTD_ERR_PARAM, "unknown weight dtype %d", (int)w_dtype);
    if (B * N_out > 0 && (!t_out || !slope || !k_idx || !grad_t_out))
        return fail(DSTD_ERR_NULL, "t_out, slope, k_idx and grad_t_out are required");
    if (B * N_in > 0 && (grad_W || grad_t_in) && !t_in) return fail(DSTD_ERR_NULL, "t_in is NULL");
    if (grad_t_in && N_in * N_out > 0 && !W) return fail(DSTD_ERR_NULL, "W is NULL");
    ExactWs L = exact_ws_layout(B, N_in, N_out, true);
    if ((s = check_ws(ws, ws_bytes, L.total)) != DSTD_OK) return s;
    LifConst C = make_const(&q);
    // B == 0: the dW kernel still runs and writes zeros; N_out == 0: the
    // dt_in kernel sums nothing and writes zeros
    hipError_t e = dstd::launch_exact_backward(
        C, B, N_in, N_out, W, w_dtype == DSTD_BF16, t_in, p->t_max, t_out, slope, k_idx,
        grad_t_out, at<float4>(ws, L.P), at<float4>(ws, L.PT), grad_W, grad_t_in,
        static_cast<hipStream_t>(stream));
    return hip_status(e, "exact backward launch");
}

}  // extern "C"

// ------------------------------------------------------------------- skip --
namespace {

dstd_status check_skip(int64_t B, int64_t C1, int64_t C2, int64_t HW) {
    if (B < 0 || C1 < 0 || C2 < 0 || HW < 0)
        return fail(DSTD_ERR_SHAPE, "sizes must be >= 0 (B=%lld C1=%lld C2=%lld HW=%lld)",
                    (long long)B, (long long)C1, (long long)C2, (long long)HW);
    if (B > 65535) return fail(DSTD_ERR_SHAPE, "B = %lld exceeds 65535", (long long)B);
    if ((C1 + C2) * HW >= ((int64_t)1 << 30))
        return fail(DSTD_ERR_SHAPE, "(C1 + C2) * HW must be below 2^30 per sample");
    return DSTD_OK;
}

}  // namespace

extern "C" {

dstd_status dstd_skip_delay_concat(int64_t B, int64_t C1, int64_t C2, int64_t HW, const float *t1,
                                   float delay, const float *t2, float *out, void *stream) {
    dstd_status s = check_skip(B, C1, C2, HW);
    if (s != DSTD_OK) return s;
    if (!isfinite(delay)) return fail(DSTD_ERR_PARAM, "delay must be finite");
    if (B * (C1 + C2) * HW == 0) return DSTD_OK;
    if (!out || (C1 * HW > 0 && !t1) || (C2 * HW > 0 && !t2))
        return fail(DSTD_ERR_NULL, "t1, t2 and out are required");
    hipError_t e = dstd::launch_skip_concat(B, C1 * HW, C2 * HW, t1, delay, t2, out,
                                            static_cast<hipStream_t>(stream));
    return hip_status(e, "skip concat launch");
}

dstd_status dstd_skip_delay_concat_backward(int64_t B, int64_t C1, int64_t C2, int64_t HW,
                                            const float *g, float *g1, int32_t accumulate,
                                            float *g2, void *stream) {
    dstd_status s = check_skip(B, C1, C2, HW);
    if (s != DSTD_OK) return s;
    if (accumulate != 0 && accumulate != 1) return fail(DSTD_ERR_PARAM, "accumulate must be 0 or 1");
    if (B * (C1 + C2) * HW == 0) return DSTD_OK;
    if (!g) return fail(DSTD_ERR_NULL, "g is NULL");
    hipError_t e = dstd::launch_skip_split(B, C1 * HW, C2 * HW, g, g1, accumulate, g2,
                                           static_cast<hipStream_t>(stream));
    return hip_status(e, "skip split launch");
}

}  // extern "C"

// ------------------------------------------------------------- multispike --
namespace {

dstd_status check_ms(const dstd_lif_params *p, int64_t B, int64_t N_in, int64_t F_in,
                     int64_t N_out, int64_t F_out) {
    dstd_status s = check_params(p);
    if (s != DSTD_OK) return s;
    if (p->M > dstd::kMsMaxM)
        return fail(DSTD_ERR_UNSUPPORTED, "multi-spike layers support M <= %d (got %d)",
                    dstd::kMsMaxM, p->M);
    if (F_in < 1 || F_out < 1 || F_in > dstd::kMsMaxF || F_out > dstd::kMsMaxF)
        return fail(DSTD_ERR_SHAPE, "F_in and F_out must be in [1, %d]", dstd::kMsMaxF);
    if ((s = check_dims(B, N_in * F_in, N_out)) != DSTD_OK) return s;
    if (N_out * F_out >= ((int64_t)1 << 24) || N_out >= ((int64_t)1 << 22) ||
        B * N_out * (p->M + 1) >= ((int64_t)1 << 31))
        return fail(DSTD_ERR_SHAPE, "N_out (< 2^22), N_out * F_out (< 2^24) or B * N_out * (M + 1) "
                    "(< 2^31) too large");
    return DSTD_OK;
}

struct MsWs {
    size_t ev, wt, G, P, part, sj, sr, sL, sR, nvalid, rs, total;
    int n_buf;
};

// forward: the records of every input spike sorted by event row (as the TTFS
// forward's lists) and W^T; backward: per-spike events, G, dW partials and
// dt_in buffers
MsWs ms_ws_layout(int M, int64_t B, int64_t N_in, int64_t F_in, int64_t N_out, bool backward) {
    MsWs w{};
    size_t off = 0;
    const size_t n = (size_t)(B * N_in * F_in);
    if (backward) {
        w.ev = off; off += align_up(n * 5 * sizeof(float));
        w.G = off; off += align_up((size_t)B * (size_t)(M + 1) * (size_t)N_out * sizeof(float));
        w.n_buf = (int)dstd::back_buf_cap(B, N_in, F_in, N_out);
        w.P = off; off += align_up(n * (size_t)w.n_buf * sizeof(float));
        const size_t cap = (size_t)dstd::back_split_cap(B, N_in, N_out);
        w.part = off; off += align_up((cap > 1 ? cap : 0) * (size_t)N_in * (size_t)N_out * sizeof(float));
        // no less than the forward's, so that one buffer serves both
        off = std::max(off, B * N_out == 0 ? 0 : ms_ws_layout(M, B, N_in, F_in, N_out, false).total);
    } else {
        const size_t ns = n + dstd::kSortPad;
        w.sj = off; off += align_up(ns * sizeof(int));
        w.sr = off; off += align_up(ns * sizeof(int));
        w.sL = off; off += align_up(ns * sizeof(float));
        w.sR = off; off += align_up(ns * sizeof(float));
        w.nvalid = off; off += align_up((size_t)B * sizeof(int));
        w.rs = off; off += align_up((size_t)B * (M + 4) * sizeof(int));
        w.wt = off; off += align_up((size_t)N_in * (size_t)N_out * sizeof(float));
    }
    w.total = off;
    return w;
}

}  // namespace

extern "C" {

size_t dstd_lif_multispike_forward_workspace_size(const dstd_lif_params *p, int64_t B,
                                                  int64_t N_in, int64_t F_in, int64_t N_out,
                                                  int64_t F_out) {
    if (check_ms(p, B, N_in, F_in, N_out, F_out) != DSTD_OK) return 0;
    if (B * N_out == 0) return 0;
    return ms_ws_layout(p->M, B, N_in, F_in, N_out, false).total;
}

size_t dstd_lif_multispike_backward_workspace_size(const dstd_lif_params *p, int64_t B,
                                                   int64_t N_in, int64_t F_in, int64_t N_out,
                                                   int64_t F_out) {
    if (check_ms(p, B, N_in, F_in, N_out, F_out) != DSTD_OK) return 0;
    return ms_ws_layout(p->M, B, N_in, F_in, N_out, true).total;
}

dstd_status dstd_lif_multispike_forward(const dstd_lif_params *p, int64_t B, int64_t N_in,
                                        int64_t F_in, int64_t N_out, int64_t F_out,
                                        const float *t_in, const void *W, dstd_dtype w_dtype,
                                        float *t_out, float *slope, int32_t *q_idx, float *cur,
                                        void *ws, size_t ws_bytes, void *stream) {
    dstd_status s = check_ms(p, B, N_in, F_in, N_out, F_out);
    if (s != DSTD_OK) return s;
    if (w_dtype != DSTD_F32 && w_dtype != DSTD_BF16)
        return fail(DSTD_ERR_PARAM, "unknown weight dtype %d", (int)w_dtype);
    if (B * N_out == 0) return DSTD_OK;
    if (!t_out || !slope || !q_idx || !cur)
        return fail(DSTD_ERR_NULL, "t_out, slope, q_idx and cur are required");
    if (N_in > 0 && !t_in) return fail(DSTD_ERR_NULL, "t_in is NULL");
    if (N_in > 0 && !W) return fail(DSTD_ERR_NULL, "W is NULL");
    MsWs L = ms_ws_layout(p->M, B, N_in, F_in, N_out, false);
    if ((s = check_ws(ws, ws_bytes, L.total)) != DSTD_OK) return s;
    LifConst C = make_const(p);
    dstd::SortedEv srt{at<int>(ws, L.sj), at<int>(ws, L.sr), at<float>(ws, L.sL),
                       at<float>(ws, L.sR), N_in * F_in, at<int>(ws, L.rs)};
    hipError_t e = dstd::launch_ms_forward(C, B, N_in, F_in, N_out, F_out, W,
                                           w_dtype == DSTD_BF16, at<void>(ws, L.wt), srt,
                                           at<int>(ws, L.nvalid), t_in, t_out, slope, q_idx, cur,
                                           static_cast<hipStream_t>(stream));
    return hip_status(e, "multi-spike forward launch");
}

dstd_status dstd_lif_multispike_backward(const dstd_lif_params *p, int64_t B, int64_t N_in,
                                         int64_t F_in, int64_t N_out, int64_t F_out,
                                         const float *t_in, const void *W, dstd_dtype w_dtype,
                                         const float *t_out, const float *slope,
                                         const int32_t *q_idx, const float *cur,
                                         const float *grad_t_out, float *grad_W,
                                         float *grad_t_in, void *ws, size_t ws_bytes,
                                         void *stream) {
    dstd_status s = check_ms(p, B, N_in, F_in, N_out, F_out);
    if (s != DSTD_OK) return s;
    if (w_dtype != DSTD_F32 && w_dtype != DSTD_BF16)
        return fail(DSTD_ERR_PARAM, "unknown weight dtype %d", (int)w_dtype);
    if (B * N_out > 0 && (!t_out || !slope || !q_idx || !cur || !grad_t_out))
        return fail(DSTD_ERR_NULL, "t_out, slope, q_idx, cur and grad_t_out are required");
    if (B * N_in > 0 && !t_in) return fail(DSTD_ERR_NULL, "t_in is NULL");
    if (grad_t_in && N_in * N_out > 0 && !W) return fail(DSTD_ERR_NULL, "W is NULL");
    MsWs L = ms_ws_layout(p->M, B, N_in, F_in, N_out, true);
    if ((s = check_ws(ws, ws_bytes, L.total)) != DSTD_OK) return s;
    LifConst C = make_const(p);
    const dstd::DenseBwdWs bw{at<float>(ws, L.ev), at<float>(ws, L.G), at<float>(ws, L.P),
                              at<float>(ws, L.part), L.n_buf};
    // B == 0: the contraction still runs and writes zeros to dW; N_out == 0:
    // dt_in sums nothing and is zeros
    hipError_t e = dstd::launch_ms_backward(C, B, N_in, F_in, N_out, F_out, W, w_dtype == DSTD_BF16,
                                            bw, t_in, t_out, slope, q_idx, cur, grad_t_out, grad_W,
                                            grad_t_in, static_cast<hipStream_t>(stream));
    return hip_status(e, "multi-spike backward launch");
}

}  // extern "C"

// ------------------------------------------------------------- optimising --
namespace {

constexpr uint32_t kListMagic = 0x4c545344;

dstd_status check_dtype(int32_t t, const char *what) {
    if (t != DSTD_F32 && t != DSTD_BF16) return fail(DSTD_ERR_PARAM, "unknown %s dtype %d", what, (int)t);
    return DSTD_OK;
}

int64_t dtype_bytes(int32_t t) { return t == DSTD_BF16 ? 2 : 4; }

// A launch takes one block of at most 512 threads per chunk, and fewer than
// 2^32 threads.
constexpr int64_t kMaxChunks = (int64_t)1 << 23;

// most chunks that the list can have, wherever its tensors lie
dstd_status check_counts(int64_t n, const dstd_tensor *t, int64_t *n_chunks) {
    if (n < 0) return fail(DSTD_ERR_SHAPE, "n_tensors must be >= 0");
    if (n > 0 && !t) return fail(DSTD_ERR_NULL, "tensors is NULL");
    if (n >= (int64_t)1 << 31) return fail(DSTD_ERR_SHAPE, "too many tensors");
    int64_t c = 0;
    for (int64_t k = 0; k < n; ++k) {
        if (t[k].n < 0 || t[k].n >= kMaxChunks * dstd::kOptChunk)
            return fail(DSTD_ERR_SHAPE, "tensor %lld: n = %lld must be in [0, 2^35)", (long long)k,
                        (long long)t[k].n);
        c += dstd::opt_chunks(t[k].n, dstd::kOptAlign - 1);
        if (c >= kMaxChunks) return fail(DSTD_ERR_SHAPE, "the list's tensors are too large together");
    }
    *n_chunks = c;
    return DSTD_OK;
}

size_t list_bytes(int64_t n_chunks) {
    return std::max(kAlign, align_up((size_t)n_chunks * sizeof(dstd::OptChunk)));
}

struct Range { uintptr_t lo, hi; int64_t k; };

dstd_status add_range(std::vector<Range> &r, const void *p, int64_t n, int64_t bytes, int64_t k,
                      const char *what) {
    const uintptr_t a = (uintptr_t)p;
    if (a % (uintptr_t)bytes != 0)
        return fail(DSTD_ERR_PARAM, "tensor %lld: %s is not aligned to its type", (long long)k, what);
    if (n > 0) r.push_back(Range{a, a + (uintptr_t)(n * bytes), k});
    return DSTD_OK;
}

dstd_status check_tensor(const dstd_tensor &t, int64_t k, std::vector<Range> &r) {
    dstd_status s;
    if (t.n == 0) return DSTD_OK;
    if (!t.g) return fail(DSTD_ERR_NULL, "tensor %lld: g is NULL", (long long)k);
    if ((s = check_dtype(t.g_dtype, "gradient")) != DSTD_OK) return s;
    if ((s = add_range(r, t.g, t.n, dtype_bytes(t.g_dtype), k, "g")) != DSTD_OK) return s;
    if (t.out) {
        if ((s = check_dtype(t.out_dtype, "out")) != DSTD_OK) return s;
        if (t.out == t.g && t.out_dtype != t.g_dtype)
            return fail(DSTD_ERR_PARAM, "tensor %lld: in place, out has the type of g", (long long)k);
        if (t.out != t.g &&
            (s = add_range(r, t.out, t.n, dtype_bytes(t.out_dtype), k, "out")) != DSTD_OK)
            return s;
    }
    if (!t.w) {
        if (t.w32 || t.m || t.v)
            return fail(DSTD_ERR_NULL, "tensor %lld: w32, m and v go with w", (long long)k);
        return DSTD_OK;
    }
    if (!t.m || !t.v) return fail(DSTD_ERR_NULL, "tensor %lld: m and v are required with w", (long long)k);
    if ((s = check_dtype(t.w_dtype, "weight")) != DSTD_OK) return s;
    if (t.w32 && t.w_dtype != DSTD_BF16)
        return fail(DSTD_ERR_PARAM, "tensor %lld: w32 goes with bf16 weights", (long long)k);
    if (!(isfinite(t.lr_scale) && t.lr_scale >= 0.f && isfinite(t.decay_scale) && t.decay_scale >= 0.f))
        return fail(DSTD_ERR_PARAM, "tensor %lld: lr_scale and decay_scale must be finite and >= 0",
                    (long long)k);
    if ((s = add_range(r, t.w, t.n, dtype_bytes(t.w_dtype), k, "w")) != DSTD_OK) return s;
    if (t.w32 && (s = add_range(r, t.w32, t.n, 4, k, "w32")) != DSTD_OK) return s;
    if ((s = add_range(r, t.m, t.n, 4, k, "m")) != DSTD_OK) return s;
    return add_range(r, t.v, t.n, 4, k, "v");
}

dstd_status check_list(const dstd_tensor_list *l) {
    if (!l) return fail(DSTD_ERR_NULL, "list is NULL");
    if (l->magic != kListMagic || !l->mem || l->n_tensors < 0 || l->n_chunks < 0 ||
        l->n_chunks >= kMaxChunks)
        return fail(DSTD_ERR_PARAM, "not a list that dstd_tensor_list_build has filled");
    return DSTD_OK;
}

// The place of a tensor's first element among kOptAlign elements that most of
// its arrays share (views at one offset of flat buffers share it; the others'
// accesses are right at any place, 5 to 25 % slower where they split lines).
uint16_t tensor_phase(const dstd_tensor &t) {
    const struct { const void *p; int64_t bytes; } arr[] = {
        {t.g, dtype_bytes(t.g_dtype)}, {t.w, dtype_bytes(t.w_dtype)}, {t.w32, 4}, {t.m, 4}, {t.v, 4},
        {t.out, dtype_bytes(t.out_dtype)}};
    const auto place = [](const void *p, int64_t bytes) {
        return (uint16_t)((uintptr_t)p / (uintptr_t)bytes % dstd::kOptAlign);
    };
    uint16_t best = 0;
    int most = 0;
    for (const auto &a : arr) {
        if (!a.p) continue;
        int n = 0;
        for (const auto &b : arr) n += b.p && place(b.p, b.bytes) == place(a.p, a.bytes);
        if (n > most) {
            most = n;
            best = place(a.p, a.bytes);
        }
    }
    return best;
}

struct OptWs {
    size_t part, at, total;
};
OptWs opt_ws_layout() {
    OptWs w{};
    w.part = 0;
    w.at = align_up(dstd::kOptMaxPart * sizeof(double));
    w.total = w.at + align_up(sizeof(dstd::OptStep));
    return w;
}

dstd::OptList opt_list(const dstd_tensor_list *l) {
    return dstd::OptList{static_cast<const dstd::OptChunk *>(l->mem), (int)l->n_chunks, l->g_bytes,
                         l->out_bytes, l->w_bytes, l->g_types};
}

// Places that a call of a list reads or writes beside the list's arrays: the
// table, the workspace, and the scalars on the device. None may lie in another
// if one of them is written: blocks that read the other would see either value
// (and addresses, where it is the table's).
struct Place {
    const void *p;  // null: none
    size_t bytes, align;
    bool written;
    const char *what;
};
template <size_t N> dstd_status check_places(const Place (&places)[N]) {
    for (size_t i = 0; i < N; ++i) {
        const Place &a = places[i];
        if (!a.p) continue;
        const uintptr_t lo = (uintptr_t)a.p;
        if (lo % a.align != 0) return fail(DSTD_ERR_PARAM, "%s is not aligned to %zu bytes", a.what, a.align);
        for (size_t k = 0; k < i; ++k) {
            const Place &b = places[k];
            const uintptr_t at = (uintptr_t)b.p;
            if (b.p && (a.written || b.written) && lo < at + b.bytes && at < lo + a.bytes)
                return fail(DSTD_ERR_PARAM, "%s and %s overlap", b.what, a.what);
        }
    }
    return DSTD_OK;
}
Place table_place(const dstd_tensor_list *l) {
    return Place{l->mem, (size_t)l->n_chunks * sizeof(dstd::OptChunk), kAlign, false, "the list's table"};
}
Place ws_place(const void *ws) { return Place{ws, opt_ws_layout().total, kAlign, true, "the workspace"}; }
Place norm_place(const float *norm, bool given) { return Place{norm, 4, 4, !given, "norm"}; }

// beta in two fp32 parts, hi below beta (the kernels' adamw_one needs lo > 0)
void split_beta(double beta, float *hi, float *lo) {
    *hi = (float)beta;
    if ((double)*hi >= beta) *hi = nextafterf(*hi, 0.f);
    *lo = (float)(beta - (double)*hi);
}

dstd_status check_max_norm(double max_norm) {
    if (!(max_norm > 0.0)) return fail(DSTD_ERR_PARAM, "max_norm must be > 0 or +inf (got %g)", max_norm);
    return DSTD_OK;
}

dstd_status check_norm(const float *norm, int32_t norm_given) {
    if (norm_given != 0 && norm_given != 1) return fail(DSTD_ERR_PARAM, "norm_given must be 0 or 1");
    if (norm_given && !norm) return fail(DSTD_ERR_NULL, "norm is NULL but said to be given");
    return DSTD_OK;
}

}  // namespace

extern "C" {

size_t dstd_tensor_list_size(int64_t n_tensors, const dstd_tensor *tensors) {
    int64_t nc;
    if (check_counts(n_tensors, tensors, &nc) != DSTD_OK) return 0;
    return list_bytes(nc);
}

dstd_status dstd_tensor_list_build(int64_t n_tensors, const dstd_tensor *tensors, void *mem,
                                   size_t mem_bytes, dstd_tensor_list *list, void *stream) try {
    int64_t nc;
    dstd_status s = check_counts(n_tensors, tensors, &nc);
    if (s != DSTD_OK) return s;
    if (!list) return fail(DSTD_ERR_NULL, "list is NULL");
    const size_t need = list_bytes(nc);
    std::vector<Range> ranges;
    ranges.reserve((size_t)n_tensors * 6 + 1);
    uint32_t has_weights = 1;
    for (int64_t k = 0; k < n_tensors; ++k) {
        if ((s = check_tensor(tensors[k], k, ranges)) != DSTD_OK) return s;
        if (tensors[k].n > 0 && !tensors[k].w) has_weights = 0;
    }
    if ((s = check_ws(mem, mem_bytes, need)) != DSTD_OK) return s;
    ranges.push_back(Range{(uintptr_t)mem, (uintptr_t)mem + need, -1});
    std::sort(ranges.begin(), ranges.end(), [](const Range &a, const Range &b) { return a.lo < b.lo; });
    for (size_t i = 1; i < ranges.size(); ++i)
        if (ranges[i].lo < ranges[i - 1].hi)
            return fail(DSTD_ERR_PARAM, "arrays of tensors %lld and %lld overlap (-1: the list's own memory)",
                        (long long)ranges[i - 1].k, (long long)ranges[i].k);
    auto *chunks = static_cast<dstd::OptChunk *>(mem);
    int64_t c = 0, gb = 0, ob = 0, wb = 0;
    uint32_t types = 0;
    for (int64_t k0 = 0; k0 < n_tensors; k0 += dstd::kOptBatch) {
        const int count = (int)std::min<int64_t>(dstd::kOptBatch, n_tensors - k0);
        dstd::OptBatch b{};
        for (int i = 0; i < count; ++i) {
            const dstd_tensor &t = tensors[k0 + i];
            dstd::OptChunk &o = b.ten[i];
            o.g = t.g;
            o.out = t.out ? t.out : t.g;
            o.w = t.w;
            o.w32 = t.w32;
            o.m = t.m;
            o.v = t.v;
            o.lr_scale = t.lr_scale;
            o.decay_scale = t.decay_scale;
            o.types = (t.g_dtype == DSTD_BF16 ? dstd::kOptGradBf16 : 0) |
                      ((t.out ? t.out_dtype : t.g_dtype) == DSTD_BF16 ? dstd::kOptOutBf16 : 0) |
                      (t.w_dtype == DSTD_BF16 ? dstd::kOptWeightBf16 : 0);
            o.lead = tensor_phase(t);
            b.n[i] = t.n;
            b.chunk0[i] = c;
            c += dstd::opt_chunks(t.n, o.lead);
            gb += t.n * dtype_bytes(t.g_dtype);
            if (t.n > 0) types |= t.g_dtype == DSTD_BF16 ? dstd::kOptListBf16 : dstd::kOptListF32;
            if (o.out != o.g) ob += t.n * dtype_bytes(t.out_dtype);
            if (t.w) wb += t.n * (8 + dtype_bytes(t.w_dtype) + (t.w32 ? 4 : 0));
        }
        hipError_t e = dstd::launch_tensor_list(b, count, chunks, static_cast<hipStream_t>(stream));
        if (e != hipSuccess) return hip_status(e, "tensor list launch");
    }
    *list = dstd_tensor_list{mem, n_tensors, c, gb, ob, wb, kListMagic, has_weights, types};
    return DSTD_OK;
} catch (const std::exception &e) {
    return fail(DSTD_ERR_UNSUPPORTED, "tensor list: %s", e.what());
}

size_t dstd_tensor_list_workspace_size(const dstd_tensor_list *list) {
    if (check_list(list) != DSTD_OK) return 0;
    return opt_ws_layout().total;
}

dstd_status dstd_grad_norm(const dstd_tensor_list *list, float *norm, void *ws, size_t ws_bytes,
                           void *stream) {
    dstd_status s = check_list(list);
    if (s != DSTD_OK) return s;
    if (!norm) return fail(DSTD_ERR_NULL, "norm is NULL");
    const OptWs w = opt_ws_layout();
    if ((s = check_ws(ws, ws_bytes, w.total)) != DSTD_OK) return s;
    if ((s = check_places({table_place(list), ws_place(ws), norm_place(norm, false)})) != DSTD_OK) return s;
    const dstd::OptList L = opt_list(list);
    const dstd::OptNorm nm{at<double>(ws, w.part), dstd::opt_norm_blocks(L.n_chunks), norm, INFINITY};
    return hip_status(dstd::launch_grad_norm(L, nm, static_cast<hipStream_t>(stream)), "grad_norm launch");
}

dstd_status dstd_grad_clip(const dstd_tensor_list *list, double max_norm, float *norm,
                           int32_t norm_given, void *ws, size_t ws_bytes, void *stream) {
    dstd_status s = check_list(list);
    if (s != DSTD_OK) return s;
    if ((s = check_max_norm(max_norm)) != DSTD_OK) return s;
    if ((s = check_norm(norm, norm_given)) != DSTD_OK) return s;
    const OptWs w = opt_ws_layout();
    if ((s = check_ws(ws, ws_bytes, w.total)) != DSTD_OK) return s;
    if ((s = check_places({table_place(list), ws_place(ws), norm_place(norm, norm_given)})) != DSTD_OK)
        return s;
    const dstd::OptList L = opt_list(list);
    const dstd::OptNorm nm{at<double>(ws, w.part), norm_given ? -1 : dstd::opt_norm_blocks(L.n_chunks),
                           norm, max_norm};
    return hip_status(dstd::launch_grad_clip(L, nm, static_cast<hipStream_t>(stream)), "grad_clip launch");
}

dstd_status dstd_adamw_step(const dstd_tensor_list *list, const dstd_adamw_params *p,
                            const float *lr, int64_t *step, float *norm, int32_t norm_given,
                            void *ws, size_t ws_bytes, void *stream) {
    dstd_status s = check_list(list);
    if (s != DSTD_OK) return s;
    if (!p) return fail(DSTD_ERR_NULL, "params is NULL");
    if (!(isfinite((float)p->lr) && p->lr >= 0.0)) return fail(DSTD_ERR_PARAM, "lr must be finite and >= 0");
    if (!(p->beta1 >= 0.0 && (float)p->beta1 < 1.f && p->beta2 >= 0.0 && (float)p->beta2 < 1.f))
        return fail(DSTD_ERR_PARAM, "need 0 <= beta1, beta2 < 1 in fp32");
    if (!(isfinite((float)p->eps) && (float)p->eps > 0.f))
        return fail(DSTD_ERR_PARAM, "eps must be finite and > 0 in fp32");
    if (!(isfinite((float)p->weight_decay) && p->weight_decay >= 0.0))
        return fail(DSTD_ERR_PARAM, "weight_decay must be finite and >= 0");
    if ((s = check_max_norm(p->max_norm)) != DSTD_OK) return s;
    if ((s = check_norm(norm, norm_given)) != DSTD_OK) return s;
    if (!step) return fail(DSTD_ERR_NULL, "step is NULL");
    if (!list->has_weights)
        return fail(DSTD_ERR_NULL, "a tensor of the list has no weights");
    const OptWs w = opt_ws_layout();
    if ((s = check_ws(ws, ws_bytes, w.total)) != DSTD_OK) return s;
    if ((s = check_places({table_place(list), ws_place(ws), norm_place(norm, norm_given),
                           Place{lr, 4, 4, false, "lr"}, Place{step, 8, 8, true, "step"}})) != DSTD_OK)
        return s;
    const dstd::OptList L = opt_list(list);
    const bool sums = !norm_given && (norm || isfinite(p->max_norm));
    const dstd::OptNorm nm{at<double>(ws, w.part), sums ? dstd::opt_norm_blocks(L.n_chunks) : -1,
                           norm, p->max_norm};
    dstd::OptAdamW hp{};
    hp.beta1 = p->beta1;
    hp.beta2 = p->beta2;
    split_beta(p->beta1, &hp.b1, &hp.b1_lo);
    split_beta(p->beta2, &hp.b2, &hp.b2_lo);
    hp.a1 = (float)(1.0 - p->beta1);
    hp.a2 = (float)(1.0 - p->beta2);
    hp.eps = (float)p->eps;
    hp.lr = (float)p->lr;
    hp.decay = (float)p->weight_decay;
    return hip_status(dstd::launch_adamw(L, nm, hp, lr, step, at<dstd::OptStep>(ws, w.at),
                                         static_cast<hipStream_t>(stream)), "adamw launch");
}

}  // extern "C"

// --------------------------------------------------------------- answers --
namespace {

dstd_status check_rows(int64_t B, int64_t N, int64_t ld, const char *what) {
    if (B < 0 || B > 65535 || N < 1 || N >= (1 << 24))
        return fail(DSTD_ERR_SHAPE, "need 0 <= B <= 65535 and 1 <= N < 2^24");
    if (ld < N || ld > (int64_t)1 << 40)
        return fail(DSTD_ERR_SHAPE, "rows of %s lie %lld elements apart, need N to 2^40", what, (long long)ld);
    return DSTD_OK;
}
size_t rows_bytes(int64_t B, int64_t N, int64_t ld, size_t elem) {
    return B > 0 ? ((size_t)(B - 1) * (size_t)ld + (size_t)N) * elem : 0;
}
dstd_status check_top(int64_t K, int64_t N) {
    if (K < 1 || K > N) return fail(DSTD_ERR_SHAPE, "need 1 <= K <= N");
    if (K > DSTD_MAX_TOP) return fail(DSTD_ERR_UNSUPPORTED, "K = %lld exceeds DSTD_MAX_TOP = %d", (long long)K, DSTD_MAX_TOP);
    return DSTD_OK;
}

dstd_status check_scores(const dstd_scores *s) {
    if (!s) return fail(DSTD_ERR_NULL, "scores are NULL");
    dstd_status st = check_rows(s->B, s->N, s->ld, "the scores");
    if (st != DSTD_OK) return st;
    if (s->dtype != DSTD_F32 && s->dtype != DSTD_BF16) return fail(DSTD_ERR_PARAM, "unknown dtype %d", s->dtype);
    if (!isfinite((float)s->scale) || (float)s->scale == 0.f)
        return fail(DSTD_ERR_PARAM, "scale must be finite and not 0 in fp32 (got %g)", s->scale);
    return DSTD_OK;
}

dstd::ScoreRows score_rows(const dstd_scores *s) {
    const bool neg = s->scale < 0.0;
    dstd::ScoreRows r{};
    r.x = s->x;
    r.B = s->B;
    r.N = s->N;
    r.ld = s->ld;
    r.bf16 = s->dtype == DSTD_BF16;
    r.cap = isfinite(s->cap) ? s->cap : neg ? INFINITY : -INFINITY;
    r.flip = neg ? 0x80000000u : 0u;
    r.scale = fabs(s->scale);
    return r;
}
Place scores_place(const dstd_scores *s) {
    const size_t elem = s->dtype == DSTD_BF16 ? 2 : 4;
    return Place{s->x, rows_bytes(s->B, s->N, s->ld, elem), elem, false, "the scores"};
}

dstd_status check_sample(const dstd_sample_params *p) {
    if (!p) return fail(DSTD_ERR_NULL, "params is NULL");
    if (p->top_k < 0) return fail(DSTD_ERR_PARAM, "top_k must be >= 0");
    if (!(p->top_p > 0.0 && p->top_p <= 1.0)) return fail(DSTD_ERR_PARAM, "need 0 < top_p <= 1 (got %g)", p->top_p);
    if (!(p->min_p >= 0.0 && p->min_p <= 1.0)) return fail(DSTD_ERR_PARAM, "need 0 <= min_p <= 1 (got %g)", p->min_p);
    return DSTD_OK;
}

}  // namespace

extern "C" {

dstd_status dstd_top_logits(const dstd_scores *s, int64_t K, int32_t *idx, float *logit, float *rest,
                            void *stream) {
    dstd_status st = check_scores(s);
    if (st != DSTD_OK) return st;
    if ((st = check_top(K, s->N)) != DSTD_OK) return st;
    // the sum's exponents are formed in base 2
    if (rest && !isfinite((float)(s->scale * 1.4426950408889634)))
        return fail(DSTD_ERR_PARAM, "scale * log2(e) must be finite in fp32 where rest is wanted (scale %g)", s->scale);
    if (s->B > 0 && (!s->x || !idx || !logit)) return fail(DSTD_ERR_NULL, "x, idx and logit are required");
    const size_t bk = (size_t)(s->B * K) * 4;
    if ((st = check_places({scores_place(s), Place{idx, bk, 4, true, "idx"}, Place{logit, bk, 4, true, "logit"},
                            Place{rest, (size_t)s->B * 4, 4, true, "rest"}})) != DSTD_OK)
        return st;
    const dstd::TopJob j{score_rows(s), (int)K, idx, logit, rest};
    return hip_status(dstd::launch_top_logits(j, static_cast<hipStream_t>(stream)), "top_logits launch");
}

size_t dstd_distill_workspace_size(int64_t B, int64_t N, int64_t K) {
    if (check_rows(B, N, N, "t_out") != DSTD_OK || check_top(K, N) != DSTD_OK) return 0;
    return align_up((size_t)(B * dstd::distill_parts(B, N)) * sizeof(float2));
}

dstd_status dstd_distill_grad(int64_t B, int64_t N, int64_t K, const float *t_out, int64_t ld_t,
                              const int32_t *idx, const void *logit, dstd_dtype logit_dtype,
                              const float *rest, float tau_soft, float t_cap, float weight,
                              int32_t accumulate, float *grad_t, int64_t ld_g, float *loss, void *ws,
                              size_t ws_bytes, void *stream) {
    dstd_status st = check_rows(B, N, ld_t, "t_out");
    if (st != DSTD_OK) return st;
    if (grad_t && (st = check_rows(B, N, ld_g, "grad_t")) != DSTD_OK) return st;
    if ((st = check_top(K, N)) != DSTD_OK) return st;
    if (logit_dtype != DSTD_F32 && logit_dtype != DSTD_BF16)
        return fail(DSTD_ERR_PARAM, "unknown dtype %d", (int)logit_dtype);
    if (!(isfinite(tau_soft) && tau_soft > 0.f && isfinite(1.4426950408889634f / tau_soft)))
        return fail(DSTD_ERR_PARAM, "tau_soft must be > 0, and 1 / tau_soft finite");
    if (!isfinite(t_cap)) return fail(DSTD_ERR_PARAM, "t_cap must be finite");
    if (!(weight >= 0.f && isfinite(weight * (1.f / tau_soft))))
        return fail(DSTD_ERR_PARAM, "weight must be >= 0, and weight / tau_soft finite");
    if (accumulate != 0 && accumulate != 1) return fail(DSTD_ERR_PARAM, "accumulate must be 0 or 1");
    if (!loss || (B > 0 && (!t_out || !idx || !logit)))
        return fail(DSTD_ERR_NULL, "t_out, idx, logit and loss are required");
    const size_t need = dstd_distill_workspace_size(B, N, K);
    if ((st = check_ws(ws, ws_bytes, need)) != DSTD_OK) return st;
    const size_t le = dtype_bytes(logit_dtype), bk = (size_t)(B * K);
    if ((st = check_places({Place{t_out, rows_bytes(B, N, ld_t, 4), 4, false, "t_out"},
                            Place{idx, bk * 4, 4, false, "idx"}, Place{logit, bk * le, le, false, "logit"},
                            Place{rest, (size_t)B * 4, 4, false, "rest"},
                            Place{grad_t, rows_bytes(B, N, ld_g, 4), 4, true, "grad_t"},
                            Place{loss, (size_t)(B + 1) * 4, 4, true, "loss"},
                            Place{need ? ws : nullptr, need, kAlign, true, "the workspace"}})) != DSTD_OK)
        return st;
    dstd::KdArgs a{};
    a.N = (int)N;
    a.K = (int)K;
    a.t = t_out;
    a.ld_t = ld_t;
    a.idx = idx;
    a.rest = rest;
    a.inv = 1.f / tau_soft;
    a.c2 = (float)(1.4426950408889634 / (double)tau_soft);
    a.t_cap = t_cap;
    a.weight = weight;
    a.accumulate = accumulate;
    a.grad = grad_t;
    a.ld_g = ld_g;
    a.loss = loss;
    a.part = static_cast<float2 *>(ws);
    return hip_status(dstd::launch_distill(a, B, logit, logit_dtype == DSTD_BF16, static_cast<hipStream_t>(stream)),
                      "distill launch");
}

dstd_status dstd_sample(const dstd_scores *s, const dstd_sample_params *p, const float *u, int32_t *choice,
                        float *logp, void *stream) {
    dstd_status st = check_scores(s);
    if (st != DSTD_OK) return st;
    if ((st = check_sample(p)) != DSTD_OK) return st;
    if (s->B > 0 && (!s->x || !u || !choice)) return fail(DSTD_ERR_NULL, "x, u and choice are required");
    const size_t b4 = (size_t)s->B * 4;
    if ((st = check_places({scores_place(s), Place{u, b4, 4, false, "u"}, Place{choice, b4, 4, true, "choice"},
                            Place{logp, b4, 4, true, "logp"}})) != DSTD_OK)
        return st;
    dstd::SampleJob j{};
    j.in = score_rows(s);
    int bits = 0;  // ceil(log2 N)
    while (((int64_t)1 << bits) < s->N) ++bits;
    j.shift = std::min(51, 62 - bits);
    j.top_k = p->top_k < s->N ? (int)p->top_k : 0;
    j.top_p = p->top_p;
    j.min_p = p->min_p;
    j.u = u;
    j.choice = choice;
    j.logp = logp;
    return hip_status(dstd::launch_sample(j, static_cast<hipStream_t>(stream)), "sample launch");
}

}  // extern "C"
