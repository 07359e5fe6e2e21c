"""Distillation of rows whose times lie far from 0 in units of tau_soft: nothing fires, only
named classes fire, times of 1e6 to 1e37 tau apart or next to each other.

Tolerances, in half steps H of fp32. A probability e^d takes the difference of two inputs, the
scale and their product with half a step each, so 3 H |d| of it (it is 0 in fp32 from |d| = 88
on, and its size bounds the error from there); exp2 is two half steps off, again at each of
the some 30 places where partial sums are joined, and a thread adds 64 terms at most one by
one. A logarithm of a sum is as far off as the sum relatively, a logit difference by 3 H of
itself, and a row's loss adds K terms, 4 of a lane one by one and 6 times over the lanes."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

H = 2.0 ** -24
FMAX = float(np.finfo(np.float32).max)


def eps(N):
    return H * (3 * math.log(N + 1) + 2 * 30 + 4 + 64)


def _torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2607_14672_amd import dstd
    return torch, dstd


def reference(t, idx, logit, rest, tau, t_cap, weight, E=None):
    """(loss, its tolerance, gradient, its tolerance) in 64 bits, differences before they are
    scaled, so that digits of huge logits that cancel are not lost here either. E: how far a
    sum may be off, relatively."""
    B, N = t.shape
    loss, ltol, grad, gtol = np.zeros(B), np.zeros(B), np.zeros((B, N)), np.zeros((B, N))
    E = eps(N) if E is None else E
    for b in range(B):
        fired = np.isfinite(t[b])
        y = -np.where(fired, t[b], np.float32(t_cap)).astype(np.float64)
        cls, l = idx[b].astype(np.int64), logit[b].astype(np.float64)
        r = -math.inf if rest is None else float(rest[b])
        lm = max(l.max(), r)
        e, er = np.exp(l - lm), math.exp(r - lm)
        P = e.sum() + er
        p, pr, lp = e / P, er / P, (l - lm) - math.log(P)
        named = np.zeros(N, dtype=bool)
        named[cls] = True
        ym, yr = y.max(), y[~named].max()
        R, Z = np.exp((y[~named] - yr) / tau).sum(), np.exp((y - ym) / tau).sum()
        lq = (y - ym) / tau - math.log(Z)
        lR = (yr - ym) / tau + math.log(R) - math.log(Z)
        loss[b] = np.sum(np.where(p > 0, p * (lp - lq[cls]), 0))
        near = lambda d: np.minimum(d, 110.0)  # where its exponential is 0 in fp32
        part = (np.abs(lp) + np.abs(lq[cls]) + 1) * (2 * E + H * (3 * near(lm - l) + 30))
        ltol[b] = np.sum(p * part + np.where(p < 2.0 ** -120, 2.0 ** -120, 0) * (np.abs(lp) + np.abs(lq[cls])))
        if pr > 0:
            lpr = (r - lm) - math.log(P)
            loss[b] += pr * (lpr - lR)
            ltol[b] += pr * (abs(lpr) + abs(lR) + 1) * (2 * E + H * (3 * near(lm - r) + 30))
        q, share = np.exp(lq), np.exp(np.minimum(y - yr, 0) / tau) / R
        pn = np.zeros(N)
        np.add.at(pn, cls, p)
        g = np.where(named, q - pn, share * (math.exp(lR) - pr))
        s = np.where(named, q + pn, share * (math.exp(lR) + pr))
        d = near((ym - y) / tau) + near((ym - yr) / tau) + near(np.where(named, 0, (yr - y) / tau).clip(0)) + \
            near(lm - (r if pr > 0 else lm))
        dn = np.zeros(N)
        np.maximum.at(dn, cls, near(lm - l))
        grad[b] = np.where(fired, -weight / tau * g, 0)
        gtol[b] = np.where(fired, weight / tau * (s * (2 * E + 3 * H * (d + dn) + 16 * H) + 2.0 ** -124), 0)
    return loss * weight, ltol * weight + 2.0 ** -140, grad, gtol + 2.0 ** -140


def _far_rows(B, N, K, tau, t_cap, rng):
    """Rows of six kinds in turn, and the K classes that a record names in each."""
    t = np.sqrt(rng.random((B, N))).astype(np.float32)
    t[rng.random((B, N)) < 0.2] = np.inf
    idx = np.stack([rng.permutation(N)[:K] for _ in range(B)]).astype(np.int32)
    for b in range(B):
        kind = b % 6
        if kind == 0:  # nothing fires
            t[b] = np.inf
        elif kind == 1:  # only named classes do
            keep = t[b, idx[b]].copy()
            t[b] = np.nan
            t[b, idx[b]] = keep
            t[b, idx[b][0]] = 0.5
        elif kind == 2:  # all do
            t[b] = np.where(np.isfinite(t[b]), t[b], 0.25)
        elif kind == 3:  # a few steps of fp32 around t_cap
            near = np.float32(t_cap)
            steps = [near]
            for _ in range(3):
                steps.append(np.nextafter(steps[-1], np.float32(0)))
            t[b] = np.array(steps, dtype=np.float32)[rng.integers(0, 4, N)]
            t[b, rng.random(N) < 0.2] = np.inf
        elif kind == 4:  # one class that is not named
            other = np.setdiff1d(np.arange(N), idx[b])[0]
            t[b] = np.inf
            t[b, other] = 0.75
    return t, idx


# tau, t_cap: from where kb is as large as 2^24, 2^32, to the ends of fp32
ENDS = [(0.1, 1e6), (0.1, 1.3e6), (0.1, 1e9), (0.1, 1e10), (0.1, 1e12), (0.1, 1e20), (0.1, 1e30), (0.1, 1e37),
        (0.1, -1e9), (1e-10, 1.5), (1e-30, 1.5), (100.0, 1e9), (1e5, 1e13), (1e30, 1e36)]


# a row in one block's registers (each size of blocks), rows in chunks
@pytest.mark.parametrize("B,N", [(6, 10), (6, 300), (6, 3000), (6, 8000), (36, 12000), (36, 20000), (36, 40000),
                                 (6, 20000), (6, 70000)])
def test_times_far_from_zero(B, N):
    torch, dstd = _torch()
    rng = np.random.default_rng(N)
    K = min(N // 3, 20)
    for tau, t_cap in ENDS:
        print(f"B={B} N={N} tau={tau} t_cap={t_cap}", flush=True)
        tau, t_cap = float(np.float32(tau)), float(np.float32(t_cap))
        t, idx = _far_rows(B, N, K, tau, t_cap, rng)
        logit = (rng.standard_normal((B, K)) * 2).astype(np.float32)
        rest = rng.standard_normal(B).astype(np.float32)
        weight = float(np.float32(1.0 / B))
        dev = [torch.from_numpy(v).cuda() for v in (t, idx, logit, rest)]
        for r in (rest, None):
            g, loss = dstd.distill_grad(dev[0], dev[1], dev[2], None if r is None else dev[3], tau_soft=tau,
                                        t_cap=t_cap, weight=weight)
            torch.cuda.synchronize()
            g, loss = g.cpu().numpy().astype(np.float64), loss.cpu().numpy().astype(np.float64)
            e_loss, ltol, e_grad, gtol = reference(t, idx, logit, r, tau, t_cap, weight)
            assert np.isfinite(g).all()
            bad = np.abs(g - e_grad) > gtol
            assert not bad.any(), (np.argwhere(bad)[:3], g[bad][:3], e_grad[bad][:3], gtol[bad][:3])
            assert np.isfinite(loss).all() and np.abs(e_loss).max() < FMAX
            bad = np.abs(loss[1:] - e_loss) > ltol
            assert not bad.any(), (np.argwhere(bad)[:3], loss[1:][bad][:3], e_loss[bad][:3], ltol[bad][:3])


@pytest.mark.parametrize("B,N,K", [(8, 10, 3), (8, 4096, 32), (8, 20000, 200), (40, 20000, 200), (1, 70000, 64)])
@pytest.mark.parametrize("size", [1e4, 1e6, 1e8])
def test_records_of_large_logits(B, N, K, size):
    """A teacher whose logits are large and near each other: only their differences count,
    which fp32 holds exactly here."""
    torch, dstd = _torch()
    rng = np.random.default_rng(N)
    tau, t_cap = 0.125, 1.5
    t, _ = _far_rows(B, N, K, tau, t_cap, rng)
    t = np.where(np.isfinite(t) & (np.abs(t) <= 1), t, np.inf).astype(np.float32)
    t[:, 0] = 0.25
    idx = np.stack([rng.permutation(N)[:K] for _ in range(B)]).astype(np.int32)
    step = float(np.spacing(np.float32(size)))
    apart = max(step, 0.25)  # of fp32 around it, or a quarter
    for sign in (1.0, -1.0):
        logit = (sign * size + apart * rng.integers(-4, 5, (B, K))).astype(np.float32)
        rest = (sign * size + apart * rng.integers(-4, 5, B)).astype(np.float32)
        dev = [torch.from_numpy(v).cuda() for v in (t, idx, logit, rest)]
        for r in (rest, None):
            g, loss = dstd.distill_grad(dev[0], dev[1], dev[2], None if r is None else dev[3], tau_soft=tau,
                                        t_cap=t_cap, weight=1.0)
            torch.cuda.synchronize()
            g, loss = g.cpu().numpy().astype(np.float64), loss.cpu().numpy().astype(np.float64)
            e_loss, ltol, e_grad, gtol = reference(t, idx, logit, r, tau, t_cap, 1.0)
            assert np.all(np.abs(g - e_grad) <= gtol)
            bad = np.abs(loss[1:] - e_loss) > ltol
            assert not bad.any(), (np.argwhere(bad)[:3], loss[1:][bad][:3], e_loss[bad][:3], ltol[bad][:3])
