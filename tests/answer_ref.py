"""Plain forms in 64 bits of what reads a network's answer, row by row."""
import math

import numpy as np


def goodness(x, scale, cap):
    """Scores as float64 (of the fp32 or bf16 values), -inf where they do not
    count, so that larger is likelier."""
    x = np.asarray(x, dtype=np.float64)
    c = cap if cap is not None and math.isfinite(cap) else -math.inf * math.copysign(1.0, scale)
    x = np.where(np.isfinite(x), x, np.float64(np.float32(c)))
    return x if scale > 0 else -x


def order_of(y):
    """Indices by falling value, equal ones by index; entries that do not count last."""
    return np.argsort(-(y + 0.0), kind="stable")


def lse(z):
    z = z[np.isfinite(z)]
    if z.size == 0:
        return -math.inf
    m = z.max()
    return m + math.log(math.fsum(np.exp(z - m)))


def top(x, K, scale, cap):
    idx = np.full((x.shape[0], K), -1, dtype=np.int64)
    logit = np.full((x.shape[0], K), -math.inf)
    rest = np.full(x.shape[0], -math.inf)
    for b, y in enumerate(goodness(x, scale, cap)):
        o = order_of(y)
        o = o[np.isfinite(y[o])]
        n = min(K, o.size)
        idx[b, :n] = o[:n]
        logit[b, :n] = y[o[:n]] * abs(scale)
        rest[b] = lse(y[o[n:]] * abs(scale))
    return idx, logit, rest


def distill(t, idx, logit, rest, tau, t_cap, weight):
    """(loss [B], gradient [B, N], size [B, N] of what the gradient is the difference of)."""
    B, N = t.shape
    loss, grad, size = np.zeros(B), np.zeros((B, N)), np.zeros((B, N))
    for b in range(B):
        fired = np.isfinite(t[b])
        z = -np.where(fired, t[b].astype(np.float64), t_cap) / tau
        ok = (idx[b] >= 0) & (idx[b] < N) & np.isfinite(logit[b])
        if not ok.any():
            continue
        cls, lp = idx[b][ok].astype(np.int64), logit[b][ok].astype(np.float64)
        r = -math.inf if rest is None or not math.isfinite(rest[b]) else float(rest[b])
        norm = lse(np.append(lp, r))
        lp, lr = lp - norm, r - norm
        named = np.zeros(N, dtype=bool)
        named[cls] = True
        lq = z - lse(z)
        p = np.zeros(N)
        np.add.at(p, cls, np.exp(lp))
        loss[b] = np.sum(np.exp(lp) * (lp - lq[cls]))
        pr = math.exp(lr)
        lR = lse(z[~named]) - lse(z) if (~named).any() else -math.inf
        if pr > 0:
            loss[b] += pr * (lr - lR)
        q = np.exp(lq)
        g, s = q - p, q + p
        if (~named).any():
            share = np.exp(lq - lR)
            g = np.where(named, g, share * (math.exp(lR) - pr))
            s = np.where(named, s, share * (math.exp(lR) + pr))
        grad[b] = np.where(fired, -weight / tau * g, 0.0)
        size[b] = np.where(fired, weight / tau * s, 0.0)
    return loss * weight, grad, size


def kept(x, scale, cap, top_k, top_p, min_p):
    """Weights [B, N] of what is kept, 0 elsewhere."""
    out = np.zeros(x.shape)
    for b, y in enumerate(goodness(x, scale, cap)):
        o = order_of(y)
        o = o[np.isfinite(y[o])]
        if o.size == 0:
            continue
        if top_k:
            o = o[:top_k]
        w = np.exp((y[o] - y[o[0]]) * abs(scale))
        if top_p < 1.0:
            before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
            keep = before < top_p * w.sum()
            o, w = o[keep], w[keep]
        keep = w >= min_p
        out[b, o[keep]] = w[keep]
    return out
