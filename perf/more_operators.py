"""Timed cases of what reads a network's answer: the softmax over its output
spike times, or over the scores of another network.

A case is a dict of plain values. ``op`` says which operator it goes through:

  top      the K largest logits of every row, and the log of what the others
           add up to: what is kept of a teacher
  distill  loss and gradient of a student's spike times against such a record
  sample   one class drawn for every row from a given random number, with
           temperature, top-k, top-p and min-p

``x`` is "times" (f32 spike times, some neurons silent), or the type of another
network's scores, "f32" or "bf16". ``soft`` is the temperature (tau_soft).
``absent`` is the share of silent neurons or masked classes; ``cap`` says that
they count as the time CAP (else they are left out). In one of ``pad`` rows
nothing is left (0: in none). ``ld`` is how many elements further than N a row
starts behind the one before.
"""
import math
import random

import torch

own = False

CAP = 1.5  # spike times lie in [0, 1): where a silent neuron enters the softmax


def _case(name, op, B, N, K=0, x="times", soft=0.1, absent=0.0, cap=True, pad=0, ld=0, rest=True,
          add=False, top_k=0, top_p=1.0, min_p=0.0):
    return dict(name=name, op=op, B=B, N=N, K=K, x=x, soft=soft, absent=absent, cap=cap, pad=pad,
                ld=ld, rest=rest, add=add, top_k=top_k, top_p=top_p, min_p=min_p)


def listed():
    return [
        # a spiking teacher's record: the wide layer's outputs, a fifth of them silent
        _case("top-wide", "top", 256, 4096, 32, absent=0.2),
        # one row of a large vocabulary, as a record is made while a stream is answered
        _case("top-row-bf16", "top", 1, 131072, 64, "bf16", 1.0),
        # a teacher's record over a whole batch of token positions, some of them padding
        _case("top-large-bf16", "top", 512, 131072, 64, "bf16", 2.0, cap=False, pad=64),
        # ten classes: launches and latency
        _case("distill-classes", "distill", 128, 10, 3, absent=0.3),
        # the wide layer as a readout
        _case("distill-wide", "distill", 256, 4096, 32, absent=0.2),
        # an odd vocabulary, the teacher's probabilities made to add to one, onto another loss's gradient
        _case("distill-ragged", "distill", 77, 50021, 100, absent=0.1, pad=16, ld=3, rest=False, add=True),
        # the largest: a batch of token positions
        _case("distill-large", "distill", 1024, 65536, 64, soft=0.07, absent=0.2, pad=32),
        # an answer for each sample of a small batch
        _case("sample-classes", "sample", 128, 10, absent=0.3),
        # one token
        _case("sample-row-bf16", "sample", 1, 131072, x="bf16", soft=0.8, top_k=50, top_p=0.9),
        # a batch of requests: the nucleus of a large vocabulary
        _case("sample-nucleus-bf16", "sample", 64, 131072, x="bf16", soft=1.0, top_p=0.95, min_p=0.002),
        # plain draws from an odd vocabulary with masked classes
        _case("sample-ragged", "sample", 300, 50021, x="f32", soft=1.3, absent=0.1, cap=False, pad=50, ld=1),
        # many rollouts at once
        _case("sample-large-bf16", "sample", 512, 131072, x="bf16", soft=1.0, top_k=1000, top_p=0.98),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["top", "distill", "sample"])
    N = _log(rng, 2, 131072)
    B = _log(rng, 1, min(4096, (1 << 25) // N))
    x = "times" if op == "distill" else rng.choice(["times", "f32", "bf16"])
    c = _case("", op, B, N, x=x, soft=rng.choice([0.05, 0.1, 0.3] if x == "times" else [0.5, 1.0, 2.0]),
              absent=rng.choice([0.0, 0.1, 0.4]), cap=op == "distill" or rng.random() < 0.5,
              pad=rng.choice([0, 0, 7]), ld=rng.choice([0, 0, 0, 1, 6]))
    if op == "sample":
        c.update(top_k=rng.choice([0, 0, _log(rng, 1, N)]), top_p=rng.choice([1.0, 0.9, 0.6, 0.99]),
                 min_p=rng.choice([0.0, 0.0, 0.01]))
    else:
        c["K"] = _log(rng, 1, min(N, 256))
        if op == "distill":
            c.update(rest=rng.random() < 0.7, add=rng.random() < 0.4)
    c.pop("name")
    return c


# ------------------------------------------------------------------ inputs --
def _dev():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _padded(c):
    """Truth values [B][1]: the rows with nothing in them."""
    b = torch.arange(c["B"], device=_dev())
    return (b % c["pad"] == c["pad"] - 1 if c["pad"] else b < 0)[:, None]


def _rows(c, x):
    """x as rows that lie N + ld elements apart."""
    if not c["ld"]:
        return x
    wide = torch.zeros(c["B"], c["N"] + c["ld"], dtype=x.dtype, device=x.device)
    wide[:, :c["N"]] = x
    return wide[:, :c["N"]]


def _inputs(c, seed):
    gen = torch.Generator(device=_dev()).manual_seed(int(seed))
    shape = (c["B"], c["N"])

    def rand():
        return torch.rand(shape, generator=gen, device=_dev())

    def normal():
        return torch.randn(shape, generator=gen, device=_dev())

    gone = rand() < c["absent"]
    if c["x"] == "times":
        # most neurons fire late, few early
        x = rand().pow_(0.5).masked_fill_(gone, math.inf)
        if c["op"] != "distill":
            x = x.masked_fill_(_padded(c), math.inf)
    else:
        # scores: a wide bulk and a few classes that stand out
        x = normal().mul_(2.0) + 7.0 * (rand() < 20.0 / c["N"])
        x = x.masked_fill_(gone | _padded(c), -math.inf).to(torch.bfloat16 if c["x"] == "bf16" else torch.float32)
    a = dict(scores=_rows(c, x))
    if c["op"] == "sample":
        a["u"] = torch.rand(c["B"], generator=gen, device=_dev())
    if c["op"] == "distill":
        # a teacher that knows the student's task better than the student
        t = torch.where(torch.isfinite(x), x, CAP)
        logits = normal().mul_(1.5).sub_(t / c["soft"])
        top, idx = logits.topk(c["K"], dim=1)
        a["logit"] = top
        a["idx"] = idx.masked_fill_(_padded(c), -1).to(torch.int32)
        if c["rest"]:
            a["other"] = logits.scatter_(1, idx.clamp_(min=0), -math.inf).logsumexp(1)
        g = normal().mul_(0.1 / c["B"]) if c["add"] else torch.zeros(shape, device=_dev())
        a["grad"] = g
    return a


def prepare(case, seed):
    return dict(case, **_inputs(case, seed))


# --------------------------------------------------------------------- run --
def _scale(c):
    return -1.0 / c["soft"] if c["x"] == "times" else 1.0 / c["soft"]


def _cap(c):
    return CAP if c["cap"] and c["x"] == "times" else None


def run(s):
    return _run_own(s) if own else globals()["_plain_" + s["op"]](s)


def _run_own(s):
    from paper_2607_14672_amd import dstd

    if s["op"] == "top":
        return dstd.top_logits(s["scores"], s["K"], scale=_scale(s), cap=_cap(s))
    if s["op"] == "sample":
        return dstd.sample(s["scores"], s["u"], scale=_scale(s), cap=_cap(s), top_k=s["top_k"],
                           top_p=s["top_p"], min_p=s["min_p"])
    return dstd.distill_grad(s["scores"], s["idx"], s["logit"], s.get("other"), tau_soft=s["soft"],
                             t_cap=CAP, weight=1.0 / s["B"], grad=s["grad"], accumulate=s["add"])


def _scores(s):
    """The scores so that larger is likelier, -inf where they do not count."""
    x = s["scores"].float()
    x = torch.where(torch.isfinite(x), x, math.inf * -_scale(s) if _cap(s) is None else _cap(s))
    return x if _scale(s) > 0 else -x


def _plain_top(s):
    K, scale = s["K"], abs(_scale(s))
    x, order = torch.sort(_scores(s), dim=1, descending=True, stable=True)
    logit = (x[:, :K].double() * scale).float()
    idx = torch.where(torch.isfinite(logit), order[:, :K], -1).to(torch.int32)
    others = x[:, K:]
    if others.shape[1] == 0:
        return idx, logit, torch.full((s["B"],), -math.inf, device=x.device)
    top = others[:, :1]
    shift = torch.where(torch.isfinite(top), top, 0.0)
    rest = (scale * (others - shift)).exp().sum(1).log() + scale * shift[:, 0]
    return idx, logit, rest


def _plain_distill(s):
    B, N, tau = s["B"], s["N"], s["soft"]
    fired = torch.isfinite(s["scores"])
    t = torch.where(fired, s["scores"], CAP)
    z = (t.amin(1, keepdim=True) - t) / tau
    e = z.exp()
    real = s["idx"] >= 0
    some = real.any(1)
    at = s["idx"].clamp(min=0).long()
    # what the teacher says: its top classes, and all others together
    logit = torch.where(real, s["logit"], -math.inf)
    rest = s["other"] if "other" in s else torch.full((B,), -math.inf, device=t.device)
    all_of = torch.cat([logit, rest[:, None]], 1)
    top = torch.where(some, all_of.amax(1), 0.0)[:, None]
    p = (all_of - top).exp()
    p = p / torch.where(some[:, None], p.sum(1, keepdim=True), 1.0)
    listed_ = torch.zeros_like(e).scatter_add_(1, at, real.float())
    teacher = torch.zeros_like(e).scatter_add_(1, at, torch.where(real, p[:, :-1], 0.0))
    R = (e * (listed_ == 0)).sum(1, keepdim=True)
    Z = e.sum(1, keepdim=True)
    logq = torch.cat([z.gather(1, at), torch.log(R)], 1) - torch.log(Z)
    terms = torch.where(p > 0, p * (torch.log(p) - logq), 0.0)
    terms = torch.where(some, terms.sum(1), 0.0) / B
    q = e / Z
    others = torch.where(R > 0, q - e * (p[:, -1:] / R), 0.0)
    grad = torch.where(listed_ > 0, q - teacher, others) * (-1.0 / (tau * B))
    grad = torch.where(fired & some[:, None], grad, 0.0)
    s["grad"] = s["grad"] + grad if s["add"] else grad
    return s["grad"], torch.cat([terms.sum().reshape(1), terms])


def _plain_sample(s):
    """In 64 bits: what is kept and drawn turns on sums next to a border."""
    x, order = torch.sort(_scores(s), dim=1, descending=True, stable=True)
    x = x.double() * abs(_scale(s))
    top = torch.where(torch.isfinite(x[:, :1]), x[:, :1], 0.0)
    w = (x - top).exp()
    if s["top_k"]:
        w[:, s["top_k"]:] = 0.0
    cum = w.cumsum(1)
    kept = w
    if s["top_p"] < 1.0:
        kept = torch.where(cum - w < s["top_p"] * cum[:, -1:], kept, 0.0)
    kept = torch.where(w >= s["min_p"], kept, 0.0)
    kept = torch.zeros_like(kept).scatter_(1, order, kept)
    cum = kept.cumsum(1)
    total = cum[:, -1]
    target = s["u"].double() * total
    choice = (cum <= target[:, None]).sum(1)
    some = total > 0
    choice = torch.where(some, choice, 0)
    logp = kept.gather(1, choice[:, None])[:, 0].log() - total.log()
    return torch.where(some, choice, -1).to(torch.int32), torch.where(some, logp, -math.inf).float()


# ------------------------------------------------------------------ floors --
def work(case):
    B, N, K = (float(case[k]) for k in ("B", "N", "K"))
    size = 2 if case["x"] == "bf16" else 4
    if case["op"] == "top":
        return {"bytes": B * (N * size + 8 * K + 4), "flops": 3 * B * N}
    if case["op"] == "sample":
        return {"bytes": B * (N * size + 12), "flops": 3 * B * N}
    return {"bytes": B * (N * (12 if case["add"] else 8) + 8 * K + 8), "flops": 6 * B * N}


# ------------------------------------------------- the same in 64 bits ----
def exact(case, seed):
    """Row by row of a few at a time, every value in 64 bits."""
    a = _inputs(case, seed)
    each = max(1, (1 << 24) // case["N"])
    parts = []
    for b in range(0, case["B"], each):
        rows = {k: v[b:b + each] for k, v in a.items()}
        parts.append(globals()["_exact_" + case["op"]](case, rows))
    out = [torch.cat(p) if p[0] is not None else None for p in zip(*parts)]
    if case["op"] == "distill":
        out[1] = torch.cat([out[1].sum().reshape(1), out[1]])
    return tuple(out)


def _logits64(case, x):
    x = x.double()
    z = x * _scale(case)
    absent = -math.inf if _cap(case) is None else _cap(case) * _scale(case)
    return torch.where(torch.isfinite(x), z, torch.full_like(z, absent))


def _exact_top(case, rows):
    z = _logits64(case, rows["scores"])
    top, at = z.topk(case["K"], dim=1)
    return None, top, z.scatter(1, at, -math.inf).logsumexp(1)


def _exact_distill(case, rows):
    """The gradient is the softmax of each side, class by class, in the logits."""
    tau, B = case["soft"], case["B"]
    t = rows["scores"].double()
    fired = torch.isfinite(t)
    logq = torch.log_softmax(torch.where(fired, t, torch.full_like(t, CAP)) * (-1.0 / tau), 1)
    idx = rows["idx"].long()
    pad = idx[:, 0] < 0
    idx = idx.clamp(min=0)
    parts = [rows["logit"].double()]
    if case["rest"]:
        parts.append(rows["other"].double()[:, None])
    logp = torch.log_softmax(torch.cat(parts, 1), 1)
    K = case["K"]
    loss = (logp[:, :K].exp() * (logp[:, :K] - logq.gather(1, idx))).sum(1)
    outside = logq.scatter(1, idx, -math.inf)
    grad = logq.exp()
    if case["rest"]:
        logr = outside.logsumexp(1)
        pr = logp[:, K].exp()
        loss += torch.where(pr > 0, pr * (logp[:, K] - logr), torch.zeros_like(pr))
        share = (outside - torch.where(torch.isfinite(logr), logr, torch.zeros_like(logr))[:, None]).exp()
        grad = grad - pr[:, None] * share
    grad = grad.scatter_add(1, idx, -logp[:, :K].exp())
    grad = torch.where(fired & ~pad[:, None], grad / (-tau * B), torch.zeros_like(grad))
    if case["add"]:
        grad = grad + rows["grad"].double()
    return grad, torch.where(pad, torch.zeros_like(loss), loss) / B


def _exact_sample(case, rows):
    z = _logits64(case, rows["scores"])
    z, at = torch.sort(z, dim=1, descending=True, stable=True)
    some = torch.isfinite(z[:, 0])
    logp = torch.log_softmax(z[:, :case["top_k"] or case["N"]], 1)
    p = logp.exp()
    before = torch.cumsum(p, 1) - p
    keep = torch.isfinite(logp)
    if case["top_p"] < 1.0:
        keep &= before < case["top_p"]
    if case["min_p"] > 0.0:
        keep &= p >= case["min_p"] * p[:, :1]
    logp = torch.log_softmax(torch.where(keep, logp, torch.full_like(logp, -math.inf)), 1)
    by_class = torch.full_like(z, -math.inf).scatter(1, at[:, :logp.shape[1]], logp)
    reached = torch.cumsum(by_class.exp(), 1) > rows["u"].double()[:, None]
    choice = reached.int().argmax(1)
    got = by_class.gather(1, choice[:, None])[:, 0]
    return None, torch.where(some, got, torch.full_like(got, -math.inf))
