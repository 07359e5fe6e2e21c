"""Top logits, distillation and sampling on the GPU against their formulas in 64 bits.

Tolerances. A term e^(scale (y - m)) of the kernels' sums takes y - m, the scale and
their product with half a step each, 3 * 2^-24 relative in an exponent d = scale (m - y),
so 3 * 2^-24 d in the term; the mean of d over a softmax of N classes is ln N at most.
exp2 is a step off (2^-23), again at each of the some 30 places where partial sums with
different m are joined, and a thread adds N / 64 terms at most one by one. EPS below adds
these up; it bounds the relative error of each sum and of each probability at d = 0."""
import math

import numpy as np
import pytest

from tests import answer_ref as ref

pytestmark = pytest.mark.gpu

H = 2.0 ** -24  # half a step of fp32


def eps(N):
    return H * (3 * math.log(N + 1) + 2 * 30 + 4 + N / 64)


def _torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2607_14672_amd import dstd
    return torch, dstd


def _put(torch, x, dtype, ld=0, shift=0):
    """x on the GPU with rows N + ld elements apart, `shift` elements off an aligned place."""
    B, N = x.shape
    flat = torch.full((shift + B * (N + ld),), math.nan, dtype=dtype, device="cuda")
    v = flat[shift:].view(B, N + ld)[:, :N]
    v.copy_(torch.from_numpy(x).to(dtype))
    return v


def _scores(kind, B, N, seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((B, N)).astype(np.float32) * 3
    if kind == "masked":
        x[rng.random((B, N)) < 0.5] = -np.inf
        x[rng.random((B, N)) < 0.1] = np.nan
        x[0] = -np.inf  # nothing is left
        if B > 1:
            x[1, 1:] = np.nan  # one class at most
    elif kind == "ties":
        x = np.round(x)
    elif kind == "equal":
        x[:] = 2.5
    elif kind == "zeros":
        x = np.where(rng.random((B, N)) < 0.5, -0.0, 0.0).astype(np.float32)
        x[:, ::7] = 1e-42
    elif kind == "huge":
        x = (rng.standard_normal((B, N)) * 1e38).astype(np.float32)
        x[:, -1] = 3e38
        x[:, 0] = -3e38
        x[~np.isfinite(x)] = 0
    elif kind == "near":  # distinct, all within a few steps
        x = (1.0 + rng.integers(0, 50, (B, N)) * 2.0 ** -23).astype(np.float32)
    elif kind == "signalling":  # NaN of the other kind, and +inf
        x[rng.random((B, N)) < 0.3] = np.inf
        x.view(np.uint32)[rng.random((B, N)) < 0.3] = 0x7f810000
    elif kind == "lowest":  # masked by the lowest value of the type
        x[rng.random((B, N)) < 0.6] = -3.3895314e38
        x[0] = -3.3895314e38
    elif kind == "tiny":  # a few values next to 0, others equal to it
        x[:, rng.integers(0, N, max(1, N // 700))] *= 1e-9
        x[:, rng.integers(0, N, max(1, N // 100))] = 0.0
        x[1 % B] = np.where(rng.random(N) < 0.9, 0.0, 1e-20 * x[1 % B])
        x[2 % B] = -np.abs(x[2 % B])
        x[2 % B, N // 3] = -1e-10
    elif kind == "sorted":  # one thread's share holds many of the largest
        x = np.sort(x, axis=1)
    elif kind == "outlier":
        x = x * 0.01
        x[:, N // 2] = 90.0
    return x


KINDS = ["plain", "masked", "ties", "equal", "zeros", "huge", "near", "sorted", "outlier", "signalling", "lowest", "tiny"]
SIZES = [1, 2, 63, 64, 65, 511, 512, 513, 1000, 4096, 4097, 20011]


def _check_top(torch, dstd, x, dtype, K, scale, cap, ld=0, shift=0):
    v = _put(torch, x, dtype, ld, shift)
    got = dstd.top_logits(v, K, scale=scale, cap=cap)
    torch.cuda.synchronize()
    idx, logit, rest = (g.cpu().numpy() for g in got)
    e_idx, e_logit, e_rest = ref.top(v.float().cpu().numpy(), K, scale, cap)
    assert np.array_equal(idx, e_idx)
    with np.errstate(invalid="ignore", over="ignore"):
        want = e_logit.astype(np.float32)
        assert np.array_equal(np.isfinite(logit), np.isfinite(want))
        f = np.isfinite(want)
        assert np.all(np.abs(logit[f] - e_logit[f]) <= H * np.abs(e_logit[f]) + 2.0 ** -150)
        assert np.array_equal(np.isneginf(rest), np.isneginf(e_rest.astype(np.float32)))
        f = np.isfinite(e_rest.astype(np.float32))
        # differences of y beyond fp32 count for nothing: the term is 0 all the same
        assert np.all(np.abs(rest[f] - e_rest[f]) <= eps(x.shape[1]) + H * np.abs(e_rest[f]))


@pytest.mark.parametrize("N", SIZES)
@pytest.mark.parametrize("kind", KINDS)
def test_top_logits(kind, N):
    torch, dstd = _torch()
    x = _scores(kind, 5, N, N)
    for K in sorted({1, min(N, 3), min(N, 64), min(N, 256)}):
        print(f"top {kind} N={N} K={K}", flush=True)
        _check_top(torch, dstd, x, torch.float32, K, -1.0 / 0.3, 1.5, ld=3, shift=1)
        _check_top(torch, dstd, x, torch.float32, K, 0.7, None)
        _check_top(torch, dstd, x, torch.bfloat16, K, 0.7, None, ld=1, shift=1)


@pytest.mark.parametrize("B,N,K,dtype", [(1, 131072, 64, "bf16"), (1, 131077, 256, "f32"), (3, 300007, 17, "f32"),
                                         (70, 65536, 64, "f32"), (1, (1 << 24) - 1, 256, "bf16"),
                                         (300, 10, 3, "f32"), (2000, 33, 33, "bf16")])
def test_top_logits_long_rows(B, N, K, dtype):
    torch, dstd = _torch()
    print(f"top B={B} N={N} K={K} {dtype}", flush=True)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    _check_top(torch, dstd, _scores("plain", B, N, 5), dt, K, 1.0, None, ld=1)
    _check_top(torch, dstd, _scores("ties", B, N, 6), dt, K, -1.0, None)
    _check_top(torch, dstd, _scores("sorted", B, N, 7), dt, K, 1.0, None)


# -------------------------------------------------------------- distillation --
def _record(rng, t, K, tau, t_cap, rest, dtype, kind):
    """A teacher's record: noisy logits of the student's classes, the K largest."""
    B, N = t.shape
    z = -np.where(np.isfinite(t), t, t_cap) / tau * 0.8 + rng.standard_normal((B, N)) * 1.5
    idx = np.argsort(-z, axis=1, kind="stable")[:, :K].astype(np.int32)
    logit = np.take_along_axis(z, idx, 1)
    other = np.array([ref.lse(np.delete(z[b], idx[b])) for b in range(B)]).astype(np.float32)
    if kind == "holes":
        gone = rng.random((B, K)) < 0.3
        idx[gone] = rng.choice([-1, N, N + 5, -(1 << 31), (1 << 31) - 1], gone.sum())
        logit[rng.random((B, K)) < 0.2] = rng.choice([np.nan, -np.inf, np.inf])
        idx[0] = -1  # a padded row
        other[-1] = np.nan
    elif kind == "twice":
        idx[:, K // 2:] = idx[:, :K - K // 2]
    elif kind == "far":  # named classes that the student thinks impossible
        idx = np.argsort(z, axis=1, kind="stable")[:, :K].astype(np.int32)
    return idx, logit.astype(np.float32), other if rest else None


def _check_distill(torch, dstd, t, idx, logit, rest, tau, t_cap, weight, dtype, accumulate=False, ld=0, shift=0):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    B, N = t.shape
    tau, t_cap, weight = (float(np.float32(v)) for v in (tau, t_cap, weight))
    tv = _put(torch, t, torch.float32, ld, shift)
    lv = torch.from_numpy(logit).to(dt).cuda()
    iv = torch.from_numpy(idx).cuda()
    rv = None if rest is None else torch.from_numpy(rest).cuda()
    rng = np.random.default_rng(9)
    g0 = rng.standard_normal((B, N)).astype(np.float32) * weight
    gv = _put(torch, g0, torch.float32, ld, shift)
    g, loss = dstd.distill_grad(tv, iv, lv, rv, tau_soft=tau, t_cap=t_cap, weight=weight, grad=gv,
                                accumulate=accumulate)
    alone = dstd.distill_grad(tv, iv, lv, rv, tau_soft=tau, t_cap=t_cap, weight=weight, need_grad=False)
    torch.cuda.synchronize()
    assert g is gv and alone[0] is None and torch.equal(alone[1], loss)
    if ld:  # what lies between the rows is left as it was
        assert torch.isnan(gv.as_strided((B - 1, ld), (N + ld, 1), gv.storage_offset() + N)).all()
    e_loss, e_grad, size = ref.distill(t, idx, lv.float().cpu().numpy(), rest, tau, t_cap, weight)
    g, loss = g.cpu().numpy(), loss.cpu().numpy()
    # a probability e^(z - ln Z) carries 3 * 2^-24 of its own exponent beside the sums'
    z = -np.where(np.isfinite(t), t.astype(np.float64), t_cap) / tau
    d = z.max(1, keepdims=True) - z
    tol = size * (2 * eps(N) + 4 * H * np.minimum(d, 100) + 16 * H) + 2.0 ** -126 * weight / tau
    if accumulate:
        e_grad = e_grad + g0
        tol = tol + H * (np.abs(e_grad) + np.abs(g0))
    assert np.all(np.isfinite(g))
    bad = np.abs(g - e_grad) > tol
    assert not bad.any(), (np.argwhere(bad)[:3], g[bad][:3], e_grad[bad][:3], tol[bad][:3])
    # a term p (ln p - ln q): both logarithms to eps, their size by half a step of each part
    zmax = np.abs(d).max(1) + np.abs(np.where(np.isfinite(logit), logit, 0)).max(1) + 2 * math.log(N + 1) + \
        (0 if rest is None else np.abs(np.where(np.isfinite(rest), rest, 0)))
    ltol = weight * (4 * eps(N) + 16 * H * zmax + len(idx[0]) * H * zmax)
    assert np.all(np.abs(loss[1:] - e_loss) <= ltol), (loss[1:], e_loss, ltol)
    assert abs(loss[0] - loss[1:].astype(np.float64).sum()) <= H * (B + 8) * np.abs(loss[1:]).sum()
    if B > 1:  # one row by itself
        one = dstd.distill_grad(tv[1:2], iv[1:2], lv[1:2], None if rv is None else rv[1:2], tau_soft=tau, t_cap=t_cap,
                                weight=weight, need_grad=False)[1].cpu().numpy()
        assert one[0] == one[1] and abs(one[1] - e_loss[1]) <= ltol[1]


def _times(B, N, seed, silent=0.2):
    rng = np.random.default_rng(seed)
    t = np.sqrt(rng.random((B, N))).astype(np.float32)
    t[rng.random((B, N)) < silent] = np.inf
    return t


@pytest.mark.parametrize("N", SIZES + [8191, 8192, 8193, 65536])
@pytest.mark.parametrize("kind", ["plain", "holes", "twice", "far"])
def test_distill(kind, N):
    torch, dstd = _torch()
    B, tau, t_cap = 5, 0.1, 1.5
    for K in sorted({1, min(N, 5), min(N, 200)}):
        for rest in (True, False):
            rng = np.random.default_rng(N + K)
            t = _times(B, N, N)
            t[B - 1] = np.nan  # nothing fires
            rec = _record(rng, t, K, tau, t_cap, rest and K < N, "f32", kind)
            print(f"distill {kind} N={N} K={K} rest={rest}", flush=True)
            _check_distill(torch, dstd, t, *rec, tau, t_cap, 1.0 / B, "f32")
            _check_distill(torch, dstd, t, *rec, tau, t_cap, 0.7, "bf16", accumulate=True, ld=5, shift=1)


@pytest.mark.parametrize("B,N,K", [(1, 131072, 64), (2, 300007, 256), (700, 10, 3), (300, 700, 9), (40, 40000, 100)])
def test_distill_sizes(B, N, K):
    torch, dstd = _torch()
    print(f"distill B={B} N={N} K={K}", flush=True)
    rng = np.random.default_rng(B)
    t = _times(B, N, 3)
    _check_distill(torch, dstd, t, *_record(rng, t, K, 0.07, 1.2, True, "f32", "plain"), 0.07, 1.2, 1.0 / B, "f32",
                   accumulate=B % 2 == 0)


def test_distill_gradient_is_the_losses_difference():
    """Central differences of the loss in 64 bits, at one class of each kind; and the
    kernel's loss moves as its gradient says."""
    torch, dstd = _torch()
    rng = np.random.default_rng(4)
    B, N, K, tau, cap = 3, 40, 6, 0.25, 1.5
    t = _times(B, N, 8)
    idx, logit, rest = _record(rng, t, K, tau, cap, True, "f32", "plain")
    g, _ = dstd.distill_grad(torch.from_numpy(t).cuda(), torch.from_numpy(idx).cuda(),
                             torch.from_numpy(logit).cuda(), torch.from_numpy(rest).cuda(), tau_soft=tau,
                             t_cap=cap, weight=1.0)
    g = g.cpu().numpy()
    h = 1e-5
    for b in range(B):
        for i in range(N):
            if not np.isfinite(t[b, i]):
                assert g[b, i] == 0
                continue
            up, dn = t.astype(np.float64), t.astype(np.float64)
            up[b, i] += h
            dn[b, i] -= h
            d = [ref.distill(v, idx, logit, rest, tau, cap, 1.0)[0][b] for v in (up, dn)]
            # third derivative of the loss: 1 / tau^3 at most
            assert abs((d[0] - d[1]) / (2 * h) - g[b, i]) <= h * h / tau ** 3 + 1e-9 / h * 1e-4 + 1e-5 / tau


def test_distill_equal_student_has_no_gradient():
    """A student that says what the teacher says: loss and gradient vanish."""
    torch, dstd = _torch()
    t = _times(4, 1000, 2, silent=0.0)
    v = torch.from_numpy(t).cuda()
    idx, logit, rest = dstd.top_logits(v, 20, scale=-1.0 / 0.2)
    g, loss = dstd.distill_grad(v, idx, logit, rest, tau_soft=0.2, t_cap=2.0, weight=1.0)
    torch.cuda.synchronize()
    # the record is rounded: 2^-24 of logits up to 5, against probabilities of 1 at most
    e = 4 * eps(1000) + 20 * 5 * H
    assert float(g.abs().max()) <= e / 0.2 and float(loss.abs().max()) <= 4 * e


# ------------------------------------------------------------------ sampling --
def _check_sample(torch, dstd, x, dtype, scale, cap, top_k, top_p, min_p, seed=0, ld=0, shift=0, u=None):
    v = _put(torch, x, dtype, ld, shift)
    B, N = x.shape
    rng = np.random.default_rng(seed)
    u = rng.random(B).astype(np.float32) if u is None else u
    c, logp = dstd.sample(v, torch.from_numpy(u).cuda(), scale=scale, cap=cap, top_k=top_k, top_p=top_p, min_p=min_p)
    torch.cuda.synchronize()
    c, logp = c.cpu().numpy(), logp.cpu().numpy()
    w = ref.kept(v.float().cpu().numpy(), scale, cap, top_k, top_p, min_p)
    cum = np.cumsum(w, axis=1)
    # N weights to 2^-(s+1) each, and the reference's own sums
    slack = N * (2.0 ** -(min(51, 62 - math.ceil(math.log2(N)))) + 2.0 ** -52 * 4)
    for b in range(B):
        C = cum[b, -1]
        if C == 0:
            assert c[b] == -1 and np.isneginf(logp[b])
            continue
        assert 0 <= c[b] < N and w[b, c[b]] > 0, (b, c[b])
        uu = min(max(float(u[b]), 0.0), 1 - 2.0 ** -24) if u[b] == u[b] else 0.0
        below = cum[b, c[b] - 1] if c[b] else 0.0
        assert below <= uu * C + slack and cum[b, c[b]] > uu * C - slack, (b, c[b], below, uu * C, cum[b, c[b]])
        want = math.log(w[b, c[b]]) - math.log(C)
        assert abs(logp[b] - want) <= H * abs(want) + 4 * slack + 1e-12


FILTERS = [(0, 1.0, 0.0), (0, 0.9, 0.0), (5, 1.0, 0.0), (300, 0.7, 0.0), (0, 1.0, 0.05), (40, 0.95, 0.02),
           (1, 0.5, 1.0), (1 << 40, 1e-6, 0.0), (3000, 0.999, 1e-4)]


@pytest.mark.parametrize("N", SIZES)
@pytest.mark.parametrize("kind", KINDS)
def test_sample(kind, N):
    torch, dstd = _torch()
    x = _scores(kind, 6, N, N + 1)
    for n, (k, p, m) in enumerate(FILTERS):
        print(f"sample {kind} N={N} top_k={k} top_p={p} min_p={m}", flush=True)
        _check_sample(torch, dstd, x, torch.float32, -1.0 / 0.3, 1.5, k, p, m, n, ld=3, shift=1)
        _check_sample(torch, dstd, x, torch.float32, 0.7, None, k, p, m, n + 20)
        _check_sample(torch, dstd, x, torch.bfloat16, 1.1, None, k, p, m, n + 40, ld=1, shift=1)
        _check_sample(torch, dstd, x, torch.bfloat16, -2.0, 1.5, k, p, m, n + 60)
        _check_sample(torch, dstd, x, torch.bfloat16, -2.0, 0.1, k, p, m, n + 80)  # no bf16 value


@pytest.mark.parametrize("B,N,dtype", [(1, 131072, "bf16"), (2, 131077, "f32"), (40, 50021, "f32"),
                                       (1, (1 << 24) - 1, "bf16"), (500, 10, "f32")])
@pytest.mark.parametrize("k,p,m", FILTERS)
def test_sample_long_rows(B, N, dtype, k, p, m):
    torch, dstd = _torch()
    print(f"sample B={B} N={N} {dtype} top_k={k} top_p={p} min_p={m}", flush=True)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    for n, kind in enumerate(["plain"] if N > 1 << 20 else ["plain", "equal", "ties", "near", "outlier"]):
        _check_sample(torch, dstd, _scores(kind, B, N, n), dt, 0.8, None, k, p, m, n)


def test_sample_ends_of_u():
    """The first kept class at u = 0, the last with a weight at the largest u; u outside
    [0, 1) is drawn in to it."""
    torch, dstd = _torch()
    x = _scores("ties", 8, 700, 3)
    u = np.array([0.0, 1 - 2.0 ** -24, 1.0, 7.0, -3.0, np.nan, np.inf, -np.inf], dtype=np.float32)
    for f in FILTERS:
        _check_sample(torch, dstd, x, torch.float32, 1.0, None, *f, u=u)


def test_sample_frequencies():
    """Draws with evenly spread u come out as often as their probability says."""
    torch, dstd = _torch()
    n = 20000
    x = _scores("plain", 1, 37, 5)
    u = (np.arange(n, dtype=np.float32) + 0.5) / n
    v = torch.from_numpy(x).cuda().expand(n, 37).contiguous()
    c, _ = dstd.sample(v, torch.from_numpy(u).cuda(), top_p=0.9)
    got = np.bincount(c.cpu().numpy(), minlength=37)
    w = ref.kept(x, 1.0, None, 0, 0.9, 0.0)[0]
    # each class's interval of u holds its length times n points, give or take one at each end
    assert np.all(np.abs(got - n * w / w.sum()) <= 2.01)


def test_top_k_of_one_is_the_first_of_top_logits():
    torch, dstd = _torch()
    x = _put(torch, _scores("ties", 50, 3001, 4), torch.bfloat16)
    idx, logit, rest = dstd.top_logits(x, 1)
    c, logp = dstd.sample(x, torch.full((50,), 0.5, device="cuda"), top_k=1)
    assert torch.equal(idx[:, 0], c) and float(logp.abs().max()) == 0.0


@pytest.mark.parametrize("op", ["top", "distill", "sample"])
def test_empty_batches(op):
    torch, dstd = _torch()
    x = torch.empty((0, 9), device="cuda")
    if op == "top":
        idx, logit, rest = dstd.top_logits(x, 4)
        assert idx.shape == logit.shape == (0, 4) and rest.shape == (0,)
    elif op == "sample":
        c, logp = dstd.sample(x, torch.empty(0, device="cuda"))
        assert c.shape == logp.shape == (0,)
    else:
        g, loss = dstd.distill_grad(x, torch.empty((0, 3), dtype=torch.int32, device="cuda"),
                                    torch.empty((0, 3), device="cuda"), t_cap=1.0)
        torch.cuda.synchronize()
        assert g.shape == (0, 9) and loss.tolist() == [0.0]


# -------------------------------------------------- calls as programs make them --
def _calls(torch, dstd, B=40, N=20011, seed=0):
    """One call of each operator on inputs of its own, as (name, call) pairs; a call
    returns its outputs."""
    rng = np.random.default_rng(seed)
    x = _put(torch, _scores("ties", B, N, seed), torch.bfloat16)
    f = _put(torch, _scores("plain", B, N, seed + 1), torch.float32)
    u = torch.from_numpy(rng.random(B).astype(np.float32)).cuda()
    t = _times(B, N, seed)
    idx, logit, rest = (torch.from_numpy(v).cuda() for v in _record(rng, t, 50, 0.1, 1.5, True, "f32", "twice"))
    tv = torch.from_numpy(t).cuda()
    return [("top", lambda: dstd.top_logits(x, 64)), ("top f32", lambda: dstd.top_logits(f, 200, scale=-2.0, cap=1.0)),
            ("picked", lambda: dstd.sample(x, u, top_k=100, top_p=0.9)),
            ("values", lambda: dstd.sample(x, u, top_p=0.9, min_p=0.01)),
            ("f32", lambda: dstd.sample(f, u, top_p=0.9)), ("f32 all", lambda: dstd.sample(f, u)),
            ("f32 count", lambda: dstd.sample(f, u, top_k=3000)),
            ("distill", lambda: dstd.distill_grad(tv, idx, logit, rest, tau_soft=0.1, t_cap=1.5)),
            ("distill rows", lambda: dstd.distill_grad(tv[:5], idx[:5], logit[:5], rest[:5], tau_soft=0.1, t_cap=1.5))]


def _same(torch, a, b):
    return all(torch.equal(p.view(torch.int32), q.view(torch.int32)) for p, q in zip(a, b))


def test_repeated_calls_give_the_same_bits():
    torch, dstd = _torch()
    for name, call in _calls(torch, dstd):
        print(f"again: {name}", flush=True)
        first = [v.clone() for v in call()]
        for _ in range(5):
            assert _same(torch, first, call()), name


def test_calls_on_another_stream_and_two_at_once():
    torch, dstd = _torch()
    calls = _calls(torch, dstd)
    want = [[v.clone() for v in call()] for _, call in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for k, (_, call) in enumerate(calls + calls):
        with torch.cuda.stream(streams[k % 2]):
            got.append(call())
    torch.cuda.synchronize()
    for k, g in enumerate(got):
        assert _same(torch, want[k % len(calls)], g), calls[k % len(calls)][0]


@pytest.mark.parametrize("B,N", [(33, 5003), (3, 20011), (1, 70001)])
def test_captured_calls_replay(B, N):
    """Each call captured, replayed between eager work, on inputs that change; two graphs
    side by side."""
    torch, dstd = _torch()
    x = torch.empty((B, N), dtype=torch.bfloat16, device="cuda")
    t = torch.empty((B, N), device="cuda")
    u = torch.empty(B, device="cuda")

    def fill(seed):
        x.copy_(torch.from_numpy(_scores("plain", B, N, seed)))
        t.copy_(torch.from_numpy(_times(B, N, seed)))
        u.copy_(torch.from_numpy(np.random.default_rng(seed).random(B).astype(np.float32)))

    def step():
        idx, logit, rest = dstd.top_logits(x, 30, scale=0.5)
        g, loss = dstd.distill_grad(t, idx, logit, rest, tau_soft=0.1, t_cap=1.5)
        g, loss2 = dstd.distill_grad(t, idx, logit, tau_soft=0.2, t_cap=1.5, grad=g, accumulate=True)
        return (idx, logit, rest, g, loss, loss2) + dstd.sample(x, u, top_p=0.8) + dstd.sample(t, u, scale=-5.0, top_k=9)

    fill(0)
    step()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    outs = []
    for g in graphs:
        with torch.cuda.graph(g):
            outs.append(step())
    for seed in range(1, 5):
        fill(seed)
        want = [v.clone() for v in step()]
        graphs[seed % 2].replay()
        torch.zeros(1000, device="cuda").sum().item()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        for o in outs:
            assert _same(torch, want, o), seed


def test_rows_far_apart():
    """Places beyond 2^32 elements."""
    torch, dstd = _torch()
    B, N, ld = 4200, 9, 1 << 20
    xs = _scores("plain", B, N, 3)
    flat = torch.empty(B * ld, dtype=torch.bfloat16, device="cuda")
    x = flat.view(B, ld)[:, :N]
    x.copy_(torch.from_numpy(xs))
    small = x.contiguous()
    for a, b in zip(dstd.top_logits(x, 3), dstd.top_logits(small, 3)):
        assert torch.equal(a, b)
    u = torch.rand(B, device="cuda")
    for a, b in zip(dstd.sample(x, u), dstd.sample(small, u)):
        assert torch.equal(a, b)
    del flat, x
    tf, gf = (torch.empty(B * ld, device="cuda") for _ in range(2))
    t, g = tf.view(B, ld)[:, :N], gf.view(B, ld)[:, :N]
    t.copy_(torch.from_numpy(_times(B, N, 4)))
    idx, logit, rest = dstd.top_logits(small, 3)
    got = dstd.distill_grad(t, idx, logit, rest, tau_soft=0.3, t_cap=1.5, grad=g)
    want = dstd.distill_grad(t.contiguous(), idx, logit, rest, tau_soft=0.3, t_cap=1.5)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("B,N,K", [(65535, 3, 2), (65535, 1, 1), (1, (1 << 24) - 1, 4)])
def test_largest_sizes(B, N, K):
    torch, dstd = _torch()
    print(f"largest B={B} N={N}", flush=True)
    t = _times(B, N, 1)
    _check_top(torch, dstd, t, torch.float32, K, -4.0, 1.5)
    _check_sample(torch, dstd, t, torch.float32, -4.0, 1.5, 0, 0.9, 0.0)
    rng = np.random.default_rng(2)
    idx = rng.integers(0, N, (B, K)).astype(np.int32)
    logit = rng.standard_normal((B, K)).astype(np.float32)
    rest = rng.standard_normal(B).astype(np.float32) if N > 3 else None
    if B * N < 1 << 20:
        t, idx, logit = t[-300:], idx[-300:], logit[-300:]
        g, loss = dstd.distill_grad(*(torch.from_numpy(v).cuda() for v in (_times(B, N, 1), np.resize(idx, (B, K)),
                                                                            np.resize(logit, (B, K)))),
                                    tau_soft=0.25, t_cap=1.5, weight=1.0)
        e_loss, e_grad, _ = ref.distill(t, np.resize(idx, (B, K))[-300:], np.resize(logit, (B, K))[-300:], None, 0.25,
                                        1.5, 1.0)
        torch.cuda.synchronize()
        assert np.allclose(g[-300:].cpu().numpy(), e_grad, rtol=0, atol=1e-4)
        assert np.allclose(loss[-300:].cpu().numpy(), e_loss, rtol=1e-4, atol=1e-5)
    else:
        _check_distill(torch, dstd, t, idx, logit, rest, 0.25, 1.5, 1.0, "f32")


@pytest.mark.parametrize("scale", [1e38, -1e38, 1e-38, -1e-42, 1e-3])
@pytest.mark.parametrize("N", [100, 3000, 20011])
def test_scales_at_the_ends_of_fp32(scale, N):
    """Logits beyond fp32 read inf; choices hold all the same."""
    torch, dstd = _torch()
    x = _scores("ties", 4, N, 5)
    scale = float(np.float32(scale))
    for dt in (torch.float32, torch.bfloat16):
        v = _put(torch, x, dt)
        idx, logit, rest = dstd.top_logits(v, 7, scale=scale)
        e_idx, e_logit, _ = ref.top(x, 7, scale, None)
        assert np.array_equal(idx.cpu().numpy(), e_idx)
        with np.errstate(over="ignore"):
            assert np.array_equal(logit.cpu().numpy(), e_logit.astype(np.float32))
        assert not torch.isnan(rest).any()
        _check_sample(torch, dstd, x, dt, scale, None, 0, 0.7, 0.0)
        _check_sample(torch, dstd, x, dt, scale, None, 5, 1.0, 0.0)


def test_record_that_names_all_classes():
    """Without a rest nothing is left outside; with one the loss says so."""
    torch, dstd = _torch()
    t = torch.from_numpy(_times(3, 8, 3)).cuda()
    idx = torch.arange(8, dtype=torch.int32, device="cuda").repeat(3, 1)
    logit = torch.randn(3, 8, device="cuda")
    g, loss = dstd.distill_grad(t, idx, logit, tau_soft=0.5, t_cap=1.5)
    h, more = dstd.distill_grad(t, idx, logit, torch.zeros(3, device="cuda"), tau_soft=0.5, t_cap=1.5)
    assert torch.isfinite(loss).all() and (loss[1:] >= 0).all()
    assert (more == math.inf).all() and torch.isfinite(g).all() and torch.isfinite(h).all()


def test_views_are_read_as_they_are():
    """Transposed, stepped and reversed-stride views give what their copies give."""
    torch, dstd = _torch()
    base = torch.from_numpy(_scores("plain", 300, 200, 6)).cuda()
    u = torch.rand(200, device="cuda")
    for v in (base.t(), base[::3], base[:, ::2], base[:, 7:50], base[5:6], base.expand(2, 300, 200)[1]):
        c = v.contiguous()
        assert all(torch.equal(a, b) for a, b in zip(dstd.top_logits(v, 5), dstd.top_logits(c, 5)))
        k = u[:v.shape[0]] if v.shape[0] <= 200 else torch.rand(v.shape[0], device="cuda")
        assert all(torch.equal(a, b) for a, b in zip(dstd.sample(v, k), dstd.sample(c, k)))
    with pytest.raises(ValueError):
        dstd.distill_grad(base, torch.zeros((300, 2), dtype=torch.int32, device="cuda"),
                          torch.zeros((300, 2), device="cuda"), t_cap=1.0,
                          grad=torch.zeros((200, 300), device="cuda").t())


def test_outputs_of_the_caller():
    torch, dstd = _torch()
    x = torch.randn(20, 500, device="cuda")
    i, l, r = torch.empty((20, 4), dtype=torch.int32, device="cuda"), torch.empty((20, 4), device="cuda"), torch.empty(20, device="cuda")
    assert [a is b for a, b in zip(dstd.top_logits(x, 4, idx=i, logit=l, rest=r), (i, l, r))] == [True] * 3
    c, p = torch.empty(20, dtype=torch.int32, device="cuda"), torch.empty(20, device="cuda")
    assert [a is b for a, b in zip(dstd.sample(x, r.clamp(0, 0.5), choice=c, logp=p), (c, p))] == [True] * 2
    with pytest.raises(dstd.DSTDError):  # the scores' own memory
        dstd.sample(x, r, choice=x.view(torch.int32).view(-1)[:20])
    with pytest.raises(dstd.DSTDError):
        dstd.distill_grad(x, i, l, r, t_cap=1.0, grad=x)
    with pytest.raises(TypeError):
        dstd.sample(x, r, choice=c.long())
    with pytest.raises(ValueError):
        dstd.top_logits(x, 4, idx=i[:, :3])
    with pytest.raises(ValueError):
        dstd.distill_grad(x, i, l, r)  # no t_cap
    with pytest.raises(ValueError):
        dstd.distill_grad(x, i, l[:, :2], r, t_cap=1.0)
    with pytest.raises(ValueError):
        dstd.distill_grad(x, i, l, r, t_cap=1.0, accumulate=True)


def test_a_student_learns_from_a_teacher():
    """A run of all three: the teacher's record from its spike times, the student's layer
    forward, its loss and gradients, an update, and a drawn answer. The weights' gradient
    is the loss's difference along a direction."""
    torch, dstd = _torch()
    rng = np.random.default_rng(3)
    B, N_in, N, M, tau, cap = 64, 96, 500, 16, 0.2, 1.6
    p = dstd.make_params(1.0, 0.3, 1.0, M, 0.0, 1.0 / M)
    t_in = torch.from_numpy(rng.random((B, N_in)).astype(np.float32)).cuda()
    W_t, W_s = (torch.from_numpy((7.0 / N_in * (1 + 0.3 * math.sqrt(N_in) * rng.standard_normal((N, N_in))))
                                 .astype(np.float32)).cuda() for _ in range(2))
    idx, logit, rest = dstd.top_logits(dstd.forward(p, t_in, W_t)[0], 40, scale=-1.0 / tau, cap=cap)
    u = torch.from_numpy(rng.random(B).astype(np.float32)).cuda()

    def loss_of(W):
        t, slope, q = dstd.forward(p, t_in, W)
        return t, slope, q, dstd.distill_grad(t, idx, logit, rest, tau_soft=tau, t_cap=cap)

    t, slope, q, (g, loss) = loss_of(W_s)
    e_loss, e_grad, _ = ref.distill(t.cpu().numpy(), idx.cpu().numpy(), logit.cpu().numpy(), rest.cpu().numpy(),
                                    float(np.float32(tau)), float(np.float32(cap)), 1.0 / B)
    assert abs(float(loss[0]) - e_loss.sum()) <= 1e-4 * abs(e_loss.sum())
    gW = torch.empty_like(W_s)
    dstd.backward(p, t_in, W_s, t, slope, q, g, need_t_in=False, grad_W=gW)
    tl = dstd.make_tensor_list([gW], weights=[W_s.clone()], m=[torch.zeros_like(W_s)], v=[torch.zeros_like(W_s)])
    norm = dstd.adamw_step(tl, dstd.make_adamw(lr=1e-3, max_norm=1.0), torch.zeros(1, dtype=torch.int64, device="cuda"))
    choice, logp = dstd.sample(t, u, scale=-1.0 / tau, cap=cap, top_k=10)
    w = ref.kept(t.cpu().numpy(), -1.0 / tau, cap, 10, 1.0, 0.0)
    torch.cuda.synchronize()
    assert math.isfinite(float(norm)) and float(norm) > 0
    assert all(w[b, c] > 0 for b, c in enumerate(choice.tolist()))
    # the layer's own gradient through its loss: only the outputs' part is checked here
    assert np.allclose(g.cpu().numpy(), e_grad, rtol=1e-3, atol=1e-6 / B)
