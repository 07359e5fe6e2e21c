"""GPU checks of the tensor lists, the global gradient norm, clipping and the
AdamW step against the same formulas in 64 bits.

Tolerances, with u = 2^-24 the half step of fp32 (relative), u16 = 2^-8 that of
bf16, and 1.01 for the products of errors that are left out:

 norm   the sum is in 64 bits (its error, below 1e-9, and the root's are in the
        1.01), then one rounding: u |norm|.
 clip   the factor is rounded once, each product once: 2 u |out|; a bf16 output
        is rounded again: u16 |out|.
 AdamW  g' = fl(g fl(c)) carries 2 u.
        m: beta1 rounded u, its product with m inside the fma; 1 - beta1
           rounded u, its product u, g' 2 u; the sum rounded u |m| <= u (both):
           u (2 beta1 |m| + 5 (1 - beta1) |g'|).
        v: likewise, with g' twice and two products: 2 u and (1 + 4 + 2 + 1) u
           of terms that are all positive: 8 u v.
        the step U = (m c1) / (sqrt(v c2) + eps): m's error; c1, the product 2 u;
           under the root 8 u + 2 u, halved 5 u, the root u, eps u, the sum u;
           the quotient u: err(m) c1 / denominator + 11 u |U|.
        w: lr rounded, times lr_scale 2 u, its product u; decay rounded, times
           decay_scale 2 u; the fma u; the difference u |w|:
           lr (err(U) + 4 u |U| + 6 u decay |w|) + u |w_new|; bf16 adds u16 |w_new|.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U, U16, MORE = 2.0 ** -24, 2.0 ** -8, 1.01
SIZES = {
    "one": [1],
    "ends": [4095, 4096, 4097],
    "empty": [0, 5, 0, 1023, 0],
    "few": [2, 3, 5, 7, 11],
    "tiny": [1 + k % 9 for k in range(700)],      # more than one batch of tensors
    "long": [1_300_003, 4096 * 1024, 77],          # more chunks than partial sums
    # the most chunks of 4096 that a step, a clip and a norm take in one launch
    # of one block, and one element more
    "step": [3 * 4096], "step+": [4096, 8193],
    "clip": [8 * 4096], "clip+": [8 * 4096 + 1],
    "norm": [5 * 4096, 15 * 4096], "norm+": [20 * 4096 + 1],
}


@pytest.fixture(scope="module")
def dev():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2607_14672_amd import dstd
    dstd._load()  # fail loudly if the HIP library is missing
    return torch.device("cuda:0")


def _dt(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


class Arena:
    """Tensors of given sizes in one buffer with gaps of sentinels between
    them, each `shift` elements off a multiple of 64."""
    MARK = -7.0

    def __init__(self, values, dtype, shift, dev):
        import torch
        at, self.slots = 0, []
        for v in values:
            self.slots.append((at + shift, v.size))
            at += -(-(v.size + shift + 1) // 64) * 64
        flat = np.full(at + 64, self.MARK, dtype=np.float32)
        for (a, n), v in zip(self.slots, values):
            flat[a:a + n] = v.reshape(-1)
        self.buf = torch.from_numpy(flat).to(dev).to(_dt(dtype))
        self.t = [self.buf[a:a + n] for a, n in self.slots]

    def get(self):
        return [x.float().cpu().numpy().astype(np.float64) for x in self.t]

    def gaps_kept(self):
        b = self.buf.float().cpu().numpy().copy()
        for a, n in self.slots:
            b[a:a + n] = self.MARK
        return bool((b == self.MARK).all())


def _normal(rng, sizes, scale=1.0, zeros=0.25):
    out = []
    for n in sizes:
        x = rng.standard_normal(n) * scale
        x[rng.random(n) < zeros] = 0.0
        out.append(x.astype(np.float32))
    return out


def _norm64(gs):
    return math.sqrt(math.fsum(float((g * g).sum()) for g in gs))


def _close(got, ref, bound, what):
    got, ref, bound = (np.asarray(x, dtype=np.float64) for x in (got, ref, bound))
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.size} beyond their bound, first at "
                           f"{int(np.argmax(bad))}: {got[bad][:1]} for {ref[bad][:1]}")


# -------------------------------------------------------------------- norm --
@pytest.mark.parametrize("shift", [0, 1, 3])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", sorted(SIZES))
def test_norm(dev, sizes, dtype, shift):
    import torch
    from paper_2607_14672_amd import dstd
    print(f"norm {sizes} {dtype} shift {shift}", flush=True)
    g = Arena(_normal(np.random.default_rng(1), SIZES[sizes]), dtype, shift, dev)
    tl = dstd.make_tensor_list(g.t)
    norm = dstd.grad_norm(tl)
    torch.cuda.synchronize()
    ref = _norm64(g.get())
    _close(norm.cpu().numpy(), [ref], [U * MORE * ref], "norm")
    again = dstd.grad_norm(tl, ws=dstd.workspace(dstd.dstd_tensor_list_workspace_size(tl.c), dev))
    assert torch.equal(norm, again)
    assert g.gaps_kept()


def test_norm_of_mixed_types_and_shapes(dev):
    import torch
    from paper_2607_14672_amd import dstd
    rng = np.random.default_rng(2)
    a = torch.from_numpy(rng.standard_normal((17, 9, 3, 3)).astype(np.float32)).to(dev)
    b = torch.from_numpy(rng.standard_normal((100, 33)).astype(np.float32)).to(dev).to(torch.bfloat16)
    c = torch.empty((0, 5), device=dev)
    norm = dstd.grad_norm(dstd.make_tensor_list([a, b, c])).item()
    ref = math.sqrt(float(a.double().square().sum() + b.double().square().sum()))
    _close([norm], [ref], [U * MORE * ref], "norm")
    # nothing at all
    assert dstd.grad_norm(dstd.make_tensor_list([c])).item() == 0.0
    assert dstd.grad_norm(dstd.make_tensor_list([torch.zeros(5000, device=dev)])).item() == 0.0


@pytest.mark.parametrize("value", [1e30, 3e37, 1e-30, 1e-42])
def test_norm_neither_overflows_nor_underflows(dev, value):
    """Squares of these values do not fit fp32."""
    import torch
    from paper_2607_14672_amd import dstd
    x = torch.full((64,), value, device=dev)
    ref = 8.0 * float(x[0].double())
    got = dstd.grad_norm(dstd.make_tensor_list([x])).item()
    _close([got], [ref], [max(U * MORE * ref, 2.0 ** -150)], "norm")


@pytest.mark.parametrize("value,where", [(math.inf, 0), (-math.inf, 4999), (math.nan, 2500)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_of_what_is_not_finite(dev, value, where, dtype):
    import torch
    from paper_2607_14672_amd import dstd
    x = torch.ones(5000, device=dev, dtype=_dt(dtype))
    x[where] = value
    got = dstd.grad_norm(dstd.make_tensor_list([torch.ones(3, device=dev), x])).item()
    assert math.isnan(got) if math.isnan(value) else got == math.inf
    # finite gradients whose norm leaves fp32
    assert dstd.grad_norm(dstd.make_tensor_list([torch.full((64,), 3e38, device=dev)])).item() == math.inf


def test_more_than_2_31_elements(dev):
    """Offsets beyond 32 bits: the norm, clipping in place and a step at the
    far end of one tensor."""
    import torch
    from paper_2607_14672_amd import dstd
    n = (1 << 31) + 4099
    g = torch.ones(n, dtype=torch.bfloat16, device=dev)
    tl = dstd.make_tensor_list([g])
    _close([dstd.grad_norm(tl).item()], [math.sqrt(n)], [U * MORE * math.sqrt(n)], "norm")
    print("norm done", flush=True)
    dstd.grad_clip(tl, math.sqrt(n) / 2)
    assert bool((g[-5000:] == 0.5).all()) and bool((g[:5000] == 0.5).all())
    assert int((g != 0.5).sum()) == 0
    print("clip done", flush=True)
    w = torch.ones(n, dtype=torch.bfloat16, device=dev)
    m, v = torch.zeros(n, device=dev), torch.zeros(n, device=dev)
    step = torch.zeros(1, dtype=torch.int64, device=dev)
    tl = dstd.make_tensor_list([g], weights=[w], m=[m], v=[v])
    dstd.adamw_step(tl, dstd.make_adamw(lr=0.25, weight_decay=0.0), step)
    torch.cuda.synchronize()
    # the first step is lr times the gradient's sign
    assert bool((w[-5000:] == 0.75).all()) and int((w != 0.75).sum()) == 0
    assert int((m != m[0]).sum()) == 0 and int((v != v[0]).sum()) == 0
    assert step.item() == 1


# -------------------------------------------------------------------- clip --
@pytest.mark.parametrize("g_type,o_type", [("f32", None), ("bf16", None), ("f32", "f32"),
                                           ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("sizes", sorted(SIZES))
def test_clip(dev, sizes, g_type, o_type):
    import torch
    from paper_2607_14672_amd import dstd
    print(f"clip {sizes} {g_type} -> {o_type}", flush=True)
    vals = _normal(np.random.default_rng(3), SIZES[sizes], zeros=0.0)
    for shift in (0, 1):
        for frac in (0.37, 2.0):  # clipped, not clipped
            g = Arena(vals, g_type, shift, dev)
            o = Arena([0 * v for v in vals], o_type, 3 - shift, dev) if o_type else None
            before = g.get()
            ref = _norm64(before)
            max_norm = frac * ref
            tl = dstd.make_tensor_list(g.t, out=o.t if o else None)
            norm = dstd.grad_clip(tl, max_norm)
            torch.cuda.synchronize()
            _close(norm.cpu().numpy(), [ref], [U * MORE * ref], "norm")
            c = min(1.0, max_norm / ref)
            half = U16 if (o_type or g_type) == "bf16" else 0.0
            for x, b in zip((o or g).get(), before):
                _close(x, b * c, np.abs(b * c) * MORE * (2 * U + half), "clipped")
                if c == 1.0 and (o_type or g_type) != "bf16":
                    assert np.array_equal(x, b)
            if o:
                assert all(np.array_equal(x, b) for x, b in zip(g.get(), before))
                assert o.gaps_kept()
            assert g.gaps_kept()


def test_clip_by_a_given_norm(dev):
    """Two lists clipped by their common norm, as ranks would be."""
    import torch
    from paper_2607_14672_amd import dstd
    rng = np.random.default_rng(4)
    a, b = (Arena(_normal(rng, s), "f32", 0, dev) for s in ([5000, 3], [12345]))
    la, lb = dstd.make_tensor_list(a.t), dstd.make_tensor_list(b.t)
    norm = (dstd.grad_norm(la).double() ** 2 + dstd.grad_norm(lb).double() ** 2).sqrt().float()
    kept = norm.clone()
    before = a.get() + b.get()
    for tl in (la, lb):
        assert dstd.grad_clip(tl, 1.5, norm=norm, norm_given=True) is norm
    torch.cuda.synchronize()
    assert torch.equal(norm, kept)
    c = 1.5 / float(norm.double())
    for x, y in zip(a.get() + b.get(), before):
        _close(x, y * c, np.abs(y * c) * MORE * 2 * U, "clipped")
    _close([_norm64(a.get() + b.get())], [1.5], [1.5 * 4 * U * MORE], "norm of the clipped")


@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_clip_leaves_gradients_whose_norm_is_not_finite(dev, value):
    import torch
    from paper_2607_14672_amd import dstd
    x, y = torch.randn(9000, device=dev), torch.randn(10, device=dev)
    y[3] = value
    kept = x.clone(), y.clone()
    norm = dstd.grad_clip(dstd.make_tensor_list([x, y]), 1e-3).item()
    assert not math.isfinite(norm)
    assert torch.equal(x, kept[0]) and torch.equal(y[:3], kept[1][:3]) and torch.equal(y[4:], kept[1][4:])
    out = [torch.zeros_like(x), torch.zeros(10, device=dev)]
    dstd.grad_clip(dstd.make_tensor_list([x, y], out=out), 1e-3)
    assert torch.equal(out[0], x) and torch.equal(out[1][:3], y[:3])
    # a norm given as not finite
    bad = torch.tensor([value], device=dev)
    dstd.grad_clip(dstd.make_tensor_list([x]), 1e-3, norm=bad, norm_given=True)
    assert torch.equal(x, kept[0])


def test_zero_gradients_clip_to_zero(dev):
    import torch
    from paper_2607_14672_amd import dstd
    x = torch.zeros(5000, device=dev)
    assert dstd.grad_clip(dstd.make_tensor_list([x]), 1.0).item() == 0.0
    assert not bool(x.any())
    dstd.grad_clip(dstd.make_tensor_list([x]), math.inf)
    assert not bool(x.any())


# ------------------------------------------------------------------- AdamW --
def _adamw64(g, w, m, v, t, hp, c, lr, ls=1.0, ds=1.0):
    """(w, m, v) after step t and the bounds of their fp32 errors."""
    g = g * c
    m1 = hp["beta1"] * m + (1 - hp["beta1"]) * g
    v1 = hp["beta2"] * v + (1 - hp["beta2"]) * g * g
    em = U * (2 * hp["beta1"] * abs(m) + 5 * (1 - hp["beta1"]) * abs(g))
    ev = U * 8 * v1
    c1, c2 = 1 / (1 - hp["beta1"] ** t), 1 / (1 - hp["beta2"] ** t)
    den = (v1 * c2) ** 0.5 + hp["eps"]
    step = m1 * c1 / den
    rate, decay = lr * ls, hp["weight_decay"] * ds
    w1 = w - rate * (step + decay * w)
    ew = rate * (em * c1 / den + 15 * U * abs(step) + 6 * U * decay * abs(w)) + U * abs(w1)
    return (w1, m1, v1), (MORE * ew, MORE * em, MORE * ev)


class Train:
    """Arenas of one training step and their list."""

    def __init__(self, dev, sizes, g_type="f32", w_type="f32", master=False, shift=0, seed=5, scales=False,
                 g_scale=0.02):
        from paper_2607_14672_amd import dstd
        rng = np.random.default_rng(seed)
        self.g = Arena(_normal(rng, sizes, g_scale), g_type, shift, dev)
        w = _normal(rng, sizes, 0.3)
        self.w = Arena(w, w_type, shift, dev)
        self.w32 = Arena(w, "f32", (shift + 1) % 4, dev) if master else None
        self.m = Arena(_normal(rng, sizes, 0.01), "f32", shift, dev)
        self.v = Arena([x * x for x in _normal(rng, sizes, 0.02)], "f32", (shift + 2) % 4, dev)
        n = len(sizes)
        self.ls = [(0.5, 1.0, 0.0)[k % 3] for k in range(n)] if scales else [1.0] * n
        self.ds = [(1.0, 0.0)[k % 2] for k in range(n)] if scales else [1.0] * n
        self.tl = dstd.make_tensor_list(self.g.t, weights=self.w.t, m=self.m.t, v=self.v.t,
                                        master=self.w32.t if master else None,
                                        lr_scale=self.ls if scales else None,
                                        decay_scale=self.ds if scales else None)
        self.arenas = [a for a in (self.g, self.w, self.w32, self.m, self.v) if a]

    def bits(self):
        return [a.buf.clone() for a in self.arenas]


HP = dict(beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.05)


def _check_step(tr, before, t, hp, c, lr):
    g, w, m, v = before
    half = U16 if tr.w.buf.dtype != tr.m.buf.dtype else 0.0
    got = (tr.w32 or tr.w).get(), tr.m.get(), tr.v.get()
    for k in range(len(g)):
        ref, err = _adamw64(g[k], w[k], m[k], v[k], t, hp, c, lr, tr.ls[k], tr.ds[k])
        more = (0.0 if tr.w32 else half) * np.abs(ref[0]) * MORE
        _close(got[0][k], ref[0], err[0] + more, f"w of tensor {k}")
        _close(got[1][k], ref[1], err[1], f"m of tensor {k}")
        _close(got[2][k], ref[2], err[2], f"v of tensor {k}")
    if tr.w32:  # the weights are the rounded copy, bit for bit
        import torch
        for a, b in zip(tr.w.t, tr.w32.t):
            assert torch.equal(a, b.to(torch.bfloat16))
    assert all(a.gaps_kept() for a in tr.arenas)


@pytest.mark.parametrize("g_type,w_type,master", [("f32", "f32", False), ("f32", "bf16", False),
                                                  ("f32", "bf16", True), ("bf16", "f32", False),
                                                  ("bf16", "bf16", False), ("bf16", "bf16", True)])
@pytest.mark.parametrize("sizes", sorted(SIZES))
def test_adamw(dev, sizes, g_type, w_type, master):
    import torch
    from paper_2607_14672_amd import dstd
    for shift, done, frac, scales in ((0, 0, 0.3, False), (1, 1, 3.0, True), (3, 1000, None, True)):
        print(f"adamw {sizes} {g_type} {w_type} master {master} shift {shift}", flush=True)
        tr = Train(dev, SIZES[sizes], g_type, w_type, master, shift, scales=scales)
        before = tr.g.get(), (tr.w32 or tr.w).get(), tr.m.get(), tr.v.get()
        ref = _norm64(before[0])
        max_norm = math.inf if frac is None else frac * ref
        hp = dstd.make_adamw(lr=2e-3, max_norm=max_norm, **HP)
        step = torch.full((1,), done, dtype=torch.int64, device=dev)
        lr = None if done == 0 else torch.tensor([2e-3], device=dev)
        norm = dstd.adamw_step(tr.tl, hp, step, lr=lr)
        torch.cuda.synchronize()
        assert step.item() == done + 1
        if frac is None:
            assert norm is None
        else:
            _close(norm.cpu().numpy(), [ref], [U * MORE * ref], "norm")
        c = 1.0 if frac is None else min(1.0, max_norm / ref)
        _check_step(tr, before, done + 1, HP, c, 2e-3)
        assert all(np.array_equal(a, b) for a, b in zip(tr.g.get(), before[0]))


@pytest.mark.parametrize("kw", [dict(beta1=0.0), dict(beta2=0.0), dict(beta1=0.0, beta2=0.0),
                                dict(weight_decay=0.0), dict(beta2=0.99999, eps=1e-3)])
def test_adamw_constants(dev, kw):
    import torch
    from paper_2607_14672_amd import dstd
    c = {**HP, **kw}
    for done in (0, 12):
        tr = Train(dev, [1000, 5001], seed=6)
        before = tr.g.get(), tr.w.get(), tr.m.get(), tr.v.get()
        step = torch.full((1,), done, dtype=torch.int64, device=dev)
        dstd.adamw_step(tr.tl, dstd.make_adamw(lr=1e-2, **c), step)
        torch.cuda.synchronize()
        _check_step(tr, before, done + 1, c, 1.0, 1e-2)


def test_adamw_silent_weights_stay(dev):
    """No gradient ever and no decay: 0 / (0 + eps) moves nothing; with decay the
    weight shrinks by lr decay."""
    import torch
    from paper_2607_14672_amd import dstd
    w = torch.randn(5000, device=dev)
    z = [torch.zeros(5000, device=dev) for _ in range(3)]
    kept, step = w.clone(), torch.zeros(1, dtype=torch.int64, device=dev)
    tl = dstd.make_tensor_list([z[0]], weights=[w], m=[z[1]], v=[z[2]])
    norm = dstd.adamw_step(tl, dstd.make_adamw(weight_decay=0.0, max_norm=1.0), step)
    assert norm.item() == 0.0 and torch.equal(w, kept)
    dstd.adamw_step(tl, dstd.make_adamw(lr=0.5, weight_decay=0.5), step)
    assert torch.equal(w, kept * 0.75) and step.item() == 2  # powers of two: exact


def test_adamw_of_empty_tensors_counts_its_step(dev):
    import torch
    from paper_2607_14672_amd import dstd
    e = [torch.empty(s, device=dev) for s in ((0,), (3, 0)) * 4]
    tl = dstd.make_tensor_list(e[:2], weights=e[2:4], m=e[4:6], v=e[6:])
    step = torch.full((1,), 7, dtype=torch.int64, device=dev)
    norm = dstd.adamw_step(tl, dstd.make_adamw(max_norm=1.0), step)
    assert norm.item() == 0.0 and step.item() == 8
    assert dstd.grad_clip(tl, 1.0).item() == 0.0


def test_scalar_tensors_and_learning_rate_zero(dev):
    """Tensors without dimensions; a rate of zero moves moments alone."""
    import torch
    from paper_2607_14672_amd import dstd
    g, w, m, v = (torch.tensor(x, device=dev) for x in (2.0, 1.0, 0.0, 0.0))
    step = torch.zeros(1, dtype=torch.int64, device=dev)
    tl = dstd.make_tensor_list([g], weights=[w], m=[m], v=[v])
    dstd.adamw_step(tl, dstd.make_adamw(beta1=0.5, beta2=0.5), step, lr=torch.zeros(1, device=dev))
    assert (w.item(), m.item(), v.item(), step.item()) == (1.0, 1.0, 2.0, 1)


@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_adamw_skips_a_step_whose_norm_is_not_finite(dev, value):
    import torch
    from paper_2607_14672_amd import dstd
    tr = Train(dev, [5000, 7], "f32", "bf16", True)
    tr.g.t[1][2] = value
    kept, step = tr.bits(), torch.full((1,), 3, dtype=torch.int64, device=dev)
    norm = dstd.adamw_step(tr.tl, dstd.make_adamw(max_norm=1.0), step)
    assert not math.isfinite(norm.item()) and step.item() == 3
    same = [torch.equal(a, b) for a, b in zip(tr.bits()[1:], kept[1:])]
    assert all(same)
    # asked for by the norm alone, without clipping
    norm = dstd.adamw_step(tr.tl, dstd.make_adamw(), step, norm=torch.zeros(1, device=dev))
    assert not math.isfinite(norm.item()) and step.item() == 3
    assert all(torch.equal(a, b) for a, b in zip(tr.bits()[1:], kept[1:]))
    # and by a given one
    dstd.adamw_step(tr.tl, dstd.make_adamw(), step, norm=norm, norm_given=True)
    assert step.item() == 3 and all(torch.equal(a, b) for a, b in zip(tr.bits()[1:], kept[1:]))
    # no norm asked for: the step is made
    assert dstd.adamw_step(tr.tl, dstd.make_adamw(), step) is None
    assert step.item() == 4 and bool(torch.isfinite(tr.w.t[0].float()).all())


def test_adamw_by_a_given_norm(dev):
    import torch
    from paper_2607_14672_amd import dstd
    tr = Train(dev, [3000, 4097])
    before = tr.g.get(), tr.w.get(), tr.m.get(), tr.v.get()
    norm = torch.tensor([8.0], device=dev)
    step = torch.zeros(1, dtype=torch.int64, device=dev)
    assert dstd.adamw_step(tr.tl, dstd.make_adamw(lr=1e-3, max_norm=2.0, **HP), step, norm=norm,
                           norm_given=True) is norm
    torch.cuda.synchronize()
    assert norm.item() == 8.0
    _check_step(tr, before, 1, HP, 0.25, 1e-3)


def test_mixed_types_in_one_list(dev):
    """Gradients, weights and outputs of both types side by side, in a list for
    one block and in one for many."""
    import torch
    from paper_2607_14672_amd import dstd
    for scale in (1, 40):
        rng = np.random.default_rng(11)
        kinds = [(g, w, ms) for g in ("f32", "bf16") for w, ms in (("f32", False), ("bf16", False), ("bf16", True))]
        sizes = [scale * (301 + 97 * k) for k in range(len(kinds))]
        vals = [_normal(rng, sizes, sc) for sc in (0.02, 0.3, 0.01, 0.02)]

        def put(v, t):
            return torch.from_numpy(v).to(dev).to(_dt(t))

        g = [put(v, k[0]) for v, k in zip(vals[0], kinds)]
        w = [put(v, k[1]) for v, k in zip(vals[1], kinds)]
        w32 = [put(v, "f32") if k[2] else None for v, k in zip(vals[1], kinds)]
        m = [put(v, "f32") for v in vals[2]]
        v2 = [put(v * v, "f32") for v in vals[3]]
        out = [None if k[2] else torch.zeros_like(x, dtype=_dt("bf16" if k[0] == "f32" else "f32"))
               for x, k in zip(g, kinds)]
        tl = dstd.make_tensor_list(g, weights=w, m=m, v=v2, master=w32, out=out)

        def f64(x):
            return x.double().cpu().numpy()

        g0, m0, v0 = ([f64(x) for x in c] for c in (g, m, v2))
        w0 = [f64(a if b is None else b) for a, b in zip(w, w32)]
        ref = _norm64(g0)
        step = torch.full((1,), 4, dtype=torch.int64, device=dev)
        norm = dstd.adamw_step(tl, dstd.make_adamw(lr=1e-3, max_norm=0.5 * ref, **HP), step)
        _close(norm.cpu().numpy(), [ref], [U * MORE * ref], "norm")
        for k, (gt, wt, ms) in enumerate(kinds):
            want, err = _adamw64(g0[k], w0[k], m0[k], v0[k], 5, HP, 0.5, 1e-3)
            more = U16 * MORE * abs(want[0]) if wt == "bf16" and not ms else 0.0
            _close(f64(w32[k] if ms else w[k]), want[0], err[0] + more, f"w of {kinds[k]}")
            _close(f64(m[k]), want[1], err[1], f"m of {kinds[k]}")
            _close(f64(v2[k]), want[2], err[2], f"v of {kinds[k]}")
        dstd.grad_clip(tl, 0.25 * ref)
        for k, (gt, wt, ms) in enumerate(kinds):
            got = f64(g[k] if ms else out[k])
            half = U16 if (gt == "bf16") == ms else 0.0  # in place, or into the other type
            _close(got, 0.25 * g0[k], abs(0.25 * g0[k]) * MORE * (2 * U + half), f"clip of {kinds[k]}")


def _gpu_close(got, ref, bound, what):
    bad = int((~((got.double() - ref).abs() <= bound)).sum())
    assert bad == 0, f"{what}: {bad} of {ref.numel()} beyond their bound"


# lists past the sizes from which their accesses are streamed: of all arrays
# (96 MB), and of the gradients alone (240 MB)
@pytest.mark.parametrize("n,g_type", [(7_000_001, "f32"), (66_000_003, "f32"), (130_000_001, "bf16")])
def test_lists_that_exceed_the_caches(dev, n, g_type):
    import torch
    from paper_2607_14672_amd import dstd
    torch.manual_seed(12)
    cut = n // 3 | 1  # the second tensor starts off every alignment
    flat = {k: torch.randn(n, device=dev) for k in "gwm"}
    flat["g"] = flat["g"].to(_dt(g_type))
    flat["v"] = torch.rand(n, device=dev)
    parts = {k: [x[:cut], x[cut:]] for k, x in flat.items()}
    out = [torch.empty_like(x, dtype=torch.bfloat16) for x in parts["g"]]
    tl = dstd.make_tensor_list(parts["g"], weights=parts["w"], m=parts["m"], v=parts["v"], out=out)
    old = {k: x.clone() for k, x in flat.items()}
    g = old["g"].double()
    ref = float(g.square().sum().sqrt())
    norm = dstd.grad_norm(tl).item()
    _close([norm], [ref], [U * MORE * ref], "norm")
    dstd.grad_clip(tl, 0.5 * ref)
    for i, sl in ((0, slice(0, cut)), (1, slice(cut, None))):
        _gpu_close(out[i], 0.5 * g[sl], 0.5 * g[sl].abs() * MORE * (2 * U + U16), "clipped")
    step = torch.full((1,), 2, dtype=torch.int64, device=dev)
    dstd.adamw_step(tl, dstd.make_adamw(lr=1e-3, max_norm=0.5 * ref, **HP), step)
    for i in range(0, n, 33_000_000):  # the reference a part at a time
        sl = slice(i, min(n, i + 33_000_000))
        want, err = _adamw64(g[sl], *(old[k][sl].double() for k in "wmv"), 3, HP, 0.5, 1e-3)
        for k, x, e in zip("wmv", want, err):
            _gpu_close(flat[k][sl], x, e, k)
    assert torch.equal(flat["g"], old["g"]) and step.item() == 3
    # in place, the last of all
    tl = dstd.make_tensor_list(parts["g"])
    dstd.grad_clip(tl, 0.5 * ref)
    half = U16 if g_type == "bf16" else 0.0
    _gpu_close(flat["g"], 0.5 * g, 0.5 * g.abs() * MORE * (2 * U + half), "clipped in place")


# --------------------------------------------------- streams, graphs, lists --
def test_a_list_dropped_while_another_stream_reads_it(dev):
    """Built and freed on one stream, used on another: its table stays until
    that stream is through, whatever is allocated meanwhile."""
    import torch
    from paper_2607_14672_amd import dstd
    g = [torch.ones(1000, device=dev) for _ in range(2000)]
    side = torch.cuda.Stream(dev)
    got = []
    for _ in range(10):
        tl = dstd.make_tensor_list(g)
        size = tl.mem.numel()
        side.wait_stream(torch.cuda.current_stream(dev))
        with torch.cuda.stream(side):
            got.append(dstd.grad_norm(tl))
        del tl
        torch.zeros(size, dtype=torch.uint8, device=dev)
    torch.cuda.synchronize()
    want = math.sqrt(2e6)
    _close([x.item() for x in got], [want] * 10, [U * MORE * want] * 10, "norm")


def test_one_list_on_two_streams_at_once(dev):
    """Norms of one list on two streams, each with its workspace."""
    import torch
    from paper_2607_14672_amd import dstd
    g = Arena(_normal(np.random.default_rng(13), [900_001, 50]), "f32", 1, dev)
    tl = dstd.make_tensor_list(g.t)
    ref = dstd.grad_norm(tl)
    streams = [torch.cuda.Stream(dev) for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        for st in streams:
            with torch.cuda.stream(st):
                got.append(dstd.grad_norm(tl))
    torch.cuda.synchronize()
    assert all(torch.equal(x, ref) for x in got)


def test_other_streams_and_two_lists_at_once(dev):
    """Each list on a stream of its own, with its own workspace, gives the bits
    that one after the other on the default stream gives."""
    import torch
    from paper_2607_14672_amd import dstd
    hp = dstd.make_adamw(max_norm=0.5, **HP)

    def steps(parallel):
        trs = [Train(dev, s, seed=8 + k) for k, s in enumerate(([500_001, 7], [60_000] * 30))]
        done = [torch.zeros(1, dtype=torch.int64, device=dev) for _ in trs]
        streams = [torch.cuda.Stream(dev) if parallel else torch.cuda.current_stream(dev) for _ in trs]
        torch.cuda.synchronize()
        for _ in range(4):
            for tr, st, d in zip(trs, streams, done):
                with torch.cuda.stream(st):
                    dstd.grad_clip(tr.tl, 3.0)
                    dstd.adamw_step(tr.tl, hp, d)
        torch.cuda.synchronize()
        assert all(d.item() == 4 for d in done)
        return [b for tr in trs for b in tr.bits()]

    assert all(torch.equal(a, b) for a, b in zip(steps(False), steps(True)))


@pytest.mark.parametrize("sizes", [[70_000, 4097, 1], [5000, 7]])
def test_graph_replays_match_eager(dev, sizes):
    """A captured step, replayed between eager work, does what eager calls do:
    its step number and learning rate are read at each replay. Two graphs share
    a list and a workspace."""
    import torch
    from paper_2607_14672_amd import dstd
    hp = dstd.make_adamw(max_norm=0.7, **HP)

    def fresh():
        tr = Train(dev, sizes, "f32", "bf16", True, seed=9)
        return dict(tr=tr, step=torch.zeros(1, dtype=torch.int64, device=dev),
                    lr=torch.full((1,), 1e-3, device=dev), norm=torch.zeros(1, device=dev),
                    ws=dstd.workspace(dstd.dstd_tensor_list_workspace_size(tr.tl.c), dev))

    def call(s):
        dstd.adamw_step(s["tr"].tl, hp, s["step"], lr=s["lr"], norm=s["norm"], ws=s["ws"])

    a, b = fresh(), fresh()
    call(a), call(b)  # both sides alike before the capture
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(b)
        graphs.append(graph)
    for k in range(6):
        for s in (a, b):
            s["lr"].mul_(1.5)
            s["tr"].g.buf.mul_(0.8)
        call(a)
        graphs[k % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(a["norm"], b["norm"]) and a["step"].item() == b["step"].item() == k + 2
        for x, y in zip(a["tr"].bits(), b["tr"].bits()):
            assert torch.equal(x, y), f"replay {k}"
        scratch = dstd.grad_norm(b["tr"].tl, ws=b["ws"])  # eager work in the same workspace
        assert torch.equal(scratch, b["norm"])


def test_a_list_can_be_built_inside_a_capture(dev):
    """The table goes to the device as kernel arguments."""
    import torch
    from paper_2607_14672_amd import dstd
    g = [torch.randn(300 + 17 * k, device=dev) for k in range(100)]
    ref = dstd.grad_norm(dstd.make_tensor_list(g))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tl = dstd.make_tensor_list(g)
        norm = dstd.grad_norm(tl)
    for _ in range(3):
        tl.mem.fill_(0)
        norm.fill_(-1.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, ref)


def test_refusals_of_the_helpers(dev):
    import torch
    from paper_2607_14672_amd import dstd
    g = torch.randn(8, 6, device=dev)
    with pytest.raises(ValueError, match="contiguous"):
        dstd.make_tensor_list([g.t()])
    with pytest.raises(ValueError, match="shape"):
        dstd.make_tensor_list([g], out=[torch.zeros(6, 8, device=dev)])
    with pytest.raises(TypeError, match="first moment"):
        dstd.make_tensor_list([g], weights=[g.clone()], m=[g.bfloat16()], v=[g.clone()])
    with pytest.raises(dstd.DSTDError, match="overlap"):
        dstd.make_tensor_list([g, g])
    with pytest.raises(dstd.DSTDError, match="required with w"):
        dstd.make_tensor_list([g], weights=[g.clone()])
    tl = dstd.make_tensor_list([g])
    with pytest.raises(dstd.DSTDError, match="no weights"):
        dstd.adamw_step(tl, dstd.make_adamw(), torch.zeros(1, dtype=torch.int64, device=dev))
    with pytest.raises(dstd.DSTDError, match="max_norm"):
        dstd.grad_clip(tl, 0.0)
    with pytest.raises(ValueError, match="norm"):
        dstd.grad_clip(tl, 1.0, norm_given=True)
    with pytest.raises(ValueError, match="norm"):
        dstd.grad_norm(tl, norm=torch.zeros(1))
    with pytest.raises(ValueError, match="ws"):
        dstd.grad_norm(tl, ws=torch.zeros(tl.ws_bytes, dtype=torch.uint8))
    w = [torch.zeros(8, 6, device=dev) for _ in range(3)]
    tl = dstd.make_tensor_list([g], weights=w[:1], m=w[1:2], v=w[2:])
    with pytest.raises(ValueError, match="step"):
        dstd.adamw_step(tl, dstd.make_adamw(), torch.zeros(1, device=dev))
    with pytest.raises(ValueError, match="lr"):
        dstd.adamw_step(tl, dstd.make_adamw(), torch.zeros(1, dtype=torch.int64, device=dev),
                        lr=torch.zeros(2, device=dev))


# ------------------------------------------------------------ all together --
def _workload(name, batch):
    """The named workload, or a small conv net of non-leaky neurons (whose
    potential stays: every layer fires)."""
    from paper_2607_14672_amd import workloads
    if name != "small-conv":
        return workloads.with_batch(workloads.get(name), batch)
    inf, M = math.inf, 16
    L = [workloads._conv_layer(1, 3, 12, 12, 8, M, inf, inf),
         workloads._conv_layer(2, 8, 12, 12, 12, M, inf, inf, pool_in=2),
         workloads._conv_layer(3, 12, 6, 6, 20, M, inf, inf, stride=2),
         workloads.LayerSpec("dense", 20 * 3 * 3, 10, M, 3.0, 1.0 / M, inf, inf)]
    return workloads.Workload(name, batch, L, "one_minus_u", seed=7, extra={"k": [2.0] * 4})


# (the 20-layer net's last layers are silent at its initial weights: no gradient
# anywhere, and the step is the decay alone)
@pytest.mark.parametrize("name,batch", [("mlp3", 16), ("small-conv", 5), ("conv20", 2), ("wide-M8", 4)])
def test_training_steps_eager_and_captured(dev, name, batch):
    """Whole training steps: every layer's forward and backward, the loss, and a
    clipped AdamW step of all weights. Each eager step's update follows the
    formula from the gradients it was given; a captured step, replayed with eager
    work between, reaches the same bits."""
    import bench
    import torch
    from paper_2607_14672_amd import dstd
    hp = dstd.make_adamw(lr=1e-3, max_norm=0.01, **HP)
    wl = _workload(name, batch)
    a, b = bench.Net(wl, dev, optimizer=hp), bench.Net(wl, dev, optimizer=hp)

    def weights(net):
        return [e["W"] if w is None else w for e, w in zip(net.L, net.opt["w32"])]

    def f64(ts):
        return [t.double().cpu().numpy().reshape(-1) for t in ts]

    losses = []
    for k in range(3):
        w, m, v = f64(weights(a)), f64(a.opt["m"]), f64(a.opt["v"])
        a.step()
        torch.cuda.synchronize()
        g = f64(e["gW"] for e in a.L)
        ref = _norm64(g)
        fires = bool((a.L[-1]["q"] >= 0).any())
        assert (ref > 0.0) == fires == (name != "conv20")
        _close(a.opt["norm"].cpu().numpy(), [ref], [U * MORE * ref], "norm")
        c = min(1.0, 0.01 / ref) if fires else 1.0
        for i, (w1, m1, v1) in enumerate(zip(f64(weights(a)), f64(a.opt["m"]), f64(a.opt["v"]))):
            want, err = _adamw64(g[i], w[i], m[i], v[i], k + 1, HP, c, 1e-3)
            # products of tiny gradients leave the normal range of fp32: each of
            # the at most four of them is off by half of 2^-149
            for got, x, e, what in zip((w1, m1, v1), want, err, "wmv"):
                _close(got, x, e + (0.0 if what == "w" else 2.0 ** -148), f"{what} of layer {i}")
        losses.append(a.loss[0].item())
        assert a.opt["steps"].item() == k + 1
    assert name == "conv20" or len(set(losses)) > 1  # the steps act on the next forward

    b.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.stream = torch.cuda.current_stream(dev).cuda_stream
        b.step()
    for k in range(2):
        graph.replay()
        dstd.grad_norm(b.opt["list"])  # eager work between the replays
        torch.cuda.synchronize()
        assert b.loss[0].item() == losses[k + 1]
    for x, y in zip(weights(a) + a.opt["m"] + a.opt["v"], weights(b) + b.opt["m"] + b.opt["v"]):
        assert torch.equal(x, y)
    assert torch.equal(a.opt["norm"], b.opt["norm"]) and b.opt["steps"].item() == 3
