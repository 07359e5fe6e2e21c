"""GPU checks of the tensor lists, the global gradient norm, clipping and the
AdamW step at the limits of their types and of their launch forms. Tolerances
as in test_gpu_optim.py, where a test says nothing else: u = 2^-24 and
u16 = 2^-8 are the half steps of fp32 and bf16."""
import math

import numpy as np
import pytest

from tests.test_gpu_optim import HP, MORE, U, U16, Arena, Train, _check_step, _close, _norm64, _normal
from tests.test_gpu_optim import dev  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ streams --
DELAY = 20_000_000  # clock ticks of a kernel that only waits: 10 to 200 ms


def test_a_list_used_on_another_stream_waits_for_its_build(dev):
    """The building stream is held up; nothing orders the other one but the call."""
    import torch
    from paper_2607_14672_amd import dstd
    g = [torch.full((3000,), float(k % 5), device=dev) for k in range(100)]
    ref = _norm64([x.double().cpu().numpy() for x in g])
    build, side = torch.cuda.Stream(dev), torch.cuda.Stream(dev)
    torch.cuda.synchronize()
    with torch.cuda.stream(build):
        torch.cuda._sleep(DELAY)
        tl = dstd.make_tensor_list(g)
    assert not tl.built.query()
    with torch.cuda.stream(side):
        norm = dstd.grad_norm(tl)
    torch.cuda.synchronize()
    _close([norm.item()], [ref], [U * MORE * ref], "norm")
    with torch.cuda.stream(side):  # the build is long done
        assert torch.equal(dstd.grad_norm(tl), norm)
    assert tl.built is None


def test_a_list_built_inside_a_capture_is_for_captures(dev):
    import torch
    from paper_2607_14672_amd import dstd
    g = [torch.ones(500, device=dev) for _ in range(40)]
    torch.cuda.synchronize()
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tl = dstd.make_tensor_list(g)
    with pytest.raises(RuntimeError, match="inside a capture"):
        dstd.grad_norm(tl)
    with torch.cuda.graph(other):
        norm = dstd.grad_norm(tl)
    graph.replay()
    for _ in range(3):
        norm.fill_(-1.0)
        other.replay()
        torch.cuda.synchronize()
        _close([norm.item()], [math.sqrt(20_000)], [U * MORE * 200], "norm")


def test_the_table_of_a_dropped_list_is_not_reused_while_it_is_read(dev):
    """The other stream is held up in front of its call: until it is through, an
    allocation of the table's size on the building stream gets other memory."""
    import torch
    from paper_2607_14672_amd import dstd
    g = [torch.ones(1000, device=dev) for _ in range(5000)]
    side = torch.cuda.Stream(dev)
    tl = dstd.make_tensor_list(g)
    size, at = tl.mem.numel(), tl.mem.data_ptr()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(DELAY)
        norm = dstd.grad_norm(tl)
        read = side.record_event()
    del tl
    blocks = [torch.empty(size, dtype=torch.uint8, device=dev) for _ in range(3)]
    assert not read.query()
    assert at not in [b.data_ptr() for b in blocks]
    torch.cuda.synchronize()
    del blocks
    want = math.sqrt(5e6)
    _close([norm.item()], [want], [U * MORE * want], "norm")
    # the delay over, its memory is there for others again
    assert at in [torch.empty(size, dtype=torch.uint8, device=dev).data_ptr()]


# ------------------------------------------------------- moments over steps --
@pytest.mark.parametrize("n", [4000, 20_000])
@pytest.mark.parametrize("beta1,beta2", [(0.9, 0.999), (0.999, 0.9999), (0.9999, 0.99999)])
def test_moments_follow_their_betas_over_many_steps(dev, beta1, beta2, n):
    """4000 steps against a 64-bit recursion that sees the gradients alone. In
    the mean over all elements only what all of them share is left: 1 - beta
    rounded (u), and at worst the two roundings of (1 - beta) g^2 (2 u). The
    roundings of a moment differ in every step and element (at most u each,
    evenly spread: u / sqrt(3) in the mean square), so that their mean over n
    elements has a deviation below u sqrt(4000 / (3 n)) = 0.6 u for n = 4000:
    3 u and six deviations, 7 u. A beta and a 1 - beta that do not add to 1
    would be off by 2^-25 / (1 - beta) once the moment is settled."""
    import torch
    from paper_2607_14672_amd import dstd
    steps, bank = 4000, 16
    gen = torch.Generator(device=dev).manual_seed(n)
    grads = 1.0 + 0.3 * torch.randn(bank, n, generator=gen, device=dev)
    g, w, m, v = (torch.zeros(n, device=dev) for _ in range(4))
    tl = dstd.make_tensor_list([g], weights=[w], m=[m], v=[v])
    hp = dstd.make_adamw(lr=0.0, beta1=beta1, beta2=beta2)
    step, ws = torch.zeros(1, dtype=torch.int64, device=dev), dstd.workspace(tl.ws_bytes, dev)
    m64, v64 = torch.zeros(2, n, dtype=torch.float64, device=dev)
    g64 = grads.double()
    for k in range(steps):
        g.copy_(grads[k % bank])
        dstd.adamw_step(tl, hp, step, ws=ws)
        m64.mul_(beta1).add_(g64[k % bank], alpha=1.0 - beta1)
        v64.mul_(beta2).addcmul_(g64[k % bank], g64[k % bank], value=1.0 - beta2)
    assert step.item() == steps
    for got, ref, what in ((m, m64, "m"), (v, v64, "v")):
        off = float(((got.double() - ref) / ref).mean())
        assert abs(off) <= 7 * U, f"{what} off by {off:.3g} in the mean"


@pytest.mark.parametrize("n", [4000, 20_000])
@pytest.mark.parametrize("beta2", [0.5, 0.999])
def test_a_second_moment_that_overflowed_stays_infinite(dev, beta2, n):
    """Its weight only decays then: m / (inf + eps) is 0."""
    import torch
    from paper_2607_14672_amd import dstd
    g, w, m = (torch.full((n,), x, device=dev) for x in (0.5, 1.0, 0.25))
    v = torch.full((n,), math.inf, device=dev)
    tl = dstd.make_tensor_list([g], weights=[w], m=[m], v=[v])
    step = torch.full((1,), 3, dtype=torch.int64, device=dev)
    dstd.adamw_step(tl, dstd.make_adamw(lr=0.5, beta2=beta2, weight_decay=0.5), step)
    assert bool((v == math.inf).all()) and bool((w == 0.75).all())


# ---------------------------------------------------------- extreme factors --
# of chunks for one launch of one block, and for many
@pytest.mark.parametrize("sizes", [[5000, 3], [60_001, 7]])
@pytest.mark.parametrize("g_type,o_type", [("f32", None), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("max_norm", [1e-3, 1e-6, 1e-12])
def test_clip_of_huge_gradients_keeps_its_bits(dev, max_norm, g_type, o_type, sizes):
    """max_norm / norm lies below the normal range of fp32 here, or below all of
    it; the results do not. Bounds as for other factors, and half of the least
    fp32 or bf16 number for results that go there."""
    import torch
    from paper_2607_14672_amd import dstd
    vals = _normal(np.random.default_rng(21), sizes, 1e35)
    g = Arena(vals, g_type, 1, dev)
    o = Arena([0 * v for v in vals], o_type, 2, dev) if o_type else None
    before = g.get()
    ref = _norm64(before)
    assert ref < 3e38 and max_norm / ref < 2.0 ** -126
    norm = dstd.grad_clip(dstd.make_tensor_list(g.t, out=o.t if o else None), max_norm)
    torch.cuda.synchronize()
    _close(norm.cpu().numpy(), [ref], [U * MORE * ref], "norm")
    c = max_norm / ref
    half, least = (U16, 2.0 ** -133) if o_type == "bf16" else (0.0, 2.0 ** -149)
    for x, b in zip((o or g).get(), before):
        _close(x, b * c, np.abs(b * c) * MORE * (2 * U + half) + least, "clipped")
    assert g.gaps_kept() and (o is None or o.gaps_kept())


@pytest.mark.parametrize("sizes", [[5000, 3], [60_001, 7]])
@pytest.mark.parametrize("g_type", ["f32", "bf16"])
@pytest.mark.parametrize("max_norm", [1e-3, 1e-6])
def test_adamw_of_huge_gradients(dev, max_norm, g_type, sizes):
    import torch
    from paper_2607_14672_amd import dstd
    tr = Train(dev, sizes, g_type, seed=22, g_scale=1e35)
    before = tr.g.get(), tr.w.get(), tr.m.get(), tr.v.get()
    ref = _norm64(before[0])
    step = torch.full((1,), 9, dtype=torch.int64, device=dev)
    norm = dstd.adamw_step(tr.tl, dstd.make_adamw(lr=2e-3, max_norm=max_norm, **HP), step)
    torch.cuda.synchronize()
    _close(norm.cpu().numpy(), [ref], [U * MORE * ref], "norm")
    _check_step(tr, before, 10, HP, max_norm / ref, 2e-3)


@pytest.mark.parametrize("n", [5000, 60_001])
@pytest.mark.parametrize("outside", [False, True])
def test_a_tiny_factor_whose_mantissa_rounds_to_one_still_clips(dev, outside, n):
    import torch
    from paper_2607_14672_amd import dstd
    g = torch.full((n,), 2.0 ** 100, device=dev)
    out = [torch.zeros(n, device=dev)] if outside else None
    norm = torch.full((1,), 2.0 ** 120, device=dev)
    dstd.grad_clip(dstd.make_tensor_list([g], out=out), 2.0 ** -10 * (1 - 2.0 ** -30), norm=norm,
                   norm_given=True)
    assert bool(((out[0] if outside else g) == 2.0 ** -30).all())


@pytest.mark.parametrize("sizes", [[5000, 3], [60_001, 7]])
@pytest.mark.parametrize("o_type", [None, "f32"])
def test_clip_of_finite_gradients_whose_norm_leaves_fp32(dev, o_type, sizes):
    import torch
    from paper_2607_14672_amd import dstd
    with np.errstate(over="ignore"):
        vals = [np.clip(v, -3.3e38, 3.3e38) for v in _normal(np.random.default_rng(23), sizes, 1.5e38)]
    g = Arena(vals, "f32", 1, dev)
    o = Arena([0 * v for v in vals], o_type, 2, dev) if o_type else None
    before = g.get()
    ref = _norm64(before)
    assert ref > 1e39
    tl = dstd.make_tensor_list(g.t, out=o.t if o else None)
    assert dstd.grad_clip(tl, 0.5).item() == math.inf
    for x, b in zip((o or g).get(), before):
        _close(x, b * (0.5 / ref), np.abs(b) * (0.5 / ref) * MORE * 2 * U, "clipped")
    assert g.gaps_kept() and (o is None or o.gaps_kept())


@pytest.mark.parametrize("sizes", [[5000, 3], [60_001, 7]])
def test_adamw_of_finite_gradients_whose_norm_leaves_fp32(dev, sizes):
    """Clipped, the step is made; without a bound in fp32 it is skipped."""
    import torch
    from paper_2607_14672_amd import dstd
    tr = Train(dev, sizes, seed=24, g_scale=3e37)
    for a, n in tr.g.slots:  # a norm beyond fp32 in the short list, too
        tr.g.buf[a:a + 2] = 3e38
    before = tr.g.get(), tr.w.get(), tr.m.get(), tr.v.get()
    ref = _norm64(before[0])
    assert ref > 3.5e38
    kept, step = tr.bits(), torch.full((1,), 9, dtype=torch.int64, device=dev)
    for max_norm in (math.inf, 1e300):  # asked for by the norm; with a bound that is none
        norm = dstd.adamw_step(tr.tl, dstd.make_adamw(max_norm=max_norm), step,
                               norm=torch.zeros(1, device=dev))
        assert norm.item() == math.inf and step.item() == 9
        assert all(torch.equal(a, b) for a, b in zip(tr.bits(), kept))
    norm = dstd.adamw_step(tr.tl, dstd.make_adamw(lr=2e-3, max_norm=0.5, **HP), step)
    assert norm.item() == math.inf and step.item() == 10
    _check_step(tr, before, 10, HP, 0.5 / ref, 2e-3)


# ------------------------------------------------- both forms of each launch --
# 4 chunks, 124 and 2199: one launch of one block for a clip, one block per
# chunk, and more chunks than a list that is clipped in place has blocks. A step
# takes one block for at most 3: the first list without its last tensor.
FORMS = {"block": [9000, 5], "blocks": [500_001, 7], "strided": [9_000_001, 20]}


def _places(sizes):
    """The first element, one in the middle, the last (of the last tensor)."""
    return [(0, 0), (0, sizes[0] // 2), (len(sizes) - 1, sizes[-1] - 1)]


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", sorted(FORMS))
def test_norm_of_what_is_not_finite_in_every_form(dev, form, dtype, value):
    from paper_2607_14672_amd import dstd
    sizes = FORMS[form]
    for k, i in _places(sizes):
        g = Arena([np.ones(n, dtype=np.float32) for n in sizes], dtype, 1, dev)
        g.t[k][i] = value
        got = dstd.grad_norm(dstd.make_tensor_list(g.t)).item()
        assert math.isnan(got) if math.isnan(value) else got == math.inf, (k, i, got)


@pytest.mark.parametrize("value", [math.inf, math.nan])
@pytest.mark.parametrize("outs", ["in place", "outside", "mixed"])
@pytest.mark.parametrize("form", sorted(FORMS))
def test_clip_with_a_norm_that_is_not_finite_in_every_form(dev, form, outs, value):
    """In place nothing changes; elsewhere the gradients are copied, bit for bit.
    Measured by the call itself, and given."""
    import torch
    from paper_2607_14672_amd import dstd
    sizes = FORMS[form]
    vals = _normal(np.random.default_rng(31), sizes)
    for k, i in _places(sizes):
        for given in (False, True):
            g, o = Arena(vals, "f32", 1, dev), Arena([0 * v for v in vals], "f32", 3, dev)
            if not given:
                g.t[k][i] = value
            kept = g.buf.clone()
            out = {"in place": None, "outside": o.t, "mixed": [None] + o.t[1:]}[outs]
            norm = torch.tensor([value], device=dev) if given else None
            got = dstd.grad_clip(dstd.make_tensor_list(g.t, out=out), 1e-3, norm=norm, norm_given=given)
            assert not math.isfinite(got.item())
            assert torch.equal(g.buf.view(torch.int32), kept.view(torch.int32))
            for a, b, into in zip(o.t, g.t, out or [None] * len(sizes)):
                if into is None:
                    assert not bool(a.any())
                else:
                    assert torch.equal(a.view(torch.int32), b.view(torch.int32))
            assert o.gaps_kept()


@pytest.mark.parametrize("outs", ["in place", "outside", "mixed"])
@pytest.mark.parametrize("form", sorted(FORMS))
def test_clip_by_a_given_norm_in_every_form(dev, form, outs):
    """Clipped, and with nothing to clip, where the gradients stay or are copied."""
    import torch
    from paper_2607_14672_amd import dstd
    sizes = FORMS[form]
    vals = _normal(np.random.default_rng(32), sizes)
    for given, max_norm in ((8.0, 2.0), (8.0, 8.0), (0.0, 1.0)):
        g, o = Arena(vals, "f32", 2, dev), Arena([0 * v for v in vals], "f32", 0, dev)
        out = {"in place": None, "outside": o.t, "mixed": [None] + o.t[1:]}[outs]
        norm = torch.tensor([given], device=dev)
        dstd.grad_clip(dstd.make_tensor_list(g.t, out=out), max_norm, norm=norm, norm_given=True)
        assert norm.item() == given
        c = 0.25 if max_norm < given else 1.0  # a power of two: exact
        for a, b, v, into in zip(o.get(), g.get(), vals, out or [None] * len(sizes)):
            want = v.astype(np.float64)
            assert np.array_equal(b, want * (c if into is None else 1.0))
            assert np.array_equal(a, want * c) if into is not None else not a.any()
        assert g.gaps_kept() and o.gaps_kept()


STEP_FORMS = {"block": [9000], "blocks": [500_001, 7], "far": [9_000_001, 20]}


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("g_type,w_type,master", [("f32", "f32", False), ("bf16", "bf16", True),
                                                  ("f32", "bf16", False)])
@pytest.mark.parametrize("form", sorted(STEP_FORMS))
def test_a_skipped_step_changes_nothing_in_every_form(dev, form, g_type, w_type, master, value):
    """A norm that is not finite: asked for by max_norm, by a place for it alone,
    and given. Weights, copies, moments, gaps and step number keep their bits."""
    import torch
    from paper_2607_14672_amd import dstd
    sizes = STEP_FORMS[form]
    tr = Train(dev, sizes, g_type, w_type, master, shift=1, seed=33)
    step = torch.full((1,), 3, dtype=torch.int64, device=dev)
    for k, i in _places(sizes):
        old = tr.g.t[k][i].clone()
        tr.g.t[k][i] = value
        kept = tr.bits()
        calls = [(1.0, None, False), (math.inf, torch.zeros(1, device=dev), False),
                 (1.0, torch.tensor([value], device=dev), True),
                 (math.inf, torch.tensor([value], device=dev), True)]
        for max_norm, norm, given in calls:
            norm = dstd.adamw_step(tr.tl, dstd.make_adamw(max_norm=max_norm), step, norm=norm,
                                   norm_given=given)
            got = norm.item()
            assert math.isnan(got) if math.isnan(value) else abs(got) == math.inf
            assert step.item() == 3
            for a, b in zip(tr.bits(), kept):
                bits = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
                assert torch.equal(a.view(bits), b.view(bits))
        tr.g.t[k][i] = old
    # no norm asked for: the step is made
    assert dstd.adamw_step(tr.tl, dstd.make_adamw(), step) is None and step.item() == 4
    assert all(a.gaps_kept() for a in tr.arenas)


@pytest.mark.parametrize("form", sorted(STEP_FORMS))
def test_adamw_by_a_given_norm_in_every_form(dev, form):
    import torch
    from paper_2607_14672_amd import dstd
    tr = Train(dev, STEP_FORMS[form], seed=34)
    before = tr.g.get(), tr.w.get(), tr.m.get(), tr.v.get()
    norm = torch.tensor([8.0], device=dev)
    step = torch.full((1,), 6, dtype=torch.int64, device=dev)
    dstd.adamw_step(tr.tl, dstd.make_adamw(lr=1e-3, max_norm=2.0, **HP), step, norm=norm, norm_given=True)
    torch.cuda.synchronize()
    assert norm.item() == 8.0 and step.item() == 7
    _check_step(tr, before, 7, HP, 0.25, 1e-3)
