"""Gradients written where the caller wants them: `grad_W` of the backward
helpers, and training steps whose tensor list holds those places."""
import math

import pytest

from tests.test_gpu_conv import _conv_case
from tests.test_gpu_dense import _layer_case
from tests.test_gpu_exact import _case as _exact_case
from tests.test_gpu_multispike import _case as _ms_case

pytestmark = pytest.mark.gpu
CONV = dict(C_in=3, H=7, W=6, C_out=5, KH=3, KW=3, stride=1, pad=1, pool_in=1)


@pytest.fixture(scope="module")
def dev():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2607_14672_amd import dstd
    dstd._load()  # fail loudly if the HIP library is missing
    return torch.device("cuda:0")


def _backward(kind, dev, bf16=False):
    """(weights, the backward as a call that takes need_W and grad_W)."""
    import torch
    from paper_2607_14672_amd import dstd

    def put(t, W):
        W = torch.from_numpy(W).to(dev)
        return torch.from_numpy(t).to(dev), W.bfloat16() if bf16 else W

    if kind == "conv":
        p, t, W = _conv_case(41, 3, CONV, 8, 1.0, 0.5)
        p, cs = dstd.make_params(**p), dstd.make_conv_shape(**CONV)
        t, W = put(t, W)
        out = dstd.conv_forward(p, cs, t, W)
        return W, lambda **kw: dstd.conv_backward(p, cs, t, W, *out, torch.ones_like(out[0]), **kw)
    if kind == "multispike":
        p, t, W = _ms_case(42, 3, 20, 2, 9, 8, 1.0, 0.5)
        p = dstd.make_params(**p)
        t, W = put(t, W)
        out = dstd.multispike_forward(p, t, W, 3)
        return W, lambda **kw: dstd.multispike_backward(p, t, W, *out, torch.ones_like(out[0]), **kw)
    if kind == "exact":
        p, t, W = _exact_case(43, 3, 33, 9, 1.0, 0.5)
        p = dstd.make_params(p["tau_m"], p["tau_s"], p["threshold"], 1, 0.0, 1.0, p["t_max"])
        t, W = put(t, W)
        out = dstd.exact_forward(p, t, W)
        return W, lambda **kw: dstd.exact_backward(p, t, W, *out, torch.ones_like(out[0]), **kw)
    p, t, W = _layer_case(44, 3, 33, 17, 8, 1.0, 0.5)
    p = dstd.make_params(**p)
    t, W = put(t, W)
    out = dstd.forward(p, t, W)
    return W, lambda **kw: dstd.backward(p, t, W, *out, torch.ones_like(out[0]), **kw)


KINDS = ["dense", "conv", "multispike", "exact"]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("kind", KINDS)
def test_gradient_goes_to_its_place(dev, kind, bf16):
    """The same gradient as in a new tensor, nothing outside the place."""
    import torch
    W, backward = _backward(kind, dev, bf16)
    want, want_t = backward()
    assert bool(want.any()) and bool(torch.isfinite(want).all())
    room = torch.full((W.numel() + 128,), -7.0, device=dev)
    place = room[64:-64].view(W.shape)
    got, got_t = backward(grad_W=place)
    assert got is place and torch.equal(place, want) and torch.equal(got_t, want_t)
    assert bool((room[:64] == -7).all()) and bool((room[-64:] == -7).all())
    # once more over what is there, without dL/dt_in
    place.fill_(math.nan)
    assert torch.equal(backward(grad_W=place, need_t_in=False)[0], want)


@pytest.mark.parametrize("kind", KINDS)
def test_places_that_do_not_fit_are_refused(dev, kind):
    import torch
    W, backward = _backward(kind, dev)
    for bad, err in ((W.double(), TypeError), (W.bfloat16(), TypeError), (1.0, TypeError),
                     (W.cpu(), ValueError), (torch.zeros(W.numel(), device=dev), ValueError),
                     (torch.zeros(W.shape + (2,), device=dev)[..., 0], ValueError), (W, ValueError)):
        with pytest.raises(err, match="grad_W"):
            backward(grad_W=bad)
    with pytest.raises(ValueError, match="need_W"):
        backward(grad_W=torch.zeros_like(W), need_W=False)


def test_training_through_the_helpers(dev):
    """A list built once, two layers, steps whose gradients all differ: each step
    applies the gradients of its own backward."""
    import torch
    from paper_2607_14672_amd import dstd
    p, t, W0 = _layer_case(45, 6, 40, 30, 8, math.inf, math.inf)
    _, _, W1 = _layer_case(46, 6, 30, 10, 8, math.inf, math.inf)
    p, t = dstd.make_params(**p), torch.from_numpy(t).to(dev)
    W = [torch.from_numpy(w).to(dev) for w in (W0, W1)]
    grads, m, v = ([torch.zeros_like(w) for w in W] for _ in range(3))
    tl = dstd.make_tensor_list(grads, weights=W, m=m, v=v)
    step, hp = torch.zeros(1, dtype=torch.int64, device=dev), dstd.make_adamw(lr=0.01, max_norm=0.1)
    target = torch.full((6, 10), 0.5, device=dev)
    seen = []
    for k in range(4):
        h = dstd.forward(p, t, W[0])
        o = dstd.forward(p, h[0], W[1])
        g, _ = dstd.mse_grad(o[0], target)
        # the same backward into new tensors: what the update has to use
        fresh1, g_h = dstd.backward(p, h[0], W[1], *o, g)
        fresh0, _ = dstd.backward(p, t, W[0], *h, g_h, need_t_in=False)
        _, g_h = dstd.backward(p, h[0], W[1], *o, g, grad_W=grads[1])
        dstd.backward(p, t, W[0], *h, g_h, need_t_in=False, grad_W=grads[0])
        assert torch.equal(grads[0], fresh0) and torch.equal(grads[1], fresh1)
        copy = dict(weights=[w.clone() for w in W], m=[x.clone() for x in m], v=[x.clone() for x in v])
        norm = dstd.adamw_step(dstd.make_tensor_list([fresh0, fresh1], **copy), hp, step.clone())
        assert torch.equal(dstd.adamw_step(tl, hp, step), norm)
        for a, b in zip(W + m + v, copy["weights"] + copy["m"] + copy["v"]):
            assert torch.equal(a, b)
        seen.append(norm.item())
    assert step.item() == 4 and len(set(seen)) == 4 and min(seen) > 0.0
