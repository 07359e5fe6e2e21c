"""Sums over long rows to their last entry, and the weights' gradient behind a distillation.

Where all others of a row are equal, their terms are one power of two and fp32 adds them
exactly, up to 2^24 of them: whatever the length of the row, the sum is off by a few half
steps (H) alone, and a vector of four that is left out shows up to some 2^21 entries."""
import math

import numpy as np
import pytest

import oracle
from tests import answer_ref as ref
from tests.parity import check_forward, check_grad, grad_err_inputs
from tests.test_gpu_distill_ends import reference
from tests.test_gpu_top_rest import _check_rest

pytestmark = pytest.mark.gpu

H = 2.0 ** -24


def _torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2607_14672_amd import dstd
    return torch, dstd


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [513, 2001, 16384, 20011, 131072, 131077, (1 << 24) - 1])
def test_rest_counts_every_entry(N, dtype):
    """K entries in different threads' shares, the others equal: rest = ln(N - K). A term is
    off by 2 H, the logarithm and its rounding by 2 H and half a step of ln N."""
    torch, dstd = _torch()
    dt, vec = (torch.bfloat16, 8) if dtype == "bf16" else (torch.float32, 4)
    for K in (1, 60):
        x = torch.zeros((2, N), dtype=dt, device="cuda")
        x[:, torch.arange(K, device="cuda") * vec % (N - 1)] = 10.0
        _, logit, rest = dstd.top_logits(x, K, scale=math.log(2.0))
        torch.cuda.synchronize()
        assert np.all(np.abs(logit.cpu().numpy() - 10 * math.log(2.0)) <= 10 * H)
        want = math.log(N - K)
        assert np.all(np.abs(rest.cpu().numpy() - want) <= H * want + 8 * H), (rest, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,N", [(4, 3000), (4, 16384), (4, 16385), (4, 131072), (1, 1 << 20)])
def test_rest_of_long_rows(B, N, dtype):
    """Ordinary rows against the tolerance of the threads that share them."""
    torch, dstd = _torch()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = (np.random.default_rng(N).standard_normal((B, N)) * 3).astype(np.float32)
    for K in (1, 64, 256):
        _check_rest(torch, dstd, x, dt, K, 0.9)
        _check_rest(torch, dstd, x, dt, K, -1.1)


@pytest.mark.parametrize("B,N", [(6, 11), (6, 299), (6, 3001), (6, 8191), (36, 12001), (36, 20003), (36, 40001),
                                 (33, 65536), (6, 20003), (6, 70001), (1, 1 << 20)])
def test_distillation_counts_every_neuron(B, N):
    """All classes outside the record at one time, or silent at that time's cap: their sum is
    exact. The record's own sum joins 20 entries, 4 H and 3 H of a distance of 10 each at most
    a join, over 6 joins and 4 entries a lane."""
    torch, dstd = _torch()
    rng = np.random.default_rng(N)
    K = min(N // 3, 20)
    tau, t_cap = 0.25, 1.5
    for silent in (False, True):
        t = np.full((B, N), t_cap, dtype=np.float32)
        if silent:
            t[rng.random((B, N)) < 0.5] = np.inf
        idx = np.stack([rng.permutation(N)[:K] for _ in range(B)]).astype(np.int32)
        np.put_along_axis(t, idx.astype(np.int64), rng.random((B, K)).astype(np.float32), 1)
        logit = rng.standard_normal((B, K)).astype(np.float32)
        rest = (math.log(N) - 2 + rng.standard_normal(B)).astype(np.float32)
        g, loss = dstd.distill_grad(*(torch.from_numpy(v).cuda() for v in (t, idx, logit, rest)), tau_soft=tau,
                                    t_cap=t_cap, weight=1.0)
        torch.cuda.synchronize()
        g, loss = g.cpu().numpy().astype(np.float64), loss.cpu().numpy().astype(np.float64)
        e_loss, ltol, e_grad, gtol = reference(t, idx, logit, rest, tau, t_cap, 1.0, E=40 * H)
        bad = np.abs(g - e_grad) > gtol
        assert not bad.any(), (np.argwhere(bad)[:3], g[bad][:3], e_grad[bad][:3], gtol[bad][:3])
        assert np.all(np.abs(loss[1:] - e_loss) <= ltol), (loss[1:], e_loss, ltol)


# ------------------------------------------------- behind the loss: the weights --
def _student(seed=3):
    rng = np.random.default_rng(seed)
    B, N_in, N, M = 16, 96, 200, 16
    p = dict(tau_m=1.0, tau_s=0.3, threshold=1.0, M=M, t0=0.0, dt=1.0 / M)
    t_in = rng.random((B, N_in)).astype(np.float32)
    W_t, W_s = ((7.0 / N_in * (1 + 0.3 * math.sqrt(N_in) * rng.standard_normal((N, N_in)))).astype(np.float32)
                for _ in range(2))
    return p, t_in, W_t, W_s, rng


def _loss64(p, t_in, W, rec, tau, t_cap):
    """The student's loss by the oracle; W in 64 bits."""
    t = oracle.dstd_forward(p, t_in, W)["t_out"]
    return ref.distill(t, *rec, tau, t_cap, 1.0 / len(t))[0].sum()


def test_weights_gradient_of_a_distilled_layer():
    """A teacher's record, a student's forward, the distillation's gradient and the layer's
    backward: the weights' gradient is the 64-bit oracle's, and that is the difference of the
    64-bit loss along directions. The student's answers are drawn from what is kept."""
    torch, dstd = _torch()
    p, t_in, W_t, W_s, rng = _student()
    tau, t_cap, K = 0.25, 1.625, 40
    prm = dstd.make_params(p["tau_m"], p["tau_s"], p["threshold"], p["M"], p["t0"], p["dt"])
    ti, Wt, Ws = (torch.from_numpy(v).cuda() for v in (t_in, W_t, W_s))
    rec = dstd.top_logits(dstd.forward(prm, ti, Wt)[0], K, scale=-1.0 / tau, cap=t_cap)
    t, slope, q = dstd.forward(prm, ti, Ws)
    g, loss = dstd.distill_grad(t, *rec, tau_soft=tau, t_cap=t_cap)
    orc = oracle.dstd_forward(p, t_in, W_s)
    fwd = dict(t_out=t.cpu().numpy(), slope=slope.cpu().numpy(), q=q.cpu().numpy())
    mask, st = check_forward(fwd, orc, t_in.shape[1], p["M"] * p["dt"], label="student", taus=(p["tau_m"], p["tau_s"]))
    gm = torch.where(torch.from_numpy(mask).cuda(), 0.0, g)
    gW, _ = dstd.backward(prm, ti, Ws, t, slope, q, gm, need_t_in=False)
    g64 = np.where(orc["q"] >= 0, gm.cpu().numpy().astype(np.float64), 0.0)
    oW, _, oWa, _, oWe, _ = oracle.dstd_backward(p, t_in, W_s, orc, g64, want_dt=False, want_abs=True,
                                                 err=grad_err_inputs(st, mask))
    check_grad(gW.cpu().numpy(), oW, "student dW", oWa, oWe, n_terms=2 * len(t_in))
    # the oracle's gradient from the loss's own, without a mask, against differences
    rec64 = [v.cpu().numpy() for v in rec]
    grad = ref.distill(orc["t_out"], *rec64, tau, t_cap, 1.0 / len(t_in))[1]
    oW = oracle.dstd_backward(p, t_in, W_s, orc, grad, want_dt=False)[0]
    h = 1e-7
    for d in [oW / np.abs(oW).max()] + [rng.standard_normal(oW.shape) for _ in range(3)]:
        near, far = ((_loss64(p, t_in, W_s + k * h * d, rec64, tau, t_cap) -
                      _loss64(p, t_in, W_s - k * h * d, rec64, tau, t_cap)) / (2 * k * h) for k in (1, 2))
        # a third of far - near is what near is off by (h^2); the losses' rounding, 2^-50 / h
        assert abs(near - np.sum(oW * d)) <= abs(far - near) + 2.0 ** -50 * 10 / h
    u = torch.from_numpy(rng.random(len(t_in)).astype(np.float32)).cuda()
    choice, _ = dstd.sample(t, u, scale=-1.0 / tau, cap=t_cap, top_k=10)
    w = ref.kept(fwd["t_out"], -1.0 / tau, t_cap, 10, 1.0, 0.0)
    assert all(0 <= c and w[b, c] > 0 for b, c in enumerate(choice.tolist()))
