"""The rest of a softmax behind its top logits where the others lie far below them, or scores
far from 0.

Tolerance: a term of the sum takes a difference, the scale and their product with half a step
(H) each, 3 H of its distance to the others' largest (ln N of them at the mean at most); exp2
is two half steps off, again at each of the some 30 places where partial sums are joined, and
a thread adds N over its block's threads (64 up to 512 scores, 256 up to 16384, 1024 beyond)
one by one. The result is rounded once."""
import math

import numpy as np
import pytest

from tests import answer_ref as ref

pytestmark = pytest.mark.gpu

H = 2.0 ** -24


def eps(N):
    T = 64 if N <= 512 else 256 if N <= 16384 else 1024
    return H * (3 * math.log(N + 1) + 2 * 30 + 4 + math.ceil(N / T))


def _torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2607_14672_amd import dstd
    return torch, dstd


def _check_rest(torch, dstd, x, dtype, K, scale, cap=None):
    v = torch.from_numpy(x).to(dtype).cuda()
    idx, logit, rest = (a.cpu().numpy() for a in dstd.top_logits(v, K, scale=scale, cap=cap))
    e_idx, e_logit, e_rest = ref.top(v.float().cpu().numpy(), K, scale, cap)
    assert np.array_equal(idx, e_idx)
    f = np.isfinite(e_logit)
    assert np.all(np.abs(logit[f] - e_logit[f]) <= H * np.abs(e_logit[f]))
    bad = np.isfinite(rest) != np.isfinite(e_rest)
    assert not bad.any(), (np.argwhere(bad)[:4].ravel(), rest[bad][:4], e_rest[bad][:4])
    bad = np.isfinite(e_rest)
    bad[bad] = np.abs(rest[bad] - e_rest[bad]) > eps(x.shape[1]) + H * np.abs(e_rest[bad])
    assert not bad.any(), (np.argwhere(bad)[:4].ravel(), rest[bad][:4], e_rest[bad][:4])


# how far below the top the others lie: around where an fp32 exponential becomes 0 (87.3) and
# where even its denormal numbers end (104)
GAPS = [50.0, 80.0, 85.0, 86.5, 87.0, 87.25, 87.5, 90.0, 100.0, 103.5, 104.5, 200.0]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [400, 2000, 20011, 131072])
def test_others_far_below_the_top(N, dtype):
    """Row by row another gap: the top K, one entry at the gap, the others half a unit and
    more behind it."""
    torch, dstd = _torch()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rng = np.random.default_rng(N)
    for K in (1, 7):
        for behind in (0.5, 3.0):
            x = np.empty((len(GAPS), N), dtype=np.float32)
            for b, gap in enumerate(GAPS):
                x[b] = -gap - behind - rng.integers(0, 3, N) * 0.5
                at = rng.permutation(N)[:K + 1]
                x[b, at[:K]] = 0.5 * rng.integers(0, 4, K)
                x[b, at[K]] = -gap
            print(f"N={N} {dtype} K={K} behind={behind}", flush=True)
            _check_rest(torch, dstd, x, dt, K, 1.0)
            _check_rest(torch, dstd, x * -0.125, dt, K, -8.0)


@pytest.mark.parametrize("N", [2000, 20011])
def test_spike_times_of_a_cold_softmax(N):
    """Spike times with tau_soft = 0.01: a class fires early, the others up to 1.5 later."""
    torch, dstd = _torch()
    rng = np.random.default_rng(N)
    for start in (0.8, 0.85, 0.9, 1.0, 1.1):
        t = (start + 0.3 * rng.random((8, N))).astype(np.float32)
        t[rng.random(t.shape) < 0.3] = np.inf
        t[:, N // 2] = 0.0
        t[:, N // 3] = 0.01
        _check_rest(torch, dstd, t, torch.float32, 2, -100.0, 1.5)
        _check_rest(torch, dstd, t, torch.float32, 2, -100.0)


@pytest.mark.parametrize("N", [400, 2000, 20011])
@pytest.mark.parametrize("power", [20, 24, 28, 34, 60])
def test_scores_whose_logits_are_beyond_the_integers_of_fp32(N, power):
    """One entry a row at the top, the others a step of fp32 below it, with logits just above
    a power of two, where the product with log2(e) is rounded by up to a step of theirs."""
    torch, dstd = _torch()
    scale = 0.7
    c2 = np.float32(scale * math.log2(math.e))
    top = np.float32(2.0 ** power / float(c2))
    x = np.empty((400, N), dtype=np.float32)
    for b in range(x.shape[0]):
        top = np.nextafter(top, np.float32(np.inf))
        x[b] = np.nextafter(top, np.float32(0))
        x[b, b * 7 % N] = top
    _check_rest(torch, dstd, x, torch.float32, 1, scale)
    _check_rest(torch, dstd, -x, torch.float32, 1, -scale)


@pytest.mark.parametrize("scale", [2.3e38, -2.3e38])
@pytest.mark.parametrize("N", [400, 2000, 20011])
def test_rest_at_the_largest_scales(N, scale):
    """Scores of a few steps of 2^-128, whose logits are 0.7 apart."""
    torch, dstd = _torch()
    scale = float(np.float32(scale))
    x = (np.random.default_rng(N).integers(-30, 30, (6, N)) * 2.0 ** -128).astype(np.float32)
    x[0] = 0.0
    for dt in (torch.float32, torch.bfloat16):
        _check_rest(torch, dstd, x, dt, 1, scale)
        _check_rest(torch, dstd, x, dt, 9, scale)


def test_scales_beyond_those_of_rest():
    """Top logits without a rest, and sampling, take every scale that is finite in fp32."""
    torch, dstd = _torch()
    scale = float(np.float32(3.3e38))
    x = (np.random.default_rng(1).integers(-30, 30, (50, 3001)) * 2.0 ** -129).astype(np.float32)
    v = torch.from_numpy(x).cuda()
    with pytest.raises(dstd.DSTDError, match="log2"):
        dstd.top_logits(v, 4, scale=scale)
    idx = torch.empty((50, 4), dtype=torch.int32, device="cuda")
    logit = torch.empty((50, 4), device="cuda")
    st = dstd.dstd_top_logits(dstd.make_scores(v, scale), 4, idx.data_ptr(), logit.data_ptr(), None,
                              torch.cuda.current_stream().cuda_stream)
    assert st == dstd.DSTD_OK
    e_idx, e_logit, _ = ref.top(x, 4, scale, None)
    torch.cuda.synchronize()
    assert np.array_equal(idx.cpu().numpy(), e_idx)
    assert np.all(np.abs(logit.cpu().numpy() - e_logit) <= H * np.abs(e_logit))
    c, logp = dstd.sample(v, torch.full((50,), 0.3, device="cuda"), scale=scale, top_p=0.9)
    w = ref.kept(x, scale, None, 0, 0.9, 0.0)
    cum = np.cumsum(w, axis=1)
    for b, k in enumerate(c.tolist()):
        # 3001 weights to 2^-51 each, and the reference's own sums
        below, goal = (cum[b, k - 1] if k else 0.0), float(np.float32(0.3)) * cum[b, -1]
        assert w[b, k] > 0 and below <= goal + 1e-10 and cum[b, k] > goal - 1e-10
