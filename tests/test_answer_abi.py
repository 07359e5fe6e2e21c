"""Contract of the top logits, the distillation and the sampling on the CPU: every
invalid argument is refused on the host, before anything touches a device."""
import ctypes as C
import math

import pytest

from paper_2607_14672_amd import dstd

OK, NULL, SHAPE, PARAM, UNSUP, WS = (dstd.DSTD_OK, dstd.DSTD_ERR_NULL, dstd.DSTD_ERR_SHAPE,
                                     dstd.DSTD_ERR_PARAM, dstd.DSTD_ERR_UNSUPPORTED,
                                     dstd.DSTD_ERR_WORKSPACE)
A = 1 << 40  # made-up addresses, far apart
X, IDX, LOGIT, REST, GRAD, LOSS, U, WSP = (A * (k + 1) for k in range(8))
BIG = 1 << 34


def test_structs_match_the_header():
    assert C.sizeof(dstd.dstd_scores) == 8 + 3 * 8 + 4 + 4 + 8
    assert C.sizeof(dstd.dstd_sample_params) == 8 + 2 * 8


def _s(**kw):
    f = dict(x=X, B=4, N=100, ld=100, dtype=dstd.DSTD_F32, cap=math.nan, scale=1.0)
    f.update(kw)
    return dstd.dstd_scores(*(f[k] for k in ("x", "B", "N", "ld", "dtype", "cap", "scale")))


def _top(s, K=5, idx=IDX, logit=LOGIT, rest=REST):
    return dstd.dstd_top_logits(s, K, idx, logit, rest, None)


def _sample(s, top_k=0, top_p=1.0, min_p=0.0, u=U, choice=IDX, logp=LOGIT):
    return dstd.dstd_sample(s, dstd.dstd_sample_params(top_k, top_p, min_p), u, choice, logp, None)


SCORES = [(dict(B=-1), SHAPE), (dict(B=65536), SHAPE), (dict(N=0), SHAPE), (dict(N=1 << 24), SHAPE),
          (dict(ld=99), SHAPE), (dict(ld=-100), SHAPE), (dict(ld=(1 << 40) + 1), SHAPE),
          (dict(dtype=2), PARAM), (dict(dtype=-1), PARAM), (dict(scale=0.0), PARAM),
          (dict(scale=math.inf), PARAM), (dict(scale=math.nan), PARAM), (dict(scale=1e39), PARAM),
          (dict(scale=1e-60), PARAM), (dict(x=None), NULL), (dict(x=X + 2), PARAM)]


@pytest.mark.parametrize("kw,status", SCORES)
def test_scores_are_checked(kw, status):
    assert _top(_s(**kw)) == status, dstd.dstd_last_error()
    assert _sample(_s(**kw)) == status, dstd.dstd_last_error()


def test_top_logits_arguments():
    assert _top(None) == NULL
    assert _top(_s(), K=0) == SHAPE
    assert _top(_s(), K=-3) == SHAPE
    assert _top(_s(), K=101) == SHAPE
    assert _top(_s(N=1000, ld=1000), K=dstd.DSTD_MAX_TOP + 1) == UNSUP
    assert _top(_s(), idx=None) == NULL
    assert _top(_s(), logit=None) == NULL
    assert _top(_s(), idx=IDX + 2) == PARAM
    # overlaps: outputs with the scores (their last row too) and each other
    assert _top(_s(), idx=X + 4 * 399) == PARAM
    assert _top(_s(ld=1000), rest=X + 4 * 3099) == PARAM
    assert _top(_s(), logit=IDX + 4 * 19) == PARAM
    assert _top(_s(), rest=LOGIT) == PARAM


def test_sample_arguments():
    p = dstd.dstd_sample_params(0, 1.0, 0.0)
    assert dstd.dstd_sample(_s(), None, U, IDX, LOGIT, None) == NULL
    assert dstd.dstd_sample(None, p, U, IDX, LOGIT, None) == NULL
    for bad in (dict(top_k=-1), dict(top_p=0.0), dict(top_p=1.0000001), dict(top_p=-0.5),
                dict(top_p=math.nan), dict(min_p=-1e-9), dict(min_p=1.1), dict(min_p=math.nan)):
        assert _sample(_s(), **bad) == PARAM, bad
    assert _sample(_s(), u=None) == NULL
    assert _sample(_s(), choice=None) == NULL
    assert _sample(_s(), choice=U) == PARAM
    assert _sample(_s(), logp=U + 12) == PARAM
    assert _sample(_s(), choice=X) == PARAM
    assert _sample(_s(), choice=IDX, logp=IDX) == PARAM


def _distill(B=4, N=100, K=5, t=X, ld_t=None, idx=IDX, logit=LOGIT, dtype=dstd.DSTD_F32, rest=REST, tau=0.1,
             cap=1.0, weight=1.0, acc=0, grad=GRAD, ld_g=None, loss=LOSS, ws=WSP, size=BIG):
    return dstd.dstd_distill_grad(B, N, K, t, N if ld_t is None else ld_t, idx, logit, dtype, rest, tau, cap,
                                  weight, acc, grad, N if ld_g is None else ld_g, loss, ws, size, None)


@pytest.mark.parametrize("kw,status", [
    (dict(B=-1), SHAPE), (dict(B=65536), SHAPE), (dict(N=0), SHAPE), (dict(N=1 << 24, K=1), SHAPE),
    (dict(K=0), SHAPE), (dict(K=101), SHAPE), (dict(N=1000, K=257), UNSUP), (dict(ld_t=99), SHAPE),
    (dict(ld_g=99), SHAPE), (dict(dtype=7), PARAM), (dict(tau=0.0), PARAM), (dict(tau=-1.0), PARAM),
    (dict(tau=math.inf), PARAM), (dict(tau=math.nan), PARAM), (dict(tau=1e-44), PARAM),
    (dict(cap=math.inf), PARAM), (dict(cap=math.nan), PARAM), (dict(weight=-1.0), PARAM),
    (dict(weight=math.inf), PARAM), (dict(weight=math.nan), PARAM), (dict(acc=2), PARAM),
    (dict(t=None), NULL), (dict(idx=None), NULL), (dict(logit=None), NULL), (dict(loss=None), NULL),
    (dict(N=100000, ws=None), NULL), (dict(N=100000, ws=WSP + 8), WS),
    (dict(N=100000, size=1), WS), (dict(t=X + 1), PARAM), (dict(weight=1e38, tau=1e-3), PARAM),
    (dict(grad=X), PARAM), (dict(grad=X + 4 * 399), PARAM), (dict(ld_t=1000, grad=X + 4 * 3000), PARAM),
    (dict(loss=GRAD + 4 * 399), PARAM), (dict(loss=REST + 8), PARAM), (dict(rest=GRAD), PARAM),
    (dict(idx=GRAD), PARAM), (dict(N=100000, ws=IDX), PARAM), (dict(logit=LOGIT + 2), PARAM),
])
def test_distill_arguments(kw, status):
    assert _distill(**kw) == status, dstd.dstd_last_error()


def test_workspace_sizes_grow_with_what_they_hold():
    assert dstd.dstd_distill_workspace_size(1, 10, 1) == 0  # none is needed
    assert dstd.dstd_distill_workspace_size(1, 1 << 20, 1) >= 128 * 8
    assert dstd.dstd_distill_workspace_size(65535, (1 << 24) - 1, 256) > 65535 * 8
    for bad in ((-1, 10, 1), (1, 0, 1), (1, 10, 11), (1, 1000, 257)):
        assert dstd.dstd_distill_workspace_size(*bad) == 0


@pytest.mark.parametrize("call", ["top", "distill", "sample"])
def test_helpers_refuse_cpu_tensors_and_wrong_types(call):
    import torch
    x = torch.zeros(4, 9)
    i = torch.zeros(4, 2, dtype=torch.int32)
    f = dict(top=lambda x: dstd.top_logits(x, 2), sample=lambda x: dstd.sample(x, torch.zeros(4)),
             distill=lambda x: dstd.distill_grad(x, i, torch.zeros(4, 2), t_cap=1.0))[call]
    with pytest.raises(ValueError, match="GPU"):
        f(x)
    with pytest.raises(TypeError, match="float32"):
        f(x.double())
    with pytest.raises(TypeError, match="tensor"):
        f([1.0, 2.0])
