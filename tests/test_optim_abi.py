"""Contract of the tensor lists, the global norm, clipping and AdamW on the CPU:
every invalid argument is refused on the host, before anything touches a device."""
import ctypes as C
import math

import pytest

from paper_2607_14672_amd import dstd

OK, NULL, SHAPE, PARAM, WS = (dstd.DSTD_OK, dstd.DSTD_ERR_NULL, dstd.DSTD_ERR_SHAPE,
                              dstd.DSTD_ERR_PARAM, dstd.DSTD_ERR_WORKSPACE)
F32, BF16 = dstd.DSTD_F32, dstd.DSTD_BF16


def _tensors(*rows):
    """Tensors with made-up addresses, far apart; each row overrides fields."""
    arr = (dstd.dstd_tensor * max(len(rows), 1))()
    for k, (t, row) in enumerate(zip(arr, rows)):
        base = (k + 1) << 32
        full = dict(g=base, out=None, w=base + (1 << 28), w32=None, m=base + (2 << 28),
                    v=base + (3 << 28), n=100, g_dtype=F32, out_dtype=F32, w_dtype=F32,
                    lr_scale=1.0, decay_scale=1.0)
        full.update(row)
        for key, val in full.items():
            setattr(t, key, val)
    return arr


def _build(arr, n=1, mem=1 << 40, size=None):
    lst = dstd.dstd_tensor_list()
    size = max(dstd.dstd_tensor_list_size(n, arr), 256) if size is None else size
    return dstd.dstd_tensor_list_build(n, arr, mem, size, lst, None), lst


def _list(has_weights=1):
    """A list as a build would have filled it (an empty one needs no device)."""
    st, lst = _build(None, 0)
    assert st == OK
    assert lst.n_tensors == lst.n_chunks == 0
    lst.has_weights = has_weights
    return lst


def test_structs_match_the_header():
    """Sizes that the header's field lists give (LP64, natural alignment)."""
    assert C.sizeof(dstd.dstd_tensor) == 6 * 8 + 8 + 3 * 4 + 2 * 4 + 4
    assert C.sizeof(dstd.dstd_tensor_list) == 8 + 5 * 8 + 3 * 4 + 4
    assert C.sizeof(dstd.dstd_adamw_params) == 6 * 8


def test_list_size_counts_tensors_and_chunks():
    one = dstd.dstd_tensor_list_size(1, _tensors(dict(n=1)))
    assert one > 0 and one % 256 == 0
    assert dstd.dstd_tensor_list_size(1, _tensors(dict(n=1 << 30))) > one
    assert dstd.dstd_tensor_list_size(0, None) > 0
    assert dstd.dstd_tensor_list_size(1, _tensors(dict(n=0))) > 0
    assert dstd.dstd_tensor_list_size(-1, _tensors({})) == 0
    assert dstd.dstd_tensor_list_size(1, None) == 0
    assert dstd.dstd_tensor_list_size(1, _tensors(dict(n=-1))) == 0
    assert dstd.dstd_tensor_list_size(1, _tensors(dict(n=1 << 35))) == 0
    big = _tensors(*[dict(n=(1 << 32) - 63)] * 8)  # 2^20 chunks each: one too many together
    assert dstd.dstd_tensor_list_size(7, big) > 0
    assert dstd.dstd_tensor_list_size(8, big) == 0
    big[7].n -= 4096
    assert dstd.dstd_tensor_list_size(8, big) > 0


@pytest.mark.parametrize("row,status", [
    (dict(g=None), NULL),
    (dict(n=-5), SHAPE),
    (dict(g_dtype=2), PARAM),
    (dict(w_dtype=-1), PARAM),
    (dict(out=7 << 33, out_dtype=9), PARAM),
    (dict(g=(1 << 32) + 2), PARAM),                 # fp32 off its alignment
    (dict(g=(1 << 32) + 1, g_dtype=BF16), PARAM),
    (dict(m=(1 << 32) + (2 << 28) + 1), PARAM),
    (dict(out=1 << 32, out_dtype=BF16), PARAM),     # in place, in another type
    (dict(m=None), NULL),
    (dict(v=None), NULL),
    (dict(w=None), NULL),                           # moments without weights
    (dict(w=None, m=None), NULL),
    (dict(w32=7 << 33), PARAM),                     # a copy of fp32 weights
    (dict(lr_scale=-1.0), PARAM),
    (dict(lr_scale=math.nan), PARAM),
    (dict(decay_scale=math.inf), PARAM),
])
def test_tensor_validation(row, status):
    st, lst = _build(_tensors(row))
    assert st == status, dstd.dstd_last_error()
    assert dstd.dstd_last_error()
    assert lst.magic == 0
    # the same as the last of several
    st, _ = _build(_tensors({}, {}, row), 3)
    assert st == status


def test_empty_tensors_need_no_arrays_and_are_not_looked_at():
    """Refused only for the missing memory: the tensors themselves pass."""
    row = dict(n=0, g=None, w=None, m=None, v=None)
    assert _build(_tensors(row), mem=None)[0] == NULL
    assert "workspace" in dstd.dstd_last_error()


@pytest.mark.parametrize("a,b", [
    (dict(g=1 << 33), dict(g=1 << 33)),                       # one gradient twice
    (dict(w=1 << 33), dict(w=(1 << 33) + 396)),               # the last element shared
    (dict(m=1 << 33), dict(v=1 << 33)),
    (dict(g=1 << 33), dict(out=(1 << 33) - 4, out_dtype=F32)),
    (dict(w=1 << 33, w_dtype=BF16), dict(g=(1 << 33) + 196)),
    (dict(g=1 << 40), {}),                                    # the list's own memory
])
def test_overlapping_arrays_are_refused(a, b):
    st, _ = _build(_tensors(a, b), 2)
    assert st == PARAM and "overlap" in dstd.dstd_last_error()


def test_neighbours_do_not_overlap():
    """Arrays that touch pass (the refusal here is the memory's)."""
    arr = _tensors(dict(g=1 << 33), dict(g=(1 << 33) + 400), dict(out=(1 << 33) + 800, out_dtype=F32))
    assert _build(arr, 3, mem=None)[0] == NULL
    assert _build(arr, 3, size=0)[0] == WS
    assert _build(arr, 3, mem=(1 << 40) + 8)[0] == WS
    # out = g is in place
    assert _build(_tensors(dict(out=1 << 32)), size=0)[0] == WS


def test_build_needs_its_arguments():
    arr = _tensors({})
    assert dstd.dstd_tensor_list_build(1, arr, 1 << 40, 1 << 20, None, None) == NULL
    assert _build(None, 1, size=1 << 20)[0] == NULL
    assert _build(arr, -1, size=1 << 20)[0] == SHAPE


def test_calls_refuse_what_is_not_a_list():
    blank = dstd.dstd_tensor_list()
    hp = dstd.make_adamw()
    for lst, st in ((None, NULL), (blank, PARAM)):
        assert dstd.dstd_tensor_list_workspace_size(lst) == 0
        assert dstd.dstd_grad_norm(lst, 4, 256, 1 << 20, None) == st
        assert dstd.dstd_grad_clip(lst, 1.0, 4, 0, 256, 1 << 20, None) == st
        assert dstd.dstd_adamw_step(lst, hp, None, 8, 4, 0, 256, 1 << 20, None) == st


def test_norm_clip_and_step_arguments():
    lst, hp = _list(), dstd.make_adamw()
    need = dstd.dstd_tensor_list_workspace_size(lst)
    assert need > 0
    assert dstd.dstd_grad_norm(lst, None, 256, need, None) == NULL
    for bad in (0.0, -1.0, math.nan, -math.inf):
        assert dstd.dstd_grad_clip(lst, bad, 4, 0, 256, need, None) == PARAM
    assert dstd.dstd_grad_clip(lst, 1.0, 4, 2, 256, need, None) == PARAM
    assert dstd.dstd_grad_clip(lst, 1.0, None, 1, 256, need, None) == NULL
    assert dstd.dstd_adamw_step(lst, None, None, 8, 4, 0, 256, need, None) == NULL
    assert dstd.dstd_adamw_step(lst, hp, None, None, 4, 0, 256, need, None) == NULL
    assert dstd.dstd_adamw_step(lst, hp, None, 8, None, 1, 256, need, None) == NULL
    assert dstd.dstd_adamw_step(lst, hp, None, 8, 4, -1, 256, need, None) == PARAM
    assert dstd.dstd_adamw_step(_list(has_weights=0), hp, None, 8, 4, 0, 256, need, None) == NULL
    for ws, size, st in ((None, need, NULL), (256, need - 1, WS), (260, need, WS)):
        assert dstd.dstd_grad_norm(lst, 4, ws, size, None) == st
        assert dstd.dstd_grad_clip(lst, 1.0, 4, 0, ws, size, None) == st
        assert dstd.dstd_adamw_step(lst, hp, None, 8, 4, 0, ws, size, None) == st


@pytest.mark.parametrize("kw", [
    dict(lr=-1e-3), dict(lr=math.nan), dict(lr=math.inf), dict(lr=1e60), dict(weight_decay=1e60), dict(beta1=-0.1), dict(beta1=1.0),
    dict(beta1=math.nan), dict(beta2=1.0), dict(beta2=2.0), dict(eps=0.0), dict(eps=-1e-8),
    dict(eps=1e-60), dict(eps=math.inf), dict(weight_decay=-0.1), dict(weight_decay=math.inf),
    dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=math.nan),
])
def test_adamw_constants(kw):
    lst = _list()
    need = dstd.dstd_tensor_list_workspace_size(lst)
    assert dstd.dstd_adamw_step(lst, dstd.make_adamw(**kw), None, 8, 4, 0, 256, need, None) == PARAM


def test_python_lists_refuse_what_is_not_on_the_gpu():
    import torch
    g = torch.zeros(4)
    with pytest.raises(ValueError, match="GPU"):
        dstd.make_tensor_list([g])
    with pytest.raises(TypeError, match="gradient 0"):
        dstd.make_tensor_list([g.double()])
    with pytest.raises(TypeError, match="tensor"):
        dstd.make_tensor_list([1.0])
    with pytest.raises(ValueError, match="needs a tensor"):
        dstd.make_tensor_list([])
    with pytest.raises(ValueError, match="2 weights for 1"):
        dstd.make_tensor_list([g], weights=[g, g])
