"""Places of the tensor lists' calls that must lie apart or be aligned, and
betas that fp32 cannot hold, on the CPU: refused on the host, before anything
touches a device."""
import pytest

from paper_2607_14672_amd import dstd

MEM, WS, NORM, STEP, LR = 1 << 40, 1 << 20, 4, 8, 16


def _list():
    """An empty list at MEM, said to hold 3 chunks of 64 bytes."""
    lst = dstd.dstd_tensor_list()
    assert dstd.dstd_tensor_list_build(0, None, MEM, 256, lst, None) == dstd.DSTD_OK
    lst.n_chunks = 3
    return lst


def _call(name, norm=NORM, step=STEP, lr=LR, ws=WS, given=0):
    lst, hp = _list(), dstd.make_adamw()
    need = dstd.dstd_tensor_list_workspace_size(lst)
    if name == "norm":
        return dstd.dstd_grad_norm(lst, norm, ws, need, None)
    if name == "clip":
        return dstd.dstd_grad_clip(lst, 1.0, norm, given, ws, need, None)
    return dstd.dstd_adamw_step(lst, hp, lr, step, norm, given, ws, need, None)


ALL = ("norm", "clip", "step")


@pytest.mark.parametrize("names,kw", [
    (ALL, dict(ws=MEM)),                        # the table itself as workspace
    (ALL, dict(norm=WS)), (ALL, dict(norm=WS + 4096)), (ALL, dict(norm=MEM)), (ALL, dict(norm=MEM + 188)),
    (("clip", "step"), dict(norm=WS, given=1)),
    (("step",), dict(step=WS + 8)), (("step",), dict(lr=WS + 16)), (("step",), dict(step=MEM + 64)),
    (("step",), dict(norm=LR)), (("step",), dict(norm=STEP)), (("step",), dict(norm=STEP + 4)),
    (("step",), dict(lr=STEP)), (("step",), dict(lr=STEP + 4)),
    (("step",), dict(norm=STEP + 4, given=1)),
], ids=str)
def test_overlapping_places_are_refused(names, kw):
    for name in names:
        assert _call(name, **kw) == dstd.DSTD_ERR_PARAM, name
        assert "overlap" in dstd.dstd_last_error()


@pytest.mark.parametrize("names,kw", [
    (ALL, dict(norm=6)), (("clip", "step"), dict(norm=5, given=1)), (("step",), dict(step=12)),
    (("step",), dict(lr=18)),
], ids=str)
def test_places_off_their_alignment_are_refused(names, kw):
    for name in names:
        assert _call(name, **kw) == dstd.DSTD_ERR_PARAM, name
        assert "aligned" in dstd.dstd_last_error()


def test_expanded_workspaces_are_refused():
    """One byte seen many times is no workspace."""
    import torch
    tl = dstd.TensorList(_list(), None, (), torch.device("cpu"), 0)
    ws = torch.empty(1, dtype=torch.uint8).expand(2 * tl.ws_bytes)
    with pytest.raises(ValueError, match="ws must be contiguous"):
        dstd._optim_args(tl, None, False, ws, False)
    ok = torch.empty(tl.ws_bytes, dtype=torch.uint8)
    assert dstd._optim_args(tl, None, False, ok, False) == (None, None, ok)


@pytest.mark.parametrize("beta", [1.0 - 2.0 ** -26, 1.0 - 1e-9, 1.0 - 2.0 ** -53])
def test_betas_that_are_one_in_fp32_are_refused(beta):
    """A moment in fp32 loses less than half a step of itself: it would stand."""
    need = dstd.dstd_tensor_list_workspace_size(_list())
    for kw in (dict(beta1=beta), dict(beta2=beta)):
        assert dstd.dstd_adamw_step(_list(), dstd.make_adamw(**kw), LR, STEP, NORM, 0, WS, need,
                                    None) == dstd.DSTD_ERR_PARAM


def test_gradient_places_are_checked():
    """The backward helpers' `grad_W`."""
    import torch
    W, cpu = torch.ones(4, 6), torch.device("cpu")

    def dest(g, need=True):
        return dstd._grad_dest(torch, g, W, (4, 6), cpu, need)

    g = torch.zeros(4, 6)
    assert dest(g) is g and dest(None, False) is None
    assert dest(None).shape == (4, 6) and dest(None).dtype == torch.float32
    for bad, err in ((g.double(), TypeError), (0.0, TypeError), (g.t(), ValueError),
                     (torch.zeros(6, 4).t(), ValueError), (torch.zeros(24), ValueError),
                     (g.to("meta"), ValueError), (W, ValueError)):
        with pytest.raises(err, match="grad_W"):
            dest(bad)
    with pytest.raises(ValueError, match="need_W"):
        dest(g, False)
    # a part of the weights' memory, in whichever order
    buf = torch.zeros(100)
    lo, hi, off = buf[:24].view(4, 6), buf[23:47].view(4, 6), buf[24:48].view(4, 6)
    for w, place in ((lo, hi), (hi, lo)):
        with pytest.raises(ValueError, match="share"):
            dstd._grad_dest(torch, place, w, (4, 6), cpu, True)
    assert dstd._grad_dest(torch, off, lo, (4, 6), cpu, True) is off


def test_scalars_that_are_no_tensors_are_refused():
    """A number in place of the tensor that holds it, in every place for one."""
    import torch
    tl = dstd.TensorList(_list(), None, (), torch.device("cpu"), 0)
    hp, step = dstd.make_adamw(max_norm=1.0), torch.zeros(1, dtype=torch.int64)
    norm, ws = torch.zeros(1), torch.empty(tl.ws_bytes, dtype=torch.uint8)
    for kw in (dict(lr=1e-3), dict(lr=torch.zeros(1, dtype=torch.float64).numpy()), dict(norm=2.0),
               dict(norm=2.0, norm_given=True), dict(step=3), dict(ws=bytearray(tl.ws_bytes))):
        args = dict(step=step, norm=norm, ws=ws)
        args.update(kw)
        with pytest.raises(TypeError, match=f"{next(iter(kw))} must be a tensor"):
            dstd.adamw_step(tl, hp, **args)
    with pytest.raises(TypeError, match="norm must be a tensor"):
        dstd.grad_norm(tl, norm=2.0, ws=ws)
    with pytest.raises(TypeError, match="norm must be a tensor"):
        dstd.grad_clip(tl, 1.0, norm=2.0, norm_given=True, ws=ws)
