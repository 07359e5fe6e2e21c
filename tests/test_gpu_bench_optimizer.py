"""bench.py --optimizer times the workload it names: the update runs in every
step and leaves the weights, and so the events, as they are."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2607_14672_amd import dstd
    dstd._load()  # fail loudly if the HIP library is missing
    return torch.device("cuda:0")


@pytest.mark.parametrize("name,batch", [("mlp3", 16), ("wide-M8", 4)])
@pytest.mark.parametrize("eager", [False, True])
def test_timed_steps_keep_the_workload(dev, name, batch, eager):
    import bench
    import torch
    from paper_2607_14672_amd import dstd, workloads
    wl = workloads.with_batch(workloads.get(name), batch)
    plain = bench.measure(torch, dstd, wl, dev, 3, 1, 1, eager)
    r = bench.measure(torch, dstd, wl, dev, 3, 1, 1, eager, hp=dstd.make_adamw(max_norm=1.0))
    net = r["net"]
    assert r["activity"] == plain["activity"]
    for a, b, w32 in zip(net.L, plain["net"].L, net.opt["w32"]):
        assert torch.equal(a["W"], b["W"]) and torch.equal(a["t_out"], b["t_out"])
        assert torch.equal(a["gW"], b["gW"])
        assert w32 is None or torch.equal(w32, b["W"].float())
    # warm-up, timed and profiled steps (a capture makes three more)
    assert net.opt["steps"].item() == 5 + (0 if eager else 3)
    assert net.opt["norm"].item() > 0.0 and any(bool(v.any()) for v in net.opt["v"])
    assert sorted(set(r["kernel_ms_per_step"]) - set(plain["kernel_ms_per_step"])) == ["adamw", "grad_squares"]
