"""Order of the tensor lists' calls behind the build of their table, on the CPU:
a list used on another stream than the one it was built on."""
import contextlib
from types import SimpleNamespace

import pytest

from paper_2607_14672_amd import dstd

BUILD, SIDE = 11, 22


class Event:
    def __init__(self, done):
        self.done = done

    def query(self):
        return self.done


def _world(monkeypatch, stream, capturing=False):
    """What a call does on `stream`, in order."""
    did = []
    current = SimpleNamespace(wait_event=lambda e: did.append(("wait", e)))
    cuda = SimpleNamespace(current_stream=lambda dev: current, current_device=lambda: 0,
                           is_current_stream_capturing=lambda: capturing,
                           device=lambda dev: contextlib.nullcontext())
    torch = SimpleNamespace(cuda=cuda, _C=SimpleNamespace(_cuda_getCurrentRawStream=lambda dev: stream))
    monkeypatch.setattr(dstd, "_torch", lambda: torch)
    mem = SimpleNamespace(record_stream=lambda s: did.append(("record", s is current)))

    def launch(tl):
        dstd._launch(tl, "call", lambda s: did.append(("launch", s)) or dstd.DSTD_OK)
        return did

    return mem, launch


def _list(mem, **kw):
    return dstd.TensorList(dstd.dstd_tensor_list(), mem, (), SimpleNamespace(index=0), BUILD, **kw)


def test_another_stream_waits_for_the_build(monkeypatch):
    mem, launch = _world(monkeypatch, SIDE)
    e = Event(False)
    did = launch(_list(mem, built=e))
    assert sorted(did[:-1], key=str) == sorted([("wait", e), ("record", True)], key=str)
    assert did[-1] == ("launch", SIDE)


def test_a_build_that_is_done_is_not_waited_for(monkeypatch):
    mem, launch = _world(monkeypatch, SIDE)
    tl = _list(mem, built=Event(True))
    assert launch(tl) == [("record", True), ("launch", SIDE)]
    assert tl.built is None


def test_the_building_stream_needs_no_order(monkeypatch):
    mem, launch = _world(monkeypatch, BUILD)
    assert launch(_list(mem, built=Event(False))) == [("launch", BUILD)]


def test_a_capture_cannot_wait_for_work_outside_it(monkeypatch):
    mem, launch = _world(monkeypatch, SIDE, capturing=True)
    assert launch(_list(mem, built=Event(False))) == [("record", True), ("launch", SIDE)]


@pytest.mark.parametrize("stream", [BUILD, SIDE])
def test_a_list_built_inside_a_capture_is_not_for_eager_calls(monkeypatch, stream):
    mem, launch = _world(monkeypatch, stream)
    with pytest.raises(RuntimeError, match="inside a capture"):
        launch(_list(mem, captured=True))
    mem, launch = _world(monkeypatch, stream, capturing=True)
    assert launch(_list(mem, captured=True))[-1] == ("launch", stream)
