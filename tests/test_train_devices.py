"""Plans of another GPU than the current one.  On the CPU: the library and torch's current device are stand-ins."""
import contextlib
import ctypes

import pytest
import torch

from paper_2603_18112_gb300 import optim as O


class Machine:
    """Two GPUs, of which one is current; calls note it, and the stream that they are given."""

    def __init__(self):
        self.current, self.calls = 0, []

    @contextlib.contextmanager
    def device(self, index):
        before, self.current = self.current, index
        yield
        self.current = before

    def __getattr__(self, name):
        def call(handle, *args):
            self.calls.append((name, self.current, args[-1].value))
            return 0
        return call


@pytest.fixture
def machine(monkeypatch):
    m = Machine()
    monkeypatch.setattr(O, "_lib", lambda: m)
    monkeypatch.setattr(O, "_get_device", lambda: m.current)
    monkeypatch.setattr(O.torch.cuda, "device", m.device)
    monkeypatch.setattr(O, "_stream_ptr", lambda s: ctypes.c_void_p(1000 + m.current if s is None else s))
    return m


def _plan(monkeypatch):
    plan = O._Planned()
    plan.device, plan.memory, plan.last, plan.handle = torch.device("cuda", 1), [], (), None
    monkeypatch.setattr(plan, "ran_on", lambda s: setattr(plan, "last", s.value), raising=False)
    return plan


def test_calls_go_to_the_plans_gpu(machine, monkeypatch):
    muon, adam, clip = (cls.__new__(cls) for cls in (O.MuonStep, O.AdamWStep, O.GradClipper))
    muon.hp, adam.hp = O.tula_muon_hparams(), O.tula_adamw_hparams()
    for o in (muon, adam):
        o._hp = ctypes.byref(o.hp)
    clip.record, clip._record = None, ctypes.c_void_p(0)
    for o in (muon, adam, clip):
        o._plan = _plan(monkeypatch)
    calls = [("tula_muon_step", lambda **kw: muon(1e-3, **kw)), ("tula_adamw_step", lambda **kw: adam(1e-3, **kw)),
             ("tula_grad_norm", lambda **kw: clip.norm(**kw)), ("tula_grad_clip", lambda **kw: clip.clip_(1.0, **kw))]
    for name, call in calls:
        machine.calls.clear()
        call()
        call(stream=77)
        assert machine.calls == [(name, 1, 1001), (name, 1, 77)] and machine.current == 0
    with machine.device(1):
        machine.calls.clear()
        calls[0][1]()
        assert machine.calls == [("tula_muon_step", 1, 1001)]


def test_a_stream_of_another_gpu(machine, monkeypatch):
    class Stream:
        device, cuda_stream = torch.device("cuda", 0), 5

    monkeypatch.setattr(O.torch.cuda, "Stream", Stream)
    plan, stream = _plan(monkeypatch), Stream()
    with pytest.raises(ValueError, match="GPU 1"):
        plan.call("tula_grad_norm", stream)
    assert machine.calls == []
