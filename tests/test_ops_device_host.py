"""Each call of Ops makes its own device the current one, and puts back the one
that was: on the CPU, with stand-ins for torch's device and for libember."""
import types

import pytest
import torch

from paper_2607_01455_gb300 import ember as E
from paper_2607_01455_gb300 import ops as module


class Machine:
    """Two devices of which 0 is current; what was current at each call into libember."""

    def __init__(self, monkeypatch):
        self.current, self.seen = 0, []
        machine = self

        class device:
            def __init__(self, d):
                self.index = d.index

            def __enter__(self):
                self.before, machine.current = machine.current, self.index

            def __exit__(self, *a):
                machine.current = self.before

        class stream(device):
            def __init__(self, s):
                self.index = s.device.index

        monkeypatch.setattr(module, "_current_device", lambda: self.current, raising=False)
        monkeypatch.setattr(module, "_raw_stream", lambda index: 1000 + index)
        monkeypatch.setattr(module, "_current_stream", lambda: 1000 + self.current, raising=False)
        monkeypatch.setattr(torch.cuda, "device", device)
        monkeypatch.setattr(torch.cuda, "stream", stream)
        o = self.ops = module.Ops.__new__(module.Ops)
        o.device, o._index, o._at, o._bytes = torch.device("cuda", 1), 1, 0, 0
        o._fast, o._lib = _Calls(self, ("a", "b", "c"), 1), _Calls(self, E.EMBER_OK)
        o._status_word = lambda: 4
        o._matrix = lambda *a: (1, 8)
        o._rows8 = lambda T, D: (torch.empty(T, D), D, torch.empty(T))


class _Calls:
    def __init__(self, machine, result, only=None):
        self.machine, self.result, self.only = machine, result, only

    def __getattr__(self, name):
        def call(*a):
            if self.only is not None and self.only != self.machine.current:
                return None  # as the binding does on another device
            self.machine.seen.append((name, self.machine.current, a))
            return self.result
        return call


X = torch.zeros(4, 8)
Y = torch.zeros(4, dtype=torch.int64)
CALLS = {
    "rmsnorm": (X, None), "rmsnorm_quant": (X, None), "rmsnorm_backward": (X, X, None), "quantize_rows": (X,),
    "dequantize_rows": (X, Y), "matmul_quant": (X, Y, X, Y), "softmax_loss": (X, Y), "grad_norm": ([X],),
    "clip_grads": ([X], 1.0), "device_status": (),
}


@pytest.mark.parametrize("name", CALLS)
def test_calls_run_on_the_objects_device(monkeypatch, name):
    m = Machine(monkeypatch)
    getattr(m.ops, name)(*CALLS[name])
    assert [device for _, device, _ in m.seen] == [1] and m.current == 0
    if name in ("device_status", "quantize_rows"):
        assert m.seen[0][2][-1] == 1001  # that device's current stream
    m.current = 1
    getattr(m.ops, name)(*CALLS[name])
    assert m.seen[1][1] == 1 and m.current == 1


@pytest.mark.parametrize("name", CALLS)
def test_calls_on_a_stream_run_on_its_device(monkeypatch, name):
    m = Machine(monkeypatch)
    s = types.SimpleNamespace(device=m.ops.device, cuda_stream=77)
    getattr(m.ops, name)(*CALLS[name], stream=s)
    assert [device for _, device, _ in m.seen] == [1] and m.current == 0


@pytest.mark.parametrize("name", [n for n in CALLS if n != "device_status"])
def test_a_stream_of_another_device_is_refused(monkeypatch, name):
    m = Machine(monkeypatch)
    s = types.SimpleNamespace(device=torch.device("cuda", 0), cuda_stream=77)
    with pytest.raises(ValueError, match="stream"):
        getattr(m.ops, name)(*CALLS[name], stream=s)
    assert m.seen == [] and m.current == 0


def test_the_handle_0_is_the_default_stream(monkeypatch):
    m = Machine(monkeypatch)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda d: types.SimpleNamespace(device=d, cuda_stream=0))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda p, device: pytest.fail("no stream has this handle"))
    m.ops.rmsnorm(X, None, stream=0)
    assert m.seen[0][1] == 1 and m.current == 0


def test_the_binding_belongs_to_the_torch_at_hand(monkeypatch):
    """One that was built for another torch is not loaded, and the message says what to do."""
    from paper_2607_01455_gb300.build import binding_path, build_binding
    path = build_binding()
    assert path == binding_path() and torch.__version__ in path
    assert E.ops_binding() is E.ops_binding()
    monkeypatch.setattr(E, "_binding", None)
    monkeypatch.setattr(torch, "__version__", "0.1")
    with pytest.raises(RuntimeError, match="torch-0.1.so is missing: build"):
        E.ops_binding()
