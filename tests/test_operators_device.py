"""The operators' binding with tensors on a device that is not the current one,
without a GPU: tensors, the current device and the library are stand-ins, and
each library call has to see the tensors' device current."""
import contextlib

import pytest
import torch

from paper_2504_13850_gb300 import api


class Tensor:
    is_cuda = True

    def __init__(self, shape, dtype, index):
        self.shape, self.dtype, self.index = torch.Size(shape), dtype, index
        self.device = torch.device("cuda", index)

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def get_device(self):
        return self.index

    def data_ptr(self):
        return 4096

    def is_contiguous(self):
        return True

    def contiguous(self):
        return self

    def stride(self, dim=None):
        s = [1]
        for n in reversed(self.shape[1:]):
            s.insert(0, s[0] * n)
        return tuple(s) if dim is None else s[dim]


class Machine:
    """Devices 0 and 1, of which 0 is current; a default stream has handle 0 on
    either.  `calls` holds each library call's name, current device and stream."""

    def __init__(self, monkeypatch):
        self.current, self.calls, self.allocated = 0, [], []

        @contextlib.contextmanager
        def device(index):
            before, self.current = self.current, getattr(index, "index", index)
            try:
                yield
            finally:
                self.current = before

        class Stream:
            cuda_stream = 0

        monkeypatch.setattr(torch.cuda, "current_device", lambda: self.current)
        monkeypatch.setattr(torch.cuda, "device", device)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda index=None: Stream)
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device: device)
        monkeypatch.setattr(torch.cuda, "stream", device)
        monkeypatch.setattr(torch, "empty", self.empty)
        monkeypatch.setattr(api, "lib", lambda: self)

    def empty(self, shape, dtype, device):
        self.allocated.append(device.index)
        return Tensor(shape if isinstance(shape, tuple) else (shape,), dtype, device.index)

    def fo_attention_workspace(self, spec, backward):
        return 256

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, self.current, args[-1]))
            return api.OK
        return call


CALLS = {
    "fo_attention_forward": lambda q, **kw: api.attention_forward(q, q, q, **kw),
    "fo_attention_backward": lambda q, **kw: api.attention_backward(
        q, q, q, q, q, Tensor((2, 4, 16), torch.float32, q.index), **kw),
    "fo_dropout_add": lambda q, **kw: api.dropout_add(q, q, 0.5, 1, 1, **kw),
}


@pytest.fixture
def machine(monkeypatch):
    return Machine(monkeypatch)


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("index", [0, 1])
@pytest.mark.parametrize("stream", [None, 77])
def test_the_tensors_device_is_current(machine, name, index, stream):
    CALLS[name](Tensor((2, 16, 4, 64), torch.bfloat16, index), stream=stream)
    assert machine.calls == [(name, index, stream or 0)]
    assert set(machine.allocated) == {index} and machine.current == 0


def test_given_outputs(machine):
    q = Tensor((2, 16, 4, 64), torch.bfloat16, 1)
    api.dropout_add(q, None, 0.5, 1, 1, out=q)
    api.dropout_grad(q, 0.5, 1, 1)
    api.attention_forward(q, q, q, out=q)
    api.attention_backward(q, q, q, q, q, Tensor((2, 4, 16), torch.float32, 1), grads=(q, q, q))
    assert [c[1] for c in machine.calls] == [1] * 4 and machine.current == 0


def test_errors_of_a_device(machine):
    api.attention_error()
    api.attention_error(device=1)
    assert machine.calls == [("fo_attention_error", 0, 0), ("fo_attention_error", 1, 0)]


def test_mixed_devices_are_refused(machine):
    q, far = (Tensor((2, 16, 4, 64), torch.bfloat16, i) for i in (1, 0))
    for call in (lambda: api.attention_forward(q, far, q), lambda: api.dropout_add(q, far, 0.5, 1, 1),
                 lambda: api.attention_forward(q, q, q, documents=Tensor((2, 16), torch.int32, 0))):
        with pytest.raises(ValueError):
            call()
    assert machine.calls == [] and machine.current == 0
