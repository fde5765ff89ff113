"""Order of streams and devices around a plan's calls (training._Plan), with torch's streams and the library played by recorders.  No GPU work."""
import ctypes as C
import types

import pytest
import torch

from paper_2503_05931_amd import binding, training as T


class Recorder:
    """torch.cuda and the library: what was done, in order"""

    def __init__(self, status=0, device=-1, stream=7):
        self.done, self.status, self.device, self.stream = [], status, device, stream
        self.lib = types.SimpleNamespace(aed_attn_forward=self.call, aed_attn_backward=self.call, aed_attn_destroy=self.destroy, aed_preference_forward=self.call,
                                         aed_preference_backward=self.call)

    def call(self, *_):
        self.done.append(("call", self.device))
        return self.status

    def destroy(self, *_):
        self.done.append(("destroy", self.device))
        return 0

    def set_device(self, n):
        self.device = n


class Stream:
    def __init__(self, recorder, raw):
        self.recorder, self.cuda_stream = recorder, raw

    def wait_stream(self, other):
        self.recorder.done.append((self.cuda_stream, "waits for", other.cuda_stream))


def plan(kind, monkeypatch, **kw):
    """A plan of stream 5 of device -1, which is what tensors of the host say theirs is"""
    rec = Recorder(**kw)
    p = kind.__new__(kind)
    p.torch = types.SimpleNamespace(uint8=torch.uint8, bool=torch.bool, float32=torch.float32, int32=torch.int32, empty_like=torch.empty_like,
                                    cuda=types.SimpleNamespace(current_stream=lambda device: Stream(rec, rec.stream), set_device=rec.set_device))
    p.lib, p.dtype, p.device = rec.lib, torch.float32, torch.device("cpu")
    p.handle, p._destroy = C.c_void_p(1), rec.lib.aed_attn_destroy
    p.stream, p.raw, p.index = Stream(rec, 5), 5, -1
    p._f32 = torch.empty(0)
    p._raw_stream = lambda index: rec.stream
    p._get_device, p._only = lambda: rec.device, False
    monkeypatch.setattr(T, "_lib", lambda: types.SimpleNamespace(aed_train_last_error=lambda: b"a launch failed"))
    return p, rec


def attention(monkeypatch, **kw):
    p, rec = plan(T.Attention, monkeypatch, **kw)
    p.cfg = T.AedAttnConfig(C.sizeof(T.AedAttnConfig), 2, 2, 64, 0, 0, 0, 0, 0, 1, 0.0)
    p.q_rows = p.k_rows = 3
    p.packed = True
    p._q_shape = p._k_shape = (3, 2, 64)
    p._lse_shape = (3, 2)
    p._at = [T.AedRows() for _ in range(8)]
    return p, rec


def forward(p):
    x = torch.zeros(3, 2, 64)
    return p.aed_attn_forward(x, x, x)


def backward(p):
    x = torch.zeros(3, 2, 64)
    return p.aed_attn_backward(x, x, x, x, x, torch.zeros(3, 2))


def preference(monkeypatch, **kw):
    p, rec = plan(T.Preference, monkeypatch, **kw)
    p.cfg = T.AedPreferenceConfig(C.sizeof(T.AedPreferenceConfig), 9, 0, 0.1, 0.0)
    p.rows, p.pairs = 4, 1
    return p, rec


def loss(p):
    return p.aed_preference_forward(torch.zeros(4, 9), torch.zeros(4, dtype=torch.int32), torch.zeros(4))


def loss_backward(p):
    return p.aed_preference_backward(torch.zeros(4, 9), torch.zeros(4, dtype=torch.int32), torch.zeros(2), torch.zeros(4, 2))


CALLS = [(attention, forward), (attention, backward), (preference, loss), (preference, loss_backward)]


@pytest.mark.parametrize("make,call", CALLS)
@pytest.mark.parametrize("status", [0, -4])
def test_the_current_stream_waits_also_for_a_call_that_fails(make, call, status, monkeypatch):
    """A first kernel may be on its way when the second's launch fails: what it writes to goes back to the current stream's memory."""
    p, rec = make(monkeypatch, status=status)
    if status:
        with pytest.raises(binding.AedError):
            call(p)
    else:
        call(p)
    assert rec.done == [(5, "waits for", 7), ("call", -1), (7, "waits for", 5)]


@pytest.mark.parametrize("make,call", CALLS)
def test_the_plans_own_stream_waits_for_nothing(make, call, monkeypatch):
    p, rec = make(monkeypatch, stream=5)
    call(p)
    assert rec.done == [("call", -1)]


@pytest.mark.parametrize("make,call", CALLS)
@pytest.mark.parametrize("status", [0, -4])
@pytest.mark.parametrize("stream", [5, 7])
def test_calls_are_made_on_the_plans_device(make, call, status, stream, monkeypatch):
    """Another device is current: the default stream's number is the same on all, and would be that device's."""
    p, rec = make(monkeypatch, status=status, device=0, stream=stream)
    if status:
        with pytest.raises(binding.AedError):
            call(p)
    else:
        call(p)
    assert ("call", -1) in rec.done and rec.device == 0
    p.close()
    assert rec.done[-1] == ("destroy", -1) and rec.device == 0
    with pytest.raises(binding.AedError):
        call(p)
