"""CPU-side checks of the C ABI of the operators on rows of logits: exported symbols, refusals on the host, limits.  No GPU work."""
import ctypes as C
import os
import re

import pytest

from paper_2503_05931_amd import binding, training as T, vocabulary as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
E, U, OK = binding.AED_EINVAL, binding.AED_EUNSUPPORTED, binding.AED_OK
FAR = 1 << 20  # a device address that nothing looks at


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2503_05931_amd import build
        build.build()
    return L._lib()


def test_every_declared_symbol_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "aed_vocab.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(aed_[a-z_0-9]+)\s*\(", text)))
    assert sorted(L.EXPORTS) == names and len(names) == 10
    for n in names:
        assert hasattr(lib, n), n


def test_structs_are_laid_out_as_in_c(tmp_path):
    import subprocess
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "aed_vocab.h"\nint main(void) { printf("%zu %zu %zu %zu %zu %zu\\n", sizeof(aed_sampler_config), '
                   'sizeof(aed_sampling), offsetof(aed_sampling, temperatures), offsetof(aed_sampling, min_ps), sizeof(aed_top_config), sizeof(aed_distill_config)); }\n')
    exe = str(tmp_path / "sizes")
    subprocess.run(["gcc", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = [int(n) for n in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(L.AedSamplerConfig), C.sizeof(L.AedSampling), L.AedSampling.temperatures.offset, L.AedSampling.min_ps.offset, C.sizeof(L.AedTopConfig),
                   C.sizeof(L.AedDistillConfig)]


def make(lib, name, cfg):
    """(status, handle); a handle has no memory on the device, so making one needs none"""
    h = C.c_void_p(None)
    return getattr(lib, f"aed_{name}_create")(C.byref(cfg), None, C.byref(h)), h


CONFIGS = {"sampler": L.AedSamplerConfig, "top": L.AedTopConfig, "distill": L.AedDistillConfig}


def config(name, **over):
    kw = dict(vocab=4096, dtype=1) | (dict(top=32, temperature=2.0) if name != "sampler" else {}) | over
    return CONFIGS[name](**{"struct_size": C.sizeof(CONFIGS[name]), **kw})


@pytest.mark.parametrize("name", CONFIGS)
def test_configs(lib, name):
    both = [(dict(struct_size=4), E), (dict(vocab=0), E), (dict(vocab=-7), E), (dict(dtype=2), E), (dict(dtype=-1), E), (dict(vocab=1 << 18), OK), (dict(vocab=(1 << 18) + 1), U)]
    lists = [(dict(top=0), E), (dict(top=-1), E), (dict(top=128), OK), (dict(top=129), U), (dict(temperature=0.0), E), (dict(temperature=-1.0), E),
             (dict(temperature=float("nan")), E), (dict(temperature=float("inf")), E)]
    for over, status in both + (lists if name != "sampler" else []):
        got, h = make(lib, name, config(name, **over))
        assert got == status and bool(h.value) == (status == OK), over
        assert status == OK or len(lib.aed_train_last_error()) > 10
    create = getattr(lib, f"aed_{name}_create")
    h = C.c_void_p(None)
    assert create(None, None, C.byref(h)) == E and create(C.byref(config(name)), None, None) == E
    assert getattr(lib, f"aed_{name}_destroy")(None) == OK


def test_lists_and_vocabularies(lib):
    assert make(lib, "top", config("top", vocab=31))[0] == E
    assert make(lib, "top", config("top", vocab=32))[0] == OK
    assert make(lib, "distill", config("distill", vocab=31))[0] == OK  # ids may come twice


def sampling(**over):
    return L.AedSampling(**({"struct_size": C.sizeof(L.AedSampling), "top_k": 0, "temperature": 1.0, "top_p": 1.0, "min_p": 0.0} | over))


def test_sample_refuses_before_a_launch(lib):
    _, h = make(lib, "sampler", config("sampler"))

    def call(logits=FAR, stride=4096, rows=4, uniforms=FAR, how=None, tokens=FAR, logp=FAR, plan=h):
        return lib.aed_sample(plan, logits, stride, rows, uniforms, how or sampling(), tokens, logp)

    for bad in (dict(logits=None), dict(logits=FAR + 1), dict(stride=4095), dict(stride=0), dict(stride=-4096), dict(stride=(1 << 38) + 1), dict(rows=-1), dict(uniforms=None),
                dict(uniforms=FAR + 2), dict(tokens=None), dict(tokens=FAR + 1), dict(logp=None), dict(logp=FAR + 3), dict(plan=None)):
        assert call(**bad) == E, bad
    for bad in (dict(struct_size=8), dict(temperature=-0.5), dict(temperature=float("inf")), dict(temperature=float("nan")), dict(top_k=-1), dict(top_p=1.01), dict(top_p=-0.01),
                dict(top_p=float("nan")), dict(min_p=1.01), dict(min_p=-1.0), dict(min_p=float("nan")), dict(temperatures=FAR + 1), dict(top_ks=FAR + 2), dict(top_ps=FAR + 3),
                dict(min_ps=FAR + 1)):
        assert call(how=sampling(**bad)) == E, bad
    assert lib.aed_sample(h, FAR, 4096, 4, FAR, None, FAR, FAR) == E
    assert call(rows=1 << 22) == U
    assert call(logits=None, stride=0, rows=0, uniforms=None, tokens=None, logp=None) == OK  # nothing to do


def test_top_refuses_before_a_launch(lib):
    _, h = make(lib, "top", config("top"))

    def call(logits=FAR, stride=4096, rows=4, values=FAR, ids=FAR, rest=FAR, plan=h):
        return lib.aed_top_logits(plan, logits, stride, rows, values, ids, rest)

    for bad in (dict(logits=None), dict(logits=FAR + 1), dict(stride=4095), dict(stride=(1 << 38) + 1), dict(rows=-1), dict(values=None), dict(values=FAR + 2), dict(ids=None),
                dict(ids=FAR + 1), dict(rest=None), dict(rest=FAR + 1), dict(plan=None)):
        assert call(**bad) == E, bad
    assert call(rows=1 << 22) == U
    assert call(logits=None, rows=0, values=None, ids=None, rest=None) == OK


def test_distill_refuses_before_a_launch(lib):
    _, h = make(lib, "distill", config("distill"))

    def forward(logits=FAR, stride=4096, rows=4, values=FAR, ids=FAR, rest=None, weights=None, loss=FAR, row_loss=FAR, stats=FAR, plan=h):
        return lib.aed_distill_forward(plan, logits, stride, rows, values, ids, rest, weights, loss, row_loss, stats)

    def backward(logits=FAR, stride=4096, rows=4, ids=FAR, weights=None, stats=FAR, d_loss=None, d_logits=2 * FAR, d_stride=4096, plan=h):
        return lib.aed_distill_backward(plan, logits, stride, rows, ids, weights, stats, d_loss, d_logits, d_stride)

    rows = (dict(logits=None), dict(logits=FAR + 1), dict(stride=4095), dict(stride=(1 << 38) + 1), dict(rows=-1), dict(ids=None), dict(ids=FAR + 2), dict(weights=FAR + 1),
            dict(stats=None), dict(stats=FAR + 2), dict(plan=None))
    for bad in rows + (dict(values=None), dict(values=FAR + 1), dict(rest=FAR + 1), dict(loss=None), dict(loss=FAR + 1), dict(row_loss=None), dict(row_loss=FAR + 2)):
        assert forward(**bad) == E, bad
    for bad in rows + (dict(d_loss=FAR + 1), dict(d_logits=None), dict(d_logits=2 * FAR + 1), dict(d_stride=4095), dict(d_logits=FAR, d_stride=4098)):
        assert backward(**bad) == E, bad
    assert forward(rows=1 << 22) == U and backward(rows=1 << 22) == U
    assert backward(logits=None, rows=0, ids=None, stats=None, d_logits=None) == OK
    assert forward(rows=0, loss=None) == E


@pytest.mark.parametrize("name", ["top", "distill"])
def test_temperatures_are_limited(lib, name):
    for t, status in ((1e-20, OK), (1e20, OK), (1e-21, U), (2e20, U), (1e-45, U), (0.0, E), (-1.0, E), (float("nan"), E), (float("inf"), E)):
        assert make(lib, name, config(name, temperature=t))[0] == status, t


def test_numbers_that_are_no_int32():
    import torch
    for call in (lambda: L._i32(1 << 31, "top_k"), lambda: L._i32(-(1 << 31) - 1, "vocab"), lambda: L.TopLogits(100, (1 << 32) + 5, torch.float32),
                 lambda: L.Distillation(100, (1 << 32) + 5, torch.float32)):
        with pytest.raises(binding.AedError, match="is not an int32"):
            call()
    assert L._i32((1 << 31) - 1, "top_k") == (1 << 31) - 1


# ---------------------------------------------------------------- the binding, with torch's streams and the library played by recorders
class HostDistillation(L.Distillation):
    """Calls of a plan, by torch on the host; no library"""

    def __init__(self):
        pass

    def __del__(self):
        pass

    def aed_distill_forward(self, logits, values, ids, rest=None, weights=None):
        import torch
        p, q = torch.log_softmax(logits, 1).gather(1, ids.long()), torch.softmax(values, 1)
        return (q * (q.log() - p)).sum(1).mean(), None, torch.zeros(logits.shape[0], 4)

    def aed_distill_backward(self, logits, ids, stats, weights=None, d_loss=None, d_logits=None):
        import torch
        with torch.enable_grad():
            leaf = logits.detach().requires_grad_(True)
            return torch.autograd.grad(self.aed_distill_forward(leaf, torch.ones(ids.shape), ids)[0], leaf, d_loss.detach())[0]


@pytest.mark.filterwarnings("ignore:Using backward")
def test_second_derivatives_are_refused():
    import torch
    z = torch.randn(3, 7, generator=torch.Generator().manual_seed(0)).requires_grad_(True)
    ids = torch.tensor([[0, 2], [1, 3], [6, 5]], dtype=torch.int32)
    loss = HostDistillation().loss(z, torch.ones(3, 2), ids)
    (plain,) = torch.autograd.grad(loss, z, retain_graph=True)
    (g,) = torch.autograd.grad(loss, z, create_graph=True)
    assert torch.equal(g, plain) and plain.abs().sum() > 0
    with pytest.raises(RuntimeError, match="second derivatives"):
        (loss + g.square().sum()).backward()


def test_constants_that_require_a_gradient_are_refused():
    """A gradient that is not computed is not silently left out; without autograd, or of a copy that is cut off, nothing is asked for."""
    import torch
    z, ids = torch.randn(3, 7, requires_grad=True), torch.tensor([[0, 2], [1, 3], [6, 5]], dtype=torch.int32)
    given = dict(values=torch.ones(3, 2), rest=torch.zeros(3), weights=torch.ones(3))
    plan = HostDistillation()
    for name in given:
        with_one = given | {name: given[name].clone().requires_grad_(True)}
        with pytest.raises(binding.AedError, match=f"{name} requires a gradient") as e:
            plan.loss(z, ids=ids, **with_one)
        assert e.value.status == E
        with torch.no_grad():
            assert torch.isfinite(plan.loss(z, ids=ids, **with_one))
        plan.loss(z, ids=ids, **(given | {name: with_one[name].detach()})).backward()
    assert z.grad.abs().sum() > 0


class Recorder:
    def __init__(self, status, device, stream):
        import types
        self.done, self.status, self.device, self.stream = [], status, device, stream
        self.lib = types.SimpleNamespace(**{n: self.call for n in ("aed_sample", "aed_top_logits", "aed_distill_forward", "aed_distill_backward")})

    def call(self, *_):
        self.done.append(("call", self.device))
        return self.status

    def set_device(self, n):
        self.device = n


class Stream:
    def __init__(self, recorder, raw):
        self.recorder, self.cuda_stream = recorder, raw

    def wait_stream(self, other):
        self.recorder.done.append((self.cuda_stream, "waits for", other.cuda_stream))


def plan_of(kind, cfg, monkeypatch, status=0, device=-1, stream=7):
    """A plan of stream 5 of device -1, which is what tensors of the host say theirs is"""
    import types

    import torch
    rec = Recorder(status, device, stream)
    p = kind.__new__(kind)
    p.torch = types.SimpleNamespace(Tensor=torch.Tensor, float32=torch.float32, int32=torch.int32,
                                    cuda=types.SimpleNamespace(current_stream=lambda device: Stream(rec, rec.stream), set_device=rec.set_device))
    p.lib, p.dtype, p.device, p.cfg, p.vocab, p.top = rec.lib, torch.float32, torch.device("cpu"), cfg, 9, 3
    p.handle, p._destroy = C.c_void_p(1), lambda _: 0
    p.stream, p.raw, p.index = Stream(rec, 5), 5, -1
    p._f32, p._i32, p._how = torch.empty(0), torch.empty(0, dtype=torch.int32), sampling()
    p._given_how = None
    p._raw_stream = lambda index: rec.stream
    p._get_device, p._only = lambda: rec.device, False
    monkeypatch.setattr(T, "_lib", lambda: types.SimpleNamespace(aed_train_last_error=lambda: b"a launch failed"))
    return p, rec


def calls():
    import torch
    z, three = torch.zeros(4, 9), torch.zeros(4, 3)
    return [(L.Sampler, lambda p: p.aed_sample(z, torch.zeros(4))), (L.TopLogits, lambda p: p.aed_top_logits(z)),
            (L.Distillation, lambda p: p.aed_distill_forward(z, three, three.int())), (L.Distillation, lambda p: p.aed_distill_backward(z, three.int(), torch.zeros(4, 5)))]


@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("status", [0, -4])
@pytest.mark.parametrize("device", [-1, 0])
@pytest.mark.parametrize("stream", [5, 7])
def test_streams_and_devices(which, status, device, stream, monkeypatch):
    """Calls are made on the plan's device; where another stream is current, each waits for the other, after a call that fails, too."""
    kind, call = calls()[which]
    p, rec = plan_of(kind, None, monkeypatch, status, device, stream)
    if status:
        with pytest.raises(binding.AedError):
            call(p)
    else:
        call(p)
    waits = [(5, "waits for", 7)] if stream == 7 else []
    assert rec.done == waits + [("call", -1)] + [(7, "waits for", 5)] * bool(waits) and rec.device == device
    p.handle = C.c_void_p(None)
    with pytest.raises(binding.AedError):
        call(p)
