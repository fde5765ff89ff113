"""ctypes binding of the operators on rows of logits (include/aed_vocab.h): sampling the next token, a row's largest logits, and
distillation from those of a teacher.

Argument marshalling only; a missing library raises.  Tensors are torch tensors on the device; rows of logits may lie any distance apart.  A plan
works on the stream that was current when it was made, or on `stream`; a call under another current stream waits for that one's
work and lets it wait for the results.  A graph that holds a plan's calls needs the plan for as long as it is replayed.
"""
from __future__ import annotations

import ctypes as C

from . import training as _t

EXPORTS = ("aed_sampler_create", "aed_sampler_destroy", "aed_sample", "aed_top_create", "aed_top_destroy", "aed_top_logits",
           "aed_distill_create", "aed_distill_destroy", "aed_distill_forward", "aed_distill_backward")


class AedSamplerConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("vocab", C.c_int32), ("dtype", C.c_int32)]


class AedSampling(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("top_k", C.c_int32), ("temperature", C.c_float), ("top_p", C.c_float), ("min_p", C.c_float),
                ("temperatures", C.c_void_p), ("top_ks", C.c_void_p), ("top_ps", C.c_void_p), ("min_ps", C.c_void_p)]


class AedTopConfig(C.Structure):
    _fields_ = AedSamplerConfig._fields_ + [("top", C.c_int32), ("temperature", C.c_float)]


class AedDistillConfig(C.Structure):
    _fields_ = AedTopConfig._fields_


_configured = False


def _lib():
    global _configured
    lib = _t._lib()
    if not _configured:
        vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        for n, cfg in (("sampler", AedSamplerConfig), ("top", AedTopConfig), ("distill", AedDistillConfig)):
            getattr(lib, f"aed_{n}_create").argtypes = [C.POINTER(cfg), vp, C.POINTER(vp)]
            getattr(lib, f"aed_{n}_destroy").argtypes = [vp]
        lib.aed_sample.argtypes = [vp, vp, i64, i32, vp, C.POINTER(AedSampling), vp, vp]
        lib.aed_top_logits.argtypes = [vp, vp, i64, i32, vp, vp, vp]
        lib.aed_distill_forward.argtypes = [vp, vp, i64, i32, vp, vp, vp, vp, vp, vp, vp]
        lib.aed_distill_backward.argtypes = [vp, vp, i64, i32, vp, vp, vp, vp, vp, i64]
        for n in EXPORTS:
            getattr(lib, n).restype = C.c_int
        _configured = True
    return lib


def _i32(value, name):
    """An int32's number: ctypes takes others modulo 2^32."""
    if not -(1 << 31) <= value < 1 << 31:
        _t._refuse(f"{name} {value} is not an int32")
    return value


def _rows(logits):
    return logits.shape[0] if logits.dim() == 2 else None  # None: refused for its shape


class _RowsPlan(_t._Plan):
    """A plan for rows of logits, any number a call."""

    def __init__(self, vocab, dtype, device, stream, name, cfg):
        super().__init__(dtype, device, stream)
        lib = self.lib = _lib()
        self.vocab = vocab
        self.cfg = cfg
        cfg.struct_size, cfg.vocab, cfg.dtype = C.sizeof(type(cfg)), _i32(vocab, "vocab"), int(dtype == self.torch.bfloat16)
        self._start(0, lambda _, st, h: getattr(lib, f"aed_{name}_create")(C.byref(cfg), st, h), getattr(lib, f"aed_{name}_destroy"))

    def _logits(self, t, name, rows=None):
        """Pointer and row stride of a tensor [rows, vocab]."""
        self._given(t, name, self.dtype, (rows, self.vocab))
        if t.stride(1) != 1 and self.vocab > 1:
            _t._refuse(f"{name}: a row is not contiguous")
        return t.data_ptr(), t.stride(0)

    def _by_row(self, t, name, dtype, rows):
        """Pointer of a tensor [rows], or None."""
        return None if t is None else self._flat(t, name, dtype, (rows,))


class Sampler(_RowsPlan):
    """The next tokens of rows of logits, such as Decoder.aed_decode_step's."""

    def __init__(self, vocab: int, dtype, device="cuda", stream=None):
        super().__init__(vocab, dtype, device, stream, "sampler", AedSamplerConfig())
        self._how = AedSampling(C.sizeof(AedSampling), 0, 1.0, 1.0, 0.0, None, None, None, None)
        self._given_how = None  # what _how was made of, if that were numbers
        self._i32 = self.torch.empty(0, dtype=self.torch.int32, device=self.device)

    def _set(self, rows, temperature, top_k, top_p, min_p):
        """The parameters: of all rows, or of each."""
        how, torch, numbers = self._how, self.torch, True
        self._given_how = None
        for name, value, dtype, default in (("temperature", temperature, torch.float32, 1.0), ("top_k", top_k, torch.int32, 0), ("top_p", top_p, torch.float32, 1.0),
                                            ("min_p", min_p, torch.float32, 0.0)):
            if isinstance(value, torch.Tensor):
                setattr(how, name, default)
                setattr(how, name + "s", self._flat(value, name, dtype, (rows,)))
                numbers = False
            else:
                setattr(how, name, _i32(value, name) if name == "top_k" else value)
                setattr(how, name + "s", None)
                numbers = numbers and type(value) in (int, float)
        self._given_how = (temperature, top_k, top_p, min_p) if numbers else None

    def aed_sample(self, logits, uniforms, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
        """logits: [rows, vocab]; uniforms: float32 [rows], random numbers in [0, 1).  temperature (0: the largest logit), top_k (0: all), top_p (1:
        all) and min_p (0: all): numbers, or tensors [rows] (top_k: int32, the others float32).
        Returns (tokens int32 [rows], logp float32 [rows]: log-probability among the tokens that were left).  Neither has a gradient by the logits."""
        f32, rows = self.torch.float32, _rows(logits)
        pz, stride = self._logits(logits, "logits", rows)
        pu = self._flat(uniforms, "uniforms", f32, (rows,))
        g = self._given_how  # the same numbers again, mostly: 1.2 us of a call's 9
        if g is None or g[0] is not temperature or g[1] is not top_k or g[2] is not top_p or g[3] is not min_p:
            self._set(rows, temperature, top_k, top_p, min_p)
        tokens, logp = self._i32.new_empty(rows), self._f32.new_empty(rows)
        entered = self._enter()
        status = self.lib.aed_sample(self.handle, pz, stride, rows, pu, self._how, tokens.data_ptr(), logp.data_ptr())
        if entered is not None:
            self._exit(entered)
        if status:
            _t._check(status)
        return tokens, logp


class TopLogits(_RowsPlan):
    """A teacher's largest logits of every row, for Distillation."""

    def __init__(self, vocab: int, top: int, dtype, temperature: float = 1.0, device="cuda", stream=None):
        super().__init__(vocab, dtype, device, stream, "top", AedTopConfig(top=_i32(top, "top"), temperature=temperature))
        self.top = top
        self._i32 = self.torch.empty(0, dtype=self.torch.int32, device=self.device)

    def aed_top_logits(self, logits):
        """Returns (values float32 [rows, top], falling; ids int32 [rows, top]; rest float32 [rows]: log of the sum of exp(logit /
        temperature) over the ids that are not listed).  None has a gradient by the logits."""
        rows = _rows(logits)
        pz, stride = self._logits(logits, "logits", rows)
        new = self._f32.new_empty
        values, ids, rest = new((rows, self.top)), self._i32.new_empty((rows, self.top)), new(rows)
        entered = self._enter()
        status = self.lib.aed_top_logits(self.handle, pz, stride, rows, values.data_ptr(), ids.data_ptr(), rest.data_ptr())
        if entered is not None:
            self._exit(entered)
        if status:
            _t._check(status)
        return values, ids, rest


class Distillation(_RowsPlan):
    """The loss of a student's rows of logits against a teacher's largest logits."""

    def __init__(self, vocab: int, top: int, dtype, temperature: float = 1.0, device="cuda", stream=None):
        super().__init__(vocab, dtype, device, stream, "distill", AedDistillConfig(top=_i32(top, "top"), temperature=temperature))
        self.top = top

    def aed_distill_forward(self, logits, values, ids, rest=None, weights=None):
        """values: float32 [rows, top]; ids: int32 [rows, top]; rest: float32 [rows] (TopLogits' of the same temperature), or None: the list adds up to
        one; weights: float32 [rows], 0 where a row is not scored, or None: the mean.
        Returns (loss, row_loss [rows], stats [rows, top + 2] for the gradient), float32."""
        f32, rows = self.torch.float32, _rows(logits)
        pz, stride = self._logits(logits, "logits", rows)
        pv, pi = self._flat(values, "values", f32, (rows, self.top)), self._flat(ids, "ids", self.torch.int32, (rows, self.top))
        pr, pw = self._by_row(rest, "rest", f32, rows), self._by_row(weights, "weights", f32, rows)
        new = self._f32.new_empty
        loss, row_loss, stats = new(()), new(rows), new((rows, self.top + 2))
        entered = self._enter()
        status = self.lib.aed_distill_forward(self.handle, pz, stride, rows, pv, pi, pr, pw, loss.data_ptr(), row_loss.data_ptr(), stats.data_ptr())
        if entered is not None:
            self._exit(entered)
        if status:
            _t._check(status)
        return loss, row_loss, stats

    def aed_distill_backward(self, logits, ids, stats, weights=None, d_loss=None, d_logits=None):
        """logits, ids, weights: as forward; stats: forward's.  Returns the gradient by the logits; d_logits: where it goes (may be the logits)."""
        f32, rows = self.torch.float32, _rows(logits)
        pz, stride = self._logits(logits, "logits", rows)
        pi, ps = self._flat(ids, "ids", self.torch.int32, (rows, self.top)), self._flat(stats, "stats", f32, (rows, self.top + 2))
        pw = self._by_row(weights, "weights", f32, rows)
        pd = None if d_loss is None else self._flat(d_loss, "d_loss", f32, tuple(d_loss.shape[:0]))
        if d_logits is None:
            d_logits = logits.new_empty((rows, self.vocab))
        pg, g_stride = self._logits(d_logits, "d_logits", rows)
        entered = self._enter()
        status = self.lib.aed_distill_backward(self.handle, pz, stride, rows, pi, pw, ps, pd, pg, g_stride)
        if entered is not None:
            self._exit(entered)
        if status:
            _t._check(status)
        return d_logits

    def loss(self, logits, values, ids, rest=None, weights=None):
        """The loss, for torch's autograd: its gradient by the logits (once: second derivatives are refused).  The teacher's list and the weights are constants:
        those that require a gradient are refused."""
        return _autograd().of(self, logits, values, ids, rest, weights)


_function = None


def _autograd():
    """The torch.autograd.Function class (made when it is first needed: torch is not imported before)."""
    global _function
    if _function is None:
        import torch

        class Loss(torch.autograd.Function):
            @classmethod
            def of(cls, plan, logits, values, ids, rest, weights):
                for name, t in (("values", values), ("rest", rest), ("weights", weights)):
                    if t is not None and t.requires_grad and torch.is_grad_enabled():
                        _t._refuse(f"{name} requires a gradient, and the loss has none by it")
                return cls.apply(plan, logits, values, ids, rest, weights)

            @staticmethod
            def forward(ctx, plan, logits, values, ids, rest, weights):
                loss, _, stats = plan.aed_distill_forward(logits, values, ids, rest, weights)
                ctx.plan = plan
                ctx.save_for_backward(logits, ids, stats, weights)
                return loss

            @staticmethod
            def backward(ctx, d_loss):
                logits, ids, stats, weights = ctx.saved_tensors
                gradient = ctx.plan.aed_distill_backward(logits, ids, stats, weights, d_loss.contiguous())
                return None, *_t._autograd()[2]((gradient,), d_loss, logits), None, None, None, None

        _function = Loss
    return _function
