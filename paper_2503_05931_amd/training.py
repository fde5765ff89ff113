"""ctypes binding of the scoring and training operators (include/aed_train.h): attention of ragged batches with many rows a
sequence, forward and backward, and the preference loss on pairs of transcripts.

Argument marshalling only; a missing library raises.  Tensors are torch tensors on the device.  A plan works on the stream
that was current when it was made, or on `stream`; a call under another current stream waits for that one's work and lets it
wait for the results.  A graph that holds a plan's calls needs the plan for as long as it is replayed.
"""
from __future__ import annotations

import ctypes as C

import numpy as np

from . import binding as _b

EXPORTS = ("aed_train_last_error", "aed_attn_workspace_bytes", "aed_attn_create", "aed_attn_destroy", "aed_attn_forward",
           "aed_attn_backward", "aed_preference_workspace_bytes", "aed_preference_create", "aed_preference_destroy",
           "aed_preference_forward", "aed_preference_backward")


class AedAttnConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_int32) for n in (
        "n_heads", "n_kv_heads", "head_dim", "dtype", "causal", "bias_buckets", "bias_max_distance", "bias_bidirectional",
        "training")] + [("scale", C.c_float)]


class AedRows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64)]


class AedPreferenceConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("vocab", C.c_int32), ("dtype", C.c_int32), ("beta", C.c_float),
                ("label_smoothing", C.c_float)]


_i32p, _i64p = C.POINTER(C.c_int32), C.POINTER(C.c_int64)
_configured = False


def _lib():
    global _configured
    lib = _b.load()
    if not _configured:
        vp, rows, size = C.c_void_p, C.POINTER(AedRows), C.POINTER(C.c_size_t)
        cfg, pcfg = C.POINTER(AedAttnConfig), C.POINTER(AedPreferenceConfig)
        lib.aed_attn_workspace_bytes.argtypes = [cfg, _i32p, _i32p, _i64p, C.c_int32, size]
        lib.aed_attn_create.argtypes = [cfg, _i32p, _i32p, _i64p, C.c_int32, vp, C.c_size_t, vp, C.POINTER(vp)]
        lib.aed_attn_destroy.argtypes = [vp]
        lib.aed_attn_forward.argtypes = [vp, rows, rows, rows, vp, vp, rows, vp]
        lib.aed_attn_backward.argtypes = [vp, rows, rows, rows, rows, rows, vp, vp, vp, rows, rows, rows, vp]
        lib.aed_preference_workspace_bytes.argtypes = [pcfg, _i32p, C.c_int32, size]
        lib.aed_preference_create.argtypes = [pcfg, _i32p, C.c_int32, vp, C.c_size_t, vp, C.POINTER(vp)]
        lib.aed_preference_destroy.argtypes = [vp]
        lib.aed_preference_forward.argtypes = [vp, vp, C.c_int64, vp, vp, vp, vp, vp]
        lib.aed_preference_backward.argtypes = [vp, vp, C.c_int64, vp, vp, vp, vp, vp, C.c_int64]
        for n in EXPORTS:
            getattr(lib, n).restype = C.c_int
        lib.aed_train_last_error.argtypes = []
        lib.aed_train_last_error.restype = C.c_char_p
        _configured = True
    return lib


def _check(status):
    if status != _b.AED_OK:
        raise _b.AedError(status, _lib().aed_train_last_error().decode())


def _lens(a):
    a = np.ascontiguousarray(a, dtype=np.int32).reshape(-1)
    return a, a.ctypes.data_as(_i32p)


def _refuse(message):
    raise _b.AedError(_b.AED_EINVAL, message)


class _Plan:
    """A handle, its workspace and its stream."""

    def __init__(self, dtype, device, stream):
        import torch
        self.torch = torch
        self.lib = _lib()
        if dtype not in (torch.bfloat16, torch.float32):
            raise _b.AedError(_b.AED_EUNSUPPORTED, f"{dtype}: tensors are bfloat16 or float32")
        self.dtype, self.device = dtype, torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.handle = C.c_void_p(None)
        self.stream = stream
        self._destroy = None
        # new tensors are made from one that is there: 1.5 us instead of 1.7 each, of 9 us for a call with one row
        self._f32 = torch.empty(0, dtype=torch.float32, device=self.device)

    def _start(self, nbytes, create, destroy):
        """create(workspace pointer, stream, handle)"""
        torch = self.torch
        with torch.cuda.device(self.device):
            if self.stream is None:
                self.stream = torch.cuda.current_stream(self.device)
            self.raw, self.index = self.stream.cuda_stream, self.device.index
            self._raw_stream, self._get_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
            self._only = torch.cuda.device_count() == 1  # no other device can be current: 0.2 us of a call's 9 are not spent on asking
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            self._enter()
            _check(create(C.c_void_p(self.workspace.data_ptr()), C.c_void_p(self.stream.cuda_stream), C.byref(self.handle)))
        self._destroy = destroy

    def close(self):
        if self.handle and self._destroy:
            back = self._to_device()
            self._destroy(self.handle)
            self.handle = C.c_void_p(None)
            if back != self.index:
                self.torch.cuda.set_device(back)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # inputs come from torch's current stream, and what follows there uses the results; of a call that fails, the memory that they were to have
    def _enter(self):
        if not self.handle and self._destroy:
            raise _b.AedError(_b.AED_ESTATE, "the plan is closed")
        if self._raw_stream(self.index) == self.raw and (self._only or self._get_device() == self.index):
            return None
        back = self._to_device()
        current = self.torch.cuda.current_stream(self.device)
        if current.cuda_stream != self.raw:
            self.stream.wait_stream(current)
        return current, back

    def _exit(self, entered):
        current, back = entered
        if current.cuda_stream != self.raw:
            current.wait_stream(self.stream)
        if back != self.index:
            self.torch.cuda.set_device(back)

    def _to_device(self):
        """Makes the plan's device the current one (a default stream is that device's) and returns which it was."""
        back = self._get_device()
        if back != self.index:
            self.torch.cuda.set_device(self.index)
        return back

    def _given(self, t, name, dtype, shape):
        if t.dtype is dtype and t.shape == shape and t.get_device() == self.index:
            return t
        if t.dtype != dtype:
            _refuse(f"{name} is {t.dtype}, the plan's is {dtype}")
        if t.device != self.device:
            _refuse(f"{name} is on {t.device}, the plan on {self.device}")
        for have, want in zip(t.shape, shape) if t.dim() == len(shape) else ((-1, 0),):
            if want is not None and have != want:
                _refuse(f"{name} has shape {tuple(t.shape)}, expected {tuple('any' if n is None else n for n in shape)}")
        return t

    def _flat(self, t, name, dtype, shape):
        if not self._given(t, name, dtype, shape).is_contiguous():
            _refuse(f"{name} is not contiguous")
        return t.data_ptr()


class Attention(_Plan):
    """Attention of one batch's lengths, for all its layers.  q: [query rows, n_heads, head_dim]; k, v: [key rows, n_kv_heads,
    head_dim]; parts of wider tensors are taken as they are (the last dimension contiguous, 16-byte aligned)."""

    def __init__(self, q_lens, k_lens, n_heads: int, head_dim: int, dtype, n_kv_heads: int = None, causal: bool = False,
                 bias_buckets: int = 0, bias_max_distance: int = 0, bias_bidirectional: bool = False, scale: float = 0.0,
                 k_starts=None, training: bool = True, device="cuda", stream=None):
        super().__init__(dtype, device, stream)
        kv = n_heads if n_kv_heads is None else n_kv_heads
        self.cfg = AedAttnConfig(C.sizeof(AedAttnConfig), n_heads, kv, head_dim, int(dtype == self.torch.bfloat16), int(causal), bias_buckets,
                                 bias_max_distance, int(bias_bidirectional), int(training), scale)
        ql, pq = _lens(q_lens)
        kl, pk = _lens(k_lens)
        if len(ql) != len(kl):
            _refuse(f"{len(ql)} query lengths and {len(kl)} key lengths")
        starts = ps = None
        if k_starts is not None:
            starts = np.ascontiguousarray(k_starts, dtype=np.int64).reshape(-1)
            if len(starts) != len(kl):
                _refuse(f"{len(starts)} key starts and {len(kl)} key lengths")
            ps = starts.ctypes.data_as(_i64p)
        n = C.c_size_t(0)
        _check(self.lib.aed_attn_workspace_bytes(C.byref(self.cfg), pq, pk, ps, len(ql), C.byref(n)))
        self.q_rows = int(ql.sum(dtype=np.int64))
        # rows that the keys' tensors need; packed keys have no others
        self.k_rows = int(kl.sum(dtype=np.int64)) if starts is None else int(np.max(np.where(kl > 0, starts + kl, 0)))
        self.packed = starts is None
        self._q_shape, self._k_shape, self._lse_shape = (self.q_rows, n_heads, head_dim), (self.k_rows, kv, head_dim), (self.q_rows, n_heads)
        # arguments of a call: q, k, v, what is returned for the queries, out, d_out, dk, dv
        self._at = [AedRows() for _ in range(8)]
        for i, h in ((3, n_heads), (6, kv), (7, kv)):
            self._at[i].row_stride, self._at[i].head_stride = h * head_dim, head_dim
        self._start(n.value, lambda ws, st, h: self.lib.aed_attn_create(C.byref(self.cfg), pq, pk, ps, len(ql), ws, n.value, st, h),
                    self.lib.aed_attn_destroy)

    def _rows(self, to, t, name, heads, rows):
        shape, (s0, s1, s2) = t.shape, t.stride() if t.dim() == 3 else (0, 0, 0)
        if (s2 != 1 or t.dtype is not self.dtype or shape[1] != heads or shape[2] != self.cfg.head_dim or t.get_device() != self.index
                or shape[0] != rows and (shape[0] < rows or self.packed or name not in ("k", "v"))):
            self._given(t, name, self.dtype, (None, heads, self.cfg.head_dim))
            if shape[0] != rows:
                _refuse(f"{name} has {shape[0]} rows, expected {rows}")
            _refuse(f"{name}: the last dimension is not contiguous")
        to.data, to.row_stride, to.head_stride = t.data_ptr(), s0, s1
        return to

    def _side(self, bias, key_mask, k_rows):
        """Pointers of the bias and the mask."""
        torch, c = self.torch, self.cfg
        pb = pm = None
        if bias is not None:
            if not c.bias_buckets:
                _refuse("the plan was made without a bias")
            pb = self._flat(bias, "bias", self.dtype, (c.bias_buckets, c.n_heads))
        if key_mask is not None:
            if key_mask.dtype == torch.bool:
                key_mask = key_mask.view(torch.uint8)
            pm = self._flat(key_mask, "key_mask", torch.uint8, (k_rows,))
        return pb, pm

    def aed_attn_forward(self, q, k, v, bias=None, key_mask=None):
        """Returns (out [query rows, n_heads, head_dim], lse float32 [query rows, n_heads])."""
        c = self.cfg
        at, H, G = self._at, c.n_heads, c.n_kv_heads
        self._rows(at[0], q, "q", H, self.q_rows)
        self._rows(at[1], k, "k", G, self.k_rows)
        self._rows(at[2], v, "v", G, self.k_rows)
        pb, pm = self._side(bias, key_mask, k.shape[0]) if bias is not None or key_mask is not None else (None, None)
        out, lse = q.new_empty(self._q_shape), self._f32.new_empty(self._lse_shape)
        at[3].data = out.data_ptr()
        entered = self._enter()
        status = self.lib.aed_attn_forward(self.handle, at[0], at[1], at[2], pb, pm, at[3], lse.data_ptr())
        if entered is not None:
            self._exit(entered)
        if status:
            _check(status)
        return out, lse

    def aed_attn_backward(self, d_out, q, k, v, out, lse, bias=None, key_mask=None):
        """Returns (dq, dk, dv, d_bias or None) in the shapes of q, k, v and bias."""
        torch, c = self.torch, self.cfg
        H, G = c.n_heads, c.n_kv_heads
        at = self._at
        self._rows(at[0], q, "q", H, self.q_rows)
        self._rows(at[1], k, "k", G, self.k_rows)
        self._rows(at[2], v, "v", G, self.k_rows)
        self._rows(at[4], out, "out", H, self.q_rows)
        self._rows(at[5], d_out, "d_out", H, self.q_rows)
        plse = self._flat(lse, "lse", torch.float32, self._lse_shape)
        pb, pm = self._side(bias, key_mask, k.shape[0]) if bias is not None or key_mask is not None else (None, None)
        dq, dk, dv = q.new_empty(self._q_shape), q.new_empty(self._k_shape), q.new_empty(self._k_shape)
        d_bias = None if bias is None else torch.empty_like(bias)
        at[3].data, at[6].data, at[7].data = dq.data_ptr(), dk.data_ptr(), dv.data_ptr()
        entered = self._enter()
        status = self.lib.aed_attn_backward(self.handle, at[5], at[0], at[1], at[2], at[4], plse, pb, pm, at[3], at[6], at[7],
                                            None if d_bias is None else d_bias.data_ptr())
        if entered is not None:
            self._exit(entered)
        if status:
            _check(status)
        return dq, dk, dv, d_bias

    def attend(self, q, k, v, bias=None, key_mask=None):
        """The output, for torch's autograd (once: second derivatives are refused)."""
        return _autograd()[0].apply(self, q, k, v, bias, key_mask)


class Preference(_Plan):
    """The loss of n pairs of transcripts.  seq_lens: rows of chosen_0, rejected_0, chosen_1, ...; logits: [rows, vocab]."""

    def __init__(self, seq_lens, vocab: int, dtype, beta: float = 0.1, label_smoothing: float = 0.0, device="cuda", stream=None):
        super().__init__(dtype, device, stream)
        self.cfg = AedPreferenceConfig(C.sizeof(AedPreferenceConfig), vocab, int(dtype == self.torch.bfloat16), beta, label_smoothing)
        lens, p = _lens(seq_lens)
        if len(lens) % 2:
            _refuse("sequences come in pairs")
        self.pairs = len(lens) // 2
        n = C.c_size_t(0)
        _check(self.lib.aed_preference_workspace_bytes(C.byref(self.cfg), p, self.pairs, C.byref(n)))
        self.rows = int(lens.sum(dtype=np.int64))
        self._start(n.value, lambda ws, st, h: self.lib.aed_preference_create(C.byref(self.cfg), p, self.pairs, ws, n.value, st, h),
                    self.lib.aed_preference_destroy)

    def _logits(self, t, name):
        self._given(t, name, self.dtype, (self.rows, self.cfg.vocab))
        if t.stride(1) != 1 and self.cfg.vocab > 1:
            _refuse(f"{name}: a row is not contiguous")
        return t.data_ptr(), t.stride(0) if self.rows > 1 else self.cfg.vocab

    def aed_preference_forward(self, logits, labels, ref_logp):
        """labels: int32 [rows], negative where a row is not scored; ref_logp: float32 [rows].
        Returns (loss, ratio [2 n], lse [rows, 2]: largest logit and log sum exp of what is left without it), float32."""
        torch = self.torch
        pz, stride = self._logits(logits, "logits")
        py, pr = self._flat(labels, "labels", torch.int32, (self.rows,)), self._flat(ref_logp, "ref_logp", torch.float32, (self.rows,))
        new = self._f32.new_empty
        loss, ratio, lse = new(()), new(2 * self.pairs), new((self.rows, 2))
        entered = self._enter()
        status = self.lib.aed_preference_forward(self.handle, pz, stride, py, pr, loss.data_ptr(), ratio.data_ptr(), lse.data_ptr())
        if entered is not None:
            self._exit(entered)
        if status:
            _check(status)
        return loss, ratio, lse

    def aed_preference_backward(self, logits, labels, ratio, lse, d_loss=None, d_logits=None):
        """Returns the gradient by the logits; d_logits: where it goes (may be the logits)."""
        torch = self.torch
        pz, stride = self._logits(logits, "logits")
        py, pl = self._flat(labels, "labels", torch.int32, (self.rows,)), self._flat(lse, "lse", torch.float32, (self.rows, 2))
        pr = self._flat(ratio, "ratio", torch.float32, (2 * self.pairs,))
        pd = None if d_loss is None else self._flat(d_loss, "d_loss", torch.float32, tuple(d_loss.shape[:0]))
        if d_logits is None:
            d_logits = logits.new_empty((self.rows, self.cfg.vocab))
        pg, g_stride = self._logits(d_logits, "d_logits")
        entered = self._enter()
        status = self.lib.aed_preference_backward(self.handle, pz, stride, py, pr, pl, pd, pg, g_stride)
        if entered is not None:
            self._exit(entered)
        if status:
            _check(status)
        return d_logits

    def loss(self, logits, labels, ref_logp):
        """The loss, for torch's autograd (once: second derivatives are refused)."""
        return _autograd()[1].apply(self, logits, labels, ref_logp)


_functions = None


def _autograd():
    """The two torch.autograd.Function classes and what makes their gradients constants (made when they are first needed: torch is not imported before)."""
    global _functions
    if _functions is None:
        import torch

        class Once(torch.autograd.Function):
            """A gradient that the library made from the other arguments.  It is a constant to autograd, so what would need its own gradient is refused.
            (torch's once_differentiable does so only where the incoming gradient has a graph: not for a loss's, which is 1.)"""

            @staticmethod
            def forward(ctx, gradient, *made_from):
                return gradient.detach()

            @staticmethod
            def backward(ctx, *_):
                raise RuntimeError("second derivatives of the library's operators are not computed")

        def once(gradients, *made_from):
            if not torch.is_grad_enabled():  # on only under create_graph
                return gradients
            return tuple(None if g is None else Once.apply(g, *made_from) for g in gradients)

        class Attend(torch.autograd.Function):
            @staticmethod
            def forward(ctx, plan, q, k, v, bias, key_mask):
                out, lse = plan.aed_attn_forward(q, k, v, bias, key_mask)
                ctx.plan = plan
                ctx.save_for_backward(q, k, v, out, lse, bias, key_mask)
                return out

            @staticmethod
            def backward(ctx, d_out):
                q, k, v, out, lse, bias, key_mask = ctx.saved_tensors
                given = d_out, q, k, v, bias
                if d_out.stride(-1) != 1 or d_out.data_ptr() % 16 or any(n * d_out.element_size() % 16 for n in d_out.stride()[:2]):
                    d_out = d_out.contiguous()
                gradients = ctx.plan.aed_attn_backward(d_out, q, k, v, out, lse, bias, key_mask)
                return None, *once(gradients, *given), None

        class Loss(torch.autograd.Function):
            @staticmethod
            def forward(ctx, plan, logits, labels, ref_logp):
                loss, ratio, lse = plan.aed_preference_forward(logits, labels, ref_logp)
                ctx.plan = plan
                ctx.save_for_backward(logits, labels, ratio, lse)
                return loss

            @staticmethod
            def backward(ctx, d_loss):
                logits, labels, ratio, lse = ctx.saved_tensors
                gradient = ctx.plan.aed_preference_backward(logits, labels, ratio, lse, d_loss.contiguous())
                return None, *once((gradient,), d_loss, logits), None, None

        _functions = Attend, Loss, once
    return _functions
