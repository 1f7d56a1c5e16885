"""The operators of include/cada_ops.h on torch tensors: argument marshalling only.

``linear_forward`` / ``linear_backward``: a layer's product with bias, activation and residual, and its gradients.
``cross_entropy``: the softmax cross-entropy over any number of classes with its gradient.
``AdamW``: the step over many tensors at once, moments in 32 or in 8 bits.

Tensors are float32 or bfloat16 on one GPU.  Work goes to ``stream``, by default the device's current stream at the call (AdamW: the one that was current when
it was made, for its steps too), and nothing synchronises the host; inputs must be ready there.  Outputs that are not handed in, and a call's workspace
unless one is, come from torch's caching allocator and belong to that stream.

The calls do not take part in autograd: operands that require gradients are read as they are, outputs have no history, and what is written in place
(outputs handed in, parameters) counts no version.  ``linear_backward`` and the gradient of ``cross_entropy`` are what a backward pass is made of.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence, Tuple, Union

import torch

from .binding import CadaError, _check, _lib

try:
    from . import _ops
except ImportError as e:
    raise ImportError("_ops.so is not built: run `python -m paper_2012_15469_amd.build` (no fallback exists)") from e
_ops.set_error_class(CadaError)

F32, BF16 = 0, 1
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
MOMENT_BLOCK = 256
_TYPES = {torch.float32: F32, torch.bfloat16: BF16}


class cada_adamw_tensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("copy", C.c_void_p), ("n", C.c_int64), ("param_type", C.c_int32), ("grad_type", C.c_int32),
                ("weight_decay", C.c_double)]


class cada_adamw_config(C.Structure):
    _fields_ = [("tensors", C.POINTER(cada_adamw_tensor)), ("n_tensors", C.c_int32), ("moment_bits", C.c_int32), ("m", C.c_void_p), ("v", C.c_void_p),
                ("m_scale", C.c_void_p), ("v_scale", C.c_void_p), ("norm", C.c_void_p), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("max_norm", C.c_double), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t), ("stream", C.c_void_p)]


for _name, _res, _args in (("cada_adamw_moment_elements", C.c_int64, [C.POINTER(cada_adamw_config)]), ("cada_adamw_workspace", C.c_int, [C.POINTER(cada_adamw_config)]),
                           ("cada_adamw_init", C.c_int, [C.POINTER(cada_adamw_config), C.POINTER(C.c_void_p)]),
                           ("cada_adamw_step", C.c_int, [C.c_void_p, C.c_int64, C.c_double, C.c_void_p]),
                           ("cada_adamw_moments", C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]), ("cada_adamw_destroy", None, [C.c_void_p])):
    _f = getattr(_lib, _name)
    _f.restype, _f.argtypes = _res, _args


def _need(ok: bool, text: str):
    if not ok:
        raise ValueError(text)


def _call(call, tensor, stream, *args):
    """call(*args, stream handle) with the tensor's device current.  (The raw handle and device index: torch.cuda's own functions make objects, 2 us of a call
    that takes six.)"""
    index = tensor.get_device() if isinstance(tensor, torch.Tensor) else -1
    if index < 0:
        return call(*args, 0)          # (refused there)
    if stream is not None:
        _need(stream.device.index == index, "stream must be one of cuda:%d's" % index)
        with torch.cuda.stream(stream):          # (so that what is allocated belongs to it)
            return call(*args, stream.cuda_stream)
    handle = torch._C._cuda_getCurrentRawStream(index)
    if index == torch._C._cuda_getDevice():
        return call(*args, handle)
    with torch.cuda.device(index):
        return call(*args, handle)


def linear_forward(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, *, residual: Optional[torch.Tensor] = None, act: str = "none",
                   keep_pre: bool = False, out: Optional[torch.Tensor] = None, pre: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(y, pre) with y = act(x w + bias) + residual and pre = x w + bias; pre is None unless ``keep_pre`` or a ``pre`` to write is given.

    x [rows, in], w [in, out] (the layout of the engine's parameters), bias [out], residual [rows, out], all of one type; rows contiguous, any
    distance apart.  ``out`` may be ``residual``."""
    if act not in ACTIVATIONS:
        raise ValueError("act must be one of %s" % ", ".join(ACTIVATIONS))
    return _call(_ops.linear_forward, x, stream, x, w, bias, residual, ACTIVATIONS[act], bool(keep_pre), out, pre, workspace)


def linear_backward(dy: torch.Tensor, x: torch.Tensor, w: torch.Tensor, *, pre: Optional[torch.Tensor] = None, act: str = "none", need_dx: bool = True,
                    need_dw: bool = True, need_db: bool = True, dx: Optional[torch.Tensor] = None, dw: Optional[torch.Tensor] = None,
                    db: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None
                    ) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor], Optional[torch.Tensor]]:
    """(dx, dw, db) of a layer from the gradient of its output; the residual's gradient is dy itself.  ``pre`` is what
    linear_forward kept (not needed for act="none").  Outputs handed in are written, not added to."""
    if act not in ACTIVATIONS:
        raise ValueError("act must be one of %s" % ", ".join(ACTIVATIONS))
    return _call(_ops.linear_backward, dy, stream, dy, x, w, pre, ACTIVATIONS[act], bool(need_dx), bool(need_dw), bool(need_db), dx, dw, db, workspace)


def cross_entropy(logits: torch.Tensor, labels: torch.Tensor, *, smoothing: float = 0.0, ignore_index: int = -100, scale: float = 1.0, need_grad: bool = True,
                  grad: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None
                  ) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """(mean loss, loss of each row, gradient of scale * mean loss with respect to the logits).

    logits [rows, classes]; labels int32 or int64 [rows].  Rows labelled ``ignore_index`` count nowhere; classes at -inf are ruled out.  ``grad`` may be
    the logits themselves.  Losses are float32, the gradient has the logits' type."""
    return _call(_ops.cross_entropy, logits, stream, logits, labels, smoothing, ignore_index, scale, bool(need_grad), grad, workspace)


class AdamW:
    """The AdamW step over ``params`` with ``grads`` (the same tensors every step: write gradients into them).

    params, grads: contiguous float32 or bfloat16 tensors, each param's type its own.  ``weight_decay``: one value or one per tensor.  ``max_norm`` > 0 clips
    the gradients to that norm over all of them (``norm`` holds the norm of the last step).  ``state_bits``: 32, or 8 for moments in
    8-bit codes.  ``copies``: bfloat16 tensors that receive the rounded parameters, or None each.  ``moments``: (m, v) to go on from, as ``m`` and ``v`` of another
    AdamW, updated in place; zeros otherwise.  Parameters, copies and moments share memory with nothing (gradients may with each other).  ``stream``: where every step runs, by
    default the stream that is current here, whichever is current at the step; gradients must be ready there, and a step in a captured graph needs that graph's stream.

    ``m`` and ``v`` hold the moments of all tensors one after the other, each tensor's filled up to whole blocks of 256 (``offsets`` says where each
    starts): float32 tensors, or pairs of codes and scales.  ``moments()`` gives their values."""

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], *, lr: float = 1e-3, beta1: float = 0.9, beta2: float = 0.999,
                 eps: float = 1e-8, weight_decay: Union[float, Sequence[float]] = 0.0, max_norm: float = 0.0, state_bits: int = 32,
                 copies: Optional[Sequence[Optional[torch.Tensor]]] = None, moments=None, stream: Optional[torch.cuda.Stream] = None):
        self.plan = None
        n = len(params)
        _need(n >= 1 and len(grads) == n and (copies is None or len(copies) == n), "params, grads and copies must be lists of one length")
        _need(state_bits in (32, 8), "state_bits must be 32 or 8")
        decay = [float(weight_decay)] * n if isinstance(weight_decay, (int, float)) else [float(d) for d in weight_decay]
        _need(len(decay) == n, "weight_decay must be one value or one per tensor")
        self.device = dev = params[0].device
        _need(dev.type == "cuda", "params must be on a GPU")
        self.params, self.grads, self.copies = list(params), list(grads), list(copies) if copies is not None else [None] * n
        self.lr, self.t, self.state_bits = lr, 0, state_bits
        self.stream = stream or torch.cuda.current_stream(dev)
        _need(self.stream.device == dev, "stream must be one of %s's" % dev)
        tensors = (cada_adamw_tensor * n)()
        self.offsets, total = [], 0
        for i, (p, g, c) in enumerate(zip(self.params, self.grads, self.copies)):
            for name, t in (("param", p), ("grad", g)):
                _need(t.device == dev and t.dtype in _TYPES and t.is_contiguous(), "%s %d must be a contiguous float32 or bfloat16 tensor on %s" % (name, i, dev))
            _need(g.shape == p.shape, "grad %d must have its param's shape" % i)
            _need(c is None or (c.device == dev and c.dtype == torch.bfloat16 and c.is_contiguous() and c.shape == p.shape),
                  "copy %d must be a contiguous bfloat16 tensor of its param's shape" % i)
            t = tensors[i]
            t.param, t.grad, t.copy, t.n = p.data_ptr(), g.data_ptr(), c.data_ptr() if c is not None else None, p.numel()
            t.param_type, t.grad_type, t.weight_decay = _TYPES[p.dtype], _TYPES[g.dtype], decay[i]
            self.offsets.append(total)
            total += -(-p.numel() // MOMENT_BLOCK) * MOMENT_BLOCK
        with torch.cuda.stream(self.stream):          # (what is made here is ready for the steps)
            self.norm = torch.zeros((), device=dev)
            if moments is None:
                moments = tuple((torch.zeros(total, dtype=dt, device=dev), torch.zeros(total // MOMENT_BLOCK, device=dev)) for dt in (torch.int8, torch.uint8)) \
                    if state_bits == 8 else (torch.zeros(total, device=dev), torch.zeros(total, device=dev))
        self.m, self.v = moments
        for name, t, dt in (("m", self.m, torch.int8), ("v", self.v, torch.uint8)):
            parts = (t[0], t[1]) if state_bits == 8 else (t,)
            want = ((dt, total), (torch.float32, total // MOMENT_BLOCK)) if state_bits == 8 else ((torch.float32, total),)
            for part, (dtype, size) in zip(parts, want):
                _need(part.device == dev and part.dtype == dtype and part.is_contiguous() and part.numel() == size,
                      "%s must hold contiguous %s of %d elements on %s" % (name, dtype, size, dev))
        cfg = cada_adamw_config()
        cfg.tensors, cfg.n_tensors, cfg.moment_bits = tensors, n, state_bits
        if state_bits == 8:
            cfg.m, cfg.m_scale, cfg.v, cfg.v_scale = (t.data_ptr() for t in (*self.m, *self.v))
        else:
            cfg.m, cfg.v = self.m.data_ptr(), self.v.data_ptr()
        cfg.norm = self.norm.data_ptr()
        cfg.beta1, cfg.beta2, cfg.eps, cfg.max_norm = beta1, beta2, eps, max_norm
        _check(_lib.cada_adamw_workspace(C.byref(cfg)))
        with torch.cuda.stream(self.stream):
            self.workspace = torch.empty(cfg.workspace_bytes, dtype=torch.uint8, device=dev)
        cfg.workspace, cfg.stream = self.workspace.data_ptr(), self.stream.cuda_stream
        plan = C.c_void_p()
        with torch.cuda.device(dev):
            _check(_lib.cada_adamw_init(C.byref(cfg), C.byref(plan)))
        self.plan = plan.value

    def step(self, t: Optional[int] = None, *, lr: Optional[float] = None, grad_scale: Optional[torch.Tensor] = None):
        """One step on the plan's stream; ``t`` (1, 2, ...) goes up by one if it is not given.  ``grad_scale``: float32 [1] on the GPU, read when the step
        runs (1 / loss scale)."""
        if grad_scale is not None:
            _need(grad_scale.device == self.device and grad_scale.dtype == torch.float32 and grad_scale.numel() == 1, "grad_scale must be a float32 scalar on %s" % self.device)
        t = self.t + 1 if t is None else t
        args = self.plan, t, self.lr if lr is None else lr, None if grad_scale is None else grad_scale.data_ptr()
        if self.device.index == torch._C._cuda_getDevice():
            _check(_lib.cada_adamw_step(*args))
        else:
            with torch.cuda.device(self.device):
                _check(_lib.cada_adamw_step(*args))
        self.t = t

    def moments(self) -> Tuple[torch.Tensor, torch.Tensor]:
        """(m, v) as float32 values, laid out as ``offsets`` says: the moments themselves with 32 bits, decoded copies with 8; ready on the plan's stream."""
        if self.state_bits == 32:
            return self.m, self.v
        if self.device.index != torch._C._cuda_getDevice() or torch._C._cuda_getCurrentRawStream(self.device.index) != self.stream.cuda_stream:
            with torch.cuda.stream(self.stream):          # (its device too; so that what is allocated belongs to it)
                return self.moments()
        m, v = (torch.empty_like(self.m[0], dtype=torch.float32) for _ in range(2))
        _check(_lib.cada_adamw_moments(self.plan, m.data_ptr(), v.data_ptr()))
        return m, v

    def close(self):
        if self.plan:
            _lib.cada_adamw_destroy(self.plan)
            self.plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
