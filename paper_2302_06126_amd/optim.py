"""Binding of include/tag_optim.h: orthogonalised updates, clipped gradients.

  Orthogonalise   Newton-Schulz products that bring the singular values of
                  matrices near one
  Clip            the norm over all gradients and, where it is above a limit,
                  the gradients scaled down to it.  ``Clip.of(trainer, limit)``
                  takes a Trainer's
  Muon            the optimiser step around them: momentum, the orthogonalised
                  update of weight matrices, momentum SGD for everything else.
                  ``Muon.of(trainer)`` takes a Trainer's parameters and
                  gradients; a training step is then ``trainer.step(feats)``
                  followed by ``muon.step()``; with ``max_norm`` the step is
                  that of the clipped gradients.

Argument checks and marshalling only; everything runs in libtag.so's HIP
kernels.  An object owns its workspace: its calls must be ordered.  It is memory
of the stream that is current when the object is made (a Muon's momentum too):
another stream that a call is given has to wait for it first.
"""
from __future__ import annotations

from typing import Optional, Sequence, Tuple

from . import TagError, _abi, _ptr, _torch
from ._abi import (C, check, tag_clip_array, tag_clip_plan, tag_muon_group, tag_muon_options, tag_newton_schulz,
                   tag_ortho_group)
from .policy import _device, _dtype, _launch, _raw_stream

__all__ = ["Orthogonalise", "orthogonalise", "Clip", "Muon", "QUINTIC"]

# coefficients of the quintic whose steps bring singular values from 0.01 and more to about [0.7, 1.2]
QUINTIC = (3.4445, -4.7750, 2.0315)


def _iteration(steps, coef, eps) -> tag_newton_schulz:
    return tag_newton_schulz(int(steps), float(coef[0]), float(coef[1]), float(coef[2]), float(eps))


def _set(arr, t, what, shape, dtype, device):
    """Fills a tag_matrices from t: [count, rows, cols], or [rows, cols] for a
    count of one, with unit column stride."""
    if t.dtype != dtype or t.device != device:
        raise ValueError(f"{what} must be {dtype} on {device}")
    if tuple(t.shape) != tuple(shape) and not (shape[0] == 1 and tuple(t.shape) == tuple(shape[1:])):
        raise ValueError(f"{what} must have the shape {list(shape)}, not {list(t.shape)}")
    if shape[2] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{what} must have unit stride along a row")
    arr.base = _ptr(t)
    arr.row_stride = t.stride(-2) if shape[1] > 1 else shape[2]
    arr.matrix_stride = t.stride(0) if t.dim() == 3 and shape[0] > 1 else shape[1] * max(arr.row_stride, shape[2])


class Orthogonalise:
    """Orthogonalises matrices of fixed shapes: ``shapes`` is a list of
    (count, rows, cols).  A call takes a tensor [count, rows, cols] for each and
    returns the results, tensors of this object unless ``out`` gives others
    (they may be the inputs, each its own; what is written shares no other
    memory with anything)."""

    def __init__(self, shapes: Sequence[Tuple[int, int, int]], dtype=None, device="cuda", steps: int = 5,
                 coef=QUINTIC, eps: float = 1e-7):
        torch = _torch()
        self.dtype = torch.float32 if dtype is None else dtype
        self._code = _dtype(self.dtype)
        self.device = _device(device)
        self.shapes = [tuple(int(v) for v in s) for s in shapes]
        self._ns = _iteration(steps, coef, eps)
        self._g = (tag_ortho_group * max(len(self.shapes), 1))()
        for g, (n, r, c) in zip(self._g, self.shapes):
            g.count, g.rows, g.cols = n, r, c
        b = C.c_size_t(0)
        check(_abi.load().tag_orthogonalise_workspace(self._g, len(self.shapes), C.byref(b)),
              "tag_orthogonalise_workspace")
        self.ws_bytes = b.value
        self.ws = torch.empty(b.value, dtype=torch.uint8, device=self.device)
        self.out = None

    def __call__(self, matrices, out=None, stream=None):
        if len(matrices) != len(self.shapes) or (out is not None and len(out) != len(self.shapes)):
            raise ValueError(f"{len(self.shapes)} tensors are wanted")
        if out is None:
            if self.out is None:
                torch = _torch()
                self.out = [torch.empty(s, dtype=self.dtype, device=self.device) for s in self.shapes]
                if stream is not None:   # (memory of the current stream)
                    stream.wait_stream(torch.cuda.current_stream(self.device))
            out = self.out
        elif len({y.data_ptr() for y in out}) != len(out) or any(
                y.data_ptr() == x.data_ptr() for i, x in enumerate(matrices) for j, y in enumerate(out) if i != j):
            raise ValueError("an output may be its own input, not another's, nor another output")
        for g, s, x, y in zip(self._g, self.shapes, matrices, out):
            _set(getattr(g, "in"), x, "a matrix", s, self.dtype, self.device)
            _set(g.out, y, "an output", s, self.dtype, self.device)
        _launch(self.device, "tag_orthogonalise", self._g, len(self.shapes), self._code, C.byref(self._ns),
                _ptr(self.ws), self.ws_bytes, _raw_stream(stream, self.device))
        return list(out)


def orthogonalise(x, steps: int = 5, coef=QUINTIC, eps: float = 1e-7):
    """The orthogonalised matrices of x [rows, cols] or [count, rows, cols], on
    the current stream."""
    shape = tuple(x.shape) if x.dim() == 3 else (1,) + tuple(x.shape)
    call = Orthogonalise([shape], dtype=x.dtype, device=x.device, steps=steps, coef=coef, eps=eps)
    return call([x])[0].reshape(x.shape)


def _pieces(g, out):
    """Runs of (g, out, rows, cols, row strides) that make up a tensor and its
    output (or None): axes that follow one another in memory are one."""
    axes = [[n, s, t] for n, s, t in zip(g.shape, g.stride(), g.stride() if out is None else out.stride()) if n != 1]
    merged = []
    for n, s, t in axes:
        if merged and merged[-1][1] == n * s and merged[-1][2] == n * t:
            merged[-1] = [merged[-1][0] * n, s, t]
        else:
            merged.append([n, s, t])
    if merged and (merged[-1][1] != 1 or merged[-1][2] != 1):
        if len(merged) > 1 and g.shape[-1] != 1:
            raise ValueError("gradients must have unit stride along a row")
        merged.append([1, 1, 1])   # (single elements)
    cols = merged.pop()[0] if merged else 1
    rows, gs, os = merged.pop() if merged else (1, cols, cols)
    starts = [(0, 0)]
    for n, s, t in merged:
        starts = [(a + i * s, b + i * t) for a, b in starts for i in range(n)]
    el = g.element_size()
    return [(_ptr(g) + a * el, None if out is None else _ptr(out) + b * el, rows, cols, gs, os) for a, b in starts]


class Clip:
    """Clips ``grads``, fp32 and bf16 tensors, by their global norm: in place, or
    into the tensors ``out`` (``out=False``: the norm and the scale alone).

    A call returns the norm [1] (fp32); ``scale`` [1] is what the gradients were
    multiplied with.  A norm that is not finite drops them: scale 0, and zeros.
    The tensors stay where they are for the object's life."""

    def __init__(self, grads, max_norm: float, out=None):
        torch = _torch()
        self.grads = list(grads)
        if not self.grads:
            raise ValueError("no gradients")
        self.device = self.grads[0].device
        if self.device.type != "cuda":
            raise ValueError("the operators run on a GPU")
        self.out = self.grads if out is None else [None] * len(self.grads) if out is False else list(out)
        if len(self.out) != len(self.grads):
            raise ValueError("one output per gradient is wanted")
        self.max_norm = float(max_norm)
        arrays = []
        for g, y in zip(self.grads, self.out):
            if g.device != self.device or (y is not None and (y.device != self.device or y.shape != g.shape
                                                              or y.dtype != g.dtype)):
                raise ValueError(f"gradients must be on {self.device}, an output of its gradient's shape and type")
            code = _dtype(g.dtype)
            arrays += [tag_clip_array(*p, code) for p in (_pieces(g, y) if g.numel() else [])]
        n = len(arrays)
        arrays = (tag_clip_array * max(n, 1))(*arrays)
        lib, b = _abi.load(), C.c_size_t(0)
        check(lib.tag_clip_table_bytes(arrays, n, C.byref(b)), "tag_clip_table_bytes")
        self.table = torch.empty(max(b.value, 16), dtype=torch.uint8, device=self.device)
        self._plan = tag_clip_plan()
        _launch(self.device, "tag_clip_prepare", arrays, n, _ptr(self.table), b.value, _raw_stream(None, self.device),
                C.byref(self._plan))
        check(lib.tag_clip_workspace(C.byref(b)), "tag_clip_workspace")
        self.ws_bytes = b.value
        self.ws = torch.empty(b.value, dtype=torch.uint8, device=self.device)
        self.result = torch.zeros(2, dtype=torch.float32, device=self.device)
        self.norm, self.scale = self.result[:1], self.result[1:]
        self._args = (_ptr(self.result), _ptr(self.ws), self.ws_bytes)

    @classmethod
    def of(cls, trainer, max_norm: float, **kw):
        """Every gradient of ``trainer``."""
        return cls(list(trainer.grads.values()), max_norm, **kw)

    def __call__(self, max_norm: Optional[float] = None, stream=None):
        """``max_norm`` in place of the object's, for this call."""
        _launch(self.device, "tag_clip", C.byref(self._plan), self.max_norm if max_norm is None else float(max_norm),
                *self._args, _raw_stream(stream, self.device))
        return self.norm


class Muon:
    """Momentum with orthogonalised updates of ``params``: (weight, gradient)
    pairs of fp32 tensors, updated in place by ``step``.  [rows, cols] and
    [count, rows, cols] are matrices; one-dimensional tensors take plain
    momentum SGD.  ``state`` gives the momentum tensors (default: zeros).  No
    weight or momentum shares memory with another tensor of them.

    With ``max_norm`` a step takes the gradients as ``Clip`` would scale them
    (the tensors themselves stay); ``norm`` [1] is their norm.  Where it is not
    finite, the step leaves weights and momentum as they are."""

    def __init__(self, params, lr: float = 0.02, momentum: float = 0.95, nesterov: bool = True,
                 weight_decay: float = 0.0, steps: int = 5, coef=QUINTIC, eps: float = 1e-7,
                 state: Optional[Sequence] = None, max_norm: Optional[float] = None):
        torch = _torch()
        self.params = [(w, g) for w, g in params]
        if not self.params:
            raise ValueError("no parameters")
        self.device = self.params[0][0].device
        if self.device.type != "cuda":
            raise ValueError("the operators run on a GPU")
        self.m = [torch.zeros_like(w) for w, _ in self.params] if state is None else list(state)
        if len(self.m) != len(self.params):
            raise ValueError("one momentum tensor per parameter is wanted")
        written = [t.data_ptr() for t in self.m] + [w.data_ptr() for w, _ in self.params]
        if len(set(written)) != len(written):
            raise ValueError("a weight or a momentum stands there twice")
        self.options = tag_muon_options(float(lr), float(momentum), float(weight_decay), 1 if nesterov else 0)
        self._ns = _iteration(steps, coef, eps)
        self._g = (tag_muon_group * len(self.params))()
        for q, (w, g), m in zip(self._g, self.params, self.m):
            if w.dim() not in (1, 2, 3) or g.shape != w.shape or m.shape != w.shape:
                raise ValueError("a weight has one to three axes, its gradient and momentum the same shape")
            q.plain = 1 if w.dim() == 1 else 0
            shape = (1,) * (3 - w.dim()) + tuple(int(v) for v in w.shape)
            q.count, q.rows, q.cols = shape
            for a, t, what in ((q.w, w, "a weight"), (q.g, g, "a gradient"), (q.m, m, "a momentum")):
                _set(a, t.reshape(1, -1) if t.dim() == 1 and t.is_contiguous() else t, what, shape, torch.float32,
                     self.device)
        b = C.c_size_t(0)
        check(_abi.load().tag_muon_workspace(self._g, len(self.params), C.byref(b)), "tag_muon_workspace")
        self.ws_bytes = b.value
        self.ws = torch.empty(max(b.value, 16), dtype=torch.uint8, device=self.device)
        self.clip = self.norm = None
        if max_norm is not None:
            self.clip = Clip([g for _, g in self.params], max_norm, out=False)
            self.norm = self.clip.norm

    @classmethod
    def of(cls, trainer, **kw):
        """The parameters of ``trainer.model`` with ``trainer.grads``: the
        encoders', the layers' ([W^h | W^e] of each link type) and the decoder's
        weight matrices, everything else as vectors."""
        d, t, g = trainer.model.dims, trainer.model.t, trainer.grads
        shapes = dict(enc_op_w=(d.f, d.f_op), enc_dev_w=(d.f, d.f_dev), layer_w=(3 * d.layers, d.f, 2 * d.f),
                      dec_w1=(d.dec_hidden, 2 * d.f + 4))
        return cls([(t[k].view(shapes[k]), g[k].view(shapes[k])) if k in shapes else (t[k], g[k]) for k in g], **kw)

    def step(self, lr: Optional[float] = None, stream=None) -> None:
        """One step with the gradients as they stand.  ``lr`` holds for this
        step and the following ones; a step captured into a graph keeps the one
        that it was captured with."""
        was = self.options.lr
        if lr is not None:
            self.options.lr = float(lr)
        try:
            name, clip = "tag_muon_step", ()
            if self.clip is not None:
                self.clip(stream=stream)
                name, clip = "tag_muon_step_clipped", (_ptr(self.clip.result),)
            _launch(self.device, name, self._g, len(self.params), C.byref(self._ns), C.byref(self.options), *clip,
                    _ptr(self.ws), self.ws_bytes, _raw_stream(stream, self.device))
        except TagError:   # (a rate that was refused is not kept)
            self.options.lr = was
            raise
