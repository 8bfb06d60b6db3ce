"""Binding of include/tag_policy.h and include/tag_beam.h: operators on the
decision head's scores (``Decide.scores``).

  Constrain  priors, argmax and best score under slice masks, biases and
             penalties for slices that a query's history took already
  Balance    the loss that spreads the decisions over the devices, with the
             slices' counts, the devices' loads and the scores' gradient
  Beam       one level of a beam search: the best continuations of all beams'
             slices, their parents and slices
  Reorder    the beams' states, brought into the order of their parents

Argument checks and marshalling only; the operators run in libtag.so's HIP
kernels.  As with the other reusable calls, an object owns its workspace and
its outputs: calls of one object must be ordered (one stream, or one after the
other), and each overwrites the outputs of the last.  They are memory of the
stream that is current when the object is made: another stream that a call is
given has to wait for it first.
"""
from __future__ import annotations

import numpy as np

from . import _abi, _ptr, _torch
from ._abi import C, TAG_BF16, TAG_F32, check, tag_beam_state, tag_constraints

__all__ = ["Constrain", "Balance", "Beam", "Reorder"]


def _device(device):
    torch = _torch()
    d = torch.device(device)
    if d.type != "cuda":
        raise ValueError("the operators run on a GPU")
    return torch.device("cuda", torch.cuda.current_device()) if d.index is None else d


def _launch(device, name: str, *args) -> None:
    """Calls the library's `name` with `device` as the current one."""
    torch = _torch()
    f = getattr(_abi.load(), name)
    if torch._C._cuda_getDevice() == device.index:
        st = f(*args)
    else:
        with torch.cuda.device(device):
            st = f(*args)
    if st != _abi.TAG_OK:
        check(st, name)


def _raw_stream(stream, device) -> int:
    """The given stream's handle, or that of `device`'s current one."""
    return int(stream.cuda_stream) if stream is not None else _torch()._C._cuda_getCurrentRawStream(device.index)


def _dtype(dtype) -> int:
    torch = _torch()
    if dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("dtype must be torch.float32 or torch.bfloat16")
    return TAG_F32 if dtype == torch.float32 else TAG_BF16


def _rows(t, what, dtypes, device, n_rows, n_cols, shared=False):
    """Row stride of t, [n_rows, n_cols] with unit column stride; with `shared`
    also [n_cols] or [1, n_cols] for every row (stride 0)."""
    shape = t.shape
    if t.dtype not in dtypes or t.device != device:
        raise ValueError(f"{what} must be {' or '.join(str(d) for d in dtypes)} on {device}")
    one = shared and (len(shape) == 1 or (len(shape) == 2 and shape[0] == 1))
    if len(shape) not in ((1, 2) if shared else (2,)) or shape[-1] != n_cols or not (one or shape[0] == n_rows):
        raise ValueError(f"{what} must have the shape [{n_rows}, {n_cols}]" + (" or one row" if shared else "")
                         + f", not {list(shape)}")
    stride = t.stride()
    if n_cols > 1 and stride[-1] != 1:
        raise ValueError(f"{what} must have unit stride along a row")
    if one:
        return 0
    # (the stride of a single row means nothing)
    return stride[0] if n_rows > 1 else max(stride[0], n_cols)


def _vector(t, what, dtype, device, n):
    if t.dtype != dtype or t.device != device or t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{what} must be {dtype} [{n}] on {device}, contiguous")
    return t.data_ptr()


class Constrain:
    """Constrained priors of ``n_query`` rows of ``n_slices`` scores.

    A call returns (prior [Q, S] fp32, argmax [Q] int32, best [Q] fp32), with
    ``want_scores`` followed by the constrained scores [Q, S]; a part that is
    not wanted (``want_prior=False``) is None."""

    def __init__(self, n_query: int, n_slices: int, dtype=None, device="cuda", want_prior: bool = True,
                 want_scores: bool = False):
        torch = _torch()
        self.dtype = torch.float32 if dtype is None else dtype
        self._code = _dtype(self.dtype)
        self.device = dev = _device(device)
        self.Q, self.S = int(n_query), int(n_slices)
        b = C.c_size_t(0)
        check(_abi.load().tag_constrain_workspace(self.Q, self.S, C.byref(b)), "tag_constrain_workspace")
        self.ws_bytes = b.value
        self.ws = torch.empty(max(b.value, 16), dtype=torch.uint8, device=dev)
        self.prior = torch.empty((self.Q, self.S), dtype=torch.float32, device=dev) if want_prior else None
        self.scores = torch.empty((self.Q, self.S), dtype=self.dtype, device=dev) if want_scores else None
        self.argmax = torch.empty(self.Q, dtype=torch.int32, device=dev)
        self.best = torch.empty(self.Q, dtype=torch.float32, device=dev)
        self._c = tag_constraints()
        self._byref = C.byref(self._c)
        self._tail = (_ptr(self.scores), self.S, _ptr(self.prior), self.S, _ptr(self.argmax), _ptr(self.best),
                      _ptr(self.ws), self.ws_bytes)
        self._out = (self.prior, self.argmax, self.best) + (() if self.scores is None else (self.scores,))

    def __call__(self, scores, allow=None, bias=None, history=None, history_len=None, repetition=None, presence=None,
                 frequency=None, stream=None):
        """scores [Q, S]; allow [Q, (S + 31) // 32] words of bits (int32 or
        uint32), bias [Q, S] and history [Q, T] (int32) may be one row for every
        query; history_len (int32), repetition, presence, frequency [Q]."""
        torch = _torch()
        Q, S, dev, c = self.Q, self.S, self.device, self._c
        f32 = torch.float32
        xs = _rows(scores, "scores", (self.dtype,), dev, Q, S)
        c.allow = c.bias = c.history = c.history_len = c.repetition = c.presence = c.frequency = None
        c.n_history = 0
        if allow is not None:
            c.allow_stride = _rows(allow, "allow", (torch.int32, torch.uint32), dev, Q, (S + 31) // 32, True)
            c.allow = allow.data_ptr()
        if bias is not None:
            c.bias_stride = _rows(bias, "bias", (f32,), dev, Q, S, True)
            c.bias = bias.data_ptr()
        if history is not None:
            T = int(history.shape[-1]) if history.dim() else 0
            c.history_stride = _rows(history, "history", (torch.int32,), dev, Q, T, True)
            if T > 0:
                c.history, c.n_history = history.data_ptr(), T
            if history_len is not None:
                c.history_len = _vector(history_len, "history_len", torch.int32, dev, Q)
        elif history_len is not None or repetition is not None or presence is not None or frequency is not None:
            raise ValueError("history_len and penalties need a history")
        if repetition is not None:
            c.repetition = _vector(repetition, "repetition", f32, dev, Q)
        if presence is not None:
            c.presence = _vector(presence, "presence", f32, dev, Q)
        if frequency is not None:
            c.frequency = _vector(frequency, "frequency", f32, dev, Q)
        _launch(dev, "tag_constrain", Q, S, self._code, scores.data_ptr(), xs, self._byref, *self._tail,
                _raw_stream(stream, dev))
        return self._out


class Balance:
    """Balance loss over ``n_query`` rows of scores for a slice table.

    A call returns the loss [1]; ``grad`` [Q, S] (the scores' type), ``count``
    [S] (int32) and ``load`` [n_dev] hold the rest of its results."""

    def __init__(self, masks, n_dev: int, n_query: int, dtype=None, device="cuda"):
        torch = _torch()
        self.dtype = torch.float32 if dtype is None else dtype
        self._code = _dtype(self.dtype)
        self.device = dev = _device(device)
        self.masks = torch.from_numpy(np.ascontiguousarray(masks, np.uint64).view(np.int64)).to(dev)
        self.Q, self.S, self.M = int(n_query), len(masks), int(n_dev)
        b = C.c_size_t(0)
        check(_abi.load().tag_balance_workspace(self.Q, self.S, C.byref(b)), "tag_balance_workspace")
        self.ws_bytes = b.value
        self.ws = torch.empty(b.value, dtype=torch.uint8, device=dev)
        self.grad = torch.empty((self.Q, self.S), dtype=self.dtype, device=dev)
        self.loss = torch.empty(1, dtype=torch.float32, device=dev)
        self.count = torch.empty(self.S, dtype=torch.int32, device=dev)
        self.load = torch.empty(self.M, dtype=torch.float32, device=dev)
        self._tail = (_ptr(self.grad), self.S, 0, _ptr(self.loss), _ptr(self.count), _ptr(self.load), _ptr(self.ws),
                      self.ws_bytes)

    def __call__(self, scores, coef: float = 1e-2, use=None, stream=None):
        """scores [Q, S]; use [Q] (uint8 or bool): 0 leaves a row out."""
        torch = _torch()
        xs = _rows(scores, "scores", (self.dtype,), self.device, self.Q, self.S)
        u = None
        if use is not None:
            u = _vector(use, "use", torch.bool if use.dtype == torch.bool else torch.uint8, self.device, self.Q)
        _launch(self.device, "tag_balance", self.Q, self.S, self._code, scores.data_ptr(), xs, _ptr(self.masks), self.M,
                u, float(coef), *self._tail, _raw_stream(stream, self.device))
        return self.loss


def _beams(t, what, dtypes, device, n, width):
    if t.dtype not in dtypes or t.device != device or tuple(t.shape) != (n, width) or not t.is_contiguous():
        raise ValueError(f"{what} must be {' or '.join(str(d) for d in dtypes)} [{n}, {width}] on {device}, contiguous")
    return t.data_ptr()


class Beam:
    """One level of ``n_search`` beam searches: ``width`` beams after it,
    ``width_in`` before it (default: as many).

    A call returns (total [n, width] fp32, parent, slice [n, width] int32), best
    first.  ``total`` may go into the next level's call as it is.  A finished
    beam goes on with slice -1; what is left over of the width has parent -1."""

    def __init__(self, n_search: int, width: int, n_slices: int, width_in=None, dtype=None, device="cuda"):
        torch = _torch()
        self.dtype = torch.float32 if dtype is None else dtype
        self._code = _dtype(self.dtype)
        self.device = dev = _device(device)
        self.n, self.W, self.S = int(n_search), int(width), int(n_slices)
        self.V = self.W if width_in is None else int(width_in)
        b = C.c_size_t(0)
        check(_abi.load().tag_beam_workspace(self.n, self.V, self.W, self.S, C.byref(b)), "tag_beam_workspace")
        self.ws_bytes = b.value
        self.ws = torch.empty(max(b.value, 16), dtype=torch.uint8, device=dev)
        self.total = torch.empty((self.n, self.W), dtype=torch.float32, device=dev)
        self.parent = torch.empty((self.n, self.W), dtype=torch.int32, device=dev)
        self.slice = torch.empty((self.n, self.W), dtype=torch.int32, device=dev)
        self._out = (self.total, self.parent, self.slice)
        self._tail = tuple(_ptr(t) for t in self._out) + (_ptr(self.ws), self.ws_bytes)

    def start(self):
        """This object's ``total`` [n, width], set to what a search starts from:
        one beam of probability one, the others not there."""
        self.total.fill_(-float("inf"))
        self.total[:, :1].zero_()
        return self.total

    def __call__(self, scores, total, done=None, stream=None):
        """scores [n width_in, S], a search's beams one after the other; total
        [n, width_in]; done [n, width_in] (uint8 or bool): finished beams."""
        torch = _torch()
        n, V, dev = self.n, self.V, self.device
        xs = _rows(scores, "scores", (self.dtype,), dev, n * V, self.S)
        t = _beams(total, "total", (torch.float32,), dev, n, V)
        d = None if done is None else _beams(done, "done", (torch.uint8, torch.bool), dev, n, V)
        _launch(dev, "tag_beam_select", n, V, self.W, self.S, self._code, scores.data_ptr(), xs, t, d, *self._tail,
                _raw_stream(stream, dev))
        return self._out


class Reorder:
    """Brings the beams' ``states`` into the order of their parents: tensors of
    any type whose first axis, or first two, are the beams, [n width_in, ...] or
    [n, width_in, ...], each beam's part contiguous.  ``out`` gives tensors
    [n width, ...] or [n, width, ...] to write; without it they are reordered in
    place.  A call takes ``parent`` [n, width] (int32); beams whose parent is not
    in [0, width_in) keep what they have."""

    def __init__(self, states, n_search: int, width: int, width_in=None, out=None):
        self.n, self.W = int(n_search), int(width)
        self.V = self.W if width_in is None else int(width_in)
        self.states = list(states)
        self.out = self.states if out is None else list(out)
        if not self.states or len(self.out) != len(self.states):
            raise ValueError("states are wanted, and as many outputs")
        if out is None and self.V != self.W:
            raise ValueError("states of another width cannot be reordered in place")
        self.device = self.states[0].device
        if self.device.type != "cuda":
            raise ValueError("the operators run on a GPU")
        self._s = (tag_beam_state * len(self.states))()
        for s, x, y in zip(self._s, self.states, self.out):
            row, s_in, b_in = self._layout(x, self.V)
            row_out, s.out_search, s.out_beam = self._layout(y, self.W)
            if x.dtype != y.dtype or row != row_out:
                raise ValueError("an output has the type of its states, and rows of their size")
            setattr(s, "in", x.data_ptr())
            s.out, s.row_bytes, s.in_search, s.in_beam = y.data_ptr(), row, s_in, b_in

    def _layout(self, t, width):
        """Bytes of a row, strides of searches and of beams."""
        if t.device != self.device:
            raise ValueError(f"states must be on {self.device}")
        shape, stride, el = tuple(t.shape), t.stride(), t.element_size()
        if len(shape) >= 1 and shape[0] == self.n * width:
            lead, search, beam = 1, width * stride[0], stride[0]
        elif len(shape) >= 2 and shape[:2] == (self.n, width):
            lead, (search, beam) = 2, stride[:2]
        else:
            raise ValueError(f"states must have the shape [{self.n * width}, ...] or [{self.n}, {width}, ...], not "
                             f"{list(shape)}")
        if t.numel() == 0:
            return 0, 0, 0
        row = 1
        for size, step in zip(shape[:lead - 1:-1], stride[:lead - 1:-1]):
            if size != 1 and step != row:
                raise ValueError("each beam's part of the states must be contiguous")
            row *= size
        return row * el, search * el, beam * el

    def __call__(self, parent, stream=None):
        p = _beams(parent, "parent", (_torch().int32,), self.device, self.n, self.W)
        _launch(self.device, "tag_beam_reorder", self.n, self.V, self.W, p, self._s, len(self.states),
                _raw_stream(stream, self.device))
        return self.out
