"""Python face of the operators at both ends of a decoder step (include/ssd.h): norms and rotary positions of query
and key heads, and sampling from the vocabulary head's logits.

No computation happens here: calls go to the library on their tensors' device and its current stream, run
asynchronously, keep nothing between calls and may be captured into a CUDA graph after a first call outside of it.
"""
from __future__ import annotations

import ctypes
from typing import Sequence

import torch

from . import _binding as B
from .lowbit import _call, _fail, _rows2, _rows3, _type


class Rotary:
    """Rotary positions of heads of `head_dim` elements (ssd_rotary): the first `rotary_dim` turn, in pairs
    (i, i + rotary_dim / 2) or, interleaved, (2 i, 2 i + 1), by theta^(-2 i / rotary_dim) radians a position.

    sections: pairs that turn with each axis, in order (images and video: time, height, width); one axis by default.
    axes: instead, the axis of every pair.  freqs: radians a position of every pair, in place of theta's."""

    def __init__(self, head_dim: int, rotary_dim: int | None = None, theta: float = 10000.0,
                 sections: Sequence[int] | None = None, interleaved: bool = False, eps: float = 1e-5,
                 axes: Sequence[int] | None = None, freqs: Sequence[float] | None = None):
        self.lib = B.load()
        turn = head_dim if rotary_dim is None else rotary_dim
        if sections is not None and axes is not None:
            _fail("sections or axes expected, not both")
        n = 1 if sections is None else len(sections)
        section = None if sections is None else (ctypes.c_int * n)(*sections)
        self._c = B.SSDRotary()
        if self.lib.ssd_rotary_init(ctypes.byref(self._c), head_dim, turn, int(interleaved), n, section, theta, eps):
            _fail(self.lib.ssd_op_last_error().decode())
        for what, values in (("axes", axes), ("freqs", freqs)):
            if values is not None and len(values) != turn // 2:
                _fail(f"{what}: one for each of {turn // 2} pairs expected, got {len(values)}")
        if axes is not None:
            n = max(axes, default=0) + 1
            if min(axes, default=0) < 0 or n > B.SSD_ROTARY_MAX_AXES:
                _fail(f"axes: 0 to {B.SSD_ROTARY_MAX_AXES - 1} expected, got {list(axes)}")
            self._c.axes = n
            for i, a in enumerate(axes):
                self._c.axis[i] = a
        if freqs is not None:
            for i, f in enumerate(freqs):
                turns = float(f) / (2 * 3.141592653589793)
                if not abs(turns) < 1 << 31:
                    _fail(f"freqs: a finite number of radians expected, got {f}")
                self._c.step[i] = int((turns % 1.0) * 2.0 ** 64) % (1 << 64)
        self.head_dim, self.axes = head_dim, n
        self._ref = ctypes.byref(self._c)

    def rotate(self, q: torch.Tensor, k: torch.Tensor | None, pos: torch.Tensor, q_gain: torch.Tensor | None = None,
               k_gain: torch.Tensor | None = None, q_out: torch.Tensor | None = None,
               k_out: torch.Tensor | None = None):
        """ssd_rotary_apply: the heads of q [rows][heads][head_dim] and k [rows][kv heads][head_dim] (or None),
        normed where a gain [head_dim] is given, turned by pos int32 [rows] or [rows][axes].  Returns (q_out, k_out),
        which may be q and k themselves."""
        i, rows, d = q.get_device(), q.shape[0], self.head_dim
        if not q.is_cuda:
            _fail(f"q: a CUDA tensor expected, got {q.device}")
        if pos.dtype is not torch.int32 or pos.get_device() != i or pos.shape != ((rows, self.axes) if pos.dim() != 1 else (rows,)) \
                or (pos.dim() == 1 and self.axes != 1):
            _fail(f"pos: int32 [{rows}][{self.axes}] on {q.device} expected, got {pos.dtype} {tuple(pos.shape)} on {pos.device}")
        code, dtype = _type(q.dtype, "q"), q.dtype
        both = (B.SSDHeads * 2)()
        outs = []
        for h, x, y, gain, what in ((both[0], q, q_out, q_gain, "q"), (both[1], k, k_out, k_gain, "k")):
            if x is None:
                if y is not None or gain is not None:
                    _fail(f"{what}: missing")
                outs.append(None)
                continue
            if x.dim() != 3:
                _fail(f"{what}: [rows][heads][{d}] expected, got {tuple(x.shape)}")
            shape = (rows, x.shape[1], d)
            xs = _rows3(x, shape, i, what)
            if y is None:
                y = torch.empty(shape, dtype=dtype, device=x.device)
            ys = _rows3(y, shape, i, what + "_out")
            if x.dtype is not dtype or y.dtype is not dtype:
                _fail(f"{what} and its output: {dtype} expected, got {x.dtype} and {y.dtype}")
            h.x, h.y, h.heads, h.x_row, h.x_head, h.y_row, h.y_head = x.data_ptr(), y.data_ptr(), shape[1], xs[0], xs[1], ys[0], ys[1]
            if gain is not None:
                if gain.shape != (d,) or gain.get_device() != i or not gain.is_contiguous():
                    _fail(f"{what}_gain: contiguous [{d}] on {q.device} expected, got {tuple(gain.shape)} on {gain.device}")
                h.gain, h.gain_type = gain.data_ptr(), _type(gain.dtype, what + "_gain")
            outs.append(y)
        st = pos.stride()
        _call(i, self.lib.ssd_rotary_apply, self._ref, both, 1 if k is None else 2, code, rows, pos.data_ptr(), st[0],
              st[1] if len(st) > 1 else 0)
        return tuple(outs)


def sample(logits: torch.Tensor, u: torch.Tensor, temperature: float | torch.Tensor = 1.0,
           top_k: int | torch.Tensor = 0, top_p: float | torch.Tensor = 1.0, min_p: float | torch.Tensor = 0.0,
           out: torch.Tensor | None = None, with_prob: bool = False):
    """ssd_sample: one token per row of logits [rows][vocab] (bfloat16 or float32) from the random numbers u
    (float32 [rows], in [0, 1)).  Each setting is a number for all rows or a tensor [rows] (top_k int32, the others
    float32).  Returns int32 [rows]; with_prob: also the tokens' probabilities among the kept ones, float32 [rows]."""
    lib = B.load()
    if logits.dim() != 2 or not logits.is_cuda:
        _fail(f"logits: [rows][vocab] on a GPU expected, got {tuple(logits.shape)} on {logits.device}")
    rows, vocab = logits.shape
    i = logits.get_device()
    stride, code = _rows2(logits, (rows, vocab), i, "logits"), _type(logits.dtype, "logits")

    def per_row(t: torch.Tensor, dtype: torch.dtype, what: str) -> int:
        if t.dtype is not dtype or t.shape != (rows,) or t.get_device() != i or not t.is_contiguous():
            _fail(f"{what}: contiguous {dtype} [{rows}] on {logits.device} expected, got {t.dtype} {tuple(t.shape)} on {t.device}")
        return t.data_ptr()

    how = B.SSDSampling()
    for name, value, dtype in (("temperature", temperature, torch.float32), ("top_p", top_p, torch.float32),
                               ("min_p", min_p, torch.float32), ("top_k", top_k, torch.int32)):
        if torch.is_tensor(value):
            setattr(how, name + "_rows", per_row(value, dtype, name))
        else:
            setattr(how, name, value)
    if out is None:
        out = torch.empty(rows, dtype=torch.int32, device=logits.device)
    prob = torch.empty(rows, dtype=torch.float32, device=logits.device) if with_prob else None
    _call(i, lib.ssd_sample, logits.data_ptr(), code, rows, vocab, stride, per_row(u, torch.float32, "u"), ctypes.byref(how),
          per_row(out, torch.int32, "out"), None if prob is None else prob.data_ptr())
    return (out, prob) if with_prob else out
