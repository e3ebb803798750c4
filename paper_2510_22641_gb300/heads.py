"""Python face of the operators at both ends of a decoder step (include/ssd.h): norms and rotary positions of query
and key heads, and sampling from the vocabulary head's logits.

No computation happens here: calls go to the library on their tensors' device and its current stream, run
asynchronously, keep nothing between calls and may be captured into a CUDA graph after a first call outside of it.
"""
from __future__ import annotations

import ctypes
import struct
from typing import Sequence

import torch

from . import _binding as B
from .lowbit import _INT, _call, _fail, _ints, _rows2, _rows3, _type


# Fields of ssd_heads and ssd_sampling as bytes: filling a ctypes structure takes longer than the call it is for.
_HEADS = "PPi4xqqqqPi4x"
_one, _two, _sampling = (struct.Struct(f).pack for f in (_HEADS, 2 * _HEADS, "fffiPPPP"))


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
        _ints(head_dim=head_dim, rotary_dim=turn, **{f"sections[{a}]": v for a, v in enumerate(sections or ())})
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
        i, d, code = q.get_device(), self.head_dim, _type(q.dtype, "q")
        rows = q.shape[0] if q.dim() else 0
        if i < 0:
            _fail(f"q: a CUDA tensor expected, got {q.device}")
        if rows > _INT:
            _fail(f"q: {rows} rows")
        ps, pst = pos.shape, pos.stride()
        if pos.dtype is not torch.int32 or pos.get_device() != i or \
                (ps != (rows, self.axes) and (self.axes != 1 or ps != (rows,))):
            _fail(f"pos: int32 [{rows}][{self.axes}] on {q.device} expected, got {pos.dtype} {tuple(ps)} on {pos.device}")
        q_out, first = self._operand(q, q_out, q_gain, rows, i, q.dtype, "q")
        if k is None:
            if k_out is not None or k_gain is not None:
                _fail("k: missing")
            both = _one(*first)
        else:
            k_out, second = self._operand(k, k_out, k_gain, rows, i, q.dtype, "k")
            both = _two(*first, *second)
        _call(i, self.lib.ssd_rotary_apply, self._ref, both, 1 if k is None else 2, code, rows, pos.data_ptr(), pst[0],
              pst[1] if len(pst) > 1 else 0)
        return q_out, k_out

    def _operand(self, x, y, gain, rows: int, index: int, dtype: torch.dtype, what: str) -> tuple:
        """The output and the fields of an ssd_heads."""
        d, shape = self.head_dim, x.shape
        if len(shape) != 3 or x.dtype is not dtype:
            _fail(f"{what}: {dtype} [rows][heads][{d}] expected, got {x.dtype} {tuple(shape)}")
        heads = shape[1]
        if heads > _INT:
            _fail(f"{what}: {heads} heads")
        xs = _rows3(x, (rows, heads, d), index, what)
        if y is None:
            y = torch.empty(shape, dtype=dtype, device=x.device)
            y_row, y_head = heads * d, d
        else:
            y_row, y_head, _ = _rows3(y, (rows, heads, d), index, what + "_out")
            if y.dtype is not dtype:
                _fail(f"{what}_out: {dtype} expected, got {y.dtype}")
        g = g_type = 0
        if gain is not None:
            if gain.shape != (d,) or gain.get_device() != index or not gain.is_contiguous():
                _fail(f"{what}_gain: contiguous [{d}] on {x.device} expected, got {tuple(gain.shape)} on {gain.device}")
            g, g_type = gain.data_ptr(), _type(gain.dtype, what + "_gain")
        return y, (x.data_ptr(), y.data_ptr(), heads, xs[0], xs[1], y_row, y_head, g, g_type)


def sample(logits: torch.Tensor, u: torch.Tensor, temperature: float | torch.Tensor = 1.0,
           top_k: int | torch.Tensor = 0, top_p: float | torch.Tensor = 1.0, min_p: float | torch.Tensor = 0.0,
           out: torch.Tensor | None = None, with_prob: bool = False):
    """ssd_sample: one token per row of logits [rows][vocab] (bfloat16 or float32) from the random numbers u
    (float32 [rows], in [0, 1)).  Each setting is a number for all rows or a tensor [rows] (top_k int32, the others
    float32).  Returns int32 [rows]; with_prob: also the tokens' probabilities among the kept ones, float32 [rows]."""
    lib, i = B.load(), logits.get_device()
    if i < 0 or logits.dim() != 2:
        _fail(f"logits: [rows][vocab] on a GPU expected, got {tuple(logits.shape)} on {logits.device}")
    rows, vocab = logits.shape
    if rows > _INT or vocab > _INT:
        _fail(f"logits: {rows} rows of {vocab}")
    one, device = (rows,), logits.device

    def per_row(t: torch.Tensor, dtype: torch.dtype, what: str) -> int:
        if t.dtype is not dtype or t.shape != one or t.get_device() != i or not t.is_contiguous():
            _fail(f"{what}: contiguous {dtype} [{rows}] on {device} expected, got {t.dtype} {tuple(t.shape)} on {t.device}")
        return t.data_ptr()

    tensor, f32, i32 = torch.Tensor, torch.float32, torch.int32
    t_rows = p_rows = m_rows = k_rows = 0
    if isinstance(temperature, tensor):
        temperature, t_rows = 0.0, per_row(temperature, f32, "temperature")
    if isinstance(top_p, tensor):
        top_p, p_rows = 0.0, per_row(top_p, f32, "top_p")
    if isinstance(min_p, tensor):
        min_p, m_rows = 0.0, per_row(min_p, f32, "min_p")
    if isinstance(top_k, tensor):
        top_k, k_rows = 0, per_row(top_k, i32, "top_k")
    try:
        how = _sampling(temperature, top_p, min_p, top_k, t_rows, p_rows, m_rows, k_rows)
    except (struct.error, OverflowError):
        _fail(f"temperature, top_p and min_p: fp32 numbers expected, top_k: a 32-bit integer, got {temperature}, {top_p}, {min_p}, "
              f"{top_k}")
    if out is None:
        out = torch.empty(one, dtype=i32, device=device)
    prob = torch.empty(one, dtype=f32, device=device) if with_prob else None
    _call(i, lib.ssd_sample, logits.data_ptr(), _type(logits.dtype, "logits"), rows, vocab,
          _rows2(logits, (rows, vocab), i, "logits"), per_row(u, f32, "u"), how, per_row(out, i32, "out"),
          None if prob is None else prob.data_ptr())
    return (out, prob) if with_prob else out
