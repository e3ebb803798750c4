"""Python face of the low-bit operators (include/ssd.h): a paged 8-bit K/V cache and 4-bit weights.

The classes own torch buffers and forward every call to the library on the current CUDA stream.  No
computation happens here.  Calls of one KV8Cache share its workspace, so calls from several streams
must be ordered by the caller.  Everything but KV8Cache.check runs asynchronously and may be captured
into a CUDA graph after a first call outside of it.
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import _binding as B

_TYPES = {torch.bfloat16: B.SSD_TYPE_BF16, torch.float32: B.SSD_TYPE_FP32}


def _fail(msg: str):
    raise B.SSDError(1, msg)


def _call(fn, *args) -> None:
    status = fn(*args)
    if status != 0:
        raise B.SSDError(status, B.load().ssd_op_last_error().decode())


def _stream(device) -> int:
    return torch._C._cuda_getCurrentRawStream(device.index)


def _type(t: torch.Tensor, what: str) -> int:
    code = _TYPES.get(t.dtype)
    if code is None:
        _fail(f"{what}: bfloat16 or float32 expected, got {t.dtype}")
    return code


def _rows3(t: torch.Tensor, shape: tuple, what: str) -> None:
    """[rows][heads][dim] with any row and head strides and contiguous elements."""
    if t.shape != shape:
        _fail(f"{what}: shape {shape} expected, got {tuple(t.shape)}")
    if t.stride(2) != 1 and t.numel():
        _fail(f"{what}: the last dimension must be contiguous")


def _int32(t: torch.Tensor, n: int, what: str) -> None:
    if t.dtype is not torch.int32 or t.shape != (n,) or not t.is_contiguous() or not t.is_cuda:
        _fail(f"{what}: a contiguous int32 CUDA tensor of {n} expected, got {t.dtype} {tuple(t.shape)} on {t.device}")


class KV8Step:
    """One step's plan: which request each new row belongs to and where its K/V goes (see ssd_kv8_step).

    row_start [batch + 1], slot [rows] and length [batch] are views of the device buffer that
    KV8Cache.plan fills."""

    def __init__(self, cache: KV8Cache, batch: int, rows: int, rows_per_request: int | None = None):
        n = B.load().ssd_kv8_step_ints(batch, rows)
        if n < 0 or batch > cache.max_batch:
            _fail(f"step of {rows} rows of {batch} requests (the cache has {cache.max_batch} seats)")
        self.batch, self.rows = batch, rows
        self.data = torch.zeros(n, dtype=torch.int32, device=cache.device)
        tile = 0
        if rows_per_request is not None:
            heads = rows_per_request * (cache.n_heads // cache.n_kv_heads)
            items = -(-heads // 32)
            tile = (-(-heads // items) + 7) // 8 * 8
        at = B.SSD_KV8_STEP_HEAD + batch + 1
        self.row_start = self.data[at:at + batch + 1]
        self.length = self.data[at + batch + 1:at + 2 * batch + 1]
        self.slot = self.data[at + 2 * batch + 1:]
        self._c = B.SSDKv8Step(batch=batch, rows=rows, row_tile=tile, data=self.data.data_ptr())
        self._ref = ctypes.byref(self._c)


class KV8Cache:
    """A paged K/V cache in 8 bits with one scale per block of tokens, kv head and K / V (ssd_kv8).

    Every decode step: plan() once (block tables and slot maps from the requests' lengths), then per
    layer append() the new K/V rows and run attention().  Lengths stay on the device; rolling rejected
    drafts back is a smaller length in the next plan().

    table [max_batch][max_blocks], pool [n_blocks] (the stack of free blocks) and state
    [1 + max_batch] (free blocks, blocks held per seat) are int32 device tensors."""

    def __init__(self, n_layers: int, n_heads: int, n_kv_heads: int, head_dim: int, block_tokens: int, n_blocks: int,
                 max_batch: int, max_blocks: int, device: torch.device | str = "cuda"):
        self.lib = B.load()
        self.n_layers, self.n_heads, self.n_kv_heads, self.head_dim = n_layers, n_heads, n_kv_heads, head_dim
        self.block_tokens, self.n_blocks, self.max_batch, self.max_blocks = block_tokens, n_blocks, max_batch, max_blocks
        self._c = B.SSDKv8(n_layers=n_layers, n_heads=n_heads, n_kv_heads=n_kv_heads, head_dim=head_dim,
                           block_tokens=block_tokens, n_blocks=n_blocks, max_batch=max_batch, max_blocks=max_blocks)
        self._ref = ctypes.byref(self._c)
        size, work = self.lib.ssd_kv8_data_bytes(self._ref), self.lib.ssd_kv8_work_bytes(self._ref)
        if size < 0 or work < 0:
            _fail(f"KV8Cache: unsupported shape ({n_layers=}, {n_heads=}, {n_kv_heads=}, {head_dim=}, {block_tokens=}, "
                  f"{n_blocks=}, {max_batch=}, {max_blocks=})")
        device = torch.device(device)
        if device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        self.device = device
        self.data = torch.full((size,), 128, dtype=torch.uint8, device=device)   # code 0 everywhere
        self.scales = torch.zeros((n_layers, n_blocks, n_kv_heads, 2), dtype=torch.float32, device=device)
        self.table = torch.full((max_batch, max_blocks), -1, dtype=torch.int32, device=device)
        self.pool = torch.arange(n_blocks - 1, -1, -1, dtype=torch.int32, device=device)
        self.state = torch.zeros(1 + max_batch, dtype=torch.int32, device=device)
        self.state[0] = n_blocks
        self.work = torch.zeros(work, dtype=torch.uint8, device=device)
        c = self._c
        c.data, c.scales, c.table = self.data.data_ptr(), self.scales.data_ptr(), self.table.data_ptr()
        c.pool, c.work = self.pool.data_ptr(), self.work.data_ptr()

    def new_step(self, batch: int, rows: int, rows_per_request: int | None = None) -> KV8Step:
        """A plan's buffer for `rows` new rows of `batch` requests.  rows_per_request: the usual number, if
        it is not rows / batch (only the attention's speed depends on it)."""
        return KV8Step(self, batch, rows, rows_per_request)

    def plan(self, step: KV8Step, length: torch.Tensor, add: torch.Tensor, state: torch.Tensor | None = None,
             state_out: torch.Tensor | None = None) -> KV8Step:
        """ssd_kv8_plan: hand out blocks for add[b] new rows after length[b] cached ones (-1: give the
        seat's blocks back) and fill `step`.  Updates self.state in place unless told otherwise."""
        _int32(length, step.batch, "length")
        _int32(add, step.batch, "add")
        state = self.state if state is None else state
        state_out = state if state_out is None else state_out
        _int32(state, 1 + self.max_batch, "state")
        _int32(state_out, 1 + self.max_batch, "state_out")
        _call(self.lib.ssd_kv8_plan, self._ref, step._ref, length.data_ptr(), add.data_ptr(), state.data_ptr(),
              state_out.data_ptr(), _stream(self.device))
        return step

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, step: KV8Step) -> None:
        """ssd_kv8_append: quantise the step's new rows k, v [rows][n_kv_heads][head_dim] into the cache."""
        shape = (step.rows, self.n_kv_heads, self.head_dim)
        _rows3(k, shape, "k")
        _rows3(v, shape, "v")
        if k.dtype is not v.dtype or k.device != self.device or v.device != self.device:
            _fail(f"k and v: one type on {self.device} expected, got {k.dtype} on {k.device}, {v.dtype} on {v.device}")
        ks, vs = k.stride(), v.stride()
        _call(self.lib.ssd_kv8_append, self._ref, layer, k.data_ptr(), v.data_ptr(), _type(k, "k"), step.rows, ks[0],
              ks[1], vs[0], vs[1], step.slot.data_ptr(), _stream(self.device))

    def read(self, layer: int, slots: torch.Tensor, dtype: torch.dtype = torch.float32):
        """ssd_kv8_read: the (k, v) values held at int32 `slots`, each [n][n_kv_heads][head_dim]."""
        _int32(slots, slots.shape[0], "slots")
        out = torch.empty((2, slots.shape[0], self.n_kv_heads, self.head_dim), dtype=dtype, device=self.device)
        _call(self.lib.ssd_kv8_read, self._ref, layer, slots.data_ptr(), slots.shape[0], out[0].data_ptr(),
              out[1].data_ptr(), _type(out, "dtype"), _stream(self.device))
        return out[0], out[1]

    def attention(self, layer: int, q: torch.Tensor, step: KV8Step, out: torch.Tensor | None = None,
                  scale: float | None = None, row_mask: torch.Tensor | None = None) -> torch.Tensor:
        """ssd_kv8_attention: softmax(scale q k^T) v of the step's rows q [rows][n_heads][head_dim] over
        their requests' cached tokens and, causally or by row_mask (int32 bits, [rows]), the step's own
        rows.  scale defaults to 1 / sqrt(head_dim)."""
        shape = (step.rows, self.n_heads, self.head_dim)
        _rows3(q, shape, "q")
        if out is None:
            out = torch.empty(shape, dtype=q.dtype, device=q.device)
        else:
            _rows3(out, shape, "out")
        if q.device != self.device or out.device != self.device or out.dtype is not q.dtype:
            _fail(f"q and out: one type on {self.device} expected, got {q.dtype} on {q.device}, {out.dtype} on {out.device}")
        if row_mask is not None:
            _int32(row_mask, step.rows, "row_mask")
        qs, os = q.stride(), out.stride()
        _call(self.lib.ssd_kv8_attention, self._ref, layer, step._ref, q.data_ptr(), out.data_ptr(), _type(q, "q"),
              qs[0], qs[1], os[0], os[1], 1.0 / math.sqrt(self.head_dim) if scale is None else scale,
              None if row_mask is None else row_mask.data_ptr(), _stream(self.device))
        return out

    def check(self) -> None:
        """Wait for the stream and raise SSDError if a call met bad lengths, slots or values (ssd_kv8_status)."""
        _call(self.lib.ssd_kv8_status, self._ref, None, _stream(self.device))


_w4_work: dict = {}   # (device, stream) -> workspace: products on different streams must not share one


class W4Weight:
    """A weight matrix [n][k] packed to 4 bits with bf16 group scales (ssd_w4_pack)."""

    def __init__(self, weight: torch.Tensor, group: int = 128):
        self.lib = B.load()
        if weight.dim() != 2 or not weight.is_cuda or (weight.stride(1) != 1 and weight.numel()):
            _fail("weight: a 2-D CUDA tensor with contiguous rows expected")
        self.n, self.k = weight.shape
        self.group, self.device = group, weight.device
        size = self.lib.ssd_w4_bytes(self.n, self.k, group)
        if size < 0:
            _fail(self.lib.ssd_op_last_error().decode())
        self._work = self.lib.ssd_w4_work_bytes(self.n, self.k)
        self.packed = torch.empty(size, dtype=torch.uint8, device=weight.device)
        _call(self.lib.ssd_w4_pack, weight.data_ptr(), _type(weight, "weight"), self.n, self.k, weight.stride(0),
              group, self.packed.data_ptr(), _stream(self.device))

    def dequantize(self) -> torch.Tensor:
        """The fp32 values [n][k] the packed codes stand for."""
        out = torch.empty((self.n, self.k), dtype=torch.float32, device=self.device)
        _call(self.lib.ssd_w4_unpack, self.packed.data_ptr(), self.n, self.k, self.group, out.data_ptr(),
              _stream(self.device))
        return out

    def matmul(self, x: torch.Tensor, out: torch.Tensor | None = None,
               residual: torch.Tensor | None = None) -> torch.Tensor:
        """x W^T (+ residual) for x [rows][k] in bfloat16 or float32, rows <= 16 (ssd_w4_matmul)."""
        if x.dim() != 2 or x.shape[1] != self.k or x.stride(1) != 1:
            _fail(f"x: [rows][{self.k}] with contiguous rows expected, got {tuple(x.shape)}")
        rows = x.shape[0]
        if out is None:
            out = torch.empty((rows, self.n), dtype=x.dtype, device=x.device)
        for t, what in ((out, "out"), (residual, "residual")):
            if t is None:
                continue
            if t.shape != (rows, self.n) or t.dtype is not x.dtype or t.device != x.device or \
                    (t.stride(1) != 1 and self.n > 1):
                _fail(f"{what}: {x.dtype} [{rows}][{self.n}] with contiguous rows expected")
        if x.device != self.device:
            _fail(f"x: on {x.device}, the weight is on {self.device}")
        stream = _stream(self.device)
        work = _w4_work.get((self.device, stream))
        if work is None or work.numel() < self._work:
            work = _w4_work[(self.device, stream)] = torch.zeros(self._work, dtype=torch.uint8, device=self.device)
        _call(self.lib.ssd_w4_matmul, self.packed.data_ptr(), self.n, self.k, self.group, x.data_ptr(), _type(x, "x"),
              rows, x.stride(0), out.data_ptr(), out.stride(0), None if residual is None else residual.data_ptr(),
              0 if residual is None else residual.stride(0), work.data_ptr(), stream)
        return out
