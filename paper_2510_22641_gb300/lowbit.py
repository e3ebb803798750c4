"""Python face of the low-bit operators (include/ssd.h): a paged 8-bit K/V cache, 4-bit weights and 4-bit floats.

The classes own torch buffers and forward every call to the library on their device's current stream.  No
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
_stream = torch._C._cuda_getCurrentRawStream   # of a device index; the public wrapper makes an object per call
_current = torch._C._cuda_getDevice            # (a tensor's device exists already, so CUDA is initialised)


def _fail(msg: str):
    raise B.SSDError(1, msg)


def _call(index: int, entry, *args):
    """Makes a library call on device `index`'s current stream.  The library launches on the current device, so
    another one is entered first."""
    if _current() == index:
        status = entry(*args, _stream(index))
    else:
        with torch.cuda.device(index):
            status = entry(*args, _stream(index))
    if status:
        raise B.SSDError(status, B.load().ssd_op_last_error().decode())


_INT = 0x7fffffff   # the library's sizes are C ints, into which ctypes cuts larger numbers without a word


def _ints(**sizes: int) -> None:
    for what, v in sizes.items():
        if not -_INT - 1 <= v <= _INT:
            _fail(f"{what}: {v} is out of range")


# The checks below run on every call of a decode loop: they compare whole shapes and device indices.

def _rows3(t: torch.Tensor, shape: tuple, index: int, what: str) -> tuple:
    """[rows][heads][dim] with any row and head strides and contiguous elements; returns its strides."""
    if t.shape != shape:
        _fail(f"{what}: shape {shape} expected, got {tuple(t.shape)}")
    if t.get_device() != index:
        _fail(f"{what}: on cuda:{index} expected, got {t.device}")
    st = t.stride()
    if st[2] != 1 and t.numel():
        _fail(f"{what}: the last dimension must be contiguous")
    return st


def _int32(t: torch.Tensor, shape: tuple, index: int, what: str) -> int:
    if t.dtype is not torch.int32 or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        _fail(f"{what}: a contiguous int32 tensor of shape {shape} on cuda:{index} expected, got {t.dtype} "
              f"{tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _type(dtype: torch.dtype, what: str) -> int:
    code = _TYPES.get(dtype)
    if code is None:
        _fail(f"{what}: bfloat16 or float32 expected, got {dtype}")
    return code


class KV8Step:
    """One step's plan: which request each new row belongs to and where its K/V goes (see ssd_kv8_step).

    row_start [batch + 1], slot [rows] and length [batch] are views of the device buffer that
    KV8Cache.plan fills."""

    def __init__(self, cache: KV8Cache, batch: int, rows: int, rows_per_request: int | None = None, row_tile: int = 0):
        _ints(batch=batch, rows=rows)
        n = B.load().ssd_kv8_step_ints(batch, rows)
        if n < 0 or batch > cache.max_batch:
            _fail(f"step of {rows} rows of {batch} requests (the cache has {cache.max_batch} seats)")
        self.batch, self.rows, self.cache = batch, rows, cache
        self.data = torch.zeros(n, dtype=torch.int32, device=cache.device)
        tile = row_tile
        if rows_per_request is not None:
            if rows_per_request < 1:
                _fail(f"rows_per_request {rows_per_request}")
            heads = rows_per_request * (cache.n_heads // cache.n_kv_heads)
            items = -(-heads // 32)
            tile = (-(-heads // items) + 7) // 8 * 8
        if tile not in (0, 8, 16, 24, 32):
            _fail(f"row_tile 0, 8, 16, 24 or 32 expected, got {row_tile}")
        at = B.SSD_KV8_STEP_HEAD + batch + 1
        self.row_start = self.data[at:at + batch + 1]
        self.length = self.data[at + batch + 1:at + 2 * batch + 1]
        self.slot = self.data[at + 2 * batch + 1:]
        self._batch, self._q, self._kv = (batch,), (rows, cache.n_heads, cache.head_dim), (rows, cache.n_kv_heads, cache.head_dim)
        self._slot = self.slot.data_ptr()
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
        _ints(n_layers=n_layers, n_heads=n_heads, n_kv_heads=n_kv_heads, head_dim=head_dim, block_tokens=block_tokens,
              n_blocks=n_blocks, max_batch=max_batch, max_blocks=max_blocks)
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
        if device.type != "cuda":
            _fail(f"KV8Cache: a CUDA device expected, got {device}")
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
        self._index, self._state, self._scale = device.index, (1 + max_batch,), 1.0 / math.sqrt(head_dim)

    def _layer(self, layer: int) -> int:
        if not 0 <= layer < self.n_layers:
            _fail(f"layer {layer} of {self.n_layers}")
        return layer

    def new_step(self, batch: int, rows: int, rows_per_request: int | None = None, row_tile: int = 0) -> KV8Step:
        """A plan's buffer for `rows` new rows of `batch` requests.  row_tile: query rows of a kv head the
        attention takes at once (8, 16, 24 or 32; 0: chosen by the cache's size), or rows_per_request: as many
        as that many rows have.  Only the attention's speed depends on it."""
        return KV8Step(self, batch, rows, rows_per_request, row_tile)

    def plan(self, step: KV8Step, length: torch.Tensor, add: torch.Tensor, state: torch.Tensor | None = None,
             state_out: torch.Tensor | None = None) -> KV8Step:
        """ssd_kv8_plan: hand out blocks for add[b] new rows after length[b] cached ones (-1: give the
        seat's blocks back) and fill `step`.  Updates self.state in place unless told otherwise."""
        i = self._index
        if step.cache is not self:
            _fail("the step was made for another cache")
        state = self.state if state is None else state
        state_in = _int32(state, self._state, i, "state")
        _call(i, self.lib.ssd_kv8_plan, self._ref, step._ref, _int32(length, step._batch, i, "length"),
              _int32(add, step._batch, i, "add"), state_in,
              state_in if state_out is None else _int32(state_out, self._state, i, "state_out"))
        return step

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, step: KV8Step) -> None:
        """ssd_kv8_append: quantise the step's new rows k, v [rows][n_kv_heads][head_dim] into the cache."""
        i = self._index
        if step.cache is not self:
            _fail("the step was made for another cache")
        ks, vs = _rows3(k, step._kv, i, "k"), _rows3(v, step._kv, i, "v")
        dtype = k.dtype
        if v.dtype is not dtype:
            _fail(f"k and v: one type expected, got {dtype} and {v.dtype}")
        _call(i, self.lib.ssd_kv8_append, self._ref, self._layer(layer), k.data_ptr(), v.data_ptr(), _type(dtype, "k"),
              step.rows, ks[0], ks[1], vs[0], vs[1], step._slot)

    def read(self, layer: int, slots: torch.Tensor, dtype: torch.dtype = torch.float32):
        """ssd_kv8_read: the (k, v) values held at int32 `slots`, each [n][n_kv_heads][head_dim]."""
        i, n = self._index, slots.numel()
        self._layer(layer), _ints(slots=n)
        at, code = _int32(slots, (n,), i, "slots"), _type(dtype, "dtype")
        shape = (n, self.n_kv_heads, self.head_dim)
        k = torch.empty(shape, dtype=dtype, device=self.device)
        v = torch.empty(shape, dtype=dtype, device=self.device)
        _call(i, self.lib.ssd_kv8_read, self._ref, layer, at, n, k.data_ptr(), v.data_ptr(), code)
        return k, v

    def attention(self, layer: int, q: torch.Tensor, step: KV8Step, out: torch.Tensor | None = None,
                  scale: float | None = None, row_mask: torch.Tensor | None = None) -> torch.Tensor:
        """ssd_kv8_attention: softmax(scale q k^T) v of the step's rows q [rows][n_heads][head_dim] over
        their requests' cached tokens and, causally or by row_mask (int32 bits, [rows]), the step's own
        rows.  scale defaults to 1 / sqrt(head_dim)."""
        i = self._index
        if step.cache is not self:
            _fail("the step was made for another cache")
        qs, dtype = _rows3(q, step._q, i, "q"), q.dtype
        self._layer(layer)
        if out is None:
            out = torch.empty(step._q, dtype=dtype, device=self.device)
            os = out.stride()
        else:
            os = _rows3(out, step._q, i, "out")
            if out.dtype is not dtype:
                _fail(f"q and out: one type expected, got {dtype} and {out.dtype}")
        _call(i, self.lib.ssd_kv8_attention, self._ref, layer, step._ref, q.data_ptr(), out.data_ptr(), _type(dtype, "q"),
              qs[0], qs[1], os[0], os[1], self._scale if scale is None else scale,
              None if row_mask is None else _int32(row_mask, (step.rows,), i, "row_mask"))
        return out

    def check(self) -> None:
        """Wait for the stream and raise SSDError if a call met bad lengths, slots or values (ssd_kv8_status)."""
        _call(self._index, self.lib.ssd_kv8_status, self._ref, None)


class W4Weight:
    """A weight matrix [n][k] packed to 4 bits with bf16 group scales (ssd_w4_pack)."""

    def __init__(self, weight: torch.Tensor, group: int = 128):
        self.lib = B.load()
        if weight.dim() != 2 or not weight.is_cuda or (weight.stride(1) != 1 and weight.numel()):
            _fail("weight: a 2-D CUDA tensor with contiguous rows expected")
        self.n, self.k = weight.shape
        _ints(n=self.n, k=self.k, group=group)
        self.group, self.device = group, weight.device
        size = self.lib.ssd_w4_bytes(self.n, self.k, group)
        if size < 0:
            _fail(self.lib.ssd_op_last_error().decode())
        self._work = self.lib.ssd_w4_work_bytes(self.n, self.k)
        self._index = weight.get_device()
        self.packed = torch.empty(size, dtype=torch.uint8, device=weight.device)
        self._packed = self.packed.data_ptr()
        _call(self._index, self.lib.ssd_w4_pack, weight.data_ptr(), _type(weight.dtype, "weight"), self.n, self.k,
              weight.stride(0), group, self._packed)

    def dequantize(self) -> torch.Tensor:
        """The fp32 values [n][k] the packed codes stand for."""
        out = torch.empty((self.n, self.k), dtype=torch.float32, device=self.device)
        _call(self._index, self.lib.ssd_w4_unpack, self._packed, self.n, self.k, self.group, out.data_ptr())
        return out

    def _rows(self, t: torch.Tensor, shape: tuple, dtype: torch.dtype, what: str) -> int:
        """Row stride of a [rows][columns] tensor with contiguous rows."""
        if t.shape != shape or t.dtype is not dtype or t.get_device() != self._index:
            _fail(f"{what}: {dtype} {shape} on {self.device} expected, got {t.dtype} {tuple(t.shape)} on {t.device}")
        st = t.stride()
        if st[1] != 1 and shape[1] > 1:
            _fail(f"{what}: contiguous rows expected")
        return st[0]

    def matmul(self, x: torch.Tensor, out: torch.Tensor | None = None,
               residual: torch.Tensor | None = None) -> torch.Tensor:
        """x W^T (+ residual) for x [rows][k] in bfloat16 or float32, rows <= 16 (ssd_w4_matmul)."""
        if x.dim() != 2:
            _fail(f"x: [rows][{self.k}] expected, got {tuple(x.shape)}")
        rows, dtype, i = x.shape[0], x.dtype, self._index
        if rows > _INT:
            _fail(f"x: {rows} rows")
        xs, code = self._rows(x, (rows, self.k), dtype, "x"), _type(dtype, "x")
        if out is None:
            out = torch.empty((rows, self.n), dtype=dtype, device=self.device)
            os = self.n
        else:
            os = self._rows(out, (rows, self.n), dtype, "out")
        # A call's own workspace, so that graphs, streams and threads share nothing.  bf16 rows that are operands
        # as they lie need none (the rule of ssd_w4_matmul).
        px, work = x.data_ptr(), None
        if code or self.k % 128 or xs % 8 or px % 16:
            work = torch.empty(self._work, dtype=torch.uint8, device=self.device)
        _call(i, self.lib.ssd_w4_matmul, self._packed, self.n, self.k, self.group, px, code, rows, xs, out.data_ptr(), os,
              None if residual is None else residual.data_ptr(),
              0 if residual is None else self._rows(residual, (rows, self.n), dtype, "residual"),
              self._packed if work is None else work.data_ptr())
        return out


def _rows2(t: torch.Tensor, shape: tuple, index: int, what: str) -> int:
    """Row stride of a [rows][columns] tensor with contiguous rows on cuda:`index`."""
    if t.shape != shape or t.get_device() != index:
        _fail(f"{what}: {shape} on cuda:{index} expected, got {tuple(t.shape)} on {t.device}")
    st = t.stride()
    if st[1] != 1 and shape[1] > 1 and shape[0]:
        _fail(f"{what}: contiguous rows expected")
    return st[0]


def _f4_buffer(lib, size: int, device) -> torch.Tensor:
    if size < 0:
        _fail(lib.ssd_op_last_error().decode())
    return torch.empty(size, dtype=torch.uint8, device=device)


class F4Rows:
    """Rows [rows][k] packed to 4-bit floats with a scale per 16 columns and one per row (ssd_f4_pack).

    F4Weight.matmul takes them in place of a tensor, so that rows that meet several weights are packed once."""

    def __init__(self, x: torch.Tensor):
        if x.dim() != 2 or not x.is_cuda:
            _fail(f"a 2-D CUDA tensor expected, got {tuple(x.shape)} on {x.device}")
        self.lib, self.shape, self.device, self._index = B.load(), x.shape, x.device, x.get_device()
        rows, k = x.shape
        _ints(rows=rows, k=k)
        self.packed = _f4_buffer(self.lib, self.lib.ssd_f4_bytes(rows, k), x.device)
        self._packed = self.packed.data_ptr()
        self.pack(x)

    def pack(self, x: torch.Tensor) -> F4Rows:
        """Packs other rows of the same shape into this buffer."""
        shape, index, dtype = self.shape, self._index, x.dtype
        _call(index, self.lib.ssd_f4_pack, x.data_ptr(), _type(dtype, "x"), shape[0], shape[1], _rows2(x, shape, index, "x"),
              self._packed)
        self.dtype = dtype
        return self

    def dequantize(self, dtype: torch.dtype = torch.float32) -> torch.Tensor:
        """The values [rows][k] that the codes stand for."""
        code, shape = _type(dtype, "dtype"), self.shape
        out = torch.empty(shape, dtype=dtype, device=self.device)
        _call(self._index, self.lib.ssd_f4_unpack, self._packed, shape[0], shape[1], out.data_ptr(), code)
        return out


class F4Weight(F4Rows):
    """A weight matrix [n][k] packed to 4-bit floats, for products with any number of rows."""

    def __init__(self, weight: torch.Tensor):
        super().__init__(weight)
        self.n, self.k = self.shape

    def matmul(self, x: torch.Tensor | F4Rows, out: torch.Tensor | None = None,
               residual: torch.Tensor | None = None) -> torch.Tensor:
        """x W^T (+ residual) for x [rows][k] in bfloat16 or float32, packed on the way, or packed already
        (ssd_f4_matmul).  The result has x's type (for F4Rows the type of the rows that were packed)."""
        i, n, k, shape, dtype = self._index, self.n, self.k, x.shape, x.dtype
        code = _type(dtype, "x")
        if len(shape) != 2 or shape[1] != k:
            _fail(f"x: [rows][{k}] expected, got {tuple(shape)}")
        rows = shape[0]
        if rows > _INT:
            _fail(f"x: {rows} rows")
        if isinstance(x, F4Rows):
            if x._index != i:
                _fail(f"x: on cuda:{i} expected, got {x.device}")
            px, xs, xcode, work = x._packed, 0, B.SSD_TYPE_F4, None
        else:
            px, xs, xcode = x.data_ptr(), _rows2(x, shape, i, "x"), code
            work, size = None, self.lib.ssd_f4_work_bytes(rows, k) if rows else 0
            if size:
                work = _f4_buffer(self.lib, size, self.device)
        if out is None:
            out, os = torch.empty((rows, n), dtype=dtype, device=self.device), n
        else:
            os = _rows2(out, (rows, n), i, "out")
            if out.dtype is not dtype:
                _fail(f"out: {dtype} expected, got {out.dtype}")
        res, rs = None, 0
        if residual is not None:
            res, rs = residual.data_ptr(), _rows2(residual, (rows, n), i, "residual")
            if residual.dtype is not dtype:
                _fail(f"residual: {dtype} expected, got {residual.dtype}")
        _call(i, self.lib.ssd_f4_matmul, self._packed, n, k, px, xcode, rows, xs, out.data_ptr(), code, os, res, rs,
              None if work is None else work.data_ptr())
        return out
