"""Low-bit operators without a GPU: struct layouts, sizes and the refusals that come before any device call."""
import contextlib
import ctypes
import os
import types

import pytest
import torch

import paper_2510_22641_gb300 as lib
from paper_2510_22641_gb300 import _binding as B
from tests.test_abi_cpu import _c_layout

INVALID = 1


@pytest.fixture(scope="module")
def l():
    lib.build()
    return B.load()


def cache(**over):
    base = dict(n_layers=2, n_heads=8, n_kv_heads=4, head_dim=128, block_tokens=32, n_blocks=10, max_batch=3,
                max_blocks=5, data=256, scales=256, table=256, pool=256, work=256)   # never dereferenced
    return B.SSDKv8(**{**base, **over})


def step(**over):
    return B.SSDKv8Step(**{**dict(batch=2, rows=4, row_tile=0, data=256), **over})


def test_structs_match_the_header(tmp_path):
    pairs = {"ssd_kv8": B.SSDKv8, "ssd_kv8_step": B.SSDKv8Step}
    c = _c_layout(tmp_path, {n: [f for f, _ in t._fields_] for n, t in pairs.items()})
    for n, t in pairs.items():
        assert c[(n, "size")] == ctypes.sizeof(t)
        for f, _ in t._fields_:
            assert c[(n, f)] == getattr(t, f).offset, (n, f)


def test_sizes(l):
    c = cache()
    assert l.ssd_kv8_data_bytes(ctypes.byref(c)) == 2 * 10 * 4 * 32 * 128 * 2
    assert l.ssd_kv8_work_bytes(ctypes.byref(c)) >= 64
    assert l.ssd_kv8_step_ints(2, 4) == B.SSD_KV8_STEP_HEAD + 3 + 3 + 2 + 4
    for bad in ((0, 4), (1025, 4), (2, -1)):
        assert l.ssd_kv8_step_ints(*bad) == -1
    # codes of whole 16 x 128 tiles, one bf16 scale per row and group
    assert l.ssd_w4_bytes(17, 130, 32) == 2 * 2 * (1024 + 16 * 4 * 2)
    assert l.ssd_w4_bytes(16, 128, 128) == 1024 + 32
    for bad in ((0, 128, 32), (16, 0, 32), (16, 128, 48)):
        assert l.ssd_w4_bytes(*bad) == -1


@pytest.mark.parametrize("over", [{"head_dim": 96}, {"block_tokens": 24}, {"block_tokens": 256}, {"n_kv_heads": 3},
                                  {"n_heads": 2}, {"n_layers": 0}, {"n_blocks": 0}, {"max_batch": 0},
                                  {"max_batch": 1025}, {"max_blocks": 0}, {"n_blocks": 1 << 27},
                                  {"max_blocks": 1 << 26}], ids=str)
def test_cache_shapes_refused(l, over):
    c = cache(**over)
    assert l.ssd_kv8_data_bytes(ctypes.byref(c)) == -1
    assert l.ssd_kv8_work_bytes(ctypes.byref(c)) == -1
    assert l.ssd_kv8_status(ctypes.byref(c), None, None) == INVALID
    assert b"shape" in l.ssd_op_last_error()


@pytest.mark.parametrize("over", [{n: None} for n in ("data", "scales", "table", "pool", "work")] +
                         [{"data": 264}, {"scales": 260}, {"work": 260}], ids=str)
def test_cache_buffers_refused(l, over):
    c, s = cache(**over), step()
    assert l.ssd_kv8_plan(ctypes.byref(c), ctypes.byref(s), 256, 256, 256, 256, None) == INVALID
    assert l.ssd_kv8_append(ctypes.byref(c), 0, 256, 256, 0, 1, 0, 0, 0, 0, 256, None) == INVALID


def test_null_structs_refused(l):
    c = cache()
    assert l.ssd_kv8_data_bytes(None) == -1
    assert l.ssd_kv8_plan(None, None, 256, 256, 256, 256, None) == INVALID
    assert l.ssd_kv8_plan(ctypes.byref(c), None, 256, 256, 256, 256, None) == INVALID
    assert l.ssd_kv8_attention(ctypes.byref(c), 0, None, 256, 256, 0, 0, 0, 0, 0, 1.0, None, None) == INVALID


@pytest.mark.parametrize("over", [{"batch": 0}, {"batch": 4}, {"rows": -1}, {"row_tile": 12}, {"data": None},
                                  {"data": 260}, {"rows": 1 << 29}], ids=str)
def test_steps_refused(l, over):
    c, s = cache(), step(**over)
    assert l.ssd_kv8_plan(ctypes.byref(c), ctypes.byref(s), 256, 256, 256, 256, None) == INVALID
    assert l.ssd_kv8_attention(ctypes.byref(c), 0, ctypes.byref(s), 256, 256, 0, 0, 0, 0, 0, 1.0, None, None) == INVALID


def test_calls_refused(l):
    c, s = cache(), step()
    r, t = ctypes.byref(c), ctypes.byref(s)
    for k in range(4):
        args = [256] * 4
        args[k] = None
        assert l.ssd_kv8_plan(r, t, *args, None) == INVALID
    append = dict(layer=0, k=256, v=256, type=0, rows=1, slot=256)
    for bad in ({"layer": 2}, {"layer": -1}, {"k": None}, {"v": None}, {"type": 2}, {"rows": -1}, {"slot": None},
                {"k": 257}, {"type": 1, "v": 258}):
        a = {**append, **bad}
        assert l.ssd_kv8_append(r, a["layer"], a["k"], a["v"], a["type"], a["rows"], 0, 0, 0, 0, a["slot"],
                                None) == INVALID, bad
    for bad in ((2, 256, 1, 256, 256, 0), (0, None, 1, 256, 256, 0), (0, 256, -1, 256, 256, 0),
                (0, 256, 1, None, 256, 0), (0, 256, 1, 256, None, 0), (0, 256, 1, 256, 256, 5)):
        assert l.ssd_kv8_read(r, *bad, None) == INVALID, bad
    for bad in ((5, 256, 256, 0), (0, None, 256, 0), (0, 256, None, 0), (0, 256, 256, 3), (0, 257, 256, 0),
                (0, 258, 256, 1)):
        assert l.ssd_kv8_attention(r, bad[0], t, bad[1], bad[2], bad[3], 0, 0, 0, 0, 1.0, None, None) == INVALID, bad
    mm = dict(packed=256, n=16, k=128, group=32, x=256, type=0, rows=1, y=256, residual=None, work=256)
    for bad in ({"packed": None}, {"packed": 264}, {"n": 0}, {"k": 0}, {"group": 16}, {"x": None}, {"type": 7},
                {"rows": 17}, {"rows": -1}, {"y": None}, {"work": None}, {"work": 264}, {"x": 257},
                {"residual": 257}, {"type": 1, "y": 258}):
        a = {**mm, **bad}
        assert l.ssd_w4_matmul(a["packed"], a["n"], a["k"], a["group"], a["x"], a["type"], a["rows"], 128, a["y"], 16,
                               a["residual"], 16, a["work"], None) == INVALID, bad
        assert l.ssd_op_last_error()
    for bad in ((None, 0, 16, 128, 128, 32, 256), (256, 3, 16, 128, 128, 32, 256), (256, 0, 16, 128, 128, 32, 264),
                (256, 0, 0, 128, 128, 32, 256)):
        assert l.ssd_w4_pack(*bad, None) == INVALID, bad
    assert l.ssd_w4_unpack(256, 16, 128, 32, None, None) == INVALID
    assert l.ssd_w4_unpack(None, 16, 128, 32, 256, None) == INVALID


def test_zero_rows_need_no_device(l):
    c, s = cache(), step(rows=0)
    assert l.ssd_kv8_append(ctypes.byref(c), 0, None, None, 0, 0, 0, 0, 0, 0, None, None) == 0
    assert l.ssd_kv8_read(ctypes.byref(c), 0, None, 0, None, None, 0, None) == 0
    assert l.ssd_kv8_attention(ctypes.byref(c), 0, ctypes.byref(s), None, None, 0, 0, 0, 0, 0, 1.0, None, None) == 0
    assert l.ssd_w4_matmul(256, 16, 128, 32, None, 0, 0, 128, None, 16, None, 0, None, None) == 0


def test_the_package_offers_the_wrappers():
    for n in ("KV8Cache", "KV8Step", "W4Weight"):
        assert n in lib.__all__ and getattr(lib, n)


def test_header_compiles_as_c(tmp_path):
    src = tmp_path / "h.c"
    src.write_text('#include "ssd.h"\nint main(void) { return SSD_W4_MAX_ROWS == 16 ? 0 : 1; }\n')
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    assert os.system(f"gcc -Wall -Werror -I{inc} {src} -o {tmp_path / 'h'} && {tmp_path / 'h'}") == 0


class _FakeTensor:
    """Enough of a contiguous tensor on GPU 1 for the wrappers' checks; its address is never followed."""
    is_cuda = True

    def __init__(self, shape, dtype):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device("cuda", 1)

    def get_device(self):
        return 1

    def numel(self):
        return self.shape.numel()

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        s = [self.shape[j + 1:].numel() for j in range(len(self.shape))]
        return tuple(s) if i is None else s[i]

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return id(self) % (1 << 30) * 4096

    def __getitem__(self, i):
        return _FakeTensor((len(range(*i.indices(self.shape[0]))),), self.dtype)

    def __setitem__(self, i, v):
        pass


class _FakeTorch:
    """torch with fake allocations, and GPU 0 current."""

    def __init__(self):
        self.current = 0
        self.cuda = types.SimpleNamespace(current_device=lambda: self.current, device=self.enter)

    def __getattr__(self, name):
        return getattr(torch, name)

    def empty(self, shape, *_, dtype, device):
        assert torch.device(device) == torch.device("cuda", 1)
        return _FakeTensor((shape,) if isinstance(shape, int) else shape, dtype)

    zeros = full = empty

    def arange(self, a, b, c, dtype, device):
        return self.empty(len(range(a, b, c)), dtype=dtype, device=device)

    @contextlib.contextmanager
    def enter(self, i):
        before, self.current = self.current, i
        yield
        self.current = before


def test_calls_on_another_device_than_the_current_one_enter_it(l, monkeypatch):
    """Kernels are launched on the current device, and a default stream is the same null handle on each."""
    from paper_2510_22641_gb300 import lowbit
    fake, calls = _FakeTorch(), []

    class Lib:
        def __getattr__(self, name):
            if name.endswith(("_bytes", "_ints")):
                return getattr(l, name)
            return lambda *a: calls.append((name, fake.current)) or 0

    monkeypatch.setattr(lowbit, "torch", fake)
    monkeypatch.setattr(lowbit, "_stream", lambda i: 0)
    monkeypatch.setattr(lowbit, "_current", lambda: fake.current, raising=False)
    monkeypatch.setattr(lowbit.B, "load", Lib)
    bf16, i32 = torch.bfloat16, torch.int32
    c = lowbit.KV8Cache(1, 4, 2, 64, 16, 8, 2, 4, device="cuda:1")
    step = c.new_step(2, 3)
    kv, q = _FakeTensor((3, 2, 64), bf16), _FakeTensor((3, 4, 64), bf16)
    c.plan(step, _FakeTensor((2,), i32), _FakeTensor((2,), i32))
    c.append(0, kv, kv, step)
    c.read(0, _FakeTensor((5,), i32))
    c.attention(0, q, step)
    c.check()
    w = lowbit.W4Weight(_FakeTensor((32, 256), bf16))
    w.dequantize()
    w.matmul(_FakeTensor((3, 256), bf16))
    w.matmul(_FakeTensor((3, 256), torch.float32))
    assert [n for n, _ in calls] == ["ssd_kv8_plan", "ssd_kv8_append", "ssd_kv8_read", "ssd_kv8_attention",
                                     "ssd_kv8_status", "ssd_w4_pack", "ssd_w4_unpack", "ssd_w4_matmul", "ssd_w4_matmul"]
    assert [d for _, d in calls] == [1] * len(calls)
    assert fake.current == 0


@pytest.mark.parametrize("device", ["cpu", "meta"])
def test_a_cache_on_no_gpu_is_refused(l, device, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)   # a GPU that it must not be moved to
    with pytest.raises(lib.SSDError) as e:
        lib.KV8Cache(1, 4, 2, 64, 16, 8, 2, 4, device=device)
    assert e.value.status == INVALID


def test_outputs_over_inputs_are_refused(l):
    """Some CTAs would read what others have written.  Slices of one buffer that lie between each other are no
    overlap (the GPU tests run them)."""
    c, s = cache(), step()   # 4 rows of 8 heads of 128 elements
    r, t = ctypes.byref(c), ctypes.byref(s)
    base = 1 << 20
    for size, type in ((2, 0), (4, 1)):
        whole = (1024, 128)
        for at, strides in ((0, whole), (127, whole), (-1023, whole), (4 * 1024 - 1, whole), (0, (2048, 128)),
                            (0, (128, 512)), (1000, (1024, 130))):
            got = l.ssd_kv8_attention(r, 0, t, base, base + at * size, type, *whole, *strides, 1.0, None, None)
            assert got == INVALID and b"overlaps" in l.ssd_op_last_error(), (at, strides)
        # every second head of q, and the heads between them moved by one element
        assert l.ssd_kv8_attention(r, 0, t, base, base + 129 * size, type, 2048, 256, 2048, 256, 1.0, None, None) == INVALID

        def matmul(y, y_row, x_row=64, residual=None, res_row=0):
            return l.ssd_w4_matmul(256, 64, 64, 32, base, type, 4, x_row, base + y * size, y_row,
                                   None if residual is None else base + residual * size, res_row, 256, None)

        for y, y_row in ((0, 64), (63, 64), (-63, 64), (255, 64), (0, 100)):
            assert matmul(y, y_row) == INVALID and b"overlaps x" in l.ssd_op_last_error(), (y, y_row)
        assert matmul(65, 128, x_row=128) == INVALID   # columns 65.. of the rows whose columns ..63 are x: row 1's
        for residual, res_row in ((4097, 64), (4096 - 64, 64), (4096, 65)):
            assert matmul(4096, 64, residual=residual, res_row=res_row) == INVALID
            assert b"residual" in l.ssd_op_last_error()
