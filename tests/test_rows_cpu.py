"""Operators on rows without a GPU: struct layouts, sizes, and the refusals that come before any device call."""
import ctypes
import math
import types

import numpy as np
import pytest
import torch

import paper_2510_22641_gb300 as lib
from paper_2510_22641_gb300 import _binding as B
from tests import rows_ref as ref
from tests.test_abi_cpu import _c_layout

INVALID = 1


@pytest.fixture(scope="module")
def l():
    lib.build()
    return B.load()


def test_structs_match_the_header(tmp_path):
    pairs = {"ssd_rotary": B.SSDRotary, "ssd_heads": B.SSDHeads, "ssd_sampling": B.SSDSampling}
    c = _c_layout(tmp_path, {n: [f for f, _ in t._fields_] for n, t in pairs.items()})
    for n, t in pairs.items():
        assert c[(n, "size")] == ctypes.sizeof(t)
        for f, _ in t._fields_:
            assert c[(n, f)] == getattr(t, f).offset, (n, f)


def test_fields_as_bytes_match_the_structs():
    from paper_2510_22641_gb300 import heads
    v = (11, 12, 13, -14, 15, -16, 17, 18, 1)
    two = (B.SSDHeads * 2).from_buffer_copy(heads._two(*v, *v))
    assert heads._one(*v) == bytes(two)[:ctypes.sizeof(B.SSDHeads)]
    for h in two:
        assert tuple(getattr(h, f) for f, _ in B.SSDHeads._fields_) == v
    s = B.SSDSampling.from_buffer_copy(heads._sampling(0.5, 0.25, 0.125, -7, 21, 22, 23, 24))
    assert [getattr(s, f) for f, _ in B.SSDSampling._fields_] == [0.5, 0.25, 0.125, -7, 21, 22, 23, 24]
    assert len(heads._sampling(0, 0, 0, 0, 0, 0, 0, 0)) == ctypes.sizeof(B.SSDSampling)


def test_packed_sizes(l):
    record = 128 * 256 // 2 + 128 * 256 // 16
    assert l.ssd_f4_bytes(1, 1) == record + 128 * 4
    assert l.ssd_f4_bytes(128, 256) == record + 128 * 4
    assert l.ssd_f4_bytes(129, 257) == 4 * record + 256 * 4
    assert l.ssd_f4_bytes(1 << 23, 1 << 20) == (1 << 16) * (1 << 12) * record + (1 << 23) * 4   # past 32 bits
    for bad in ((0, 16), (16, 0), (-1, 16), ((1 << 23) + 1, 16), (16, (1 << 20) + 1)):
        assert l.ssd_f4_bytes(*bad) == -1


def test_work_sizes(l):
    """Few short rows are packed by the product itself."""
    for rows, k in ((1, 1), (1, 16384), (4, 4096)):
        assert l.ssd_f4_work_bytes(rows, k) == 0
    for rows, k in ((1, 16385), (4, 4097), (5, 64), (300, 4096)):
        assert l.ssd_f4_work_bytes(rows, k) == l.ssd_f4_bytes(rows, k) > 0
    assert l.ssd_f4_work_bytes(0, 5) == -1 and l.ssd_f4_work_bytes(5, 0) == -1


def pack(l, **over):
    a = dict(x=4096, type=0, rows=4, k=64, stride=64, packed=1 << 20) | over
    return l.ssd_f4_pack(a["x"], a["type"], a["rows"], a["k"], a["stride"], a["packed"], None)


@pytest.mark.parametrize("over", [{"x": None}, {"packed": None}, {"packed": (1 << 20) + 8}, {"x": 4097}, {"type": 2},
                                  {"type": 1, "x": 4098}, {"rows": 0}, {"k": 0}, {"rows": (1 << 23) + 1},
                                  {"packed": 4096 + 128}, {"x": (1 << 20) + 16384}, {"packed": 4096 - 16}], ids=str)
def test_pack_refused(l, over):
    assert pack(l, **over) == INVALID
    assert l.ssd_op_last_error()


@pytest.mark.parametrize("over", [{"packed": None}, {"out": None}, {"packed": 4104}, {"out": 4098, "type": 1}, {"type": 2},
                                  {"out": 4096 + 18432}, {"out": 4096 - 512},
                                  {"rows": 0}, {"k": -1}], ids=str)
def test_unpack_refused(l, over):
    a = dict(packed=4096, rows=4, k=64, out=1 << 20, type=1) | over
    assert l.ssd_f4_unpack(a["packed"], a["rows"], a["k"], a["out"], a["type"], None) == INVALID


MB = 1 << 20


def matmul(l, **over):
    a = dict(w=MB, n=100, k=64, x=8 * MB, x_type=0, rows=5, xs=64, y=16 * MB, type=0, ys=100, res=None, rs=0,
             work=24 * MB) | over
    return l.ssd_f4_matmul(a["w"], a["n"], a["k"], a["x"], a["x_type"], a["rows"], a["xs"], a["y"], a["type"], a["ys"],
                           a["res"], a["rs"], a["work"], None)


@pytest.mark.parametrize("over", [{n: None} for n in ("w", "x", "y", "work")] +
                         [{"w": MB + 8}, {"work": MB * 24 + 4}, {"x": 8 * MB + 1}, {"y": 16 * MB + 1}, {"n": 0}, {"k": 0},
                          {"rows": -1}, {"type": 2}, {"x_type": 3}, {"x_type": 2, "x": 8 * MB + 8}, {"y": 8 * MB + 128},
                          {"y": MB + 64}, {"y": 24 * MB}, {"work": 8 * MB}, {"work": MB}, {"res": 16 * MB + 2, "rs": 100},
                          {"res": 16 * MB, "rs": 101}, {"res": 24 * MB, "rs": 100}, {"x_type": 2, "y": 8 * MB + 16},
                          {"ys": 0}, {"ys": 99}, {"ys": -99}], ids=str)
def test_matmul_refused(l, over):
    assert matmul(l, **over) == INVALID
    assert l.ssd_op_last_error()


def test_matmul_of_no_rows_is_nothing(l):
    assert matmul(l, rows=0, x=None, y=None, work=None) == 0


@pytest.mark.parametrize("args", [(0, 0), (3, 2), (258, 2), (64, 66), (64, 3), (64, -2)], ids=str)
def test_rotary_shapes_refused(l, args):
    r = B.SSDRotary()
    assert l.ssd_rotary_init(ctypes.byref(r), *args, 0, 1, None, 1e4, 1e-5) == INVALID


def test_rotary_settings_refused(l):
    r = ctypes.byref(B.SSDRotary())
    three = (ctypes.c_int * 3)(8, 12, 12)
    assert l.ssd_rotary_init(r, 64, 64, 0, 3, three, 1e4, 1e-5) == 0
    for axes, section in ((0, None), (5, three), (2, None), (2, three), (3, (ctypes.c_int * 3)(8, 12, 13)),
                          (3, (ctypes.c_int * 3)(-1, 20, 13)), (1, (ctypes.c_int * 1)(31))):
        assert l.ssd_rotary_init(r, 64, 64, 0, axes, section, 1e4, 1e-5) == INVALID, axes
    for theta, eps in ((0.5, 1e-5), (math.inf, 1e-5), (math.nan, 1e-5), (1e4, -1.0), (1e4, math.nan), (1e4, math.inf)):
        assert l.ssd_rotary_init(r, 64, 64, 0, 1, None, theta, eps) == INVALID
    assert l.ssd_rotary_init(None, 64, 64, 0, 1, None, 1e4, 1e-5) == INVALID


def test_rotary_steps_are_fractions_of_a_turn(l):
    r = B.SSDRotary()
    assert l.ssd_rotary_init(ctypes.byref(r), 96, 48, 1, 2, (ctypes.c_int * 2)(10, 14), 5e5, 1e-6) == 0
    assert list(r.axis[:24]) == [0] * 10 + [1] * 14 and r.turn == 48 and r.interleaved == 1
    for i in range(24):
        want = 5e5 ** (-2 * i / 48) / (2 * math.pi)
        assert abs(r.step[i] / 2 ** 64 - want) <= 2 ** -51 * want + 2 ** -63


def heads(**over):
    return B.SSDHeads(**({"x": MB, "y": 2 * MB, "heads": 4, "x_row": 256, "x_head": 64, "y_row": 256, "y_head": 64} | over))


def apply(l, r, ops, type=0, rows=5, pos=4 * MB):
    return l.ssd_rotary_apply(ctypes.byref(r), (B.SSDHeads * len(ops))(*ops), len(ops), type, rows, pos, 1, 0, None)


def test_rotary_calls_refused(l):
    r = B.SSDRotary()
    assert l.ssd_rotary_init(ctypes.byref(r), 64, 64, 0, 1, None, 1e4, 1e-5) == 0
    bad = [[heads(x=None)], [heads(y=None)], [heads(heads=0)], [heads(x=MB + 1)], [heads(gain=8, gain_type=2)],
           [heads(gain=9, gain_type=0)], [heads(), heads()], [heads(y=MB + 128)], [heads(y=MB, y_head=32)],
           [heads(), heads(x=3 * MB, y=MB)], [heads(), heads(x=2 * MB, y=3 * MB)], [],
           [heads(gain=2 * MB + 64, gain_type=1)], [heads(), heads(x=3 * MB, y=5 * MB, gain=2 * MB + 256 * 8 + 500, gain_type=0)],
           [heads(y=4 * MB - 2)], [heads(y_row=0)], [heads(y_head=0)], [heads(y_row=255)], [heads(y_head=63)], [heads(y_row=64, y_head=64 * 4)],
           [heads(y_row=-255)]]
    for i, ops in enumerate(bad):
        assert apply(l, r, ops) == INVALID, i
    for over in ({"type": 2}, {"rows": -1}, {"pos": None}, {"pos": 4 * MB + 2}, {"rows": (1 << 26) + 1}):
        assert apply(l, r, [heads()], **over) == INVALID, over
    assert apply(l, r, [heads()], rows=0, pos=None) == 0
    assert l.ssd_rotary_apply(None, None, 1, 0, 1, MB, 1, 0, None) == INVALID
    for field, value in (("head_dim", 258), ("head_dim", 3), ("turn", 66), ("axes", 0), ("axes", 5), ("eps", -1.0)):
        c = B.SSDRotary.from_buffer_copy(r)
        setattr(c, field, value)
        assert apply(l, c, [heads()]) == INVALID, field
    c = B.SSDRotary.from_buffer_copy(r)
    c.axis[5] = 1
    assert apply(l, c, [heads()]) == INVALID


@pytest.mark.parametrize("over", [{n: None} for n in ("logits", "u", "token", "how")] +
                         [{"type": 2}, {"rows": -1}, {"vocab": 0}, {"vocab": 262145}, {"logits": MB + 1},
                          {"logits": MB + 2, "type": 1}, {"u": MB + 2}, {"token": MB + 1}, {"prob": MB + 1},
                          {"token": MB + 396}, {"token": 2 * MB + 4}, {"prob": 2 * MB - 4}, {"prob": 3 * MB + 4}, {"prob": MB}],
                         ids=str)
def test_sample_refused(l, over):
    how = B.SSDSampling(temperature=1.0, top_p=1.0)
    a = dict(logits=MB, type=0, rows=2, vocab=100, stride=100, u=2 * MB, how=ctypes.byref(how), token=3 * MB, prob=None) | over
    assert l.ssd_sample(a["logits"], a["type"], a["rows"], a["vocab"], a["stride"], a["u"], a["how"], a["token"], a["prob"],
                        None) == INVALID
    assert l.ssd_sample(None, 0, 0, 10, 10, None, None, None, None, None) == 0


def test_sample_settings_refused(l):
    how = B.SSDSampling(temperature=1.0, top_p=1.0)
    for name in ("temperature_rows", "top_p_rows", "min_p_rows", "top_k_rows"):
        c = B.SSDSampling.from_buffer_copy(how)
        setattr(c, name, MB + 2)
        assert l.ssd_sample(MB, 0, 2, 100, 100, 2 * MB, ctypes.byref(c), 3 * MB, None, None) == INVALID
        setattr(c, name, 3 * MB + 4)
        assert l.ssd_sample(MB, 0, 2, 100, 100, 2 * MB, ctypes.byref(c), 3 * MB, None, None) == INVALID


def test_wrappers_refuse_cpu_tensors(l):
    x = torch.zeros(4, 32)
    calls = [lambda: lib.F4Rows(x), lambda: lib.F4Weight(x), lambda: lib.F4Rows(x[0]), lambda: lib.sample(x, x[:, 0]),
             lambda: lib.Rotary(32).rotate(x[:, None], None, torch.zeros(4, dtype=torch.int32)),
             lambda: lib.Rotary(31), lambda: lib.Rotary(32, sections=(8, 9)), lambda: lib.Rotary(32, axes=[0] * 15),
             lambda: lib.Rotary(32, axes=[4] * 16), lambda: lib.Rotary(32, axes=[-1] + [0] * 15),
             lambda: lib.Rotary(32, sections=(16,), axes=[0] * 16), lambda: lib.Rotary(32, freqs=[1.0]),
             lambda: lib.Rotary(32, freqs=[math.nan] * 16)]
    for i, f in enumerate(calls):
        with pytest.raises(lib.SSDError) as e:
            f()
        assert e.value.status == INVALID, i


def test_rotary_of_given_frequencies(l):
    freqs = [1.0, -0.5, 100.0, 0.0]
    r = lib.Rotary(8, axes=[2, 0, 1, 2], freqs=freqs)
    assert r.axes == 3 and list(r._c.axis[:4]) == [2, 0, 1, 2]
    for i, f in enumerate(freqs):
        assert abs(r._c.step[i] / 2 ** 64 - f / (2 * math.pi) % 1) < 1e-14 * max(1, abs(f))


def test_reference_of_4_bit_floats_on_values_worked_by_hand():
    x = np.zeros((3, 32))
    x[0, 0], x[0, 1], x[0, 2], x[0, 3], x[0, 16] = 2688, 448 * 2.5, -448 * 5, 100, 1
    # rho 1, scales 448 and e4m3(1 / 6) = 0.171875: 2.5 -> 2, 5 -> 4, 100 / 448 -> 0; 1 / 0.171875 = 5.8 -> 6
    x[1, 0] = 2689   # rho 2
    x[2, 5] = 6 * 2.0 ** -100
    v = ref.f4_values(x)
    assert v[0, 0] == 2688 and v[0, 1] == 896 and v[0, 2] == -1792 and v[0, 3] == 0 and v[0, 16] == 6 * 0.171875
    assert v[1, 0] == 2 * 6 * 224 and v[2, 5] == 6 * 2.0 ** -100
    assert (ref._nearest(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7]), ref.FLOATS4) == [0, 1, 1, 2, 2, 4, 4, 6]).all()
    assert ref.E4M3[1] == 2.0 ** -9 and ref.E4M3[126] == 448


def test_reference_of_sampling_on_rows_worked_by_hand():
    z = [0.0, math.log(2), math.log(4), math.log(1)]   # weights 1, 2, 4, 1 of 8
    s = lambda u, **o: ref.sample(z, u, *(o.get(n, d) for n, d in (("t", 1.0), ("k", 0), ("p", 1.0), ("m", 0.0))))  # noqa: E731
    assert [s(u)[0] for u in (0.0, 0.124, 0.126, 0.374, 0.376, 0.874, 0.876)] == [0, 0, 1, 1, 2, 2, 3]
    assert abs(s(0.5)[1] - 0.5) < 1e-12
    assert [s(u, k=2)[0] for u in (0.0, 0.3, 0.4)] == [1, 1, 2] and s(0.9, k=1) == (2, 1.0)
    assert [s(u, p=0.8)[0] for u in (0.0, 0.142, 0.144, 0.99)] == [0, 0, 1, 2]   # 4, 2, and the first of the ones
    assert [s(u, m=0.5)[0] for u in (0.0, 0.99)] == [1, 2] and s(0.1, m=2.0)[0] == 2 and s(0.9, p=0.0)[0] == 2
    assert s(0.9, t=0.0) == (2, 1.0) and ref.sample([math.nan, -math.inf], 0.5, 1.0, 0, 1.0, 0.0) == (-1, 0.0)
