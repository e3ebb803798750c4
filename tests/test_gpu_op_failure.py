"""Operators with bounded waits, when one runs out: the documented NaN or -1 where it was waited for, everything else as ever,
and the next call whole.  The wait is made to run out on the host: one copy is left out and waits are short."""
import contextlib

import pytest
import torch

import paper_2510_22641_gb300 as lib
from tests.test_gpu_rows import DT, logits_of, normal, uneven

pytestmark = pytest.mark.gpu


@contextlib.contextmanager
def injected(kind):
    lib.set_fault_injection(kind, 1)
    try:
        yield
    finally:
        lib.set_fault_injection(lib.SSD_FAULT_NONE, 0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,n,k", [(1, 700, 1000), (3, 10000, 2560), (5, 700, 200), (20, 700, 1000), (40, 700, 8192),
                                      (96, 10000, 2560), (128, 300, 4096), (129, 700, 1000), (300, 700, 3000), (700, 5000, 600),
                                      (3001, 3000, 600)])
def test_product_whose_wait_runs_out(rows, n, k, dtype):
    w, x = lib.F4Weight(normal((n, k), 1, 0.02)), uneven(rows, k, 2, DT[dtype])
    res = normal((rows, n), 3, 1.0, DT[dtype])
    want = w.matmul(x, residual=res)
    with injected(lib.SSD_FAULT_COPY):
        y = w.matmul(x, residual=res)
    torch.cuda.synchronize()
    assert torch.equal(w.matmul(x, residual=res), want)
    lost = torch.zeros_like(y, dtype=torch.bool)
    if rows <= 128:   # tiles of 128 weight rows
        lost[:, :128] = True
    else:             # or of 256 by 256 rows, x rows fastest, dealt out to 76 pairs of CTAs, of which the first one gives up
        down = -(-rows // 256)
        for t in range(0, down * -(-n // 256), 76):
            lost[t % down * 256:, t // down * 256:][:256, :256] = True
    assert torch.isnan(y[lost]).all() and torch.equal(y[~lost], want[~lost])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,vocab", [(1, 300), (5, 40000), (300, 9000)])
def test_draw_whose_wait_runs_out(rows, vocab, dtype):
    z, u = logits_of(rows, vocab, 5, DT[dtype]), torch.rand(rows, generator=torch.Generator().manual_seed(2)).cuda()
    want = lib.sample(z, u, 0.9, 60, 0.9, with_prob=True)
    with injected(lib.SSD_FAULT_COPY):
        token, prob = lib.sample(z, u, 0.9, 60, 0.9, with_prob=True)
    torch.cuda.synchronize()
    again = lib.sample(z, u, 0.9, 60, 0.9, with_prob=True)
    assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])
    assert token[0] == -1 and torch.isnan(prob[0])
    assert torch.equal(token[1:], want[0][1:]) and torch.equal(prob[1:], want[1][1:])


def test_short_waits_are_long_enough():
    """What the injection of short waits alone leaves: every result."""
    w = lib.F4Weight(normal((700, 1000), 1, 0.02))
    for rows in (1, 40, 300):
        x = uneven(rows, 1000, 2)
        want = w.matmul(x)
        with injected(lib.SSD_FAULT_WAIT):
            y = w.matmul(x)
        assert torch.equal(y, want)
    z, u = logits_of(5, 40000, 5), torch.full((5,), 0.5, device="cuda")
    want = lib.sample(z, u)
    with injected(lib.SSD_FAULT_WAIT):
        t = lib.sample(z, u)
    assert torch.equal(t, want)


@pytest.mark.parametrize("rows", [1, 40])
def test_waits_begin_after_the_launch_before(rows):
    """A product may take its place on the GPU while the launch before it still runs; that time is not its own.  Here that
    launch takes more than a millisecond on two SMs, and the waits behind it last a quarter of one."""
    k = 1 << 20
    big, wide = lib.F4Weight(normal((200, k), 1, 0.02)), lib.F4Rows(normal((200, k), 2))
    w, x = lib.F4Weight(normal((300, 2560), 3, 0.02)), lib.F4Rows(uneven(rows, 2560, 4))
    want = w.matmul(x)
    for _ in range(3):
        torch.cuda.synchronize()
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        big.matmul(wide)
        b.record()
        torch.cuda.synchronize()
        assert a.elapsed_time(b) > 0.5, "the launch before is too short for this test"
        big.matmul(wide)
        with injected(lib.SSD_FAULT_WAIT):
            y = w.matmul(x)
        assert torch.equal(y, want)
