"""4-bit weights on the GPU: packing equals the reference bit for bit, products against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2510_22641_gb300 as lib
from tests import lowbit_ref as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def normal(shape, seed, scale=1.0, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def check(y, x, w, residual=None):
    """fp32: 22 bits of x (2^-22) and fp32 sums of k products, taken as (k / 8 + 64) 2^-24 of sum |x w|; the
    residual's addition one rounding; bf16 rows round once more at the end."""
    xd, wd = x.double(), w.double()
    want, size = xd @ wd.T, xd.abs() @ wd.abs().T
    if residual is not None:
        want, size = want + residual.double(), size + residual.double().abs()
    bound = (x.shape[1] / 8 + 64) * 2.0 ** -24 * size
    rms = 2.0 ** -18
    if y.dtype is torch.bfloat16:
        bound = bound + 2.0 ** -8 * want.abs()
        rms = 2.0 ** -8
    err = (y.double() - want).abs()
    assert (err <= bound).all(), f"{(err > bound).sum().item()} of {err.numel()}, worst {(err / bound).max().item()}"
    assert err.square().mean().sqrt() <= rms * want.square().mean().sqrt() + 1e-30


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,k", [(1, 1), (16, 128), (17, 129), (5, 333), (130, 640), (48, 96), (100, 2050)])
def test_pack_equals_the_reference(n, k, group):
    for dtype in DT.values():
        w = normal((n, k), n + k, 0.02, dtype)
        got = lib.W4Weight(w, group).dequantize().cpu().numpy()
        assert np.array_equal(got, ref.quantize4(w.float().cpu().numpy(), group))


def test_pack_of_zeros_extremes_and_views():
    w = torch.zeros(20, 256, device="cuda")
    w[1, 5], w[2, 0], w[2, 1], w[3] = 1e-30, 3e38, -1e38, -7.0
    w[4, ::2], w[4, 1::2] = 1e-40, 0
    got = lib.W4Weight(w, 64).dequantize().cpu().numpy()
    assert np.array_equal(got, ref.quantize4(w.cpu().numpy(), 64)) and np.isfinite(got).all()
    base = normal((33, 400), 3)
    view = base[1:30, 7:7 + 200]
    assert np.array_equal(lib.W4Weight(view, 32).dequantize().cpu().numpy(), ref.quantize4(view.cpu().numpy(), 32))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [1, 2, 4, 5, 8, 9, 16])
@pytest.mark.parametrize("n,k,group", [(1, 1, 32), (16, 128, 128), (33, 130, 64), (512, 1000, 32), (4096, 512, 128),
                                       (250, 4096, 64), (11008, 256, 128), (20001, 384, 32), (64, 14336, 128)])
def test_matmul(n, k, group, rows, dtype):
    w = lib.W4Weight(normal((n, k), 1, 0.02, torch.bfloat16), group)
    x = normal((rows, k), 2) * torch.exp(1.5 * normal((1, k), 3))
    x = x.to(DT[dtype])
    y = w.matmul(x, out=torch.full((rows, n), float("nan"), dtype=x.dtype, device="cuda"))
    check(y, x, w.dequantize())
    assert torch.equal(y, w.matmul(x))   # the same bits every time


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_matmul_adds_a_residual_and_takes_views(dtype):
    n, k, m = 300, 520, 6
    w = lib.W4Weight(normal((n, k), 1, 0.02), 64)
    xs = normal((m, k + 9), 2, 1.0, DT[dtype])
    res = normal((m, n + 5), 3, 1.0, DT[dtype])
    out = torch.full((m, n + 3), float("nan"), dtype=DT[dtype], device="cuda")
    for x in (xs[:, :k], xs[:, 1:k + 1], xs[:, 8:k + 8]):
        w.matmul(x, out=out[:, 1:n + 1], residual=res[:, 2:n + 2])
        check(out[:, 1:n + 1], x, w.dequantize(), res[:, 2:n + 2])
        assert torch.isnan(out[:, 0]).all() and torch.isnan(out[:, n + 1:]).all()
    y = res[:, :n].contiguous()
    before = y.clone()
    w.matmul(xs[:, :k], out=y, residual=y)   # in place
    check(y, xs[:, :k], w.dequantize(), before)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_matmul_over_the_range_of_the_type(dtype):
    """Rows of very different size, values fp16 does not hold, zeros; NaN and infinity stay in their row."""
    n, k = 200, 1024
    w = lib.W4Weight(normal((n, k), 1, 0.02), 128)
    x = normal((7, k), 2)
    x[0] *= 1e30
    x[1] *= 1e-30
    x[2, ::3] *= 1e6
    x[3] = 0
    x[4, :128] *= 1e-12
    x = x.to(DT[dtype])
    y = w.matmul(x)
    check(y[:1], x[:1], w.dequantize())
    check(y[1:2], x[1:2], w.dequantize())
    check(y[2:], x[2:], w.dequantize())
    assert (y[3] == 0).all()
    x2 = x.clone()
    x2[4, 77], x2[5, 300] = float("nan"), float("inf")
    y2 = w.matmul(x2)
    assert torch.isnan(y2[4]).all() and not torch.isfinite(y2[5]).any()
    keep = [0, 1, 2, 3, 6]
    assert torch.equal(y2[keep], y[keep])


def test_matmul_shows_non_finite_weights():
    w = normal((40, 256), 1, 0.02)
    w[3, 200], w[7, 1] = float("nan"), float("inf")
    y = lib.W4Weight(w, 64).matmul(normal((2, 256), 2))
    bad = ~torch.isfinite(y).all(0)
    assert bad.nonzero().flatten().tolist() == [3, 7]


def test_matmul_on_two_streams():
    ws = [lib.W4Weight(normal((3000, 2048), i, 0.02), 128) for i in range(2)]
    x = normal((3, 2048), 5)
    want = [w.matmul(x) for w in ws]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(ws[i].matmul(x))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, want[i]) for y in got[i])


def test_wrapper_refusals():
    w = lib.W4Weight(normal((20, 64), 1), 32)
    x = normal((2, 64), 2)
    calls = [lambda: lib.W4Weight(normal((20, 64), 1), 16), lambda: lib.W4Weight(normal((20, 64), 1).half()),
             lambda: lib.W4Weight(normal((20, 64), 1).cpu()), lambda: lib.W4Weight(normal((20, 64), 1).T),
             lambda: w.matmul(x[:, :63]), lambda: w.matmul(x.half()), lambda: w.matmul(normal((17, 64), 1)),
             lambda: w.matmul(x, out=torch.zeros(2, 21, device="cuda")), lambda: w.matmul(x.cpu()),
             lambda: w.matmul(x, residual=torch.zeros(2, 20, dtype=torch.bfloat16, device="cuda")),
             lambda: w.matmul(x.T.contiguous().T)]
    for i, f in enumerate(calls):
        with pytest.raises(lib.SSDError) as e:
            f()
        assert e.value.status == 1, i
    assert w.matmul(x[:0]).shape == (0, 20)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_captured_product_shares_nothing_with_later_calls(dtype):
    """A graph's replays after larger products on its stream: neither its values nor other tensors change."""
    x, w = normal((5, 130), 1, dtype=DT[dtype]), normal((96, 130), 2, 0.05)
    big_x, big_w = normal((16, 5000), 3, dtype=DT[dtype]), lib.W4Weight(normal((64, 5000), 4, 0.05))
    p = lib.W4Weight(w, 32)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        p.matmul(x)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            y = p.matmul(x)
        big = big_w.matmul(big_x)
        others = [torch.full((1 << e,), 7, dtype=torch.uint8, device="cuda") for e in range(9, 21) for _ in range(8)]
        for _ in range(3):
            g.replay()
            again = big_w.matmul(big_x)
    s.synchronize()
    check(y, x, p.dequantize())
    assert torch.equal(big, again) and all((o == 7).all() for o in others)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", ["inf", "-inf", "nan"])
def test_a_group_with_a_non_finite_weight_is_nan(bad, dtype):
    w = normal((20, 256), 1, 0.02, DT[dtype])
    w[3, 70] = float(bad)
    p = lib.W4Weight(w, 64)
    d = p.dequantize()
    assert torch.isnan(d[3, 64:128]).all() and torch.isfinite(d).sum() == d.numel() - 64
    assert torch.isnan(p.matmul(normal((3, 256), 2, 1.0, DT[dtype]))[:, 3]).all()


def test_pack_of_groups_whose_scale_has_no_finite_inverse():
    """bf16 scales below 2^-128 (their inverse passes fp32): zeros, for the group's zeros too."""
    w = torch.zeros(16, 128, device="cuda")
    w[0, 3], w[1, ::2], w[2, 5] = 2.0 ** -129 * 7, -(2.0 ** -130) * 7, 2.0 ** -120 * 7
    p = lib.W4Weight(w, 32)
    want = torch.zeros_like(w)
    want[2, 5] = 2.0 ** -120 * 7
    assert torch.equal(p.dequantize(), want)
    assert torch.isfinite(p.matmul(normal((2, 128), 1))).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [1, 5, 16])
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("size", [1e4, 1e6])
def test_matmul_beside_an_outlier_that_the_weights_do_not_see(size, group, rows, dtype):
    """An activation that is much larger than the others, at a column whose codes are 0, adds nothing and costs
    the others nothing: the bound is that of sum |x w|, without it.  fp32 rows are held to 2^-39 of a chunk's
    largest magnitude."""
    w = normal((200, 384), 1, 0.02)
    w[:, 70], w[:, 301] = 0, 0
    p = lib.W4Weight(w, group)
    x = normal((rows, 384), 2, 1.0)
    x[:, 70], x[:, 301] = size, -size
    x = x.to(DT[dtype])
    y, d = p.matmul(x), p.dequantize().double()
    assert (d[:, 70] == 0).all() and (d[:, 301] == 0).all()
    want, total = x.double() @ d.T, x.double().abs() @ d.abs().T
    bound = (384 / 8 + 64) * 2.0 ** -24 * total
    if dtype == "fp32":
        bound = bound + 2.0 ** -39 * size * d.abs().sum(1)
    else:
        bound = bound + 2.0 ** -8 * want.abs()
    err = (y.double() - want).abs()
    assert (err <= bound).all(), f"{(err > bound).sum().item()} of {err.numel()}, worst {(err / bound).max().item()}"


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_matmul_into_the_buffer_of_its_rows(dtype):
    """Columns beside x and the residual are fine; columns of theirs are refused."""
    w = lib.W4Weight(normal((128, 128), 1, 0.05), 64)
    buf = normal((5, 3 * 128), 2, 1.0, DT[dtype])
    x, out, res = buf[:, :128], buf[:, 128:256], buf[:, 256:]
    before = buf.clone()
    w.matmul(x, out=out, residual=res)
    check(out, before[:, :128], w.dequantize(), before[:, 256:])
    assert torch.equal(x, before[:, :128]) and torch.equal(res, before[:, 256:])
    keep = buf.clone()
    for f in (lambda: w.matmul(x, out=x), lambda: w.matmul(x, out=buf[:, 127:255]), lambda: w.matmul(x[:3], out=x[2:]),
              lambda: w.matmul(x, out=out, residual=buf[:, 129:257])):
        with pytest.raises(lib.SSDError) as e:
            f()
        assert e.value.status == 1 and "overlaps" in str(e.value)
    assert torch.equal(buf, keep)
    w.matmul(x[:2], out=buf[2:4, :128])   # other rows of the same columns
    check(buf[2:4, :128], keep[:2, :128], w.dequantize())
