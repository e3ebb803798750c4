"""Operators on rows on the GPU: 4-bit floats, head norms with rotary positions, sampling, against 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2510_22641_gb300 as lib
from tests import rows_ref as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def normal(shape, seed, scale=1.0, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def uneven(rows, k, seed, dtype=torch.float32):
    """Rows and channels of very different size."""
    return (normal((rows, k), seed) * torch.exp(normal((rows, 1), seed + 1)) * torch.exp(normal((1, k), seed + 2))).to(dtype)


# ----------------------------------------------------------------------------------------- 4-bit floats

def check_packed(x):
    """Every quotient and rounding is defined, so the values are equal; c * s has 6 bits, which bf16 holds."""
    p = lib.F4Rows(x)
    want = ref.f4_values(x.float().cpu().numpy())
    got = p.dequantize().cpu().numpy()
    with np.errstate(over="ignore"):
        assert np.array_equal(got, want.astype(np.float32), equal_nan=True)
    assert np.array_equal(p.dequantize(torch.bfloat16).float().cpu().numpy(), got, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,k", [(1, 1), (1, 16), (3, 17), (16, 256), (7, 257), (130, 512), (129, 1000), (5, 2055),
                                    (300, 48), (2, 14336), (1, 40000), (33, 1001), (17, 3001), (9, 513), (300, 2)])
def test_pack_equals_the_reference(rows, k, dtype):
    check_packed(uneven(rows, k, rows + k, DT[dtype]))


def test_pack_of_many_rows():
    x = uneven(70001, 24, 1)
    got = lib.F4Rows(x).dequantize().cpu().numpy()
    some = np.r_[0:200, 65500:65600, 69900:70001]
    assert np.array_equal(got[some], ref.f4_values(x[torch.from_numpy(some).cuda()].cpu().numpy()).astype(np.float32))


def test_pack_of_zeros_extremes_and_ties():
    x = torch.zeros(14, 288, device="cuda")
    x[1, 5], x[2, 0], x[2, 1] = 1e-30, 3.4e38, -1e38
    x[3] = -7.0
    x[4, ::2] = 1e-40
    x[5, 3], x[5, 40] = 2688, 1e-3
    x[6, 3] = 2688.0002
    x[7, 100] = float("inf")
    x[8, 200], x[8, 3] = float("nan"), 1.0
    x[9, 0], x[9, 32:40] = 2688, torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6]).cuda()   # codes between two
    x[10, 0], x[10, 16], x[10, 32], x[10, 48] = 2688, 6 * 2.0 ** -10, 6 * 3 * 2.0 ** -10, 6 * 2.0 ** -11  # scales between two
    x[11, 287] = 1.0
    x[12, 0], x[12, 16:32] = 6 * 2.0 ** -100, 2.0 ** -109
    x[13, :4] = torch.tensor([-0.0, 1e-45, 2.0 ** -126, -(2.0 ** -100)]).cuda()
    check_packed(x)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_pack_of_views(dtype):
    base = uneven(40, 700, 3, DT[dtype])
    for v in (base[1:30, 7:507], base[::2, 8:520], base[:, 1:17], base.flip(0)[3:9, :300]):
        check_packed(v)


def check_product(y, x, w, residual=None):
    """fp32 sums of k exact products (taken as (k / 8 + 64) 2^-24 of sum |x w|), a residual's addition, and bf16's
    rounding at the end."""
    xd, wd = x.double(), w.double()
    want, size = xd @ wd.T, xd.abs() @ wd.abs().T
    if residual is not None:
        want, size = want + residual.double(), size + residual.double().abs()
    bound = (x.shape[1] / 8 + 64) * 2.0 ** -24 * size
    if y.dtype is torch.bfloat16:
        bound = bound + 2.0 ** -8 * want.abs()
    err = (y.double() - want).abs()
    assert (err <= bound).all(), f"{(err > bound).sum().item()} of {err.numel()}, worst {(err / bound).max().item()}"


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [1, 2, 7, 16, 17, 33, 64, 96, 129, 256, 257, 515])
@pytest.mark.parametrize("n,k", [(1, 1), (16, 64), (100, 300), (129, 257), (513, 1000), (4096, 512), (250, 4096)])
def test_product(rows, n, k, dtype):
    w = lib.F4Weight(normal((n, k), 1, 0.02, torch.bfloat16))
    x = uneven(rows, k, 2, DT[dtype])
    y = w.matmul(x, out=torch.full((rows, n), float("nan"), dtype=x.dtype, device="cuda"))
    packed = lib.F4Rows(x)
    check_product(y, packed.dequantize(), w.dequantize())
    assert torch.equal(y, w.matmul(x))           # the same bits every time
    assert torch.equal(y, w.matmul(packed))      # and from rows that were packed before


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("n,k", [(1, 16), (130, 255), (4096, 4096), (20000, 4096), (70, 16384), (300, 5000)])
def test_product_that_packs_its_rows(rows, n, k, dtype):
    """Few short rows have no launch of their own: the same bits as of rows packed before, any alignment."""
    w = lib.F4Weight(normal((n, k), 1, 0.02, torch.bfloat16))
    base = uneven(rows, k + 8, 2, DT[dtype])
    for x in (base[:, :k], base[:, 1:k + 1], base[:, 8:k + 8]):
        packed = lib.F4Rows(x)
        y = w.matmul(x)
        assert torch.equal(y, w.matmul(packed))
        check_product(y, packed.dequantize(), w.dequantize())


@pytest.mark.parametrize("rows,n,k", [(1, 30000, 2048), (5, 64, 14336), (40, 11000, 5120), (640, 4096, 2048), (3001, 1300, 768),
                                      (1000, 9001, 1040), (8192, 200, 160)])
def test_product_of_large_shapes(rows, n, k):
    w = lib.F4Weight(normal((n, k), 1, 0.02, torch.bfloat16))
    x = uneven(rows, k, 2)
    check_product(w.matmul(x), lib.F4Rows(x).dequantize(), w.dequantize())


@pytest.mark.parametrize("n,k", [(4096, 1000), (300, 5120), (22016, 512)])
def test_rows_of_a_product_do_not_depend_on_their_company(n, k):
    w, x = lib.F4Weight(normal((n, k), 1, 0.02)), uneven(700, k, 2)
    few, many = w.matmul(x[:128]), w.matmul(x)
    for m in (1, 3, 5, 16, 17, 40, 64, 65, 100):
        assert torch.equal(w.matmul(x[:m]), few[:m]) and torch.equal(w.matmul(x[128 - m:128]), few[128 - m:])
    for m in (129, 150, 256, 257, 500):
        assert torch.equal(w.matmul(x[:m]), many[:m])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [1, 6, 150, 300])
def test_product_adds_a_residual_and_takes_views(rows, dtype):
    n, k = 300, 520
    w = lib.F4Weight(normal((n, k), 1, 0.02))
    xs = normal((rows, k + 9), 2, 1.0, DT[dtype])
    res = normal((rows, n + 5), 3, 1.0, DT[dtype])
    out = torch.full((rows + 2, n + 3), float("nan"), dtype=DT[dtype], device="cuda")
    for x in (xs[:, :k], xs[:, 1:k + 1], xs[:, 8:k + 8]):
        w.matmul(x, out=out[1:rows + 1, 1:n + 1], residual=res[:, 2:n + 2])
        check_product(out[1:rows + 1, 1:n + 1], lib.F4Rows(x).dequantize(), w.dequantize(), res[:, 2:n + 2])
        edge = out.clone()
        edge[1:rows + 1, 1:n + 1] = float("nan")
        assert torch.isnan(edge).all()
    y = res[:, :n].contiguous()
    want = w.matmul(xs[:, :k], residual=y.clone())
    assert torch.equal(w.matmul(xs[:, :k], out=y, residual=y), want)   # in place
    wide = w.matmul(xs[:, :k], residual=y.expand(rows, n), out=out[1:rows + 1, 2:n + 2])
    assert wide.data_ptr() == out[1:, 2:].data_ptr()


def test_product_of_rows_that_are_not_finite():
    """Such a row is NaN in full, of x and of w, and leaves the others alone."""
    x, wt = normal((40, 300), 1), normal((200, 300), 2, 0.02)
    clean = lib.F4Weight(wt).matmul(x)
    x[3, 5], x[39, 299], wt[130, 0] = float("nan"), float("inf"), float("-inf")
    y = lib.F4Weight(wt).matmul(x)
    bad = torch.zeros_like(y, dtype=torch.bool)
    bad[[3, 39]] = True
    bad[:, 130] = True
    assert torch.isnan(y[bad]).all() and torch.equal(y[~bad], clean[~bad])


def test_product_of_extreme_sizes():
    """Neither factor alone may carry a sum out of range: 2^120 rows times 2^-90 weights, and back."""
    for e, f in ((110, -90), (-90, 110), (120, 0), (-60, -60)):
        x, wt = normal((5, 64), 1) * 2.0 ** e, normal((20, 64), 2) * 2.0 ** f
        w = lib.F4Weight(wt)
        check_product(w.matmul(x), lib.F4Rows(x).dequantize(), w.dequantize())


def test_product_of_no_rows():
    assert lib.F4Weight(normal((20, 64), 1)).matmul(torch.empty(0, 64, device="cuda")).shape == (0, 20)


def test_other_rows_in_the_same_buffer():
    a, b = normal((20, 100), 1), normal((20, 100), 2, 3.0, torch.bfloat16)
    p = lib.F4Rows(a)
    first = p.dequantize()
    assert torch.equal(p.pack(b).dequantize(), lib.F4Rows(b).dequantize()) and p.dtype is torch.bfloat16
    assert torch.equal(p.pack(a).dequantize(), first)


def test_streams_and_graphs_of_products():
    """Products on two streams at once, and one captured into a graph and replayed over other values."""
    w = lib.F4Weight(normal((700, 600), 1, 0.02))
    xs = [normal((m, 600), m) for m in (1, 40, 300)]
    want = [w.matmul(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    for _ in range(20):
        got = []
        for s, x in zip(streams, xs):
            with torch.cuda.stream(s):
                got.append(w.matmul(x))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    buf = [x.clone() for x in xs]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = [w.matmul(b) for b in buf]
    for b in buf:
        b.mul_(-2)
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, -2 * b) for a, b in zip(out, want))   # powers of two move the row scales alone


# ----------------------------------------------------------------------------------------- rotary positions

def check_heads(y, want, size, dtype):
    """Against |a| + |b| of the pair: sine and cosine 2^-22, three roundings, and 16 for a norm (13 additions of
    positive squares, half of whose error the root leaves, the root, the quotient, two products): 23 * 2^-24."""
    bound = torch.from_numpy(2.0 ** -19 * size + (2.0 ** -8 * np.abs(want) if dtype is torch.bfloat16 else 0)).cuda()
    err = (y.double() - torch.from_numpy(want).cuda()).abs()
    assert (err <= bound + 1e-40).all(), f"{(err > bound).sum().item()} of {err.numel()}, worst {(err / bound).max().item()}"


def freqs(turn, theta):
    return [theta ** (-2 * i / turn) for i in range(turn // 2)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("rows,heads,kv,dim,turn", [(1, 1, 1, 2, 2), (1, 32, 32, 128, 128), (96, 32, 8, 128, 128), (7, 5, 1, 80, 40),
                                                    (33, 8, 8, 64, 64), (5, 40, 40, 96, 48), (300, 4, 1, 256, 256),
                                                    (3, 7, 3, 80, 80), (4, 3, 2, 6, 4), (9, 2, 1, 100, 100), (2, 64, 8, 64, 0),
                                                    (6, 3, 1, 24, 24), (1200, 16, 2, 128, 64), (5, 3, 3, 250, 30)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary(rows, heads, kv, dim, turn, norm, dtype, interleaved):
    axes = 1 + (rows + dim) % 3 if turn >= 6 else 1
    cut = [turn // 2 // axes] * (axes - 1)
    sections = cut + [turn // 2 - sum(cut)]
    r = lib.Rotary(dim, turn, 5e5, sections, interleaved, 1e-6)
    qkv = (normal((rows, heads + 2 * kv, dim), 1) * torch.exp(normal((rows, heads + 2 * kv, 1), 2))).to(DT[dtype])
    q, k = qkv[:, :heads], qkv[:, heads:heads + kv]
    pos = torch.randint(0, 1 << 20, (rows, axes), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    qg = (1 + 0.1 * normal((dim,), 4)).to(torch.bfloat16) if norm else None
    kg = 1 + 0.1 * normal((dim,), 5) if norm else None
    qo, ko = r.rotate(q, k, pos, qg, kg)
    axis = sum(([a] * n for a, n in enumerate(sections)), [])
    for x, y, g in ((q, qo, qg), (k, ko, kg)):
        want, size = ref.rotary(x.double().cpu().numpy(), pos.cpu().numpy(), freqs(turn, 5e5), axis, turn, interleaved,
                                None if g is None else g.double().cpu().numpy(), 1e-6)
        check_heads(y, want, size, x.dtype)
    before = qkv[:, heads + kv:].clone()
    q2, k2 = r.rotate(q, k, pos, qg, kg, q_out=q, k_out=k)   # in place; v between the rows' heads stays
    assert torch.equal(q2, qo) and torch.equal(k2, ko) and torch.equal(qkv[:, heads + kv:], before)


@pytest.mark.parametrize("pos", [0, 1, -1, 131071, 2 ** 31 - 1, -2 ** 31])
def test_rotary_at_any_position(pos):
    """Far positions keep their angles: the reference turns by integers of 2^-80 of a turn."""
    dim, theta = 64, 1e4
    x = normal((1, 2, dim), 1)
    y, none = lib.Rotary(dim, theta=theta).rotate(x, None, torch.tensor([pos], dtype=torch.int32, device="cuda"))
    assert none is None
    for i in range(dim // 2):
        # theta^(-2 i / dim) = 10^(-i / 8): exact decimal digits by integers
        f = 10.0 ** (-(i / 8))
        turn = math.fmod(pos * f, 2 * math.pi)     # f to 2^-53: 2^31 * 2^-53 = 2^-22 of a radian
        c, s = math.cos(turn), math.sin(turn)
        a, b = x[0, :, i].double(), x[0, :, i + dim // 2].double()
        bound = (2.0 ** -21 + 2.0 ** -20 * (abs(pos) > 1 << 20)) * (a.abs() + b.abs())
        assert ((y[0, :, i].double() - (a * c - b * s)).abs() <= bound).all(), i
        assert ((y[0, :, i + dim // 2].double() - (b * c + a * s)).abs() <= bound).all(), i


def test_rotary_layouts():
    """Heads before rows, broadcast rows, positions of one axis as a column, queries alone, given axes."""
    x = normal((4, 9, 64), 1).transpose(0, 1)           # [9 rows][4 heads][64], head stride > row stride
    one = normal((1, 4, 64), 2).expand(9, 4, 64)
    pos = torch.arange(9, dtype=torch.int32, device="cuda")
    r = lib.Rotary(64)
    a, b = r.rotate(x, one, pos)
    c, d = r.rotate(x.contiguous(), one.contiguous(), torch.stack([pos, pos], 1)[:, :1])
    assert torch.equal(a, c) and torch.equal(b, d)
    again, _ = lib.Rotary(64, axes=[0] * 32, freqs=freqs(64, 1e4)).rotate(x, None, pos)
    assert (again - a).abs().max() < 1e-5
    odd = torch.empty(9 * 4 * 64 + 1, device="cuda")[1:].view(9, 4, 64).copy_(x)   # not aligned to 16 bytes
    assert torch.equal(r.rotate(odd, None, pos)[0], a)
    assert r.rotate(x[:0], None, pos[:0])[0].shape == (0, 4, 64)
    with pytest.raises(lib.SSDError):
        r.rotate(one, None, pos, q_out=one)
    with pytest.raises(lib.SSDError):
        r.rotate(x, None, pos.long())
    with pytest.raises(lib.SSDError):
        lib.Rotary(64, sections=[16, 16]).rotate(x, None, pos)


def test_rotary_leaves_values_that_are_not_finite_in_their_pairs():
    x = normal((2, 3, 64), 1)
    x[1, 2, 5], x[0, 0, 40] = float("nan"), float("inf")
    pos = torch.tensor([3, 7], dtype=torch.int32, device="cuda")
    y, _ = lib.Rotary(64).rotate(x, None, pos)
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[1, 2, [5, 37]] = want[0, 0, [8, 40]] = True
    assert torch.equal(bad, want)
    z, _ = lib.Rotary(64).rotate(x, None, pos, torch.ones(64, device="cuda"))
    assert torch.isnan(z[1, 2]).all() and torch.isfinite(z[1, :2]).all() and torch.isfinite(z[0, 1:]).all()


# ----------------------------------------------------------------------------------------- sampling

def check_tokens(logits, u, how, got):
    """Tokens equal the 64-bit reference's, but where the draw or a border is within 2^-30 of a token's edge."""
    token, prob = (x.cpu().numpy() for x in got)
    z = logits.float().cpu().numpy()
    for r in range(len(z)):
        # settings are 32-bit numbers: 1.3 as one is 2^-25 off, which times (z - max z) / T shows in prob
        t, k, p, m = (h[r].item() if torch.is_tensor(h) else h if isinstance(h, int) else float(np.float32(h)) for h in how)
        ur = u[r].item()
        want, share = ref.sample(z[r], ur, t, k, p, m)
        if token[r] != want:
            near = {ref.sample(z[r], ur + d, t, k, p + e, m)[0] for d in (-2.0 ** -30, 2.0 ** -30) for e in (-2.0 ** -30, 2.0 ** -30)}
            assert token[r] in near, (r, token[r], want, t, k, p, m)
        else:
            assert abs(prob[r] - share) <= 2.0 ** -23 * share, (r, prob[r], share)


def logits_of(rows, vocab, seed, dtype=torch.float32):
    z = 2.5 * normal((rows, vocab), seed)
    z[:, :: max(1, vocab // 20)] += 6 * normal((rows, len(range(0, vocab, max(1, vocab // 20)))), seed + 1).abs()
    return z.to(dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (40, 7), (5, 1000), (33, 4097), (2, 32000), (3, 70001), (1, 262144)])
@pytest.mark.parametrize("how", [(0.0, 0, 1.0, 0.0), (1.0, 0, 1.0, 0.0), (0.7, 0, 0.9, 0.0), (1.3, 40, 1.0, 0.0),
                                 (1.0, 300, 0.5, 0.0), (0.9, 0, 0.97, 0.05), (1.5, 0, 1.0, 0.01), (1.0, 1, 0.3, 0.9),
                                 (2.0, 5000, 0.999, 0.0), (1.0, 0, 0.0, 0.0), (1.0, -3, 1.5, 2.0), (0.01, 50, 0.9, 0.0)], ids=str)
def test_sample(rows, vocab, how, dtype):
    z, u = logits_of(rows, vocab, rows + vocab, DT[dtype]), torch.rand(rows, generator=torch.Generator().manual_seed(9)).cuda()
    check_tokens(z, u, how, lib.sample(z, u, *how, with_prob=True))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_sample_with_settings_for_each_row(dtype):
    rows, vocab = 60, 5003
    g = torch.Generator().manual_seed(1)
    pick = lambda *v: torch.tensor(v)[torch.randint(0, len(v), (rows,), generator=g)].cuda()  # noqa: E731
    how = (pick(0.0, 0.6, 1.0, 1.7), pick(0, 1, 50, 2000).int(), pick(1.0, 0.95, 0.5), pick(0.0, 0.02, 0.3))
    wide = logits_of(rows, vocab + 30, 4, DT[dtype])
    u = torch.rand(rows, generator=g).cuda()
    for z in (wide[:, :vocab], wide[:, 3:vocab + 3]):     # rows longer than the vocabulary, any alignment
        a = lib.sample(z, u, *how, with_prob=True)
        check_tokens(z, u, how, a)
        b = lib.sample(z.contiguous(), u, *how, with_prob=True)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    out = torch.empty(rows, dtype=torch.int32, device="cuda")
    assert lib.sample(z, u, *how, out=out).data_ptr() == out.data_ptr() and torch.equal(out, a[0])


@pytest.mark.parametrize("vocab", [50, 5000, 100001])
def test_sample_of_equal_logits(vocab):
    """Borders inside a run of equal logits fall by index."""
    z = torch.zeros(6, vocab, device="cuda")
    z[1, vocab // 2] = 1.0
    z[2, ::3] = -0.0
    z[3] = torch.arange(vocab, device="cuda") % 3
    z[4] = 300.0
    z[5, 7:] = -1e30
    for how in ((1.0, 0, 1.0, 0.0), (1.0, 10, 1.0, 0.0), (1.0, 0, 0.301, 0.0), (1.0, vocab - 7, 0.77, 0.2)):
        for v in (0.0, 0.29, 0.6181, 0.9999):
            u = torch.full((6,), v, device="cuda")
            check_tokens(z, u, how, lib.sample(z, u, *how, with_prob=True))


def test_sample_of_values_that_are_not_finite():
    inf, nan = float("inf"), float("nan")
    rows = [[nan, nan, nan, nan], [-inf] * 4, [nan, 1.0, -inf, 1.0], [inf, 0.0, inf, nan], [-inf, -1e38, nan, -inf],
            [3e38, -3e38, 3e38, 0.0], [1e-45, 0.0, -1e-45, nan], [nan, inf, -inf, 5.0]]
    z = torch.tensor(rows, device="cuda")
    for v in (0.0, 0.3, 0.6, 0.99):
        u = torch.full((len(rows),), v, device="cuda")
        for how in ((1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (2.0, 2, 0.9, 0.1), (1e30, 0, 0.7, 0.0), (1e-30, 3, 1.0, 0.0)):
            check_tokens(z, u, how, lib.sample(z, u, *how, with_prob=True))


def test_sample_of_random_numbers_and_settings_out_of_range():
    z = logits_of(5, 3000, 2)
    nan = float("nan")
    for v, as_if in ((1.0, None), (7.0, None), (-1.0, 0.0), (nan, 0.0)):
        t, p = lib.sample(z, torch.full((5,), v, device="cuda"), with_prob=True)
        if as_if is None:
            assert (t > 2900).all() and (p > 0).all()
        else:
            assert torch.equal(t, lib.sample(z, torch.zeros(5, device="cuda")))
    u = torch.full((5,), 0.4, device="cuda")
    assert torch.equal(lib.sample(z, u, nan), lib.sample(z, u, 0.0))
    assert torch.equal(lib.sample(z, u, 1.0, 0, nan, nan), lib.sample(z, u))
    assert torch.equal(lib.sample(z, u, -1.0), z.argmax(1).int())


def test_sample_follows_the_distribution():
    """Over a grid of u every token comes as often as its mass says, to one step of the grid."""
    z = logits_of(1, 40, 3).expand(4096, 40)
    u = (torch.arange(4096, device="cuda") + 0.5) / 4096
    t = lib.sample(z, u, 1.2)
    share = torch.bincount(t.long(), minlength=40).double() / 4096
    assert ((share - (z[0].double() / 1.2).softmax(0)).abs() <= 1.01 / 4096).all()


def test_streams_and_graphs_of_sampling():
    z, u = logits_of(20, 9000, 5), torch.rand(20, generator=torch.Generator().manual_seed(2)).cuda()
    want = lib.sample(z, u, 0.9, 60, 0.9)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = lib.sample(z, u, 0.9, 60, 0.9)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    zb, ub = torch.zeros_like(z), torch.zeros_like(u)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = lib.sample(zb, ub, 0.9, 60, 0.9)
    zb.copy_(z), ub.copy_(u)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


# ----------------------------------------------------------------------------------------- large operands

def test_offsets_past_32_bits():
    """More than 2^31 elements in every operand that can have them; the last rows are looked at."""
    some = normal((40, 16384), 1).to(torch.bfloat16)
    x = torch.zeros(132000, 16384, dtype=torch.bfloat16, device="cuda")
    x[-40:] = some
    p = lib.F4Rows(x)
    w = lib.F4Weight(normal((32, 16384), 2))
    want = lib.F4Rows(some).dequantize()
    y = w.matmul(p)
    check_product(y[-40:], want, w.dequantize())
    assert not y[:-40].any()
    assert torch.equal(p.dequantize(torch.bfloat16)[-40:].float(), want)
    del x, p, y
    xs, wide = normal((8200, 64), 3), lib.F4Weight(normal((263000, 64), 4))
    y = wide.matmul(xs)
    check_product(y[-2:], lib.F4Rows(xs).dequantize()[-2:], wide.dequantize())
    del y, wide
    torch.cuda.empty_cache()
    heads = torch.zeros(300000, 64, 128, dtype=torch.bfloat16, device="cuda")
    heads[-3:] = normal((3, 64, 128), 5)
    pos = torch.arange(300000, dtype=torch.int32, device="cuda")
    last = lib.Rotary(128).rotate(heads[-3:].contiguous(), None, pos[-3:])[0]
    assert torch.equal(lib.Rotary(128).rotate(heads, None, pos, q_out=heads)[0][-3:], last)
    del heads
    torch.cuda.empty_cache()
    z = torch.zeros(8200, 262144, device="cuda")
    z[-5:] = logits_of(5, 262144, 6)
    u = torch.rand(8200, generator=torch.Generator().manual_seed(7)).cuda()
    token, prob = lib.sample(z, u, 1.0, 0, 0.9, 0.0, with_prob=True)
    check_tokens(z[-5:], u[-5:], (1.0, 0, 0.9, 0.0), (token[-5:], prob[-5:]))
    flat = token[:-5].cpu().numpy()
    kept = math.ceil(float(np.float32(0.9)) * 262144)   # equal logits: the first of them by index
    assert np.array_equal(flat, np.minimum(np.floor(u[:-5].cpu().double().numpy() * kept), kept - 1).astype(np.int32))


def test_two_large_products_at_once():
    w = [lib.F4Weight(normal((3000, 2048), s, 0.02)) for s in (1, 2)]
    x = [normal((m, 2048), m) for m in (900, 700)]
    want = [a.matmul(b) for a, b in zip(w, x)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in w]
    for _ in range(10):
        got = []
        for s, a, b in zip(streams, w, x):
            with torch.cuda.stream(s):
                got.append(a.matmul(b))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
