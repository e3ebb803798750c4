"""The paged 8-bit K/V cache on the GPU: block tables and slots, quantising appends, reads and attention
against the plain references of tests/lowbit_ref.py."""
import numpy as np
import pytest
import torch

import paper_2510_22641_gb300 as lib
from tests import lowbit_ref as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def rows(shape, seed, dtype, spread=0.7):
    """K / V rows whose size varies from token to token, so that block scales grow."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp(spread * torch.randn(shape[:2] + (1,), generator=g))
    return x.to(dtype).cuda()


# ------------------------------------------------------------------------------------------ plan

class Planned:
    """A cache beside the reference's lists."""

    def __init__(self, block, n_blocks, seats, wide, seed=0):
        self.cache = lib.KV8Cache(1, 1, 1, 64, block, n_blocks, seats, wide)
        self.free = np.random.RandomState(seed).permutation(n_blocks).tolist()
        self.cache.pool.copy_(ints(self.free))
        self.table, self.held = [[-1] * wide for _ in range(seats)], [0] * seats
        self.block, self.wide, self.seats = block, wide, seats

    def step(self, length, add, rows=None, state=None):
        n = len(length)
        rows = sum(a for l, a in zip(length, add) if l >= 0) if rows is None else rows
        step = self.cache.new_step(n, rows)
        self.cache.plan(step, ints(length), ints(add))
        table, held, self.free, start, slot = ref.plan(length, add, self.held[:n], self.free, self.table[:n], self.block,
                                                       self.wide, rows)
        self.table[:n], self.held[:n] = table, held
        assert step.row_start.tolist() == start
        assert step.slot.tolist() == slot[:rows]
        got = self.cache.table.tolist()
        for b in range(self.seats):
            assert got[b][:self.held[b]] == self.table[b][:self.held[b]], b
        assert self.cache.state.tolist() == [len(self.free)] + self.held
        assert self.cache.pool[:len(self.free)].tolist() == self.free
        assert step.length.tolist() == [max(l, 0) for l in length]
        return step


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("seats", [1, 3, 33, 300, 1024])
def test_plan_follows_the_reference_over_steps(block, seats):
    rng = np.random.RandomState(block + seats)
    wide = 9
    p = Planned(block, seats * 6 + 3, seats, wide, seed=block)
    length = [0] * seats
    for it in range(6):
        n = seats if it % 2 == 0 else max(1, seats - 2)
        most = 5 * block if it == 0 else 17
        add = [int(rng.randint(0, most)) for _ in range(n)]
        add = [min(a, wide * block - l) if l >= 0 else a for l, a in zip(length, add)]
        now = [-1 if it in (2, 4) and rng.rand() < 0.3 else l for l in length[:n]]
        p.step(now, add, rows=sum(a for l, a in zip(now, add) if l >= 0) + (5 if it == 1 else 0))
        for b in range(n):
            if now[b] < 0:
                length[b] = 0
            else:   # some of the new rows are rolled back
                length[b] = now[b] + int(rng.randint(0, add[b] + 1)) if it else now[b] + add[b]
        bits = status(p.cache)
        assert bits & ~1 == 0   # running out of blocks is part of the test


def status(cache):
    try:
        cache.check()
    except lib.SSDError as e:
        assert e.status == 7
        text = str(e)
        return 1 * ("out of blocks" in text) + 2 * ("length" in text) + 4 * ("slot" in text) + 8 * ("non-finite" in text)
    return 0


def test_plan_runs_out_of_blocks_and_recovers():
    p = Planned(16, 4, 3, 4)
    step = p.step([0, 0, 0], [33, 16, 20])   # 3 + 1 + 2 blocks of 4
    assert step.slot.tolist()[-20:] == [-1] * 20
    assert status(p.cache) == 1
    p.step([33, -1, 0], [0, 0, 20])          # seat 1 gives its block back, seat 2 takes it
    assert status(p.cache) == 1              # one block is still missing
    p.step([-1, 0, 0], [0, 0, 20])
    assert status(p.cache) == 0
    p.step([0, 0, 20], [0, 0, 1])
    assert status(p.cache) == 0


def test_plan_flags_and_clamps_bad_input():
    for length, add, rows, bits in (([70], [0], 0, 2), ([60], [9], 9, 2), ([0], [-3], 0, 2), ([0, 0], [3, 3], 4, 2),
                                    ([-7], [1], 1, 2), ([2 ** 31 - 1], [2 ** 31 - 1], 4, 2)):
        c = lib.KV8Cache(1, 1, 1, 64, 16, 10, 2, 4)
        step = c.new_step(len(length), rows)
        c.plan(step, ints(length), ints(add))
        assert status(c) == bits, (length, add)
        assert step.row_start[-1].item() <= rows
        assert all(-1 <= s < 160 for s in step.slot.tolist())
        assert status(c) == 0   # read once, cleared
    c = lib.KV8Cache(1, 1, 1, 64, 16, 4, 2, 4)
    c.pool.fill_(77)            # ids outside the cache are not handed out
    step = c.new_step(1, 5)
    c.plan(step, ints([0]), ints([5]))
    assert status(c) == 4 and step.slot.tolist() == [-1] * 5
    c.state.fill_(99)
    c.plan(step, ints([0]), ints([5]))
    assert status(c) & 2


def test_plan_with_states_apart_repeats():
    c = lib.KV8Cache(1, 1, 1, 64, 16, 20, 3, 6)
    out = torch.full_like(c.state, -5)
    before = c.state.clone()
    step = c.new_step(2, 40)
    seen = []
    for _ in range(3):
        c.plan(step, ints([0, 0]), ints([17, 23]), state=c.state, state_out=out)
        seen.append((out.tolist(), step.slot.tolist(), c.table.tolist()))
    assert seen[0] == seen[1] == seen[2]
    assert torch.equal(c.state, before) and out.tolist() == [20 - 4, 2, 2, 0]


# ------------------------------------------------------------------------------------------ append / read

class Filled:
    """A cache and its reference, filled by steps of ragged rows."""

    def __init__(self, block, heads, kv_heads, dim, seats, wide, dtype, layers=1, layer=0, extra=3, seed=0):
        n_blocks = seats * wide + extra
        self.cache = lib.KV8Cache(layers, heads, kv_heads, dim, block, n_blocks, seats, wide)
        self.cache.pool.copy_(ints(np.random.RandomState(seed).permutation(n_blocks).tolist()))
        self.ref = [ref.Cache(n_blocks, block, kv_heads, dim) for _ in range(2)]
        self.shape, self.dtype, self.layer, self.block = (kv_heads, dim), dtype, layer, block
        self.length, self.seed = [0] * seats, seed

    def append(self, add, kv=None, **step_args):
        n = sum(add)
        self.step = self.cache.new_step(len(add), n, **step_args)
        self.cache.plan(self.step, ints(self.length[:len(add)]), ints(add))
        self.seed += 2
        self.kv = kv or [rows((n,) + self.shape, self.seed + i, self.dtype) for i in range(2)]
        self.cache.append(self.layer, self.kv[0], self.kv[1], self.step)
        slot = self.step.slot.tolist()
        for r, x in zip(self.ref, self.kv):
            r.append(x.float().cpu().numpy(), slot)
        self.before = list(self.length)
        for b, a in enumerate(add):
            self.length[b] += a
        self.add = list(add)
        return slot

    def slots_of(self, b, n=None):
        t = self.cache.table[b].tolist()
        n = self.length[b] if n is None else n
        return [t[i // self.block] * self.block + i % self.block for i in range(n)]

    def check_values(self):
        slots = sum((self.slots_of(b) for b in range(len(self.length))), [])
        k, v = self.cache.read(self.layer, ints(slots))
        for got, r in zip((k, v), self.ref):
            assert np.array_equal(got.cpu().numpy(), r.values(slots))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim,heads,block", [(128, 3, 16), (64, 1, 16), (128, 2, 32), (64, 5, 64), (128, 1, 128),
                                             (64, 4, 128)])
def test_append_equals_the_reference(dim, heads, block, dtype):
    f = Filled(block, heads, heads, dim, 4, 5, DT[dtype])
    for add in ([1, 0, block, 2 * block + 5], [1, 3, 1, 16], [block - 2, 7, 0, 1], [1, 1, 1, 1], [17, 0, 2, 0]):
        f.append(add)
        f.check_values()
    f.length = [max(0, l - 5) for l in f.length]   # rejected drafts: shorter lengths, rows overwritten
    f.append([4, 4, 4, 4])
    f.check_values()
    assert status(f.cache) == 0


def test_append_of_a_long_prompt_and_its_error_bound():
    """More than 4096 rows; every value is within half a step of its scale of what was appended."""
    f = Filled(64, 2, 2, 128, 2, 80, torch.bfloat16)
    f.append([4500, 1003])
    f.check_values()
    slots = f.step.slot.tolist()
    k, _ = f.cache.read(0, f.step.slot)
    scale = f.ref[0].scales[np.array(slots) // 64][:, :, None].astype(np.float64)
    err = np.abs(k.double().cpu().numpy() - f.kv[0].double().cpu().numpy())
    assert (err <= scale * (0.5 + 127 * 2.0 ** -22)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append_takes_views_and_unaligned_rows(dtype):
    h, d, n = 2, 64, 21
    fused = rows((n, 3 * h, d + 1), 5, DT[dtype])
    wide = rows((n, 2 * h, 2 * d), 6, DT[dtype])
    for k, v in ((fused[:, h:2 * h, 1:], fused[:, 2 * h:, :d]), (wide[:, ::2, d:], wide[:, 1::2, :d]),
                 (wide[:, :h, 3:3 + d], wide[:, h:, 1:1 + d])):
        f = Filled(16, h, h, d, 1, 4, DT[dtype])
        f.append([n], kv=[k, v])
        f.check_values()


def test_append_and_read_of_layers_do_not_mix():
    fs = [Filled(32, 2, 2, 64, 2, 2, torch.float32, layers=3, layer=1)]
    other = rows((9, 2, 64), 77, torch.float32)
    f = fs[0]
    f.append([4, 5])
    f.cache.append(0, other, other, f.step)
    f.cache.append(2, other * 2, other, f.step)
    f.check_values()
    k, _ = f.cache.read(2, f.step.slot)
    assert (k - 2 * other).abs().max() <= 2 * other.abs().max() / 127


def test_append_of_values_no_scale_fits():
    """Zeros, denormals, the largest values, NaN and infinities; a later larger token scales them again."""
    f = Filled(16, 1, 1, 64, 1, 1, torch.float32)
    x = torch.zeros(5, 1, 64, device="cuda")
    x[1, 0, 3], x[2, 0, 0], x[2, 0, 1] = 1e-42, 1e-20, -3e-21
    f.append([5], kv=[x, x.clone()])
    f.check_values()
    assert status(f.cache) == 0
    y = torch.zeros(3, 1, 64, device="cuda")
    y[0, 0, :4] = torch.tensor([float("nan"), float("inf"), -float("inf"), 2.0])
    y[2] = torch.randn(64, device="cuda")
    f.append([3], kv=[y, y.clone()])
    f.check_values()
    assert status(f.cache) == 8
    k, _ = f.cache.read(0, f.step.slot)
    assert torch.isfinite(k).all() and k[0, 0, 0] == 0 and k[0, 0, 1] == -k[0, 0, 2] == k.max()
    f.append([1], kv=[torch.full((1, 1, 64), 3.4e38, device="cuda")] * 2)
    f.check_values()


@pytest.mark.parametrize("n", [2, 20])
def test_append_of_infinities_beside_the_largest_value(n):
    """127 times the scale of the largest fp32 value rounds to infinity; infinities still get the codes 127 and
    -127.  20 rows of one seat take the prompts' kernel, 2 the decode steps'."""
    f = Filled(16, 1, 1, 64, 1, 2, torch.float32)
    x = torch.ones(n, 1, 64, device="cuda")
    x[0, 0, :3] = torch.tensor([torch.finfo(torch.float32).max, float("inf"), -float("inf")])
    f.append([n], kv=[x, x.clone()])
    f.check_values()
    for got in f.cache.read(0, f.step.slot):
        assert got[0, 0, 1] == got[0, 0, 0] == -got[0, 0, 2] == got.max()


def test_append_and_read_skip_bad_slots():
    c = lib.KV8Cache(1, 1, 1, 64, 16, 3, 1, 3)
    step = c.new_step(1, 4)
    step.slot.copy_(ints([5, -1, 48, 2 ** 31 - 1]))
    x = torch.ones(4, 1, 64, device="cuda")
    c.append(0, x, x, step)
    assert status(c) == 4
    k, v = c.read(0, ints([5, -1, 48, 4]), torch.bfloat16)
    assert status(c) == 4
    assert k[:, 0, 0].tolist() == [1, 0, 0, 0] == v[:, 0, 63].tolist()


def test_blocks_past_four_gigabytes():
    """Offsets into data pass 32 bits: the last blocks of a cache of 5.2 GB."""
    n = 2100
    c = lib.KV8Cache(2, 40, 40, 128, 128, n, 1, 4)
    assert c.data.numel() > 5 << 30
    step = c.new_step(1, 300)
    c.pool.copy_(torch.arange(n, dtype=torch.int32, device="cuda"))   # handed out from the end
    c.plan(step, ints([0]), ints([300]))
    assert step.slot.max().item() >= (n - 1) * 128
    k, v = rows((300, 40, 128), 1, torch.bfloat16), rows((300, 40, 128), 2, torch.bfloat16)
    c.append(1, k, v, step)
    got = c.read(1, step.slot)
    for g, x in zip(got, (k, v)):
        assert ((g - x.float()).abs() <= x.float().abs().amax() / 127).all()
    q = rows((300, 40, 128), 3, torch.float32, 0.0)[-5:]
    one = c.new_step(1, 5)
    c.plan(one, ints([295]), ints([5]))
    o = c.attention(1, q, one)
    s = torch.einsum("rhd,khd->hrk", q.double(), got[0].double()) / 128 ** 0.5
    s.masked_fill_(torch.arange(300, device="cuda")[None] > torch.arange(295, 300, device="cuda")[:, None], -torch.inf)
    want = torch.einsum("hrk,khd->rhd", s.softmax(2), got[1].double())
    assert (o.double() - want).abs().max() < 1e-4


# ------------------------------------------------------------------------------------------ attention

def check_attention(f, q, o, scale, masks=None, heads=None, drop=()):
    """Bounds: scores carry q's 22 bits and fp32 sums over head_dim, so |ds| <= 2^-18 * sum|q k| (in units
    where the softmax is exp(s)); the weights' sums 2^-18 more and n 2^-26 for n keys; bf16 rows add fp16
    probabilities (2^-11, taken as 2^-10) and the output's own rounding (2^-9, taken as 2^-8).  Formats end
    below: an fp16 probability times scale, held relative to the largest one up to a factor of two, is off
    by up to 2^-24 of that (2^-24 floor), and the output by its type's smallest step (2^-149, bf16 2^-133)."""
    kv_heads, dim = f.shape

    def kv_of(b):
        n = f.before[b] + f.add[b]
        slots = f.slots_of(b, n)
        return (f.ref[0].values(slots), f.ref[1].values(slots), np.array([s not in drop for s in slots]),
                f.ref[1].scales[np.array(slots) // f.block])

    want, weight, size, floor = ref.attention(q.float().cpu().numpy(), kv_of, f.before, f.add, q.shape[1], kv_heads,
                                              scale, masks)
    n = max(a + b for a, b in zip(f.before, f.add))
    rel = 2.0 ** -18 * (1 + size[:, :, None]) + n * 2.0 ** -26
    bound = rel * weight + 2.0 ** -24 * floor + 2.0 ** (-133 if o.dtype is torch.bfloat16 else -149)
    if o.dtype is torch.bfloat16:
        bound = bound + 2.0 ** -10 * weight + 2.0 ** -8 * np.abs(want)
    got = o.double().cpu().numpy()[:len(want)]
    bad = np.abs(got - want) > bound
    assert not bad.any(), f"{bad.sum()} of {bad.size}; worst {np.max(np.abs(got - want) / (bound + 1e-300))} of the bound"


CASES = [  # dim, heads, kv_heads, block, history, new rows
    (128, 2, 2, 64, [0], [1]),
    (128, 2, 2, 16, [1], [1]),
    (64, 3, 1, 16, [0, 15, 16, 17], [1, 1, 1, 1]),
    (128, 4, 4, 32, [33, 0, 640, 7], [6, 6, 3, 0]),
    (64, 8, 8, 64, [129, 1, 63], [16, 1, 7]),
    (128, 8, 1, 128, [200, 127], [16, 5]),
    (128, 8, 2, 16, [1000, 3, 511], [1, 2, 3]),
    (64, 16, 4, 32, [300] * 9, [2] * 9),
    (128, 32, 4, 64, [2049, 77], [7, 9]),
    (128, 1, 1, 16, [5003], [5]),
    (64, 40, 40, 32, [31, 32, 33, 65, 97], [1, 1, 1, 1, 1]),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"d{c[0]}_h{c[1]}_{c[2]}_b{c[3]}_n{max(c[4])}_r{max(c[5])}")
def test_attention(case, dtype):
    dim, heads, kv, block, hist, add = case
    wide = max(-(-(a + b) // block) for a, b in zip(hist, add))
    f = Filled(block, heads, kv, dim, len(hist), wide, DT[dtype])
    f.append(hist)
    f.append(add)
    q = rows((sum(add), heads, dim), 9, DT[dtype], 0.5) * 2
    o = f.cache.attention(0, q, f.step)
    check_attention(f, q, o, dim ** -0.5)
    again = f.cache.attention(0, q, f.step, out=torch.full_like(o, float("nan")))
    assert torch.equal(o, again)
    assert status(f.cache) == 0


@pytest.mark.parametrize("tile", [1, 3, 8, 16])
def test_attention_is_right_for_any_row_tile(tile):
    f = Filled(32, 8, 4, 128, 3, 8, torch.float32)
    f.append([100, 0, 201])
    f.append([9, 16, 1], rows_per_request=tile)
    q = rows((26, 8, 128), 3, torch.float32, 0.2)
    check_attention(f, q, f.cache.attention(0, q, f.step, scale=0.2), 0.2)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tile", [16, 24, 32])
@pytest.mark.parametrize("case", CASES[2:10], ids=lambda c: f"d{c[0]}_h{c[1]}_{c[2]}_b{c[3]}_n{max(c[4])}_r{max(c[5])}")
def test_attention_row_tiles(case, tile, dtype):
    """Items of 16 to 32 query rows, which the size of the cache would choose only for large ones."""
    dim, heads, kv, block, hist, add = case
    wide = max(-(-(a + b) // block) for a, b in zip(hist, add))
    f = Filled(block, heads, kv, dim, len(hist), wide, DT[dtype])
    f.append(hist)
    f.append(add, row_tile=tile)
    q = rows((sum(add), heads, dim), 9, DT[dtype], 0.5) * 2
    masks = [(0x9e3779b9 * (i + 1) >> 3 | 1 << 31) & 0xffffffff for i in range(sum(add))]
    m = torch.tensor(np.array(masks, np.uint32).view(np.int32)).cuda()
    check_attention(f, q, f.cache.attention(0, q, f.step), dim ** -0.5)
    check_attention(f, q, f.cache.attention(0, q, f.step, row_mask=m), dim ** -0.5, masks)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tile", [8, 16, 24, 32])
def test_attention_of_many_short_contexts(tile, dtype):
    """More segments than teams, each shorter than a team's usual span; some of one token, some empty."""
    f = Filled(32, 32, 16, 64, 37, 3, DT[dtype])
    f.append([i * 5 % 41 for i in range(37)])
    f.append([i % 17 for i in range(37)], row_tile=tile)
    q = rows((sum(f.add), 32, 64), 8, DT[dtype], 0.5)
    check_attention(f, q, f.cache.attention(0, q, f.step), 0.125)
    assert status(f.cache) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_with_row_masks(dtype):
    """Trees of drafts: a row sees the prefix and some of the step's rows; rows of a request without a
    prefix may see nothing, and give zeros."""
    f = Filled(16, 4, 2, 64, 3, 6, DT[dtype])
    f.append([40, 0, 16])
    f.append([5, 6, 32])
    masks = [1, 3, 5, 11, 21] + [0, 2, 0b111111, 0, 0b100000, 1] + [(1 << 31) >> (i % 32) | 1 for i in range(32)]
    q = rows((43, 4, 64), 4, DT[dtype], 0.2)
    m = torch.tensor(np.array(masks, np.uint32).view(np.int32)).cuda()
    o = f.cache.attention(0, q, f.step, row_mask=m, out=torch.full_like(q, float("nan")))
    check_attention(f, q, o, 64 ** -0.5, masks)
    assert (o[5] == 0).all() and (o[8] == 0).all()


def test_attention_zeroes_rows_past_the_last_request():
    f = Filled(16, 2, 2, 64, 2, 3, torch.float32)
    f.append([20, 3])
    step = f.cache.new_step(2, 9)
    f.cache.plan(step, ints([20, 3]), ints([0, 0]))
    q = rows((9, 2, 64), 1, torch.float32)
    o = f.cache.attention(0, q, step, out=torch.full_like(q, float("nan")))
    assert (o == 0).all()
    f.cache.plan(step, ints([-1, 3]), ints([4, 2]))   # a released seat has no rows
    kv = rows((9, 2, 64), 2, torch.float32)
    f.cache.append(0, kv, kv, step)
    o = f.cache.attention(0, q, step, out=torch.full_like(q, float("nan")))
    assert torch.isfinite(o).all() and (o[:2] != 0).any() and (o[2:] == 0).all()


def test_attention_skips_keys_without_a_block():
    f = Filled(16, 2, 2, 128, 1, 4, torch.float32)
    f.append([40])
    f.append([3])
    slots = f.slots_of(0, 43)
    gone = set(slots[16:32])
    f.cache.table[0, 1] = -1
    f.slots_of = lambda b, n=None: slots
    q = rows((3, 2, 128), 8, torch.float32)
    check_attention(f, q, f.cache.attention(0, q, f.step), 128 ** -0.5, drop=gone)
    f.cache.table[0, 1] = 10 ** 6    # an id outside the cache is not followed
    check_attention(f, q, f.cache.attention(0, q, f.step), 128 ** -0.5, drop=gone)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_takes_views_and_unaligned_rows(dtype):
    f = Filled(32, 4, 2, 64, 2, 3, DT[dtype])
    f.append([50, 9])
    f.append([3, 4])
    base = rows((7, 9, 64 + 3), 3, DT[dtype])
    out = torch.full((7, 4, 200), float("nan"), dtype=DT[dtype], device="cuda")
    for q, o in ((base[:, 1:5, 3:], out[:, :, 1:65]), (base[:, ::2, :64][:, :4], out[:, :, 64:128])):
        f.cache.attention(0, q, f.step, out=o)
        check_attention(f, q, o, 64 ** -0.5)
    assert torch.isnan(out[:, :, 128:]).all() and torch.isnan(out[:, :, 0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_with_scales_far_apart(dtype):
    """Neighbouring blocks whose K and V differ by many orders of magnitude, with the softmax on the small
    ones, on the large ones and on both; large and tiny queries."""
    f = Filled(16, 2, 1, 128, 1, 12, DT[dtype])
    n = 180
    size = torch.tensor([10.0 ** ((i // 16) * 3 % 11 - 7) for i in range(n)], device="cuda")[:, None, None]
    k = rows((n, 1, 128), 1, torch.float32, 0.1)
    k[96:112] *= 8
    v = rows((n, 1, 128), 2, torch.float32, 0.1) * size
    f.append([n], kv=[k.to(DT[dtype]), v.to(DT[dtype])])
    f.append([6])
    for qs in (1e-30, 0.05, 1.0, 6.0, 1e4):
        q = (rows((6, 2, 128), 3, torch.float32, 0.1) * qs).to(DT[dtype])
        q[2, 0] = k[100, 0].to(DT[dtype]) * 4   # points at one key of one block
        o = f.cache.attention(0, q, f.step)
        assert torch.isfinite(o).all()
        check_attention(f, q, o, 128 ** -0.5)


def test_attention_keeps_a_bad_query_to_its_row():
    f = Filled(32, 2, 2, 64, 1, 3, torch.float32)
    f.append([60])
    f.append([5])
    q = rows((5, 2, 64), 3, torch.float32)
    want = f.cache.attention(0, q, f.step)
    q2 = q.clone()
    q2[1, 0, 7], q2[3, 1, 0] = float("nan"), float("inf")
    got = f.cache.attention(0, q2, f.step)
    assert torch.isnan(got[1, 0]).all() and torch.isnan(got[3, 1]).any()
    keep = torch.ones(5, 2, dtype=torch.bool)
    keep[1, 0] = keep[3, 1] = False
    assert torch.equal(got[keep], want[keep])


def test_attention_splits_long_contexts_the_same_way_every_time():
    """One request over many CTAs, twice the same bits; and next to short requests."""
    f = Filled(64, 4, 2, 128, 3, 400, torch.bfloat16)
    f.append([25000, 40, 0])
    f.append([4, 1, 2])
    q = rows((7, 4, 128), 3, torch.bfloat16, 0.3)
    o = f.cache.attention(0, q, f.step)
    check_attention(f, q, o, 128 ** -0.5)
    for _ in range(5):
        assert torch.equal(o, f.cache.attention(0, q, f.step))


def test_steps_in_a_graph_follow_the_lengths():
    """plan + append + attention captured once and replayed on growing lengths, on a stream of its own."""
    f = Filled(16, 4, 2, 64, 2, 6, torch.float32)
    f.append([21, 2])
    n, length, add = 4, ints(f.length), ints([2, 2])
    step = f.cache.new_step(2, n)
    k, v = rows((n, 2, 64), 1, torch.float32), rows((n, 2, 64), 2, torch.float32)
    q = rows((n, 4, 64), 3, torch.float32)
    o = torch.zeros_like(q)
    f.cache.attention(0, q, f.cache.plan(f.cache.new_step(2, n), length, ints([0, 0])))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        f.cache.plan(step, length, add)
        f.cache.append(0, k, v, step)
        f.cache.attention(0, q, step, out=o)
    for it in range(9):
        k.copy_(rows((n, 2, 64), 10 + it, torch.float32))
        q.copy_(rows((n, 4, 64), 20 + it, torch.float32))
        length.copy_(ints(f.length))
        graph.replay()
        torch.cuda.synchronize()
        f.before, f.add = list(f.length), [2, 2]
        for r, x in zip(f.ref, (k, v)):
            r.append(x.cpu().numpy(), step.slot.tolist())
        f.length = [x + 2 for x in f.length]
        f.check_values()
        check_attention(f, q, o, 64 ** -0.5)


def test_wrapper_refusals():
    c = lib.KV8Cache(1, 4, 2, 64, 16, 8, 2, 4)
    step = c.new_step(2, 3)
    good_kv, good_q = torch.zeros(3, 2, 64, device="cuda"), torch.zeros(3, 4, 64, device="cuda")
    l, a = ints([0, 0]), ints([1, 2])
    calls = [lambda: lib.KV8Cache(1, 4, 3, 64, 16, 8, 2, 4), lambda: c.new_step(3, 1), lambda: c.new_step(2, -1),
             lambda: c.plan(step, l.long(), a), lambda: c.plan(step, l[:1], a), lambda: c.plan(step, l, a.cpu()),
             lambda: c.plan(step, l, a, state=l),
             lambda: c.append(0, good_kv[:2], good_kv, step), lambda: c.append(0, good_kv, good_kv.bfloat16(), step),
             lambda: c.append(0, good_kv.half(), good_kv.half(), step), lambda: c.append(1, good_kv, good_kv, step),
             lambda: c.append(0, good_kv.cpu(), good_kv.cpu(), step),
             lambda: c.append(0, good_kv.transpose(1, 2).contiguous().transpose(1, 2), good_kv, step),
             lambda: c.attention(0, good_kv, step), lambda: c.attention(0, good_q, step, out=good_q.bfloat16()),
             lambda: c.attention(0, good_q, step, row_mask=ints([1, 2])), lambda: c.attention(-1, good_q, step),
             lambda: c.read(0, l.long()), lambda: c.read(0, l, torch.float16),
             lambda: lib.KV8Cache(1, 4, 2, 64, 16, 8, 2, 4).plan(step, l, a),
             lambda: lib.KV8Cache(1, 4, 2, 64, 16, 8, 2, 4).attention(0, good_q, step)]
    for i, f in enumerate(calls):
        with pytest.raises(lib.SSDError) as e:
            f()
        assert e.value.status == 1, i


def test_steps_refused_by_the_wrapper():
    """A step of a cache of another shape (its rows are fewer bytes than this cache would read), tiles and
    row counts that no kernel has."""
    c, other = lib.KV8Cache(1, 8, 8, 64, 16, 8, 2, 4), lib.KV8Cache(1, 2, 2, 64, 16, 8, 2, 4)
    step = other.new_step(1, 3)
    x = torch.zeros(3, 2, 64, device="cuda")
    for i, f in enumerate([lambda: c.append(0, x, x, step), lambda: c.new_step(1, 3, row_tile=12),
                           lambda: c.new_step(1, 3, row_tile=-8), lambda: c.new_step(1, 3, rows_per_request=0)]):
        with pytest.raises(lib.SSDError) as e:
            f()
        assert e.value.status == 1, i
    other.append(0, x, x, step)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tile", [8, 16])
def test_attention_of_queries_with_an_outlier_that_no_key_sees(tile, dtype):
    """One dimension of the queries is a million times the others, where all keys are 0: it adds nothing to the
    scores and costs the other dimensions nothing."""
    f = Filled(32, 4, 2, 64, 2, 4, DT[dtype])
    for add in ([90, 20], [5, 2]):
        kv = [rows((sum(add), 2, 64), 50 + i + sum(add), DT[dtype], 0.3) for i in range(2)]
        kv[0][:, :, 9] = 0
        f.append(add, kv=kv, row_tile=tile)
    q = rows((7, 4, 64), 3, torch.float32, 0.2)
    q[:, :, 9] = 1e6
    q = q.to(DT[dtype])
    check_attention(f, q, f.cache.attention(0, q, f.step), 64 ** -0.5)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_where_scores_rise_slowly_after_large_values(dtype):
    """The scores of one query head rise steeply from tile to tile, those of its neighbours slowly, and the first
    tile's values are 2^40 times the others': at the end it weighs little in every row, and the later values
    need their bits.  Enough segments that a warp takes a whole one (60 tiles)."""
    batch, kv, group, dim, block, tiles = 61, 40, 8, 64, 16, 60
    n = tiles * block
    c = lib.KV8Cache(1, kv * group, kv, dim, block, batch * (tiles + 1), batch, tiles + 1)
    g = torch.Generator(device="cuda").manual_seed(1)
    k = torch.zeros(n, kv, dim, device="cuda")
    k[:, :, 0] = (torch.arange(n, device="cuda") // block)[:, None]
    step = c.new_step(batch, batch * n)
    c.plan(step, ints([0] * batch), ints([n] * batch))
    v = torch.randn(batch, n, kv, dim, device="cuda", generator=g)
    v[:, :block] *= 2.0 ** 40
    c.append(0, k.to(DT[dtype]).repeat(batch, 1, 1), v.view(batch * n, kv, dim).to(DT[dtype]), step)
    one = c.new_step(batch, batch)
    c.plan(one, ints([n] * batch), ints([1] * batch))
    last = torch.zeros(batch, kv, dim, device="cuda", dtype=DT[dtype])
    c.append(0, last, last, one)
    q = torch.zeros(batch, kv, group, dim, device="cuda")
    rise = torch.full((group,), 0.9, device="cuda")
    rise[0] = 9
    q[..., 0] = rise * float(np.log(2.0))
    q = q.to(DT[dtype])
    o = c.attention(0, q.view(batch, kv * group, dim), one, scale=1.0).view(batch, kv, group, dim)
    slots = torch.cat([step.slot.view(batch, n), one.slot[:, None]], 1)
    for b in (0, 30, 60):
        kk, vv = (x.double() for x in c.read(0, slots[b].contiguous()))
        s = torch.einsum("hgd,nhd->hgn", q[b].double(), kk)
        p = s.softmax(2)
        want, weight = torch.einsum("hgn,nhd->hgd", p, vv), torch.einsum("hgn,nhd->hgd", p, vv.abs())
        # as in check_attention
        size = s.abs().amax(2)[:, :, None]
        bound = (2.0 ** -18 * (1 + size) + n * 2.0 ** -26) * weight
        scale = c.scales[0, slots[b].long() // block, :, 1].double()
        floor = (p * scale.T[:, None]).amax(2)[:, :, None] * (vv.abs() / scale[:, :, None]).sum(0)[:, None]
        bound = bound + 2.0 ** -24 * floor
        if dtype == "bf16":
            bound = bound + 2.0 ** -10 * weight + 2.0 ** -8 * want.abs()
        err = (o[b].double() - want).abs()
        assert (err <= bound).all(), f"{(err > bound).sum().item()} of {err.numel()}, worst {(err / bound).max().item()}"


def test_attention_flags_requests_of_more_rows_than_a_mask_has_bits():
    f = Filled(16, 2, 2, 64, 2, 5, torch.float32)
    f.append([4, 20])
    f.append([33, 3])
    q = rows((36, 2, 64), 4, torch.float32)
    want = f.cache.attention(0, q, f.step)
    assert status(f.cache) == 0   # without masks any number of rows is right
    mask = ints([-1] * 36)
    got = f.cache.attention(0, q, f.step, row_mask=mask)
    assert status(f.cache) == 2
    assert torch.isfinite(got).all() and torch.equal(got[35], want[35])   # the request of three rows is as it was
    f.append([32, 32])
    q = rows((64, 2, 64), 5, torch.float32)
    f.cache.attention(0, q, f.step, row_mask=ints([-1] * 64))
    assert status(f.cache) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_into_the_buffer_of_its_queries(dtype):
    """Heads, dimensions or rows beside the queries are fine; theirs are refused."""
    f = Filled(32, 4, 2, 64, 2, 3, DT[dtype])
    f.append([50, 9])
    f.append([3, 4])
    for q_of, o_of in ((lambda b: b[:, :4, :64], lambda b: b[:, 4:, :64]), (lambda b: b[:, ::2, 64:], lambda b: b[:, 1::2, 64:]),
                       (lambda b: b[:, :4, :64], lambda b: b[:, :4, 64:])):
        buf = rows((7, 8, 128), 3, DT[dtype])
        q = q_of(buf).clone()
        o = f.cache.attention(0, q_of(buf), f.step, out=o_of(buf))
        check_attention(f, q, o, 64 ** -0.5)
        assert torch.equal(q_of(buf), q)
    keep = buf.clone()
    for o in (buf[:, :4, :64], buf[:, 1:5, :64], buf[:, :4, 1:65]):
        with pytest.raises(lib.SSDError) as e:
            f.cache.attention(0, buf[:, :4, :64], f.step, out=o)
        assert e.value.status == 1 and "overlaps" in str(e.value)
    assert torch.equal(buf, keep)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_append_of_prompts_that_go_on_in_a_block(block, dim, dtype):
    """The prompts' kernel (one seat, more than 16 rows a call) where the first rows go to a block that holds
    older ones: in the middle of a tile or on a tile's edge, with scales that grow or stay."""
    f = Filled(block, 3, 3, dim, 1, 5 + 260 // block, DT[dtype])
    for add, size in ((block + 5, 1.0), (40, 30.0), (17, 0.01), (block + 19, 100.0), (33, 100.0)):
        kv = [rows((add, 3, dim), f.seed + i + add, torch.float32) * size for i in range(2)]
        kv[0][:, 1] *= 1e-3
        f.append([add], kv=[x.to(DT[dtype]) for x in kv])
        f.check_values()
        if add == 17:   # rejected rows: the next call starts at a tile's edge
            f.length[0] = f.length[0] // 16 * 16
    assert status(f.cache) == 0


@pytest.mark.parametrize("few", [True, False])
def test_values_rounded_again_stay_within_their_bound(few):
    """A value appended at scale s_0 and rounded again at each of r growths is off by at most half of each of the
    scales it was rounded at, so by (r + 1) / 2 of the block's scale: 1 / 2 for exact products, 2^-14 more a
    rounding for fp32 ones (codes up to 127, a few roundings to 24 bits each)."""
    block, n = 128, 8 if few else 18   # few: the decode steps' kernel
    f = Filled(block, 2, 2, 64, 1, 1, torch.float32)
    at, scales = [], []
    for i in range(7):
        f.append([n], kv=[rows((n, 2, 64), 7 + i + j, torch.float32) * 1.3 ** i for j in range(2)])
        at.append(f.kv)
        scales.append([r.scales[f.step.slot[0].item() // block].astype(np.float64) for r in f.ref])
    got = f.cache.read(0, ints(f.slots_of(0)))
    most = 0
    for j in range(2):
        for i in range(7):
            total, r = scales[i][j].copy(), 0
            for t in range(i + 1, 7):
                grown = scales[t][j] > scales[t - 1][j]
                total += np.where(grown, scales[t][j], 0)
                r = r + grown
            most = max(most, np.max(r))
            assert (total <= (r + 1) * scales[6][j]).all()
            err = (got[j][i * n:(i + 1) * n].double() - at[i][j].double()).abs().amax((0, 2)).cpu().numpy()
            assert (err <= (0.5 + 2.0 ** -14) * total).all()
    assert most >= 2
