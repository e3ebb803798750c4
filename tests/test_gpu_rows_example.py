"""The operators on rows together with the 8-bit cache: a decoder layer, its head and the draw, as a decode loop calls
them, and the loop itself (examples/lowbit_decode.py) with 4-bit floats."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2510_22641_gb300 as lib
import synth
from examples.lowbit_decode import LowBitDecoder
from tests import rows_ref as ref
from tests.gpu_util import device_weights
from tests.test_gpu_rows import check_heads, check_product, check_tokens, freqs, normal

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADS, KV, D, VOCAB, BLOCK = 8, 2, 64, 3001, 32
WIDTH = HEADS * D
HOW = (0.8, 60, 0.9, 0.01)


class Layer:
    """Weights and caller's buffers of one layer with grouped heads, norms of heads and two position axes."""

    def __init__(self, batch, dtype):
        self.qkv = lib.F4Weight(normal((WIDTH + 2 * KV * D, WIDTH), 1, 0.05))
        self.o, self.head = lib.F4Weight(normal((WIDTH, WIDTH), 2, 0.05)), lib.F4Weight(normal((VOCAB, WIDTH), 3, 0.2))
        self.gains = [(1 + 0.1 * normal((D,), s)).to(torch.bfloat16) for s in (4, 5)]
        self.rotary = lib.Rotary(D, 32, 1e4, (6, 10))
        self.cache = lib.KV8Cache(1, HEADS, KV, D, BLOCK, 8 * batch, batch, 8)

    def __call__(self, x, pos, length, add, last, u, step):
        rows = len(x)
        heads = self.qkv.matmul(x).view(rows, HEADS + 2 * KV, D)
        q, k = self.rotary.rotate(heads[:, :HEADS], heads[:, HEADS:HEADS + KV], pos, *self.gains)
        self.cache.plan(step, length, add)
        self.cache.append(0, k, heads[:, HEADS + KV:], step)
        o = self.cache.attention(0, q, step)
        y = self.o.matmul(o.view(rows, -1), residual=x)
        logits = self.head.matmul(y[last])
        return (heads, q, k, o, y, logits, *lib.sample(logits, u, *HOW, with_prob=True))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_layer_step_by_step(dtype):
    """Each result against 64 bits of the operator before it: three prompts, then a token each, eager and captured."""
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    prompts = [37, 1, 130]
    batch = len(prompts)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    layer, length = Layer(batch, t), i32([0] * batch)
    for add in (prompts, [1, 1, 1]):
        rows = sum(add)
        x, u = normal((rows, WIDTH), rows, 1.0, t), torch.rand(batch, generator=torch.Generator().manual_seed(rows)).cuda()
        where = torch.cat([torch.arange(n) + int(l) for n, l in zip(add, length.tolist())])
        pos = torch.stack([where, 3 * where // 2], 1).int().cuda()
        last = (torch.tensor(add).cumsum(0) - 1).cuda()
        step = layer.cache.new_step(batch, rows)
        args = (x, pos, length, i32(add), last, u, step)
        heads, q, k, o, y, logits, token, prob = layer(*args)
        check_product(heads.view(rows, -1), lib.F4Rows(x).dequantize(), layer.qkv.dequantize())
        axis = [0] * 6 + [1] * 10
        for got, part, gain in ((q, heads[:, :HEADS], layer.gains[0]), (k, heads[:, HEADS:HEADS + KV], layer.gains[1])):
            want, size = ref.rotary(part.double().cpu().numpy(), pos.cpu().numpy(), freqs(32, 1e4), axis, 32, False,
                                    gain.double().cpu().numpy())
            check_heads(got, want, size, t)
        table = layer.cache.table.tolist()
        for b, n in enumerate(add):
            held = int(length[b]) + n
            slots = i32([table[b][i // BLOCK] * BLOCK + i % BLOCK for i in range(held)])
            kk, vv = (c.double().repeat_interleave(HEADS // KV, 1) for c in layer.cache.read(0, slots))
            r = slice(sum(add[:b]), sum(add[:b]) + n)
            s = torch.einsum("rhd,khd->hrk", q[r].double(), kk) / math.sqrt(D)
            s.masked_fill_(torch.ones(n, held, dtype=torch.bool, device="cuda").triu(held - n + 1), -torch.inf)
            want = torch.einsum("hrk,khd->rhd", s.softmax(2), vv)
            err = (o[r].double() - want).square().mean().sqrt() / want.square().mean().sqrt()
            assert err <= (2.0 ** -8 if dtype == "bf16" else 1e-5), (b, err.item())
        check_product(y, lib.F4Rows(o.reshape(rows, -1)).dequantize(), layer.o.dequantize(), x)
        check_product(logits, lib.F4Rows(y[last]).dequantize(), layer.head.dequantize())
        check_tokens(logits, u, HOW, (token, prob))
        length = length + i32(add)
    layer.cache.check()
    # a step of single tokens, captured: the values that its buffers hold when it is replayed
    g = torch.cuda.CUDAGraph()
    args = [torch.zeros_like(a) if a.dtype is t or a.dtype is torch.float32 else a.clone() for a in args[:-1]] + [args[-1]]
    args[2] = length.clone()
    with torch.cuda.graph(g):
        out = layer(*args)
    x, u = normal((batch, WIDTH), 99, 1.0, t), torch.rand(batch, device="cuda")
    args[0].copy_(x), args[5].copy_(u)
    g.replay()
    torch.cuda.synchronize()
    heads, q, k, o, y, logits, token, prob = out
    check_product(heads.view(batch, -1), lib.F4Rows(x).dequantize(), layer.qkv.dequantize())
    check_product(y, lib.F4Rows(o.reshape(batch, -1)).dequantize(), layer.o.dequantize(), x)
    check_tokens(logits, u, HOW, (token, prob))
    again = layer(*args)   # the same step once more: the same rows go to the same slots
    assert torch.equal(again[0], heads) and torch.equal(again[1], q) and torch.equal(again[2], k)


def test_decode_loop_with_4_bit_floats():
    """Greedy tokens are the logits' largest, drawn ones those of the rules, and the same seed draws the same."""
    w = synth.TINY
    dev = device_weights(synth.make_weights(w))
    g = torch.Generator().manual_seed(3)
    prompts = [torch.randn(n, w.shape.d_model, generator=g).cuda() for n in (37, 1, 16)]
    run = lambda **how: LowBitDecoder(dev, w.shape, 3, 80, 32, floats=True).generate(prompts, 7, **how)  # noqa: E731
    tokens, logits = run()
    assert tokens == logits.argmax(2).tolist() and torch.isfinite(logits).all()
    how = {"temperature": 1.0, "top_k": 40, "top_p": 0.9}
    a, za = run(seed=5, **how)
    b, zb = run(seed=5, **how)
    assert a == b and torch.equal(za, zb)
    u = torch.Generator(device="cuda").manual_seed(5)
    for step in range(7):
        z = za[:, step].cpu().numpy()
        for r, v in enumerate(torch.rand(3, device="cuda", generator=u).tolist()):
            near = {ref.sample(z[r], v + e, 1.0, 40, float(np.float32(0.9)), 0.0)[0] for e in (-2.0 ** -30, 0, 2.0 ** -30)}
            assert a[r][step] in near


def test_example_runs_with_4_bit_floats_and_draws():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "lowbit_decode.py"), "--new", "5", "--floats",
                        "--temperature", "0.7", "--top-k", "20", "--top-p", "0.95"],
                       capture_output=True, text=True, timeout=300, cwd=ROOT)
    assert r.returncode == 0, r.stderr[-2000:]
    assert r.stdout.count("tokens as in full precision") == 3 and "of bf16" in r.stdout
