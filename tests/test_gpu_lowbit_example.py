"""The low-bit operators together: the decode loop of examples/lowbit_decode.py against a plain torch decoder
of the same low-bit values."""
import math
import os
import subprocess
import sys

import pytest
import torch

import synth
from examples.lowbit_decode import LowBitDecoder
from tests.gpu_util import device_weights

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def plain_logits(dec: LowBitDecoder, x, tables):
    """fp64 forward of one request's rows x [n][d] over the values the packed weights and the cache hold
    (attention reads K/V of every row back from the cache)."""
    s = dec.shape
    x = x.double()
    n = x.shape[0]
    norm = lambda v, g: v * torch.rsqrt(v.square().mean(-1, keepdim=True) + s.rms_eps) * g.double()  # noqa: E731
    freq = s.rope_theta ** (-torch.arange(0, s.head_dim, 2, device="cuda", dtype=torch.float64) / s.head_dim)
    angle = torch.arange(n, device="cuda", dtype=torch.float64)[:, None, None] * freq
    cos, sin = angle.cos(), angle.sin()
    for i, (w, lw) in enumerate(zip(dec.layers, dec.weights["layers"])):
        qkv = norm(x, lw["attn_norm"]) @ w["qkv"].dequantize().double().T
        q = qkv.view(n, 3, s.n_heads, s.head_dim)[:, 0]
        a, b = q.chunk(2, -1)
        q = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        k, v = dec.cache.read(i, tables)
        p = torch.einsum("rhd,khd->hrk", q, k.double()) / math.sqrt(s.head_dim)
        p.masked_fill_(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -torch.inf)
        o = torch.einsum("hrk,khd->rhd", p.softmax(2), v.double()).reshape(n, -1)
        x = x + o @ w["o"].dequantize().double().T
        gate, up = (norm(x, lw["ffn_norm"]) @ w["gate_up"].dequantize().double().T).chunk(2, 1)
        x = x + (torch.nn.functional.silu(gate) * up) @ w["down"].dequantize().double().T
    return norm(x, dec.weights["final_norm"]) @ dec.head.dequantize().double().T


@pytest.mark.parametrize("block,group", [(16, 32), (64, 128)])
def test_decode_loop_against_a_plain_decoder(block, group):
    """Three ragged requests, one of them a single row.  While they decode, block scales grow and old codes
    are rounded again, so the comparison is at the last step, whose row read the cache as it is at the end:
    its logits depend on earlier rows through the cached K/V alone, and only fp32 arithmetic (4 layers, sums
    of up to 1024 products, 1e-6 each) separates the two."""
    w = synth.TINY
    dev = device_weights(synth.make_weights(w))
    dec = LowBitDecoder(dev, w.shape, 3, 80, block, group)
    g = torch.Generator().manual_seed(3)
    prompts = [torch.randn(n, w.shape.d_model, generator=g).cuda() for n in (37, 1, 16)]
    tokens, logits = dec.generate(prompts, 9)
    table = dec.cache.table.tolist()
    for b, p in enumerate(prompts):
        rows = torch.cat([p, dev["embed"][torch.tensor(tokens[b][:-1]).cuda()].float()])
        slots = torch.tensor([table[b][i // block] * block + i % block for i in range(len(rows))], dtype=torch.int32).cuda()
        want = plain_logits(dec, rows, slots)[-1]
        err = (logits[b, -1].double() - want).square().mean().sqrt() / want.square().mean().sqrt()
        assert err < 1e-4, (b, err.item())


def test_prompt_alone_equals_the_plain_decoder():
    """No rounding happens twice in a prompt: only fp32 arithmetic separates the two."""
    w = synth.TINY
    dev = device_weights(synth.make_weights(w))
    dec = LowBitDecoder(dev, w.shape, 2, 64, 32, 64)
    g = torch.Generator().manual_seed(4)
    prompts = [torch.randn(n, w.shape.d_model, generator=g).cuda() for n in (45, 12)]
    _, logits = dec.generate(prompts, 1)
    table = dec.cache.table.tolist()
    for b, p in enumerate(prompts):
        slots = torch.tensor([table[b][i // 32] * 32 + i % 32 for i in range(len(p))], dtype=torch.int32).cuda()
        want = plain_logits(dec, p, slots)[-1]
        err = (logits[b, 0].double() - want).square().mean().sqrt() / want.square().mean().sqrt()
        assert err < 1e-4, (b, err.item())


def test_example_runs():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "lowbit_decode.py"), "--new", "6"],
                       capture_output=True, text=True, timeout=300, cwd=ROOT)
    assert r.returncode == 0, r.stderr[-2000:]
    assert r.stdout.count("tokens as in full precision") == 3 and "of bf16" in r.stdout
