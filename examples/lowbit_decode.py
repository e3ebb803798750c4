"""Greedy decoding of a ragged batch with 4-bit weights and an 8-bit paged K/V cache.

The low-bit operators run together as a decode loop uses them.  Every step: one plan (block tables and
slots of the new rows, from the lengths on the device), then per layer the 4-bit projections, the append
of the new K/V rows, attention over the cache and the 4-bit MLP.  Norms, rotary positions and the gate are
torch operations.  The model is a small LLaMA-style decoder with the library's synthetic weights; its tokens
and logits are compared with the full-precision engine's.

    python examples/lowbit_decode.py [--batch 3] [--new 16] [--group 64] [--block 32]
"""
from __future__ import annotations

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch

import paper_2510_22641_gb300 as lib


class LowBitDecoder:
    """A LLaMA-style decoder whose projections are W4Weights and whose K/V live in a KV8Cache.

    weights: the dict lib.SSDModel takes (bf16 CUDA tensors); shape: an object with n_layers, d_model, n_heads,
    head_dim, rms_eps and rope_theta."""

    def __init__(self, weights: dict, shape, max_batch: int, max_seq: int, block_tokens: int = 32, group: int = 64):
        self.shape, self.weights = shape, weights
        self.layers = [{"qkv": lib.W4Weight(torch.cat([lw["wq"], lw["wk"], lw["wv"]]), group),
                        "o": lib.W4Weight(lw["wo"], group),
                        "gate_up": lib.W4Weight(torch.cat([lw["w_gate"], lw["w_up"]]), group),
                        "down": lib.W4Weight(lw["w_down"], group)} for lw in weights["layers"]]
        self.head = lib.W4Weight(weights["lm_head"], group)
        per_seat = -(-max_seq // block_tokens)
        self.cache = lib.KV8Cache(shape.n_layers, shape.n_heads, shape.n_heads, shape.head_dim, block_tokens,
                                  max_batch * per_seat, max_batch, per_seat)

    def _norm(self, x, gain):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + self.shape.rms_eps) * gain.float()

    def _rotate(self, x, cos, sin):
        """Rotate-half pairing (i, i + head_dim / 2) of [rows][heads][head_dim]."""
        a, b = x.chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    @staticmethod
    def _product(w: lib.W4Weight, x, residual=None):
        """w.matmul takes up to 16 rows at a time: decode steps are one call, prompts several."""
        if x.shape[0] <= 16:
            return w.matmul(x, residual=residual)
        out = torch.empty((x.shape[0], w.n), dtype=x.dtype, device=x.device)
        for i in range(0, x.shape[0], 16):
            w.matmul(x[i:i + 16], out=out[i:i + 16], residual=None if residual is None else residual[i:i + 16])
        return out

    def step(self, x: torch.Tensor, length: torch.Tensor, add: torch.Tensor, row_mask: torch.Tensor | None = None):
        """Runs the rows x fp32 [sum(add)][d_model] of all requests, add[b] of request b at positions
        length[b] .. (int32 CUDA tensors), and returns their logits [rows][vocab]."""
        s, cache = self.shape, self.cache
        rows = x.shape[0]
        step = cache.plan(cache.new_step(len(length), rows), length, add)
        r = torch.arange(rows, device=x.device, dtype=torch.int32)
        request = torch.searchsorted(step.row_start[1:], r, right=True)
        pos = (length[request] + r - step.row_start[request]).double()
        freq = s.rope_theta ** (-torch.arange(0, s.head_dim, 2, device=x.device, dtype=torch.float64) / s.head_dim)
        angle = pos[:, None, None] * freq
        cos, sin = angle.cos().float(), angle.sin().float()
        for i, (w, lw) in enumerate(zip(self.layers, self.weights["layers"])):
            qkv = self._product(w["qkv"], self._norm(x, lw["attn_norm"])).view(rows, 3, s.n_heads, s.head_dim)
            cache.append(i, self._rotate(qkv[:, 1], cos, sin), qkv[:, 2], step)
            o = cache.attention(i, self._rotate(qkv[:, 0], cos, sin), step, row_mask=row_mask)
            x = self._product(w["o"], o.view(rows, -1), residual=x)
            gate, up = self._product(w["gate_up"], self._norm(x, lw["ffn_norm"])).chunk(2, 1)
            x = self._product(w["down"], torch.nn.functional.silu(gate) * up, residual=x)
        return self._product(self.head, self._norm(x, self.weights["final_norm"]))

    def generate(self, prompts: list, max_new: int):
        """Greedy tokens of each request and the logits of every step.  prompts: fp32 rows [n_b][d_model]
        (visual rows and embedded ids).  Lengths and tokens stay on the device until the end."""
        n = [len(p) for p in prompts]
        add = torch.tensor(n, dtype=torch.int32, device="cuda")
        length = torch.zeros_like(add)
        logits = self.step(torch.cat(prompts), length, add)[add.cumsum(0) - 1]
        tokens, seen = [], []
        one = torch.ones_like(add)
        for t in range(max_new):
            seen.append(logits)
            tokens.append(logits.argmax(1))
            if t + 1 < max_new:
                length = length + add
                add = one
                logits = self.step(self.weights["embed"][tokens[-1]].float(), length, add)
        self.cache.check()
        return torch.stack(tokens, 1).tolist(), torch.stack(seen, 1)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--batch", type=int, default=3)
    ap.add_argument("--new", type=int, default=16)
    ap.add_argument("--group", type=int, default=64, choices=(32, 64, 128))
    ap.add_argument("--block", type=int, default=32, choices=(16, 32, 64, 128))
    a = ap.parse_args()
    import synth
    w = synth.TINY
    bits = synth.make_weights(w)
    up = lib.bf16_bits_to_device
    weights = {k: up(bits[k]) for k in ("embed", "lm_head", "final_norm", "in_norm", "in_w1", "in_w2")}
    weights["layers"] = [{n: up(v) for n, v in lw.items()} for lw in bits["layers"]]
    cfg = lib.config_dict(w.shape, w.draft_exit_k, w.in_kind, w.in_hidden, w.gamma, w.n_vis + w.n_prompt + a.new + 8)
    engine = lib.SSDModel(cfg, weights, torch.ones(w.shape.n_layers, device="cuda"), torch.ones(1, device="cuda"))
    prompts, want = [], []
    for b in range(a.batch):
        vis, ids = synth.make_inputs(w, seed=b + 1)
        ids = ids[:max(1, len(ids) - 3 * b)]   # ragged
        want.append(engine.greedy_generate(vis, ids, a.new)[0])
        prompts.append(torch.cat([up(vis).float(), weights["embed"][torch.from_numpy(ids).cuda().long()].float()]))
    low = LowBitDecoder(weights, w.shape, a.batch, max(map(len, prompts)) + a.new, a.block, a.group)
    got, _ = low.generate(prompts, a.new)
    for b in range(a.batch):
        same = next((i for i, (x, y) in enumerate(zip(got[b], want[b])) if x != y), a.new)
        print(f"request {b}: {len(prompts[b])} rows, {same} of {a.new} tokens as in full precision before the first difference")
    full = sum(t.numel() * 2 for lw in weights["layers"] for t in lw.values()) + weights["lm_head"].numel() * 2
    packed = sum(x.packed.numel() for lw in low.layers for x in lw.values()) + low.head.packed.numel()
    c = low.cache
    print(f"weights {packed / full:.3f} of bf16; K/V {(c.data.numel() + 4 * c.scales.numel()) / (4 * c.data.numel()):.3f} of fp32")
    engine.close()


if __name__ == "__main__":
    main()
