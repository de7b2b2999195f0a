"""A transformer layer that serves drafted tokens, built of the library's calls: quantized products, norms around the blocks, attention of
a tree of tokens over a paged cache, and the cache's upkeep -- accepted tokens appended, attention weights added up, entries evicted when a
sequence grows past its budget.

    python examples/decode_layer.py            # Llama-2-7B's layer: 8 sequences, trees of 8 drafted tokens, caches held to 512 slots

PyTorch supplies device memory, rotary angles and the choice of accepted tokens; weights are random, and rows whose draft would be verified are
picked at random, since nothing here is trained.
"""
from __future__ import annotations

import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2504_14152_amd import fgmp  # noqa: E402


def pack(w: torch.Tensor, fraction: float = 0.1) -> fgmp.Packed:
    """Weights with a tenth of their blocks in FP8 (sensitivities all alike: there is no model to calibrate on)."""
    fisher, scale = torch.ones(w.shape[1], device=w.device), float(w.abs().max()) / 448.0
    _, scores = fgmp.quantize_weights(w, fisher, math.inf, scale, want_scores=True)
    return fgmp.quantize_weights(w, fisher, fgmp.threshold_for_fraction(scores, fraction), scale)


class Linear:
    """Packed weights, and what its activations are quantized with; the workspace serves up to `rows` rows."""

    def __init__(self, w: torch.Tensor, rows: int, act_scale: float, threshold: float):
        self.packed, self.fisher = pack(w), torch.ones(w.shape[1], device=w.device)
        self.scale, self.threshold = act_scale, threshold
        self.workspace = fgmp.new_workspace(fgmp.workspace_bytes(rows, *w.shape), w.device)

    def __call__(self, x: torch.Tensor, out: torch.Tensor) -> torch.Tensor:
        return fgmp.quant_gemm_fused(x, self.fisher, self.threshold, self.scale, self.packed, out=out, workspace=self.workspace)


def rotate(x: torch.Tensor, positions: torch.Tensor) -> torch.Tensor:
    """Rotary positions on batch x tokens x heads x dim."""
    half = x.shape[-1] // 2
    angle = positions[:, :, None, None] * 10000.0 ** (-torch.arange(half, device=x.device) / half)
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1)


class Layer:
    def __init__(self, batch, tokens, hidden=4096, heads=32, kv_heads=32, ffn=11008, page=64, budget=512, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.batch, self.tokens, self.hidden, self.heads, self.kv_heads = batch, tokens, hidden, heads, kv_heads
        self.dim, self.budget, rows = hidden // heads, budget, batch * tokens

        def w(n, k):
            return torch.randn(n, k, generator=g, device=device) / math.sqrt(k)

        self.qkv = Linear(w((heads + 2 * kv_heads) * self.dim, hidden), rows, 6.0 / 448, 1e-3)
        self.o = Linear(w(hidden, hidden), rows, 6.0 / 448, 1e-3)
        self.down, self.gate_up = pack(w(hidden, ffn)), Linear(w(2 * ffn, hidden), rows, 6.0 / 448, 1e-3)   # (gate and up rows in groups of 32 + 32)
        self.ffn, self.hidden_fisher = ffn, torch.ones(ffn, device=device)
        self.norm = [torch.ones(hidden, device=device) for _ in range(3)]      # before attention, before the MLP, before the next layer
        slots = -(-(budget + 2 * tokens) // page) * page
        pages = batch * slots // page
        table = torch.randperm(pages, generator=g, device=device).view(batch, -1).int()
        kv = [torch.empty(pages, page, kv_heads, self.dim, dtype=torch.bfloat16, device=device) for _ in range(2)]
        zeros = torch.zeros(batch, dtype=torch.int32, device=device)
        self.cache = fgmp.Cache(kv[0], kv[1], zeros.clone(), table)
        self.lengths = [zeros.clone() for _ in range(2)]                       # (taken in turn: no call's lengths are its own result)
        self.seen, self.held = zeros, 0                                        # tokens so far; the longest sequence's slots, known here without asking the GPU
        self.weights = torch.zeros(batch, kv_heads, slots, device=device)
        self.positions = torch.zeros(batch, kv_heads, slots, dtype=torch.int32, device=device)
        # buffers of a step
        def f32(n):
            return torch.empty(rows, n, device=device)
        self.b_qkv, self.b_o, self.b_z = f32((heads + 2 * kv_heads) * self.dim), f32(hidden), f32(hidden)
        self.b_out = torch.empty(batch, tokens, heads, self.dim, dtype=torch.bfloat16, device=device)
        self.b_lse = torch.empty(batch, tokens, heads, device=device)
        self.b_h = [torch.empty(rows, hidden, dtype=torch.bfloat16, device=device) for _ in range(2)]
        gate = fgmp.EPILOGUE_SILU_GATE
        self.packed_h = fgmp.Packed(torch.empty(fgmp.packed_bytes(rows, ffn), dtype=torch.uint8, device=device), rows, ffn)
        self.ws_up = fgmp.new_workspace(fgmp.workspace_bytes_packed_out(rows, 2 * ffn, hidden, gate), device)
        self.ws_down = fgmp.new_workspace(fgmp.workspace_bytes(rows, hidden, ffn), device)
        self.ws_attend = fgmp.new_workspace(fgmp.tree_attention_workspace_bytes(batch, tokens, heads, kv_heads, self.dim, slots), device)
        self.ws_evict = fgmp.new_workspace(fgmp.cache_evict_workspace_bytes(batch, kv_heads, slots, budget), device)

    def attend(self, x: torch.Tensor, depth: torch.Tensor, tree: torch.Tensor | None = None) -> tuple[torch.Tensor, torch.Tensor]:
        """One pass of the layer over batch * tokens rows of the residual stream (FP32, changed in place): (x, the next layer's input).  `depth`,
        batch x tokens: how many drafted tokens come before each one; `tree`: fgmp.tree_words of their parents, None for a chain."""
        B, T, D = self.batch, self.tokens, self.dim
        positions = self.seen[:, None] + depth
        _, h = fgmp.block_norm(x, pre_weight=self.norm[0], h=self.b_h[0])
        q, k, v = self.qkv(h, self.b_qkv).view(B, T, -1, D).split([self.heads, self.kv_heads, self.kv_heads], 2)
        self.q, self.k, self.v = rotate(q, positions).bfloat16(), rotate(k, positions).bfloat16(), v.bfloat16()
        self.new_positions = positions.int()
        out, self.lse = fgmp.tree_attention(self.q, self.k, self.v, self.cache, tree=tree, scale=D ** -0.5, max_length=max(1, self.held),
                                            out=self.b_out, lse=self.b_lse, workspace=self.ws_attend)
        o = self.o(out.view(B * T, -1), self.b_o)
        x, h = fgmp.block_norm(x, o, pre_weight=self.norm[1], out=x, h=self.b_h[1])
        fgmp.quant_gemm_fused_packed_out(h, self.gate_up.fisher, self.gate_up.threshold, self.gate_up.scale, self.gate_up.packed, self.hidden_fisher,
                                         1e-3, 6.0 / 448, out=self.packed_h, workspace=self.ws_up, epilogue=fgmp.EPILOGUE_SILU_GATE)
        z = fgmp.gemm(self.packed_h, self.down, out=self.b_z, workspace=self.ws_down)
        return fgmp.block_norm(x, z, pre_weight=self.norm[2], out=x, h=self.b_h[0])

    def accept(self, rows: torch.Tensor | None = None, counts: torch.Tensor | None = None, most: int | None = None) -> None:
        """Keeps the tokens of the last pass that were accepted (`rows`, `counts`; all unless given; `most`: no sequence more than that)."""
        old = self.cache.lengths
        new = fgmp.cache_append(self.k, self.v, self.cache, rows=rows, counts=counts, positions=self.new_positions, slot_positions=self.positions,
                                slot_weights=self.weights, lengths_out=self.lengths[0] if old is not self.lengths[0] else self.lengths[1])
        self.seen = self.seen + (self.tokens if counts is None else counts)
        self.cache.lengths = new
        self.held += self.tokens if most is None else most
        fgmp.attention_weights(self.q, self.lse, self.cache, self.weights, rows=rows, counts=counts, scale=self.dim ** -0.5, max_length=self.held)
        if self.held > self.budget:
            after = self.lengths[0] if new is not self.lengths[0] else self.lengths[1]
            self.cache.lengths = fgmp.cache_evict(self.cache, self.weights, self.positions, self.seen.int(), self.budget, sinks=4, recent=self.budget // 4,
                                                  lengths_out=after, workspace=self.ws_evict)[2]
            self.held = self.budget


def main() -> None:
    batch, tokens, steps = 8, 8, 300
    layer = Layer(batch, tokens)
    g = torch.Generator(device="cuda").manual_seed(1)
    parents = torch.tensor([[-1, 0, 0, 1, 1, 2, 3, 5]]).repeat(batch, 1)
    tree = fgmp.tree_words(parents).cuda()
    depth = torch.tensor([[0, 1, 1, 2, 2, 2, 3, 3]], device="cuda").repeat(batch, 1)
    paths = torch.tensor([[0, 1, 3, 6], [0, 2, 5, 7], [0, 1, 4, -1]], device="cuda", dtype=torch.int32)   # from the root to each leaf
    x = torch.randn(batch * tokens, layer.hidden, generator=g, device="cuda")
    began = time.perf_counter()
    for step in range(steps):
        if step == steps // 2:
            torch.cuda.synchronize()
            began = time.perf_counter()
        layer.attend(x.copy_(torch.randn(x.shape, generator=g, device="cuda")), depth, tree)
        rows = paths[torch.randint(0, 3, (batch,), generator=g, device="cuda")]
        counts = torch.minimum(torch.randint(1, 5, (batch,), generator=g, device="cuda"), (rows >= 0).sum(1)).int()
        layer.accept(rows.contiguous(), counts, most=4)
    torch.cuda.synchronize()
    us = (time.perf_counter() - began) / (steps - steps // 2) * 1e6
    print(f"{steps} steps of {batch} sequences x {tokens} drafted tokens: {us:.0f} us a layer and step")
    print("slots:", layer.cache.lengths.tolist(), "tokens seen:", layer.seen.tolist())


if __name__ == "__main__":
    main()
