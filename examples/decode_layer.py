"""A transformer layer that serves drafted tokens, built of the library's calls: quantized products, norms around the blocks, rotated queries
and keys with norms of their own, attention of a tree of tokens over a paged cache, the choice of the tokens that are kept, and the cache's
upkeep -- accepted tokens appended, attention weights added up, entries evicted when a sequence grows past its budget.  A cache in 8 bits
holds what it is given instead: twice the slots in the same memory.

    python examples/decode_layer.py            # Llama-2-7B's layer: 8 sequences, trees of 8 drafted tokens, caches held to 256 slots
    python examples/decode_layer.py 8          # the same with caches of 4096 slots in 8 bits

PyTorch supplies device memory and the softmax over the vocabulary; weights are random, and the drafted tokens are likely ones of the target's own,
since nothing here is trained.
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


class Head:
    """What follows the last layer: the target's distribution behind each row, and which drafted tokens it keeps."""

    def __init__(self, batch, tokens, hidden, vocab, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.product = Linear(torch.randn(vocab, hidden, generator=g, device=device) * (3.0 / math.sqrt(hidden)), batch * tokens, 6.0 / 448, 1e-3)
        self.logits = torch.empty(batch * tokens, vocab, device=device)
        self.shape, self.workspace = (batch, tokens, vocab), fgmp.new_workspace(fgmp.verify_drafts_workspace_bytes(batch, tokens, vocab), device)

    def distributions(self, h: torch.Tensor) -> torch.Tensor:
        return torch.softmax(self.product(h, self.logits), -1).view(self.shape)

    def verify(self, target, tokens, uniforms, parents=None, counts=None):
        """(rows, accepted, next tokens) of drafted tokens that were not drawn from a distribution."""
        return fgmp.verify_drafts(target, tokens, uniforms, parents=parents, counts=counts, workspace=self.workspace)


class Layer:
    def __init__(self, batch, tokens, hidden=4096, heads=32, kv_heads=32, ffn=11008, page=64, budget=512, seed=0, device="cuda", bits=16):
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
        self.head_norm = [torch.ones(self.dim, device=device) for _ in range(2)]   # of queries and keys
        self.inv_freq = (10000.0 ** (-torch.arange(self.dim // 2, device=device) / (self.dim // 2))).float()
        self.bits, slots = bits, -(-(budget + 2 * tokens) // page) * page           # (8 bits: the budget is what a sequence may hold)
        pages = batch * slots // page
        table = torch.randperm(pages, generator=g, device=device).view(batch, -1).int()
        kind = torch.bfloat16 if bits == 16 else torch.float8_e4m3fn
        kv = [torch.empty(pages, page, kv_heads, self.dim, dtype=kind, device=device) for _ in range(2)]
        zeros = torch.zeros(batch, dtype=torch.int32, device=device)
        if bits == 16:
            self.cache = fgmp.Cache(kv[0], kv[1], zeros.clone(), table)
        else:
            scales = [torch.empty(pages, kv_heads, page, dtype=torch.uint8, device=device) for _ in range(2)]
            self.cache = fgmp.QuantCache(kv[0], kv[1], scales[0], scales[1], zeros.clone(), table)
        self.lengths = [zeros.clone() for _ in range(2)]                       # (taken in turn: no call's lengths are its own result)
        self.seen, self.held = zeros, 0                                        # tokens so far; the longest sequence's slots, known here without asking the GPU
        self.weights = torch.zeros(batch, kv_heads, slots, device=device)
        self.positions = torch.zeros(batch, kv_heads, slots, dtype=torch.int32, device=device)
        # buffers of a step
        def f32(n):
            return torch.empty(rows, n, device=device)
        self.b_qkv, self.b_o, self.b_z = f32((heads + 2 * kv_heads) * self.dim), f32(hidden), f32(hidden)
        self.q, self.k, self.v, self.b_out = (torch.empty(batch, tokens, n, self.dim, dtype=torch.bfloat16, device=device)
                                              for n in (heads, kv_heads, kv_heads, heads))
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
        self.new_positions = positions.int()
        fgmp.rotate_heads(q, k, v, self.new_positions, self.inv_freq, q_weight=self.head_norm[0], k_weight=self.head_norm[1], q_out=self.q, k_out=self.k,
                          v_out=self.v)
        out, self.lse = fgmp.tree_attention(self.q, self.k, self.v, self.cache, tree=tree, scale=D ** -0.5, max_length=max(1, self.held),
                                            out=self.b_out, lse=self.b_lse, workspace=self.ws_attend)
        o = self.o(out.view(B * T, -1), self.b_o)
        x, h = fgmp.block_norm(x, o, pre_weight=self.norm[1], out=x, h=self.b_h[1])
        fgmp.quant_gemm_fused_packed_out(h, self.gate_up.fisher, self.gate_up.threshold, self.gate_up.scale, self.gate_up.packed, self.hidden_fisher,
                                         1e-3, 6.0 / 448, out=self.packed_h, workspace=self.ws_up, epilogue=fgmp.EPILOGUE_SILU_GATE)
        z = fgmp.gemm(self.packed_h, self.down, out=self.b_z, workspace=self.ws_down)
        return fgmp.block_norm(x, z, pre_weight=self.norm[2], out=x, h=self.b_h[0])

    def accept(self, rows: torch.Tensor | None = None, counts: torch.Tensor | None = None, most: int | None = None) -> None:
        """Keeps the tokens of the last pass that were accepted (`rows`, `counts`; all unless given; `most`: no sequence more than that).  A cache in
        8 bits is never cut: RuntimeError, and nothing is kept, where a sequence has no room left."""
        old = self.cache.lengths
        if self.bits == 8:
            most = self.tokens if most is None else most
            if self.held + most > self.cache.slots:     # (that is a bound; from here on the GPU has to be asked)
                self.held = int(old.max())
                if int((old + (self.tokens if counts is None else counts)).max()) > self.cache.slots:
                    raise RuntimeError(f"the cache is full: a sequence has {self.cache.slots} slots")
            self.cache.lengths = fgmp.cache_append(self.k, self.v, self.cache, rows=rows, counts=counts,
                                                   lengths_out=self.lengths[0] if old is not self.lengths[0] else self.lengths[1])
            self.seen = self.seen + (self.tokens if counts is None else counts)
            self.held = min(self.cache.slots, self.held + most)
            return
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
    batch, tokens, steps, vocab = 8, 8, 300, 32000
    bits = 8 if sys.argv[1:] == ["8"] else 16
    layer = Layer(batch, tokens, bits=bits, budget=256 if bits == 16 else 4096)
    head = Head(batch, tokens, layer.hidden, vocab)
    g = torch.Generator(device="cuda").manual_seed(1)
    parents = torch.tensor([[-1, 0, 0, 1, 1, 2, 3, 5]], dtype=torch.int32).repeat(batch, 1)
    tree, parents = fgmp.tree_words(parents).cuda(), parents.cuda()
    depth = torch.tensor([[0, 1, 1, 2, 2, 2, 3, 3]], device="cuda").repeat(batch, 1)
    rank = torch.tensor([[0, 0, 1, 0, 1, 0, 0, 0]], device="cuda").repeat(batch, 1)      # of a drafted token among its parent's likeliest
    x = torch.randn(batch * tokens, layer.hidden, generator=g, device="cuda")
    began, kept = time.perf_counter(), torch.zeros((), device="cuda")
    for step in range(steps):
        if step == steps // 2:
            torch.cuda.synchronize()
            began = time.perf_counter()
        _, h = layer.attend(x.copy_(torch.randn(x.shape, generator=g, device="cuda")), depth, tree)
        target = head.distributions(h)
        likely = target.topk(2, -1).indices
        drafted = likely[torch.arange(batch, device="cuda")[:, None], parents.clamp(min=0).long(), rank].int()
        rows, accepted, _ = head.verify(target, drafted, torch.rand(batch, tokens, generator=g, device="cuda"), parents=parents)
        layer.accept(rows, accepted, most=4)
        kept += accepted.float().mean()
    torch.cuda.synchronize()
    us = (time.perf_counter() - began) / (steps - steps // 2) * 1e6
    print(f"{steps} steps of {batch} sequences x {tokens} drafted tokens: {us:.0f} us a layer, head and step, {float(kept) / steps:.2f} tokens kept a step")
    print("slots:", layer.cache.lengths.tolist(), "tokens seen:", layer.seen.tolist())


if __name__ == "__main__":
    main()
