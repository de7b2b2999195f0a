"""The example layer on the GPU: verifying drafted tokens as a tree gives what decoding the accepted path token by token does, and a cache
held to a budget keeps what it is meant to keep."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _layer():
    spec = importlib.util.spec_from_file_location("decode_layer", os.path.join(ROOT, "examples", "decode_layer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


SMALL = dict(hidden=512, heads=8, kv_heads=2, ffn=1024, page=16)


def test_a_tree_is_the_path_that_was_accepted():
    m = _layer()
    g = torch.Generator(device="cuda").manual_seed(5)
    tree_layer, one = m.Layer(2, 6, budget=64, **SMALL), m.Layer(2, 1, budget=64, **SMALL)
    prompt = torch.randn(2, 6, 512, generator=g, device="cuda")
    depth = torch.arange(6, device="cuda").repeat(2, 1)
    # the prompt as a chain of six, and token by token
    chain, _ = tree_layer.attend(prompt.reshape(12, 512).clone(), depth)
    chain = chain.view(2, 6, 512).clone()
    tree_layer.accept()
    zero = torch.zeros(2, 1, dtype=torch.long, device="cuda")
    for t in range(6):
        x, _ = one.attend(prompt[:, t].clone(), zero)
        # rounding moves a code of a quantized activation now and then; a token that saw other tokens is off by as much as itself
        assert float((x - chain[:, t]).norm() / x.norm()) < 0.02, t
        one.accept()
    assert one.cache.lengths.tolist() == tree_layer.cache.lengths.tolist() == [6, 6]
    # a tree: 0 -> 1 -> 3, 0 -> 2 -> 4 -> 5; the second path is accepted in one sequence, two tokens of the first in the other
    words = m.fgmp.tree_words([[-1, 0, 0, 1, 2, 4]] * 2).cuda()
    depth = torch.tensor([[0, 1, 1, 2, 2, 3]] * 2, device="cuda")
    drafts = torch.randn(2, 6, 512, generator=g, device="cuda")
    out, _ = tree_layer.attend(drafts.reshape(12, 512).clone(), depth, words)
    out = out.view(2, 6, 512).clone()
    rows = torch.tensor([[0, 2, 4, 5], [0, 1, -1, -1]], dtype=torch.int32, device="cuda")
    tree_layer.accept(rows, torch.tensor([4, 2], dtype=torch.int32, device="cuda"), most=4)
    assert tree_layer.cache.lengths.tolist() == [10, 8]
    for i in range(4):
        x, _ = one.attend(torch.stack([drafts[0, int(rows[0, i])], drafts[1, max(0, int(rows[1, i]))]]), zero)
        for b in range(2 if i < 2 else 1):
            assert float((x[b] - out[b, int(rows[b, i])]).norm() / x[b].norm()) < 0.02, (i, b)
        one.accept()
    # every accepted token gave a weight of one for each query head
    for layer, n in ((tree_layer, [10, 8]), (one, [10, 10])):
        w = torch.stack([layer.weights[b, :, :n[b]].sum(-1) for b in range(2)])
        assert bool((w - torch.tensor(n, device="cuda")[:, None] * 4.0).abs().max() < 1e-3)


def test_a_budget_is_kept_and_the_ends_stay():
    m = _layer()
    layer = m.Layer(2, 4, budget=32, **SMALL)
    g = torch.Generator(device="cuda").manual_seed(6)
    depth = torch.arange(4, device="cuda").repeat(2, 1)
    for step in range(20):
        layer.attend(torch.randn(8, 512, generator=g, device="cuda"), depth)
        layer.accept(None, torch.tensor([4, 3], dtype=torch.int32, device="cuda"))
    assert layer.cache.lengths.tolist() == [32, 32] and layer.seen.tolist() == [80, 60]
    for b, seen in enumerate((80, 60)):
        for h in range(2):
            kept = sorted(layer.positions[b, h, :32].tolist())
            assert len(set(kept)) == 32 and kept[:4] == [0, 1, 2, 3] and kept[-8:] == list(range(seen - 8, seen))
