"""The example layer with its cache in 8 bits and its drafted tokens verified: what a tree gives is what decoding the kept path token by token
does, and steps of everything together keep what the definition keeps."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from test_layer_example import SMALL, _layer  # noqa: E402
from test_serving_ops import _verified  # noqa: E402

pytestmark = pytest.mark.gpu


def test_a_tree_over_8_bits_is_the_path_that_was_kept():
    m = _layer()
    g = torch.Generator(device="cuda").manual_seed(5)
    tree_layer, one = m.Layer(2, 6, budget=64, bits=8, **SMALL), m.Layer(2, 1, budget=64, bits=8, **SMALL)
    wide = m.Layer(2, 6, budget=64, bits=16, **SMALL)
    prompt = torch.randn(2, 6, 512, generator=g, device="cuda")
    depth = torch.arange(6, device="cuda").repeat(2, 1)
    chain, _ = tree_layer.attend(prompt.reshape(12, 512).clone(), depth)
    chain = chain.view(2, 6, 512).clone()
    same, _ = wide.attend(prompt.reshape(12, 512).clone(), depth)
    # (the cache is empty, new tokens are BF16 either way: the same numbers, for all that 8 bits are none of them)
    assert torch.equal(same.view(2, 6, 512), chain)
    tree_layer.accept(), wide.accept()
    zero = torch.zeros(2, 1, dtype=torch.long, device="cuda")
    for t in range(6):
        x, _ = one.attend(prompt[:, t].clone(), zero)
        # earlier tokens come from the cache here: off by 2^-4 of an element at most, by 2^-5 or so of what a head sums up, of which the
        # residual stream is many times the size
        assert float((x - chain[:, t]).norm() / x.norm()) < 0.05, t
        one.accept()
    assert one.cache.lengths.tolist() == tree_layer.cache.lengths.tolist() == [6, 6]
    words = m.fgmp.tree_words([[-1, 0, 0, 1, 2, 4]] * 2).cuda()
    depth = torch.tensor([[0, 1, 1, 2, 2, 3]] * 2, device="cuda")
    drafts = torch.randn(2, 6, 512, generator=g, device="cuda")
    out, _ = tree_layer.attend(drafts.reshape(12, 512).clone(), depth, words)
    out = out.view(2, 6, 512).clone()
    near, _ = wide.attend(drafts.reshape(12, 512).clone(), depth, words)
    assert float((near.view(2, 6, 512) - out).norm() / out.norm()) < 0.05
    rows = torch.tensor([[0, 2, 4, 5], [0, 1, -1, -1]], dtype=torch.int32, device="cuda")
    tree_layer.accept(rows, torch.tensor([4, 2], dtype=torch.int32, device="cuda"), most=4)
    assert tree_layer.cache.lengths.tolist() == [10, 8]
    for i in range(4):
        x, _ = one.attend(torch.stack([drafts[0, int(rows[0, i])], drafts[1, max(0, int(rows[1, i]))]]), zero)
        for b in range(2 if i < 2 else 1):
            assert float((x[b] - out[b, int(rows[b, i])]).norm() / x[b].norm()) < 0.05, (i, b)
        one.accept()


@pytest.mark.parametrize("bits", [8, 16])
def test_steps_keep_what_the_definition_keeps(bits):
    m = _layer()
    batch, tokens, vocab = 3, 8, 1111
    layer = m.Layer(batch, tokens, budget=48, bits=bits, **SMALL)
    head = m.Head(batch, tokens, 512, vocab)
    g = torch.Generator(device="cuda").manual_seed(9)
    parents = torch.tensor([[-1, 0, 0, 1, 1, 2, 3, 5]], dtype=torch.int32).repeat(batch, 1)
    tree, depth = m.fgmp.tree_words(parents).cuda(), torch.tensor([[0, 1, 1, 2, 2, 2, 3, 3]], device="cuda").repeat(batch, 1)
    counts = torch.tensor([8, 3, 8], dtype=torch.int32, device="cuda")
    expected = [0] * batch
    for step in range(6):
        _, h = layer.attend(torch.randn(batch * tokens, 512, generator=g, device="cuda"), depth, tree)
        target = head.distributions(h)
        assert bool((target.sum(-1) - 1).abs().max() < 1e-4)
        likely = target.topk(3, -1).indices
        drafted = likely[torch.arange(batch, device="cuda")[:, None], parents.cuda().clamp(min=0).long(), torch.randint(0, 3, (batch, tokens), generator=g, device="cuda")].int()
        u = torch.rand(batch, tokens, generator=g, device="cuda") * 0.3
        rows, accepted, behind = head.verify(target, drafted, u, parents.cuda(), counts)
        want = _verified(target, drafted, u, None, parents, counts.tolist())
        assert (rows.tolist(), accepted.tolist(), behind.tolist()) == want
        layer.accept(rows, accepted, most=4)
        expected = [min(48 if bits == 16 else 64, n + c) for n, c in zip(expected, want[1])]
        assert layer.cache.lengths.tolist() == expected, step
    assert max(expected) > 6
