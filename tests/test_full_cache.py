"""The example layer at the end of its cache: in 16 bits it keeps to its budget, in 8 bits it says that the cache is full and keeps what it has,
rather than drop tokens whose positions later ones count."""
import os
import sys
import types

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from test_layer_example import SMALL, _layer  # noqa: E402


def _bare(monkeypatch, slots, lengths, tokens):
    """A layer with a cache in 8 bits and nothing else, whose appends do what fgmp_quant_cache_append does to lengths, on the CPU."""
    m = _layer()

    def append(k, v, cache, rows=None, counts=None, lengths_out=None):
        grown = tokens if counts is None else counts
        return lengths_out.copy_((cache.lengths + grown).clamp(max=cache.slots))

    monkeypatch.setattr(m.fgmp, "cache_append", append)
    layer = m.Layer.__new__(m.Layer)
    n = torch.tensor(lengths, dtype=torch.int32)
    layer.bits, layer.tokens, layer.k, layer.v = 8, tokens, None, None
    layer.cache, layer.lengths = types.SimpleNamespace(lengths=n.clone(), slots=slots), [n.clone(), n.clone()]
    layer.seen, layer.held = n.long(), int(n.max())
    return layer


def test_a_full_cache_in_8_bits_is_said_to_be_full(monkeypatch):
    layer = _bare(monkeypatch, 32, [25, 3], 4)
    layer.accept()
    assert layer.cache.lengths.tolist() == layer.seen.tolist() == [29, 7]
    with pytest.raises(RuntimeError, match="full"):
        layer.accept()
    assert layer.cache.lengths.tolist() == layer.seen.tolist() == [29, 7]      # (nothing was kept in part)
    layer.accept(torch.zeros(2, 4, dtype=torch.int32), torch.tensor([3, 4], dtype=torch.int32))
    assert layer.cache.lengths.tolist() == layer.seen.tolist() == [32, 11]
    with pytest.raises(RuntimeError, match="full"):
        layer.accept(torch.zeros(2, 4, dtype=torch.int32), torch.tensor([1, 0], dtype=torch.int32), most=1)
    layer.accept(torch.zeros(2, 4, dtype=torch.int32), torch.tensor([0, 2], dtype=torch.int32), most=4)
    assert layer.cache.lengths.tolist() == layer.seen.tolist() == [32, 13] and layer.held == 32


def test_it_is_not_full_before_a_sequence_is(monkeypatch):
    """What is known without asking the GPU is a bound: one token a step of at most four."""
    layer = _bare(monkeypatch, 32, [0, 0], 4)
    one = torch.ones(2, dtype=torch.int32)
    for step in range(32):
        layer.accept(torch.zeros(2, 4, dtype=torch.int32), one, most=4)
        assert step < layer.held <= 32 and layer.seen.tolist() == [step + 1] * 2
    with pytest.raises(RuntimeError, match="full"):
        layer.accept(torch.zeros(2, 4, dtype=torch.int32), one, most=4)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 16])
def test_steps_up_to_the_budget_and_past_it(bits):
    m = _layer()
    batch, tokens, budget = 3, 4, 48
    layer = m.Layer(batch, tokens, budget=budget, bits=bits, **SMALL)
    most = layer.cache.slots if bits == 8 else budget
    g = torch.Generator(device="cuda").manual_seed(11)
    depth = torch.arange(tokens, device="cuda").repeat(batch, 1)
    counts = torch.tensor([4, 1, 3], dtype=torch.int32, device="cuda")
    rows = torch.arange(tokens, dtype=torch.int32, device="cuda").repeat(batch, 1)
    held, seen = [0] * batch, [0] * batch
    for step in range(20):
        x, _ = layer.attend(torch.randn(batch * tokens, 512, generator=g, device="cuda"), depth)
        assert bool(torch.isfinite(x).all()), step
        full = bits == 8 and held[0] + 4 > most
        if full:
            with pytest.raises(RuntimeError, match="full"):
                layer.accept(rows, counts, most=4)
        else:
            layer.accept(rows, counts, most=4)
            held, seen = [min(most, n + c) for n, c in zip(held, (4, 1, 3))], [n + c for n, c in zip(seen, (4, 1, 3))]
        assert layer.cache.lengths.tolist() == held and layer.seen.tolist() == seen, step
    assert held[0] == most and (seen[0] == (most if bits == 8 else 80))
