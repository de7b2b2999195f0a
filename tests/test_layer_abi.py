"""Host-side checks of the entry points between a layer's products, without a GPU: sizes, and refusals before anything is launched."""
import ctypes

import pytest
import torch

from paper_2504_14152_amd import fgmp

OK, INVALID, SHAPE, ALIGN, SMALL, UNSUPPORTED = 0, -1, -2, -3, -4, -5
AT = 4096   # an address, aligned


def _cache(**change):
    c = dict(k=AT, v=AT, dtype=1, batch=2, heads=2, head_dim=128, page_size=64, pages_per_sequence=4, pages=10, page_stride=64 * 256,
             token_stride=256, head_stride=128, page_table=AT, table_stride=4, lengths=AT)
    c.update(change)
    return ctypes.byref(fgmp._CacheStruct(*(c[n] for n, _ in fgmp._CacheStruct._fields_)))


def _heads(data=AT, strides=(1024, 512, 128)):
    return ctypes.byref(fgmp._HeadsStruct(data, *strides))


def _attend(cache=None, q=None, k=None, v=None, out=None, tokens=2, q_heads=4, scale=0.5, max_length=0, lse=AT, ws=AT, ws_n=1 << 30):
    q, k, v, out = q or _heads(), k or _heads(), v or _heads(), out or _heads()
    return fgmp.lib().fgmp_tree_attention(q, k, v, tokens, q_heads, cache or _cache(), None, None, scale, max_length, out, lse, ws, ws_n, None)


CACHES = [(dict(k=None), INVALID), (dict(v=None), INVALID), (dict(lengths=None), INVALID), (dict(dtype=7), INVALID), (dict(batch=0), INVALID),
          (dict(heads=-1), INVALID), (dict(page_size=0), INVALID), (dict(pages=0), INVALID), (dict(pages_per_sequence=0), INVALID),
          (dict(head_dim=96), UNSUPPORTED), (dict(page_size=24), SHAPE), (dict(table_stride=3), SHAPE), (dict(page_table=None), SHAPE),
          (dict(page_table=None, pages_per_sequence=1, pages=1), SHAPE), (dict(token_stride=64), SHAPE), (dict(head_stride=64), SHAPE),
          (dict(page_stride=0), SHAPE), (dict(token_stride=260), ALIGN), (dict(head_stride=132), ALIGN), (dict(page_stride=64 * 256 + 4), ALIGN),
          (dict(k=AT + 8), ALIGN), (dict(v=AT + 2), ALIGN), (dict(lengths=AT + 2), ALIGN), (dict(token_stride=1 << 27), UNSUPPORTED),
          (dict(page_size=1 << 20, pages_per_sequence=1 << 12, table_stride=1 << 12), UNSUPPORTED)]


@pytest.mark.parametrize("change,code", CACHES)
def test_a_cache_that_does_not_hold_together_is_refused_everywhere(change, code):
    L = fgmp.lib()
    c = _cache(**change)
    assert _attend(cache=c) == code
    assert L.fgmp_attention_weights(_heads(), AT, 2, 4, c, None, 2, None, 0.5, 0, AT, AT, 256, None) == code
    assert L.fgmp_cache_append(_heads(), _heads(), 1, 2, c, None, 2, None, None, None, None, 0, AT + 64, None) == code
    assert L.fgmp_cache_evict(c, AT, AT, 256, AT, 10, 0, 0, AT, AT, AT + 64, AT, 1 << 30, None) == code


def test_attention_refuses():
    L = fgmp.lib()
    assert _attend(tokens=0) == INVALID and _attend(q_heads=0) == INVALID and _attend(lse=None) == INVALID
    assert _attend(scale=0.0) == INVALID and _attend(scale=-1.0) == INVALID and _attend(scale=float("nan")) == INVALID and _attend(scale=float("inf")) == INVALID
    assert _attend(max_length=-1) == INVALID and _attend(q_heads=5) == SHAPE and _attend(tokens=1025) == UNSUPPORTED
    assert _attend(q=_heads(None)) == INVALID and _attend(q=_heads(AT + 8)) == ALIGN and _attend(q=_heads(strides=(1024, 516, 128))) == ALIGN
    assert _attend(out=_heads(strides=(1024, 0, 128))) == SHAPE and _attend(out=_heads(strides=(1024, 512, 64))) == SHAPE
    assert _attend(q=_heads(strides=(-1024, 512, 128))) == SHAPE
    for bad in (_heads(None), _heads(AT + 8)):
        assert _attend(k=bad) in (INVALID, ALIGN) and _attend(v=bad) in (INVALID, ALIGN)
    assert L.fgmp_tree_attention(_heads(), None, _heads(), 2, 4, _cache(), None, None, 0.5, 0, _heads(), AT, AT, 1 << 30, None) == INVALID
    assert L.fgmp_tree_attention(None, None, None, 2, 4, _cache(), None, None, 0.5, 0, _heads(), AT, AT, 1 << 30, None) == INVALID
    assert L.fgmp_tree_attention(_heads(), None, None, 2, 4, None, None, None, 0.5, 0, _heads(), AT, AT, 1 << 30, None) == INVALID
    need = fgmp.tree_attention_workspace_bytes(2, 2, 4, 2, 128, 256)
    assert need > 16
    assert _attend(ws_n=need - 1) == SMALL and _attend(ws=None) == INVALID and _attend(ws=AT + 4) == ALIGN


def test_sizes():
    wb = fgmp.tree_attention_workspace_bytes
    assert wb(0, 1, 8, 8, 128, 10) == 0 and wb(1, 1, 8, 3, 128, 10) == 0 and wb(1, 1, 8, 8, 96, 10) == 0 and wb(1, 2000, 8, 8, 128, 10) == 0
    for shape in [(1, 1, 32, 32, 128), (8, 25, 64, 8, 128), (3, 64, 16, 16, 64), (1, 1000, 8, 1, 256), (64, 1, 64, 8, 128)]:
        sizes = [wb(*shape, n) for n in (0, 1, 100, 128, 129, 1000, 5000, 40000, 131072, 1 << 20)]
        assert sizes == sorted(sizes) and sizes[0] >= 16      # one workspace serves all shorter sequences
        assert sizes[-1] < 1 << 30
    ev = fgmp.cache_evict_workspace_bytes
    assert ev(0, 1, 10, 5) == 0 and ev(1, 1, 10, 0) == 0
    assert ev(2, 8, 1000, 1000) >= 2 * 8 * 4 and ev(2, 8, 1000, 400) >= 2 * 8 * (4 + 8 * 400)


def test_weights_append_and_evict_refuse():
    L = fgmp.lib()

    def weights(q=None, lse=AT, tokens=2, q_heads=4, rows=None, accepted=2, scale=0.5, w=AT, out=AT, stride=256):
        return L.fgmp_attention_weights(q or _heads(), lse, tokens, q_heads, _cache(), rows, accepted, None, scale, 0, w, out, stride, None)

    assert weights(lse=None) == INVALID and weights(w=None) == INVALID and weights(out=None) == INVALID and weights(accepted=0) == INVALID
    assert weights(q_heads=3) == SHAPE and weights(accepted=3) == SHAPE and weights(stride=255) == SHAPE and weights(scale=0.0) == INVALID
    assert weights(tokens=2000, accepted=2) == UNSUPPORTED and weights(q=_heads(AT + 4)) == ALIGN

    def append(k=None, v=None, dt=1, tokens=2, rows=None, accepted=2, positions=None, sp=None, sw=None, stride=256, out=AT + 64):
        return L.fgmp_cache_append(k or _heads(), v or _heads(), dt, tokens, _cache(), rows, accepted, None, positions, sp, sw, stride, out, None)

    assert append(out=None) == INVALID and append(out=AT) == INVALID        # (the cache's own lengths)
    assert append(dt=9) == INVALID and append(tokens=0) == INVALID and append(accepted=3) == SHAPE and append(sp=AT) == INVALID
    assert append(sw=AT, stride=255) == SHAPE and append(k=_heads(None)) == INVALID and append(v=_heads(AT + 8)) == ALIGN

    def evict(w=AT, p=AT, seen=AT, budget=10, sinks=0, recent=0, wo=AT, po=AT, lo=AT + 64, ws=AT, n=1 << 30, stride=256):
        return L.fgmp_cache_evict(_cache(), w, p, stride, seen, budget, sinks, recent, wo, po, lo, ws, n, None)

    for missing in ("w", "p", "seen", "wo", "po", "lo", "ws"):
        assert evict(**{missing: None}) == INVALID, missing
    assert evict(lo=AT) == INVALID and evict(budget=0) == INVALID and evict(sinks=-1) == INVALID and evict(recent=-1) == INVALID
    assert evict(stride=255) == SHAPE and evict(ws=AT + 8) == ALIGN and evict(n=fgmp.cache_evict_workspace_bytes(2, 2, 256, 10) - 1) == SMALL


def test_norms_refuse():
    L = fgmp.lib()

    def norm(x=AT, xd=1, ldx=256, o=AT, od=0, ldo=256, gate=AT, ldg=256, gr=1, act=0, M=4, K=256, pw=AT, pb=AT, qw=AT, qb=AT, kind=0, eps=1e-5, y=AT,
             ldy=256, h=AT, hd=1, ldh=256):
        return L.fgmp_block_norm(x, xd, ldx, o, od, ldo, gate, ldg, gr, act, M, K, pw, pb, qw, qb, kind, eps, 1.0, 1.0, y, ldy, h, hd, ldh, None)

    assert norm(x=None) == INVALID and norm(M=0) == INVALID and norm(K=0) == INVALID and norm(kind=2) == INVALID and norm(act=3) == INVALID
    assert norm(eps=-1.0) == INVALID and norm(eps=float("nan")) == INVALID and norm(o=None) == INVALID and norm(y=None) == INVALID
    assert norm(h=None) == INVALID and norm(qw=None) == INVALID and norm(pw=None) == INVALID and norm(gr=0) == INVALID
    assert norm(o=None, y=None) == INVALID                   # a gate and a post norm without a block
    assert norm(o=None, y=None, gate=None, pw=None, pb=None, h=None, qw=None, qb=None) == INVALID   # nothing to do
    assert norm(xd=3) == INVALID and norm(od=3) == INVALID and norm(hd=-1) == INVALID
    assert norm(K=24) == SHAPE and norm(K=32784, ldx=1 << 16, ldo=1 << 16, ldg=1 << 16, ldy=1 << 16, ldh=1 << 16) == UNSUPPORTED
    for name in ("ldx", "ldo", "ldg", "ldy", "ldh"):
        assert norm(**{name: 240}) == SHAPE, name
        assert norm(**{name: 257}) == ALIGN, name
    for name in ("x", "o", "gate", "pw", "pb", "qw", "qb", "y", "h"):
        assert norm(**{name: AT + 8}) == ALIGN, name


def test_trees_from_parents():
    words = fgmp.tree_words([[-1, 0, 0, 1, -1]])
    assert words.tolist() == [[[0b1], [0b11], [0b101], [0b1011], [0b10000]]]
    chain = fgmp.tree_words([list(range(-1, 69))])
    assert chain.shape == (1, 70, 2)
    for t in (0, 62, 63, 64, 69):
        both = (chain[0, t, 0].item() & (1 << 64) - 1) | (chain[0, t, 1].item() & (1 << 64) - 1) << 64
        assert both == (1 << t + 1) - 1
    for bad in ([[0]], [[-1, 1]], [[-2]]):
        with pytest.raises(fgmp.FgmpError):
            fgmp.tree_words(bad)


def test_the_binding_wants_gpu_tensors():
    x = torch.zeros(1, 16, 1, 64)
    n = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(fgmp.FgmpError):
        fgmp.Cache(x, x, n)
    with pytest.raises(fgmp.FgmpError):
        fgmp.block_norm(torch.zeros(1, 16), pre_weight=torch.ones(16))
