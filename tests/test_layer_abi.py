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


def test_more_workgroups_than_a_grid_counts_are_refused():
    L, many = fgmp.lib(), 65535
    c = _cache(batch=many, heads=many)
    assert _attend(cache=c, q_heads=many, ws_n=1 << 62) == UNSUPPORTED
    assert L.fgmp_attention_weights(_heads(), AT, 2, many, c, None, 2, None, 0.5, 0, AT, AT, 256, None) == UNSUPPORTED
    assert L.fgmp_cache_append(_heads(), _heads(), 1, 1 << 20, c, None, 1 << 20, None, None, None, None, 0, AT + 64, None) == UNSUPPORTED
    assert L.fgmp_cache_evict(c, AT, AT, 256, AT, 10, 0, 0, AT, AT, AT + 64, AT, 1 << 62, None) == UNSUPPORTED


@pytest.mark.parametrize("slots,heads", [(64, 129), (2048, 129), (4096, 65), (16384, 65)])
def test_an_eviction_of_more_threads_than_a_launch_counts_is_refused(slots, heads):
    """A launch counts its threads in 32 bits: 512 for a sequence and head up to 2048 slots, 1024 above.  The launch that moves has fewer: it
    must not run over moves that the one before it has not written."""
    c = _cache(batch=65535, heads=heads, pages_per_sequence=slots // 64, table_stride=slots // 64)
    assert 65535 * (heads - 1) * (512 if slots <= 2048 else 1024) < 1 << 32 <= 65535 * heads * (512 if slots <= 2048 else 1024)
    assert fgmp.lib().fgmp_cache_evict(c, AT, AT, slots, AT, 10, 0, 0, AT, AT, AT + 64, AT, 1 << 62, None) == UNSUPPORTED


def test_more_threads_than_a_launch_counts_are_refused():
    """2^32 threads, in workgroups of 256 or 512, are too many: each call just past that."""
    L, many = fgmp.lib(), 65535
    # attention: one workgroup of 256 for each head of a sequence, 512 where a head has more than 128 rows
    assert _attend(cache=_cache(batch=many, heads=257), tokens=1, q_heads=257, max_length=1) == UNSUPPORTED
    wide = _cache(batch=many, heads=129)
    assert _attend(cache=wide, tokens=129, q_heads=129, max_length=1, q=_heads(strides=(1 << 16, 128, 1 << 12)), out=_heads(strides=(1 << 16, 128, 1 << 12)),
                   k=_heads(strides=(1 << 16, 128, 1 << 12)), v=_heads(strides=(1 << 16, 128, 1 << 12))) == UNSUPPORTED
    # weights: at least one workgroup of 256 for each head of a sequence
    assert L.fgmp_attention_weights(_heads(), AT, 2, 257, _cache(batch=many, heads=257), None, 2, None, 0.5, 0, AT, AT, 256, None) == UNSUPPORTED
    # append: one of 256 for each token of up to 16 heads
    assert L.fgmp_cache_append(_heads(), _heads(), 1, 257, _cache(batch=many), None, 257, None, None, None, None, 0, AT + 64, None) == UNSUPPORTED

    def norm(M, K):
        return L.fgmp_block_norm(AT, 1, K, None, 1, 0, None, 0, 1, 0, M, K, None, None, AT, None, 0, 1e-5, 1.0, 1.0, None, 0, AT, 1, K, None)

    # norms: as many threads as a row has
    for K, threads in [(64, 16), (128, 16), (144, 32), (512, 64), (1024, 64), (2048, 256), (4096, 256), (8192, 512), (16384, 1024), (32768, 1024)]:
        assert norm((1 << 32) // threads, K) == UNSUPPORTED, K


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


# ---- the extension module's way ----

class _Tensor:
    """What the binding asks of a GPU tensor, without one."""

    def __init__(self, at, shape, dtype=torch.float32, stride=None, cuda=True):
        self.at, self.shape, self.dtype, self.is_cuda = at, torch.Size(shape), dtype, cuda
        self._stride = stride or torch.empty(shape, device="meta").stride()

    def data_ptr(self):
        return self.at

    def stride(self):
        return self._stride


class _Handle:
    def __init__(self):
        self.struct = fgmp._CacheStruct()
        self.fast = (ctypes.addressof(self.struct), 2, 3, 64, 40, torch.bfloat16)


I64, VP, F, SZ, I = ctypes.c_int64, ctypes.c_void_p, ctypes.c_float, ctypes.c_size_t, ctypes.c_int
HEADS = ctypes.POINTER(fgmp._HeadsStruct)
_NUMBERS = {ctypes.c_int64, ctypes.c_float, ctypes.c_size_t, ctypes.c_int}


def _told(name, given, *argtypes):
    """What the entry point is called with when the extension is given `given`, and the answer; heads as tuples."""
    got = []

    def entry(*a):
        got.append(tuple((x.contents.data, x.contents.batch_stride, x.contents.token_stride, x.contents.head_stride) if t is HEADS and x else
                         None if t is HEADS else x for x, t in zip(a, argtypes)))
        return -4

    f = ctypes.CFUNCTYPE(ctypes.c_int, *argtypes)(entry)
    fgmp.lib()
    rc = getattr(fgmp._call, name)(ctypes.cast(f, VP).value, fgmp._TYPES, *given, 0x77)
    assert (rc is None) == (not got) and rc in (None, -4)
    return got[0] if got else None


def _t(at, *shape, dtype=torch.float32, **more):
    return _Tensor(at, shape, dtype, **more)


BF, I32 = torch.bfloat16, torch.int32


def test_the_extension_hands_on_attention():
    h = _Handle()
    q, out = _t(16, 2, 5, 6, 64, dtype=BF, stride=(4000, 800, 64, 1)), _t(32, 2, 5, 6, 64, dtype=BF)
    k, v = _t(48, 2, 5, 3, 64, dtype=BF), _t(64, 2, 5, 3, 64, dtype=BF, stride=(9000, 1000, 128, 1))
    tree, counts, lse, ws = _t(80, 2, 5, 1, dtype=torch.int64), _t(96, 2, dtype=I32), _t(112, 2, 5, 6), _t(128, 999, dtype=torch.uint8)
    types = (HEADS, HEADS, HEADS, I64, I64, VP, VP, VP, F, I64, HEADS, VP, VP, SZ, VP)
    given = [q, k, v, h.fast, tree, counts, 0.25, 33, out, lse, ws]
    want = ((16, 4000, 800, 64), (48, 960, 192, 64), (64, 9000, 1000, 128), 5, 6, h.fast[0], 80, 96, 0.25, 33, (32, 1920, 384, 64), 112, 128, 999, 0x77)
    assert _told("tree_attention", given, *types) == want
    assert _told("tree_attention", given[:1] + [None, None] + given[3:4] + [None, None] + given[6:], *types) == want[:1] + (None, None) + want[3:6] + (None, None) + want[8:]
    bad = {0: [_t(16, 2, 5, 6, 64), _t(16, 2, 5, 6, 32, dtype=BF), _t(16, 3, 5, 6, 64, dtype=BF), _t(16, 2, 5, 6, 64, dtype=BF, cuda=False),
               _t(16, 2, 5, 6, 64, dtype=BF, stride=(1920, 384, 1, 6)), None, 7],
           1: [_t(48, 2, 4, 3, 64, dtype=BF), _t(48, 2, 5, 6, 64, dtype=BF), None], 4: [_t(80, 2, 5, 2, dtype=torch.int64), _t(80, 2, 5, 1, dtype=I32)],
           5: [_t(96, 2, dtype=torch.int64), _t(96, 3, dtype=I32), _t(96, 2, dtype=I32, stride=(2,))], 6: [None, "x"], 7: [1.5, None],
           8: [_t(32, 2, 5, 6, 64)], 9: [_t(112, 2, 6, 5), _t(112, 2, 5, 6, stride=(60, 12, 2)), None], 10: [None, _t(128, 9, dtype=I32)]}
    for at, values in bad.items():
        for value in values:
            assert _told("tree_attention", given[:at] + [value] + given[at + 1:], *types) is None, (at, value)
    # 70 tokens take two words
    g70 = [_t(16, 2, 70, 6, 64, dtype=BF), None, None, h.fast, _t(80, 2, 70, 2, dtype=torch.int64), None, 1, 0, _t(32, 2, 70, 6, 64, dtype=BF), _t(112, 2, 70, 6), ws]
    assert _told("tree_attention", g70, *types)[3:9] == (70, 6, h.fast[0], 80, None, 1.0)


def test_the_extension_hands_on_weights_append_and_evict():
    h = _Handle()
    types = (HEADS, VP, I64, I64, VP, VP, I64, VP, F, I64, VP, VP, I64, VP)
    given = [_t(16, 2, 5, 6, 64, dtype=BF), _t(32, 2, 5, 6), h.fast, _t(48, 2, 3, 50), _t(64, 2, 4, dtype=I32), _t(80, 2, dtype=I32), 0.5, 0, _t(96, 2, 3, 50)]
    want = ((16, 1920, 384, 64), 32, 5, 6, h.fast[0], 64, 4, 80, 0.5, 0, 48, 96, 50, 0x77)
    assert _told("attention_weights", given, *types) == want
    assert _told("attention_weights", given[:4] + [None, None] + given[6:], *types)[5:8] == (None, 5, None)
    for at, value in [(3, _t(48, 2, 4, 50)), (8, _t(96, 2, 3, 51)), (4, _t(64, 3, 4, dtype=I32)), (1, _t(32, 2, 5, 6, dtype=BF))]:
        assert _told("attention_weights", given[:at] + [value] + given[at + 1:], *types) is None, at

    types = (HEADS, HEADS, I, I64, VP, VP, I64, VP, VP, VP, VP, I64, VP, VP)
    given = [_t(16, 2, 5, 3, 64), _t(32, 2, 5, 3, 64), h.fast, None, _t(48, 2, dtype=I32), _t(64, 2, 5, dtype=I32), _t(80, 2, 3, 41, dtype=I32), _t(96, 2, 3, 41), _t(112, 2, dtype=I32)]
    want = ((16, 960, 192, 64), (32, 960, 192, 64), 0, 5, h.fast[0], None, 5, 48, 64, 80, 96, 41, 112, 0x77)
    assert _told("cache_append", given, *types) == want
    both = _told("cache_append", [_t(16, 2, 5, 3, 64, dtype=BF), _t(32, 2, 5, 3, 64, dtype=BF)] + given[2:5] + [None, None, None] + given[8:], *types)
    assert both[2] == 1 and both[8:12] == (None, None, None, 0)
    for at, value in [(0, _t(16, 2, 5, 3, 64, dtype=BF)), (1, _t(32, 2, 5, 4, 64)), (6, _t(80, 2, 3, 40, dtype=I32)), (8, None)]:
        assert _told("cache_append", given[:at] + [value] + given[at + 1:], *types) is None, at

    types = (VP, VP, VP, I64, VP, I64, I64, I64, VP, VP, VP, VP, SZ, VP)
    given = [h.fast, _t(16, 2, 3, 40), _t(32, 2, 3, 40, dtype=I32), _t(48, 2, dtype=I32), 30, 4, 5, _t(64, 2, 3, 40), _t(80, 2, 3, 40, dtype=I32),
             _t(96, 2, dtype=I32), _t(112, 77, dtype=torch.uint8)]
    assert _told("cache_evict", given, *types) == (h.fast[0], 16, 32, 40, 48, 30, 4, 5, 64, 80, 96, 112, 77, 0x77)
    for at, value in [(1, _t(16, 2, 3, 39)), (2, _t(32, 2, 3, 40)), (4, 1.0), (7, None), (9, _t(96, 3, dtype=I32)), (10, None)]:
        assert _told("cache_evict", given[:at] + [value] + given[at + 1:], *types) is None, at


def test_the_extension_hands_on_norms():
    types = (VP, I, I64, VP, I, I64, VP, I64, I64, I, I64, I64, VP, VP, VP, VP, I, F, F, F, VP, I64, VP, I, I64, VP)
    vec = [_t(200 + 16 * i, 32) for i in range(4)]
    given = [_t(16, 5, 32, dtype=BF, stride=(40, 1)), _t(32, 5, 32), _t(48, 3, 32, stride=(48, 1)), 2, 1, *vec, 1, 0.5, 0.25, 2, _t(64, 5, 32, dtype=BF), _t(80, 5, 32)]
    want = (16, 1, 40, 32, 0, 32, 48, 48, 2, 1, 5, 32, 200, 216, 232, 248, 1, 0.5, 0.25, 2.0, 64, 32, 80, 0, 32, 0x77)
    assert _told("block_norm", given, *types) == want
    first = _told("block_norm", [given[0], None, None, 1, 0, None, None, vec[2], None, 0, 1e-5, 1.0, 1.0, None, given[14]], *types)
    assert first[3] is None and first[6] is None and first[12:16] == (None, None, 232, None) and first[20] is None
    for at, value in [(0, _t(16, 5, 32, dtype=I32)), (1, _t(32, 4, 32)), (2, _t(48, 2, 32)), (2, _t(48, 3, 32, dtype=BF)), (2, _t(48, 32)), (3, 0), (5, _t(200, 31)),
                      (5, _t(200, 32, dtype=BF)), (13, _t(64, 5, 32)), (14, _t(80, 5, 32, stride=(1, 5)))]:
        assert _told("block_norm", given[:at] + [value] + given[at + 1:], *types) is None, (at, value)


@pytest.mark.parametrize("name,count", [("tree_attention", 14), ("attention_weights", 12), ("cache_append", 12), ("cache_evict", 14), ("block_norm", 18)])
def test_the_extension_counts_its_arguments(name, count):
    fgmp.lib()
    f = getattr(fgmp._call, name)
    with pytest.raises(TypeError):
        f(*[None] * (count - 1))
    assert f(*[None] * count) is None and f(0, (1, 2), *[None] * (count - 2)) is None
