"""Host-side checks of rotated heads, the cache in 8 bits and the verification of drafted tokens, without a GPU: sizes, refusals before
anything is launched, and the extension module's way."""
import ctypes
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from paper_2504_14152_amd import fgmp  # noqa: E402
from test_layer_abi import ALIGN, AT, BF, CACHES, F, HEADS, I, I32, I64, INVALID, SHAPE, SMALL, SZ, UNSUPPORTED, VP, _heads, _t, _told  # noqa: E402

MANY = 65535


def _quant(k_scales=AT, v_scales=AT, scale_page_stride=128, scale_head_stride=64, **change):
    c = dict(k=AT, v=AT, dtype=2, batch=2, heads=2, head_dim=128, page_size=64, pages_per_sequence=4, pages=10, page_stride=64 * 256,
             token_stride=256, head_stride=128, page_table=AT, table_stride=4, lengths=AT)
    c.update(change)
    codes = fgmp._CacheStruct(*(c[n] for n, _ in fgmp._CacheStruct._fields_))
    return ctypes.byref(fgmp._QuantCacheStruct(codes, k_scales, v_scales, scale_page_stride, scale_head_stride))


def _attend(cache=None, q=None, k=None, v=None, out=None, tokens=2, q_heads=4, scale=0.5, max_length=0, lse=AT, ws=AT, ws_n=1 << 30):
    q, k, v, out = q or _heads(), k or _heads(), v or _heads(), out or _heads()
    return fgmp.lib().fgmp_quant_cache_attention(q, k, v, tokens, q_heads, cache or _quant(), None, None, scale, max_length, out, lse, ws, ws_n, None)


def _append(cache=None, k=None, v=None, dt=1, tokens=2, rows=None, accepted=2, out=AT + 64):
    return fgmp.lib().fgmp_quant_cache_append(k or _heads(), v or _heads(), dt, tokens, cache or _quant(), rows, accepted, None, out, None)


def _read(cache=None, first=0, tokens=2, k=None, v=None, dt=1):
    return fgmp.lib().fgmp_quant_cache_read(cache or _quant(), first, tokens, k or _heads(), v or _heads(), dt, None)


QUANT = [(change, code) for change, code in CACHES if not any(n in change for n in ("dtype", "token_stride", "head_stride", "page_stride", "page_table"))] + [
    (dict(dtype=1), INVALID), (dict(dtype=0), INVALID), (dict(dtype=7), INVALID), (dict(k_scales=None), INVALID), (dict(v_scales=None), INVALID),
    (dict(k_scales=AT + 4), ALIGN), (dict(v_scales=AT + 8), ALIGN), (dict(scale_page_stride=48), SHAPE), (dict(scale_head_stride=48), SHAPE),
    (dict(scale_page_stride=136), ALIGN), (dict(scale_head_stride=72), ALIGN), (dict(scale_page_stride=1 << 41), UNSUPPORTED),
    (dict(token_stride=64), SHAPE), (dict(head_stride=64), SHAPE), (dict(page_stride=0), SHAPE), (dict(token_stride=264), ALIGN), (dict(head_stride=136), ALIGN),
    (dict(page_stride=64 * 256 + 8), ALIGN), (dict(token_stride=1 << 27), UNSUPPORTED), (dict(page_table=None), SHAPE),
    (dict(page_table=None, pages_per_sequence=1, page_size=72), SHAPE), (dict(page_table=None, pages_per_sequence=1, pages=1), SHAPE)]


@pytest.mark.parametrize("change,code", QUANT)
def test_a_cache_in_8_bits_that_does_not_hold_together_is_refused_everywhere(change, code):
    c = _quant(**change)
    assert _attend(cache=c) == code and _append(cache=c) == code and _read(cache=c) == code


def test_a_cache_in_8_bits_is_no_other_cache():
    L = fgmp.lib()
    c = ctypes.cast(_quant(), ctypes.POINTER(fgmp._CacheStruct))
    assert L.fgmp_tree_attention(_heads(), _heads(), _heads(), 2, 4, c, None, None, 0.5, 0, _heads(), AT, AT, 1 << 30, None) == INVALID
    assert L.fgmp_attention_weights(_heads(), AT, 2, 4, c, None, 2, None, 0.5, 0, AT, AT, 256, None) == INVALID
    assert L.fgmp_cache_append(_heads(), _heads(), 1, 2, c, None, 2, None, None, None, None, 0, AT + 64, None) == INVALID
    assert L.fgmp_cache_evict(c, AT, AT, 256, AT, 10, 0, 0, AT, AT, AT + 64, AT, 1 << 30, None) == INVALID
    assert L.fgmp_quant_cache_read(None, 0, 2, _heads(), _heads(), 1, None) == INVALID


def test_attention_over_8_bits_refuses():
    assert _attend(tokens=0) == INVALID and _attend(q_heads=0) == INVALID and _attend(lse=None) == INVALID and _attend(max_length=-1) == INVALID
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert _attend(scale=scale) == INVALID
    assert _attend(q_heads=5) == SHAPE and _attend(tokens=1025) == UNSUPPORTED
    assert _attend(q=_heads(None)) == INVALID and _attend(q=_heads(AT + 8)) == ALIGN and _attend(q=_heads(strides=(1024, 516, 128))) == ALIGN
    assert _attend(out=_heads(strides=(1024, 0, 128))) == SHAPE and _attend(k=_heads(AT + 8)) == ALIGN
    long = _quant(pages_per_sequence=64, table_stride=64)
    need = fgmp.tree_attention_workspace_bytes(2, 2, 4, 2, 128, 64 * 64)
    assert _attend(cache=long, ws_n=need - 1) == SMALL and _attend(cache=long, ws=None) == INVALID and _attend(cache=long, ws=AT + 4) == ALIGN
    assert _attend(cache=_quant(batch=MANY, heads=257), tokens=1, q_heads=257, max_length=1) == UNSUPPORTED


def test_append_and_read_refuse():
    assert _append(out=None) == INVALID and _append(out=AT) == INVALID and _append(dt=2) == INVALID and _append(tokens=0) == INVALID
    assert _append(accepted=3) == SHAPE and _append(accepted=0) == INVALID and _append(k=_heads(None)) == INVALID and _append(v=_heads(AT + 8)) == ALIGN
    assert _append(cache=_quant(batch=MANY), tokens=1 << 20, accepted=1 << 20) == UNSUPPORTED     # (2^32 threads and more)
    assert _read(first=-1) == INVALID and _read(tokens=0) == INVALID and _read(dt=2) == INVALID and _read(first=255) == SHAPE and _read(tokens=257) == SHAPE
    assert _read(first=(1 << 63) - 1, tokens=2) == SHAPE and _read(first=0, tokens=(1 << 63) - 1) == SHAPE
    assert _read(k=_heads(None)) == INVALID and _read(v=_heads(AT + 8)) == ALIGN and _read(k=_heads(strides=(1024, 0, 128))) == SHAPE
    big = _quant(batch=MANY, pages_per_sequence=1 << 14, table_stride=1 << 14, heads=64, token_stride=64 * 128, page_stride=64 * 64 * 128)
    far = _heads(strides=(1 << 38, 64 * 128, 128))
    assert _read(cache=big, tokens=1 << 20, k=far, v=far) == UNSUPPORTED


def _rotate(q=None, k="same", v="same", dt=0, batch=2, tokens=3, q_heads=4, heads=2, dim=128, qw=AT, kw=AT, kind=0, eps=1e-5, positions=AT, axes=1, axis_of=None,
            inv_freq=AT, rotary=128, interleaved=0, qo=None, ko="same", vo="same", odt=1):
    wide = _heads(strides=(4096, 1024, 128))
    q, k, v, qo, ko, vo = q or wide, wide if k == "same" else k, wide if v == "same" else v, qo or wide, wide if ko == "same" else ko, wide if vo == "same" else vo
    return fgmp.lib().fgmp_rotate_heads(q, k, v, dt, batch, tokens, q_heads, heads, dim, qw, kw, kind, eps, positions, axes, axis_of, inv_freq, rotary, interleaved,
                                        qo, ko, vo, odt, None)


def test_rotated_heads_refuse():
    L = fgmp.lib()
    assert L.fgmp_rotate_heads(None, None, None, 0, 1, 1, 1, 0, 64, None, None, 0, 1e-5, AT, 1, None, AT, 64, 0, _heads(), None, None, 1, None) == INVALID
    for bad in (dict(k=None), dict(ko=None), dict(v=None), dict(vo=None), dict(k=None, ko=None), dict(dt=2), dict(odt=5), dict(batch=0), dict(tokens=-1), dict(q_heads=0),
                dict(heads=0), dict(dim=0), dict(rotary=-8), dict(kind=2), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(positions=None),
                dict(inv_freq=None), dict(axes=0), dict(axes=2), dict(k=None, ko=None, v=None, vo=None), dict(q=_heads(None)), dict(qo=_heads(None))):
        assert _rotate(**bad) == INVALID, bad
    for bad in (dict(dim=124), dict(rotary=100), dict(rotary=136), dict(qo=_heads(strides=(4096, 1024, 64))), dict(ko=_heads(strides=(4096, 0, 128)))):
        assert _rotate(**bad) == SHAPE, bad
    for bad in (dict(dim=520, rotary=8, q=_heads(strides=(1 << 20, 1 << 16, 1024))), dict(batch=MANY + 1), dict(axes=1 << 17, axis_of=AT), dict(tokens=(1 << 30) + 1),
                dict(batch=MANY, tokens=1 << 20)):
        assert _rotate(**bad) == UNSUPPORTED, bad
    for bad in (dict(qw=AT + 8), dict(kw=AT + 4), dict(positions=AT + 2), dict(inv_freq=AT + 1), dict(axis_of=AT + 2), dict(q=_heads(AT + 8)), dict(vo=_heads(AT + 8)),
                dict(q=_heads(strides=(4096, 1026, 128)))):
        assert _rotate(**bad) == ALIGN, bad


def _verify(target=AT, dt=0, tb=1 << 20, tr=1 << 16, draft=None, db=1 << 20, dr=1 << 16, batch=2, tokens=4, vocab=1000, ids=AT, parents=None, counts=None, u=AT, rows=AT,
            accepted=AT, nxt=AT, ws=AT, n=1 << 30):
    return fgmp.lib().fgmp_verify_drafts(target, dt, tb, tr, draft, db, dr, batch, tokens, vocab, ids, parents, counts, u, rows, accepted, nxt, ws, n, None)


def test_verification_refuses():
    for bad in ("target", "ids", "u", "rows", "accepted", "nxt", "ws"):
        assert _verify(**{bad: None}) == INVALID, bad
    for bad in (dict(dt=2), dict(batch=0), dict(tokens=0), dict(vocab=-5), dict(draft=AT, parents=AT)):
        assert _verify(**bad) == INVALID, bad
    assert _verify(batch=16385) == UNSUPPORTED and _verify(tokens=1025) == UNSUPPORTED and _verify(vocab=(1 << 24) + 1) == UNSUPPORTED
    assert _verify(tb=-1) == SHAPE and _verify(tr=-4) == SHAPE and _verify(draft=AT, db=-1) == SHAPE and _verify(draft=AT, dr=-1) == SHAPE
    assert _verify(tr=1 << 41) == UNSUPPORTED
    for bad in (dict(target=AT + 2), dict(draft=AT + 2), dict(ids=AT + 1), dict(parents=AT + 2), dict(counts=AT + 2), dict(u=AT + 2), dict(rows=AT + 1), dict(accepted=AT + 2),
                dict(nxt=AT + 2), dict(ws=AT + 8)):
        assert _verify(**bad) == ALIGN, bad
    need = fgmp.verify_drafts_workspace_bytes(2, 4, 1000)
    assert _verify(n=need - 1) == SMALL


def test_sizes():
    wb = fgmp.verify_drafts_workspace_bytes
    assert wb(0, 1, 10) == 0 and wb(1, 0, 10) == 0 and wb(1, 1, 0) == 0 and wb(1, 1025, 10) == 0 and wb(16385, 1, 1) == 0 and wb(1, 1, (1 << 24) + 1) == 0
    sizes = [wb(4, 8, v) for v in (1, 1000, 1024, 1025, 32000, 151937, 1 << 24)]
    assert sizes == sorted(sizes) and sizes[0] > fgmp.WORKSPACE_CONTROL_BYTES and sizes[-1] < 1 << 22


def test_the_binding_wants_gpu_tensors_of_the_right_kinds():
    n = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(fgmp.FgmpError):
        fgmp.QuantCache(*(torch.zeros(1, 16, 1, 64, dtype=torch.float8_e4m3fn),) * 2, *(torch.zeros(1, 1, 16, dtype=torch.uint8),) * 2, n)
    with pytest.raises(fgmp.FgmpError):
        fgmp.rotate_heads(torch.zeros(1, 1, 1, 64))
    with pytest.raises(fgmp.FgmpError):
        fgmp.verify_drafts(torch.zeros(1, 1, 8), torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, 1))
    with pytest.raises(fgmp.FgmpError):
        fgmp.cache_read(object())


class _Gpu(torch.Tensor):
    """A CPU tensor that says it is on the GPU: for checks that come before any call of the library."""
    is_cuda = True


def _gpu(t):
    return t.as_subclass(_Gpu)


def _quant_cache(pages=4, size=32, heads=2, dim=64, codes=torch.float8_e4m3fn, scales=torch.uint8, **change):
    k, v = (_gpu(torch.zeros(pages, size, heads, dim).to(codes)) for _ in range(2))
    ks, vs = (_gpu(torch.zeros(pages, heads, size, dtype=scales)) for _ in range(2))
    given = dict(k=k, v=v, k_scales=ks, v_scales=vs, lengths=_gpu(torch.zeros(2, dtype=torch.int32)), page_table=_gpu(torch.zeros(2, 2, dtype=torch.int32)))
    given.update(change)
    return fgmp.QuantCache(**given)


def test_the_binding_checks_a_cache_in_8_bits():
    c = _quant_cache()
    assert c.slots == 64 and c.batch == 2 and c.dtype == BF
    for bad in (dict(codes=torch.uint8), dict(codes=BF), dict(scales=torch.int8), dict(k_scales=_gpu(torch.zeros(4, 32, 2, dtype=torch.uint8))),
                dict(v_scales=_gpu(torch.zeros(4, 2, 48, dtype=torch.uint8)[..., :32])), dict(lengths=_gpu(torch.zeros(2))), dict(page_table=_gpu(torch.zeros(2, 2))),
                dict(page_table=_gpu(torch.zeros(3, 2, dtype=torch.int32))), dict(v=_gpu(torch.zeros(4, 32, 2, 128).to(torch.float8_e4m3fn)))):
        with pytest.raises(fgmp.FgmpError):
            _quant_cache(**bad)
    weights, seen = _gpu(torch.zeros(2, 2, 64)), _gpu(torch.zeros(2, dtype=torch.int32))
    q = _gpu(torch.zeros(2, 1, 2, 64, dtype=BF))
    with pytest.raises(fgmp.FgmpError, match="no QuantCache"):
        fgmp.cache_evict(c, weights, seen, seen, 10)
    with pytest.raises(fgmp.FgmpError, match="no QuantCache"):
        fgmp.attention_weights(q, weights, c, weights)
    with pytest.raises(fgmp.FgmpError, match="slot_positions"):
        fgmp.cache_append(q, q, c, slot_weights=weights)
    for bad in (dict(first=64), dict(first=-1, tokens=2), dict(tokens=65), dict(tokens=0)):
        with pytest.raises(fgmp.FgmpError):
            fgmp.cache_read(c, **bad)


def test_the_binding_checks_rotations_and_verifications(monkeypatch):
    monkeypatch.setattr(fgmp, "_stream", lambda: 0)      # (asked for before the extension looks at the arguments)
    q, k = _gpu(torch.zeros(2, 3, 4, 64)), _gpu(torch.zeros(2, 3, 2, 64))
    f, p = _gpu(torch.zeros(32)), _gpu(torch.zeros(2, 3, dtype=torch.int32))
    p3 = _gpu(torch.zeros(2, 3, 3, dtype=torch.int32))
    for bad in (dict(inv_freq=f), dict(inv_freq=f, positions=p3), dict(inv_freq=f, positions=p.long()), dict(inv_freq=f.double(), positions=p), dict(kind="max", positions=p, inv_freq=f),
                dict(v=k, positions=p, inv_freq=f), dict(k_out=k, positions=p, inv_freq=f), dict(q_weight=f, positions=p, inv_freq=f),
                dict(positions=p3, inv_freq=f, axes=_gpu(torch.zeros(31, dtype=torch.int32))), dict(positions=p, inv_freq=f, k=k.to(BF)),
                dict(positions=p, inv_freq=f, q_out=k), dict(positions=p, inv_freq=f, k=k, q_out=q, k_out=k.to(BF))):
        with pytest.raises(fgmp.FgmpError):
            fgmp.rotate_heads(q, **bad)
    target, ids, u = _gpu(torch.zeros(2, 3, 50)), _gpu(torch.zeros(2, 3, dtype=torch.int32)), _gpu(torch.zeros(2, 3))
    for bad in (dict(draft=target), dict(draft=target[:, 1:], parents=ids), dict(draft=target[:, 1:].to(BF)), dict(parents=ids.long()), dict(parents=ids[:, 1:]),
                dict(counts=ids), dict(rows=ids[:, 1:]), dict(accepted=ids), dict(next_tokens=u[:, 0])):
        with pytest.raises(fgmp.FgmpError):
            fgmp.verify_drafts(target, ids, u, **bad)
    with pytest.raises(fgmp.FgmpError):
        fgmp.verify_drafts(target.transpose(1, 2), ids, u)
    with pytest.raises(fgmp.FgmpError):
        fgmp.verify_drafts(target, ids.long(), u)


# ---- the extension module's way ----

class _Handle:
    def __init__(self):
        self.struct = fgmp._QuantCacheStruct()
        self.fast = (ctypes.addressof(self.struct), 2, 3, 64, 40, BF)


def _swap(given, at, value):
    return given[:at] + [value] + given[at + 1:]


def test_the_extension_hands_on_the_cache_in_8_bits():
    h = _Handle()
    types = (HEADS, HEADS, HEADS, I64, I64, VP, VP, VP, F, I64, HEADS, VP, VP, SZ, VP)
    given = [_t(16, 2, 5, 6, 64, dtype=BF), _t(32, 2, 5, 3, 64, dtype=BF), _t(48, 2, 5, 3, 64, dtype=BF), h.fast, None, None, 0.25, 33, _t(64, 2, 5, 6, 64, dtype=BF),
             _t(80, 2, 5, 6), _t(96, 999, dtype=torch.uint8)]
    want = ((16, 1920, 384, 64), (32, 960, 192, 64), (48, 960, 192, 64), 5, 6, h.fast[0], None, None, 0.25, 33, (64, 1920, 384, 64), 80, 96, 999, 0x77)
    assert _told("quant_cache_attention", given, *types) == want
    assert _told("quant_cache_attention", _swap(given, 0, _t(16, 2, 5, 6, 64)), *types) is None

    types = (HEADS, HEADS, I, I64, VP, VP, I64, VP, VP, VP)
    given = [_t(16, 2, 5, 3, 64), _t(32, 2, 5, 3, 64, stride=(9000, 1000, 128, 1)), h.fast, None, _t(48, 2, dtype=I32), _t(64, 2, dtype=I32)]
    assert _told("quant_cache_append", given, *types) == ((16, 960, 192, 64), (32, 9000, 1000, 128), 0, 5, h.fast[0], None, 5, 48, 64, 0x77)
    both = _told("quant_cache_append", [_t(16, 2, 5, 3, 64, dtype=BF), _t(32, 2, 5, 3, 64, dtype=BF), h.fast, _t(80, 2, 4, dtype=I32), None, given[5]], *types)
    assert both[2] == 1 and both[5:9] == (80, 4, None, 64)
    for at, value in [(0, _t(16, 2, 5, 3, 64, dtype=BF)), (1, _t(32, 2, 5, 4, 64)), (3, _t(80, 3, 4, dtype=I32)), (4, _t(48, 3, dtype=I32)), (5, None)]:
        assert _told("quant_cache_append", _swap(given, at, value), *types) is None, at

    types = (VP, I64, I64, HEADS, HEADS, I, VP)
    given = [h.fast, 7, _t(16, 2, 33, 3, 64), _t(32, 2, 33, 3, 64)]
    assert _told("quant_cache_read", given, *types) == (h.fast[0], 7, 33, (16, 6336, 192, 64), (32, 6336, 192, 64), 0, 0x77)
    for at, value in [(1, 8), (1, -1), (1, None), (2, _t(16, 2, 34, 3, 64)), (2, _t(16, 2, 33, 3, 64, dtype=BF)), (3, _t(32, 2, 33, 3, 32))]:
        assert _told("quant_cache_read", _swap(given, at, value), *types) is None, (at, value)


def test_the_extension_hands_on_rotations():
    types = (HEADS, HEADS, HEADS, I, I64, I64, I64, I64, I64, VP, VP, I, F, VP, I64, VP, VP, I64, I, HEADS, HEADS, HEADS, I, VP)
    given = [_t(16, 2, 5, 6, 64, stride=(4000, 800, 64, 1)), _t(32, 2, 5, 3, 64), _t(48, 2, 5, 3, 64), _t(64, 2, 5, 3, dtype=I32), _t(80, 30), _t(96, 30, dtype=I32), _t(112, 64), None,
             1, 0.5, True, _t(128, 2, 5, 6, 64, dtype=BF), _t(144, 2, 5, 3, 64, dtype=BF), _t(160, 2, 5, 3, 64, dtype=BF)]
    want = ((16, 4000, 800, 64), (32, 960, 192, 64), (48, 960, 192, 64), 0, 2, 5, 6, 3, 64, 112, None, 1, 0.5, 64, 3, 96, 80, 60, 1, (128, 1920, 384, 64), (144, 960, 192, 64),
            (160, 960, 192, 64), 1, 0x77)
    assert _told("rotate_heads", given, *types) == want
    one = _told("rotate_heads", [given[0], None, None, _t(64, 2, 5, dtype=I32), given[4], None, None, None, 0, 1e-5, False, given[11], None, None], *types)
    assert one[1:3] == (None, None) and one[7] == 0 and one[14:18] == (1, None, 80, 60) and one[18] == 0 and one[20:22] == (None, None)
    for at, value in [(0, None), (1, None), (1, _t(32, 2, 5, 3, 64, dtype=BF)), (2, _t(48, 2, 5, 4, 64)), (3, _t(64, 2, 5, dtype=I32)), (3, None), (4, None), (5, None), (5, _t(96, 31, dtype=I32)),
                      (6, _t(112, 32)), (10, 1), (11, None), (12, None), (12, _t(144, 2, 5, 3, 64)), (13, None), (13, _t(160, 2, 4, 3, 64, dtype=BF))]:
        assert _told("rotate_heads", _swap(given, at, value), *types) is None, (at, value)


def test_the_extension_hands_on_verifications():
    types = (VP, I, I64, I64, VP, I64, I64, I64, I64, I64, VP, VP, VP, VP, VP, VP, VP, VP, SZ, VP)
    given = [_t(16, 2, 5, 50, stride=(300, 53, 1)), _t(32, 2, 5, dtype=I32), _t(48, 2, 5), _t(64, 2, 4, 50), None, _t(80, 2, dtype=I32), _t(96, 2, 5, dtype=I32), _t(112, 2, dtype=I32),
             _t(128, 2, dtype=I32), _t(144, 77, dtype=torch.uint8)]
    assert _told("verify_drafts", given, *types) == (16, 0, 300, 53, 64, 200, 50, 2, 5, 50, 32, None, 80, 48, 96, 112, 128, 144, 77, 0x77)
    tree = _told("verify_drafts", given[:3] + [None, _t(64, 2, 5, dtype=I32), None] + given[6:], *types)
    assert tree[4:7] == (None, 0, 0) and tree[11:13] == (64, None)
    for at, value in [(0, _t(16, 2, 5, 50, stride=(300, 1, 6))), (0, _t(16, 2, 5, 50, dtype=BF)), (1, _t(32, 2, 5)), (2, _t(48, 2, 4)), (3, _t(64, 2, 5, 50)), (4, _t(64, 2, 5, dtype=I32)),
                      (5, _t(80, 3, dtype=I32)), (6, None), (7, _t(112, 2)), (8, None), (9, _t(144, 7, dtype=I32))]:
        assert _told("verify_drafts", _swap(given, at, value), *types) is None, (at, value)
    one = [_t(16, 2, 1, 50), _t(32, 2, 1, dtype=I32), _t(48, 2, 1), _t(64, 2, 0, 50), None, None, _t(96, 2, 1, dtype=I32)] + given[7:]
    assert _told("verify_drafts", one, *types) is None       # (the general path leaves a draft without rows out)


@pytest.mark.parametrize("name,count", [("quant_cache_attention", 14), ("quant_cache_append", 9), ("quant_cache_read", 7), ("rotate_heads", 17), ("verify_drafts", 13)])
def test_the_extension_counts_its_arguments(name, count):
    fgmp.lib()
    f = getattr(fgmp._call, name)
    with pytest.raises(TypeError):
        f(*[None] * (count - 1))
    assert f(*[None] * count) is None and f(0, (1, 2), *[None] * (count - 2)) is None


def test_tensors_are_looked_into_where_that_was_compiled_for_this_torch(monkeypatch, tmp_path):
    """The way into a tensor's C++ object is taken for the torch it was compiled for alone; plain tensors of the CPU, subclasses and objects that are
    no tensors are left to their attributes."""
    from paper_2504_14152_amd import build
    fgmp.lib()
    tensors = ctypes.PyDLL(build.TENSORS)
    tensors.fgmp_tensors_torch.restype = ctypes.c_char_p
    assert tensors.fgmp_tensors_torch().decode() == torch.__version__.split("+")[0]
    sizes, strides, kind, data = (I64 * 4)(), (I64 * 4)(), I(), VP()
    look = tensors.fgmp_tensors_look
    look.argtypes = [ctypes.py_object, I, ctypes.POINTER(I64), ctypes.POINTER(I64), ctypes.POINTER(I), ctypes.POINTER(VP)]
    for o in (torch.zeros(3), _gpu(torch.zeros(3)), _t(16, 3), None, 7):
        assert look(o, 4, sizes, strides, ctypes.byref(kind), ctypes.byref(data)) == -1
    told = []
    module = type("Module", (), {"look_into_tensors": staticmethod(told.append)})
    fgmp._load_tensors(module)
    assert len(told) == 1 and told[0]
    monkeypatch.setattr(torch, "__version__", "9.9.9")
    fgmp._load_tensors(module)
    monkeypatch.undo()
    monkeypatch.setattr(build, "TENSORS", str(tmp_path / "none.so"))
    monkeypatch.setenv("CXX", str(tmp_path / "no-compiler"))
    fgmp._load_tensors(module)          # (nothing to compile with)
    assert len(told) == 1


@pytest.mark.gpu
def test_a_tensor_says_the_same_either_way():
    from paper_2504_14152_amd import build
    tensors = ctypes.PyDLL(build.TENSORS)
    sizes, strides, kind, data = (I64 * 4)(), (I64 * 4)(), I(), VP()
    look = tensors.fgmp_tensors_look
    look.argtypes = [ctypes.py_object, I, ctypes.POINTER(I64), ctypes.POINTER(I64), ctypes.POINTER(I), ctypes.POINTER(VP)]
    base = torch.zeros(4, 6, 8, 10, device="cuda")
    for t in (base, base[1:, ::2], base.transpose(1, 2), base[0, 0, 0], base[:0], base.bfloat16(), base.int(), base.long(), base.byte(), base.half(), base[..., 3],
              base[:1].expand(9, 6, 8, 10), torch.nn.Parameter(base)):
        n = look(t, 4, sizes, strides, ctypes.byref(kind), ctypes.byref(data))
        types = {torch.float32: 0, torch.bfloat16: 1, torch.int32: 2, torch.int64: 3, torch.uint8: 4}
        assert n == t.dim() and tuple(sizes[:n]) == t.shape and tuple(strides[:n]) == t.stride() and kind.value == types.get(t.dtype, -1)
        assert (data.value or 0) == t.data_ptr()
    assert look(base[None], 4, sizes, strides, ctypes.byref(kind), ctypes.byref(data)) == -1


def test_tensors_of_another_device_are_refused(monkeypatch):
    monkeypatch.setattr(fgmp, "_stream", lambda: 0)
    monkeypatch.setattr(fgmp, "_several_devices", lambda: True)
    monkeypatch.setattr(fgmp, "_current_device", lambda: 1)

    class On(torch.Tensor):
        is_cuda = True
        device_of = 1

        def get_device(self):
            return self.device_of

    def on(device, t):
        t = t.as_subclass(On)
        t.device_of = device
        return t

    here, there = (on(d, torch.zeros(2, 3, 4, 64)) for d in (1, 0))
    with pytest.raises(fgmp.FgmpError, match="current device, 1"):
        fgmp.rotate_heads(here, there)
    with pytest.raises(fgmp.FgmpError, match="^k: "):        # (of this device: looked at further)
        fgmp.rotate_heads(here, on(1, torch.zeros(2, 3, 4, 32)))
    with pytest.raises(fgmp.FgmpError, match="current device, 1"):
        fgmp.verify_drafts(here[0], on(0, torch.zeros(3, 4, dtype=torch.int32)), here[0, :, :, 0])
