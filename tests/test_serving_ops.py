"""Rotated heads, a cache in 8 bits (append, read, attention over it) and the verification of drafted tokens, on the GPU against their
definitions in 64 bits.

Tolerances are bounds on rounding, as in test_layer_ops: u is half an ulp, 2^-24 for FP32, 2^-8 for BF16.  Codes, scales, copies, kept tokens
and drawn ones have to be equal."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import test_layer_ops as layer  # noqa: E402
from paper_2504_14152_amd import fgmp  # noqa: E402
from test_layer_ops import BF16, DEV, F32, U32, _chain, _compare_attention, _gen, _i32, _randn, _random_tree, _say, _unit  # noqa: E402

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


# ---- rotated heads ----

def _rotated(x, weight, kind, eps, positions, inv_freq, axes, interleaved):
    """The formula in 64 bits, and a bound on what rounding may make of it before the output's: x batch x tokens x heads x dim."""
    x = x.double().cpu()
    D, size = x.shape[-1], x.abs()
    err = torch.zeros_like(x)
    if weight is not None:
        w = weight.double().cpu()
        mean = x.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(x[..., :1])
        scale = 1.0 / ((x - mean).square().mean(-1, keepdim=True) + eps).sqrt()
        # a sum of D terms: relative D u of its terms' magnitudes; the mean's error goes into every term
        off = (D + 4) * U32 * size.mean(-1, keepdim=True) if kind == "layer" else 0.0
        x = (x - mean) * scale * w
        err = (off + U32 * size) * scale * w.abs() + x.abs() * ((D / 2 + 8) * U32)
        if kind == "layer":   # (through the scale: sum |x - mean| off / sum (x - mean)^2, at most off * scale)
            err = err + x.abs() * off * scale
    pairs = 0 if inv_freq is None else inv_freq.shape[0]
    if pairs:
        pos = positions.double().cpu().view(*x.shape[:2], -1)
        f = inv_freq.double().cpu()
        if axes is None:
            angle = pos * f
        else:
            at = axes.long().cpu()
            fine = (at >= 0) & (at < pos.shape[-1])
            angle = torch.where(fine, pos[..., at.clamp(0, pos.shape[-1] - 1)], 0.0) * f
        cos, sin = angle.cos()[:, :, None], angle.sin()[:, :, None]
        if interleaved:
            first, second = torch.arange(pairs) * 2, torch.arange(pairs) * 2 + 1
        else:
            first, second = torch.arange(pairs), torch.arange(pairs) + pairs
        a, b, ea, eb = x[..., first], x[..., second], err[..., first], err[..., second]
        y, e = x.clone(), err.clone()
        y[..., first], y[..., second] = a * cos - b * sin, a * sin + b * cos
        # sines and cosines off by 4 u (their argument's rounding, the series'), two products and a sum
        e[..., first] = e[..., second] = ea + eb + 8 * U32 * (a.abs() + b.abs())
        return y, e
    return x, err


def _check_rotated(got, want_err, dtype, what):
    want, err = want_err
    tol = err + _unit(dtype) * (want.abs() + err) + 1e-30
    off = (got.double().cpu() - want).abs()
    assert got.dtype == dtype and bool((off <= tol).all()), (what, float((off / tol).max()))


ROTATE = [
    # source, out, B, T, heads, kv heads, dim, pairs, axes, kind ("none": no weights), interleaved, first position
    (F32, BF16, 1, 1, 1, 1, 64, 32, 1, "rms", False, 0),
    (F32, BF16, 2, 7, 8, 2, 128, 64, 1, "rms", False, 4090),
    (BF16, BF16, 3, 5, 5, 1, 128, 48, 3, "layer", True, 131072),
    (BF16, F32, 1, 33, 6, 3, 80, 40, 2, "none", False, -17),
    (F32, F32, 2, 3, 24, 4, 96, 20, 1, "layer", False, (1 << 29) - 3),
    (F32, F32, 1, 2, 3, 1, 192, 96, 1, "rms", True, 1000003),
    (F32, F32, 1, 300, 2, 2, 256, 128, 3, "rms", False, 77777),
    (BF16, F32, 1, 4, 7, 7, 512, 256, 1, "layer", True, 12),
    (F32, BF16, 1, 2, 3, 2, 8, 4, 1, "rms", False, 5),
    (F32, F32, 1, 3, 40, 1, 16, 4, 1, "none", True, 9),
    (F32, F32, 2, 2, 4, 2, 64, 0, 1, "rms", False, 0),
    (F32, BF16, 5, 700, 4, 1, 64, 32, 1, "none", False, 1),
]


@pytest.mark.parametrize("source,out,B,T,H,G,D,pairs,n_axes,kind,interleaved,start", ROTATE)
def test_rotated_heads_against_their_formula(source, out, B, T, H, G, D, pairs, n_axes, kind, interleaved, start):
    _say("rotate", source, out, B, T, H, G, D, pairs, n_axes, kind, interleaved, start)
    g = _gen(D + T + H)
    q, k, v = ((_randn(g, B, T, H + 2 * G, D) * 1.5 + 0.2).to(source)).split([H, G, G], 2)
    inv_freq = (10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / max(1, pairs))).float().to(DEV) if pairs else None
    positions = (start + torch.randint(0, 3, (B, T, n_axes), generator=g) + torch.arange(T)[None, :, None]).int().to(DEV)
    axes = None
    if n_axes > 1:
        axes = torch.randint(0, n_axes, (pairs,), generator=g).int().to(DEV)
        axes[1], axes[-1] = n_axes, -1                    # no such axes: position 0
    else:
        positions = positions[:, :, 0].contiguous()
    qw, kw = ((1.0 + 0.2 * _randn(g, D)) if kind != "none" else None for _ in range(2))
    norm = "rms" if kind == "none" else kind
    got = fgmp.rotate_heads(q, k, v, positions, inv_freq, axes, qw, kw, norm, 1e-5, interleaved, dtype=out)
    for name, x, w, y in (("q", q, qw, got[0]), ("k", k, kw, got[1])):
        _check_rotated(y, _rotated(x, w, kind, 1e-5, positions, inv_freq, axes, interleaved), out, name)
    assert torch.equal(got[2], v.to(out))
    # into the places of others, and with buffers of the caller's
    wide = torch.full((B, H + 2 * G, T, D + 8), 7.0, dtype=out, device=DEV)
    parts = [x[..., :D].transpose(1, 2) for x in wide.split([H, G, G], 1)]
    again = fgmp.rotate_heads(q, k, v, positions, inv_freq, axes, qw, kw, norm, 1e-5, interleaved, *parts)
    assert all(torch.equal(x, y) for x, y in zip(again, got)) and bool((wide[..., D:] == 7.0).all())
    if source == out:
        copy = torch.cat([q, k, v], 2)
        parts = copy.split([H, G, G], 2)
        fgmp.rotate_heads(*parts, positions, inv_freq, axes, qw, kw, norm, 1e-5, interleaved, *parts)
        assert all(torch.equal(x, y) for x, y in zip(parts, got))
    # queries alone, and without values
    one = fgmp.rotate_heads(q, positions=positions, inv_freq=inv_freq, axes=axes, q_weight=qw, kind=norm, interleaved=interleaved, dtype=out)
    assert torch.equal(one[0], got[0]) and one[1] is None and one[2] is None
    two = fgmp.rotate_heads(q, k, None, positions, inv_freq, axes, qw, kw, norm, 1e-5, interleaved, dtype=out)
    assert torch.equal(two[1], got[1]) and two[2] is None


def test_rotations_of_vectors_that_are_not_finite_and_of_zeros():
    g = _gen(2)
    q = _randn(g, 1, 4, 2, 64)
    q[0, 1, 0], q[0, 2, 1, 5], q[0, 3] = 0.0, math.inf, 0.0
    f = torch.ones(32, device=DEV)
    w = torch.ones(64, device=DEV)
    out, _, _ = fgmp.rotate_heads(q, positions=_i32([[0, 1, 2, 3]]), inv_freq=f, q_weight=w, dtype=F32)
    assert bool((out[0, 1, 0] == 0).all()) and bool((out[0, 3] == 0).all())
    assert not bool(torch.isfinite(out[0, 2, 1, 5])) and bool(torch.isfinite(out[0, 2, 0]).all()) and bool(torch.isfinite(out[0, 0]).all())
    plain, _, _ = fgmp.rotate_heads(q, positions=_i32([[0, 0, 0, 0]]), inv_freq=f, dtype=F32)
    assert torch.equal(plain[0, 0], q[0, 0])               # position 0 turns nothing


def test_a_rotation_of_both_keeps_their_products():
    """<q at p, k at p'> depends on p - p' alone."""
    g = _gen(3)
    q, k = _randn(g, 1, 1, 1, 128).expand(1, 64, 1, 128), _randn(g, 1, 1, 1, 128).expand(1, 64, 1, 128)
    f = (500000.0 ** (-torch.arange(64, device=DEV) / 64)).float()
    near, _, _ = fgmp.rotate_heads(q, positions=(torch.arange(64, device=DEV) + 13)[None].int(), inv_freq=f, dtype=F32)
    here, _, _ = fgmp.rotate_heads(k, positions=torch.arange(64, device=DEV)[None].int(), inv_freq=f, dtype=F32)
    s = (near.double() * here.double()).sum(-1).flatten()
    size = float((q[0, 0, 0].double().norm() * k[0, 0, 0].double().norm()))
    assert float((s - s[0]).abs().max()) <= 40 * U32 * size


def test_sections_become_axes():
    assert fgmp.rotary_axes([2, 0, 3]).tolist() == [0, 0, 2, 2, 2]


# ---- a cache in 8 bits ----

_TABLE = torch.tensor([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127], dtype=torch.float64)


def _quantized(x):
    """Codes and scale bytes of vectors (the last dimension), from the definition: on the CPU in 64 bits."""
    x = x.double().cpu()
    finite = torch.isfinite(x)
    most = torch.where(finite, x.abs(), 0.0).amax(-1)
    e = torch.full(most.shape, -100, dtype=torch.int64)
    for p in range(-100, 121):
        e = torch.where(most > 448.0 * 2.0 ** p, p + 1, e)
    y = torch.where(finite, x, 0.0) / torch.pow(2.0, e.double())[..., None]
    high = torch.searchsorted(_TABLE, y.abs().contiguous()).clamp(1, 126)
    up, down = _TABLE[high] - y.abs(), y.abs() - _TABLE[high - 1]
    code = torch.where((up < down) | ((up == down) & (high % 2 == 0)), high, high - 1)
    code = torch.where(finite, code + 128 * torch.signbit(x).long(), 127)
    return code.to(torch.uint8), (e + 127).to(torch.uint8)


def _is_code(got, want):
    """Equal codes; a NaN of either sign is one."""
    got, want = got.cpu(), want.cpu()
    return bool(((got == want) | (((got & 127) == 127) & ((want & 127) == 127))).all())


class Made8:
    """A cache in 8 bits of given lengths whose unused slots hold codes of NaN and scales of infinity."""

    def __init__(self, g, lengths, heads, dim, page, room=0, outside=False):
        self.lens, B = list(lengths), len(lengths)
        most = max(max(lengths) + room, 1)
        each = -(-most // page) if page else 1
        size = page or -(-most // 16) * 16 + 16
        pages = B * each + 2 if page else B
        shape = (pages, size, heads, dim)
        self.k, self.v = (torch.full((pages, heads, size, dim) if outside else shape, 0x7F, dtype=torch.uint8, device=DEV) for _ in range(2))
        if outside:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.ks, self.vs = (torch.full((pages, heads, size + (16 if outside else 0)), 0xFF, dtype=torch.uint8, device=DEV)[..., :size] for _ in range(2))
        self.table = None
        if page:
            self.table = torch.randperm(pages, generator=g)[: B * each].view(B, each).int()
            used = self.table.clone()
            for b, n in enumerate(lengths):
                used[b, -(-(n + room) // page):] = -1 if b % 2 else 1 << 30
        self.page, self.size, self.slots = page, size, size * each
        self.keys, self.values = [], []     # as the cache holds them, BF16 (exact)
        for b, n in enumerate(lengths):
            for pages_, scales, to in ((self.k, self.ks, self.keys), (self.v, self.vs, self.values)):
                c, s = _quantized(_randn(g, n, heads, dim) * (0.1 + 3 * torch.rand(n, heads, 1, generator=g).to(DEV)))
                to.append((c.view(E4M3).float() * torch.pow(2.0, s.float() - 127)[..., None]).bfloat16().to(DEV))
                for j in range(0, n, size):
                    at = b if not page else int(self.table[b, j // size])
                    pages_[at, : min(size, n - j)] = c[j:j + size].to(DEV)
                    scales[at, :, : min(size, n - j)] = s[j:j + size].t().to(DEV)
        self.cache = fgmp.QuantCache(self.k.view(E4M3), self.v.view(E4M3), self.ks, self.vs, _i32(self.lens), None if not page else used.to(DEV))


def _vectors(g, *shape, dtype):
    """Vectors of all sizes, some with elements that have to be right to the last bit."""
    x = torch.randn(*shape, generator=g) * torch.pow(2.0, torch.randint(-20, 20, shape[:-1], generator=g).float())[..., None]
    flat = x.view(-1, shape[-1])
    special = [torch.zeros(shape[-1]), torch.full((shape[-1],), -0.0), torch.full((shape[-1],), 448.0), torch.full((shape[-1],), 1e-42),
               torch.full((shape[-1],), 2.0 ** -100 * 448), torch.full((shape[-1],), 3.0e38), torch.full((shape[-1],), -1e-30)]
    tie = torch.zeros(shape[-1])
    tie[: 8] = torch.tensor([1.75 * 256, 17.0, -19.0, 2.0 ** -10, 3 * 2.0 ** -10, -(2.0 ** -7 + 2.0 ** -10), 1.0625, 1.1875])     # half-way between codes
    above = tie.clone()
    above[0] = 450.0 if dtype == BF16 else 448.00003
    bad = torch.randn(shape[-1], generator=g)
    bad[3], bad[7] = math.nan, -math.inf
    all_bad = torch.full((shape[-1],), math.inf)
    for i, s in enumerate((special + [tie, above, bad, all_bad])[: flat.shape[0]]):
        flat[i] = s
    return x.to(dtype).to(DEV)


@pytest.mark.parametrize("source", [BF16, F32])
@pytest.mark.parametrize("G,D,page,T,lens,counts,outside", [(2, 64, 16, 9, [0, 15, 30], [9, 3, 0], False), (8, 128, 0, 1, [9], None, True),
                                                            (3, 256, 48, 9, [47, 48], [1, 9], False), (1, 128, 64, 200, [1, 60], None, True)])
def test_append_quantizes(source, G, D, page, T, lens, counts, outside):
    _say("append8", source, G, D, page, T, lens, counts)
    g = _gen(T + D)
    B = len(lens)
    made = Made8(g, lens, G, D, page, room=T, outside=outside)
    k, v = _vectors(g, B, T, 2 * G, D, dtype=source)[:, :, ::2], _vectors(g, B, T, G, D, dtype=source)
    rows = torch.stack([torch.randperm(T, generator=g) for _ in range(B)]).int()
    if T > 4:
        rows[0, 1], rows[0, 2] = T, -3      # no such rows: their slots stay as they are
    want = [x.clone() for x in (made.k, made.v, made.ks, made.vs)]
    lengths = fgmp.cache_append(k, v, made.cache, rows=rows.to(DEV), counts=None if counts is None else _i32(counts))
    use = [T] * B if counts is None else counts
    for b in range(B):
        for i in range(use[b]):
            r, slot = int(rows[b, i]), lens[b] + i
            if 0 <= r < T:
                at = b if not page else int(made.table[b, slot // page])
                for x, c, s in ((k, want[0], want[2]), (v, want[1], want[3])):
                    code, scale = _quantized(x[b, r])
                    c[at, slot % made.size], s[at, :, slot % made.size] = code.to(DEV), scale.to(DEV)
    assert _is_code(made.k, want[0]) and _is_code(made.v, want[1])
    assert torch.equal(made.ks, want[2]) and torch.equal(made.vs, want[3])
    assert lengths.tolist() == [n + c for n, c in zip(lens, use)]


@pytest.mark.parametrize("source", [BF16, F32])
@pytest.mark.parametrize("G,D,page,T,lens,counts", [(1, 64, 64, 9001, [0, 77], None), (1, 128, 0, 4097, [3, 0, 50], [4097, 0, 4000]), (3, 256, 48, 811, [47, 1], [811, 805]),
                                                    (8, 128, 16, 300, [5, 0, 16, 31], [300, 299, 1, 300]), (5, 64, 32, 1300, [31, 0, 1], [1300, 1299, 3]),
                                                    (20, 128, 64, 130, [0, 9], None)])
def test_append_of_many_tokens_quantizes(source, G, D, page, T, lens, counts):
    """As many as workgroups have several of: rows in any order, some that are none, a page that is none, more tokens than slots."""
    _say("append8 many", source, G, D, page, T, lens, counts)
    g = _gen(T + G)
    B = len(lens)
    use = [T] * B if counts is None else counts
    made = Made8(g, lens, G, D, page, room=T - 20)          # (the first sequence's slots may end before its tokens)
    k, v = _vectors(g, B, T, G, D, dtype=source), _vectors(g, B, T, 2 * G, D, dtype=source)[:, :, ::2]
    rows = torch.stack([torch.randperm(T, generator=g) for _ in range(B)]).int()
    rows[0, 1], rows[0, 17], rows[-1, 0] = T, -3, T - 1
    cache, lost = made.cache, -1
    if page:
        lost = max(1, lens[0] // page + 1)
        table = made.table.clone()
        table[0, lost] = 1 << 30                            # what falls there is dropped
        cache = fgmp.QuantCache(made.k.view(E4M3), made.v.view(E4M3), made.ks, made.vs, _i32(lens), table.to(DEV))
    want = [x.cpu() for x in (made.k, made.v, made.ks, made.vs)]
    lengths = fgmp.cache_append(k, v, cache, rows=rows.to(DEV), counts=None if counts is None else _i32(counts))
    for x, c, s in ((k, want[0], want[2]), (v, want[1], want[3])):
        code, scale = _quantized(x)
        for b in range(B):
            i = torch.arange(min(use[b], made.slots - lens[b]))
            r, slot = rows[b, i].long(), lens[b] + i
            entry = slot // page if page else torch.zeros_like(slot)
            fine = (r >= 0) & (r < T) & ((entry != lost) if b == 0 else True)
            r, slot, entry = r[fine], slot[fine], entry[fine]
            at = made.table[b, entry].long() if page else torch.full_like(slot, b)
            c[at, slot % made.size], s[at, :, slot % made.size] = code[b, r], scale[b, r]
    assert _is_code(made.k, want[0]) and _is_code(made.v, want[1])
    assert torch.equal(made.ks.cpu(), want[2]) and torch.equal(made.vs.cpu(), want[3])
    assert lengths.tolist() == [min(n + c, made.slots) for n, c in zip(lens, use)]


def test_append_into_8_bits_drops_what_has_no_slot_and_no_page():
    g = _gen(10)
    made = Made8(g, [30, 32], 1, 64, 16)       # 32 slots each
    before = made.v.clone(), made.vs.clone()
    k = _randn(g, 2, 4, 1, 64, dtype=BF16)
    assert fgmp.cache_append(k, k, made.cache).tolist() == [32, 32]
    changed = (made.v != before[0]).flatten(1).any(-1).nonzero().flatten().tolist()
    assert changed == [int(made.table[0, 1])] == (made.vs != before[1]).flatten(1).any(-1).nonzero().flatten().tolist()
    made = Made8(g, [16], 1, 64, 16)
    table = torch.cat([made.table, torch.tensor([[1 << 20]], dtype=torch.int32)], 1)
    cache = fgmp.QuantCache(made.k.view(E4M3), made.v.view(E4M3), made.ks, made.vs, _i32([16]), table.to(DEV))
    before = [x.clone() for x in (made.k, made.v, made.ks, made.vs)]
    assert fgmp.cache_append(k[:1, :2], k[:1, :2], cache).tolist() == [18]
    assert all(torch.equal(x, y) for x, y in zip(before, (made.k, made.v, made.ks, made.vs)))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("G,D,page,lens,first,tokens,outside", [(2, 64, 16, [40, 3, 0], 0, 48, False), (8, 128, 0, [700], 333, 100, True), (3, 256, 48, [100, 47], 17, 1, False),
                                                               (1, 128, 64, [130], 130, 2, False), (16, 128, 32, [95, 64, 65], 31, 40, True),
                                                               (1, 128, 64, [9000, 8003], 5, 8995, False), (3, 128, 48, [4000, 3999, 0], 17, 3983, True), (8, 64, 0, [3001], 0, 3001, False),
                                                               (5, 256, 16, [2000, 17], 1, 1999, False), (8, 128, 64, [2100], 3, 2090, False)])
def test_reading_back(dtype, G, D, page, lens, first, tokens, outside):
    _say("read8", dtype, G, D, page, lens, first, tokens)
    g = _gen(D + first)
    made = Made8(g, lens, G, D, page, outside=outside)
    wide = [torch.full((len(lens), tokens, G, D + 8), 5.0, dtype=dtype, device=DEV) for _ in range(2)]
    k, v = fgmp.cache_read(made.cache, first=first, k_out=wide[0][..., :D], v_out=wide[1][..., :D])
    zk, zv = fgmp.cache_read(made.cache, first=first, tokens=tokens, dtype=dtype)
    for out, zeros, held, w in ((k, zk, made.keys, wide[0]), (v, zv, made.values, wide[1])):
        for b, n in enumerate(lens):
            m = max(0, min(n - first, tokens))
            assert torch.equal(out[b, :m], held[b][first:first + m].to(dtype)) and bool((out[b, m:] == 5.0).all())
            assert torch.equal(zeros[b, :m], out[b, :m]) and bool((zeros[b, m:] == 0.0).all())
        assert bool((w[..., D:] == 5.0).all())


def test_what_is_appended_reads_back_as_the_nearest_values():
    """Half a step of the format at most, 2^-4 of an element or 2^-10 of the scale, and zeros stay zeros."""
    g = _gen(12)
    made = Made8(g, [0, 5], 4, 128, 16, room=50)
    k, v = _randn(g, 2, 50, 4, 128), _randn(g, 2, 50, 4, 128) * 1e-3
    k[0, 3] = 0.0
    made.cache.lengths = fgmp.cache_append(k, v, made.cache)
    got_k, got_v = fgmp.cache_read(made.cache, tokens=55, dtype=F32)
    for b, n in ((0, 0), (1, 5)):
        for got, x in ((got_k, k), (got_v, v)):
            most = x[b].abs().amax(-1, keepdim=True)
            step = torch.maximum(x[b].abs() * 2.0 ** -4, most / 224.0 * 2.0 ** -10)
            assert bool(((got[b, n:n + 50] - x[b]).abs() <= step).all())


def test_a_scale_at_the_top_of_the_range():
    """The largest numbers round up to 2^128, which is no FP32 number."""
    made = Made8(_gen(1), [0], 1, 64, 16, room=2)
    k = torch.full((1, 2, 1, 64), torch.finfo(F32).max, device=DEV)
    k[0, 1] = 2.0 ** 127
    made.cache.lengths = fgmp.cache_append(k, k, made.cache)
    x, _ = fgmp.cache_read(made.cache, tokens=2, dtype=F32)
    assert bool((x[0, 0] == math.inf).all()) and torch.equal(x[0, 1], k[0, 1])


# ---- attention over 8 bits ----

LONGER = [
    (BF16, 64, 20, 1, 2, [1000, 16], 64, False, None),
    (BF16, 128, 8, 2, 3, [3000, 0, 1500, 33], 64, True, [3, 2, 0, 1]),
    (BF16, 64, 4, 4, 1, [2500, 1], 0, False, None),
    (BF16, 256, 4, 2, 2, [2300, 129], 16, True, None),
    (BF16, 128, 16, 1, 2, [2100, 64], 48, False, [2, 1]),
    (BF16, 128, 8, 8, 1, [700] * 9, 32, False, [1, 0, 1, 1, 1, 1, 1, 0, 1]),
    # 33 to 64 rows (17 to 64 of head_dim 256), over caches on either side of what the kernel for many rows begins with
    (BF16, 128, 8, 1, 6, [2500, 300], 64, True, None),
    (BF16, 128, 8, 1, 7, [1000, 3, 0], 64, True, [7, 6, 2]),
    (BF16, 64, 8, 1, 8, [4100], 0, False, None),
    (BF16, 64, 16, 2, 5, [2047, 33], 16, True, [5, 3]),
    (BF16, 256, 8, 1, 4, [4200, 5], 16, True, None),
    (BF16, 256, 16, 2, 7, [90, 17] * 8 + [0], 16, False, None),
    (BF16, 256, 16, 2, 8, [1700, 0, 64], 64, True, [8, 1, 5]),
]


@pytest.mark.parametrize("dtype,D,H,G,T,lens,page,tree,counts", [c for c in layer.ATTEND if c[0] == BF16] + LONGER)
def test_attention_over_8_bits_against_its_formula(dtype, D, H, G, T, lens, page, tree, counts):
    _say("attention8", D, H, G, T, lens, page, tree, counts)
    g = _gen(D + T + H + len(lens))
    B = len(lens)
    made = Made8(g, lens, G, D, page, outside=T % 2 == 1)
    q, k, v = _randn(g, B, T, H, D, dtype=dtype), _randn(g, B, T, G, D, dtype=dtype), _randn(g, B, T, G, D, dtype=dtype)
    words, sees = _random_tree(g, B, T) if tree else (None, _chain(B, T))
    use = [T] * B if counts is None else counts
    for b in range(B):   # tokens that do not count are no numbers
        k[b, use[b]:], v[b, use[b]:], q[b, use[b]:] = math.nan, math.inf, math.nan
    scale = 1.0 / math.sqrt(D)
    out, lse = fgmp.tree_attention(q, k, v, made.cache, tree=words, counts=None if counts is None else _i32(counts))
    _compare_attention(out, lse, q, made, k, v, sees, use, scale, H // G)
    out, lse = fgmp.tree_attention(q, None, None, made.cache, counts=None if counts is None else _i32(counts), scale=0.37 * scale)
    _compare_attention(out, lse, q, made, None, None, None, use, 0.37 * scale, H // G)


@pytest.mark.parametrize("D,H,G,T,lens,page,tree", [(128, 2, 1, 1024, [100], 16, False), (64, 4, 2, 512, [0, 70], 0, True), (256, 1, 1, 600, [33], 48, True)])
def test_attention_over_8_bits_of_a_chunk_of_a_prompt(D, H, G, T, lens, page, tree):
    _say("chunk8", D, H, G, T, lens, page, tree)
    g = _gen(T + D)
    B = len(lens)
    made = Made8(g, lens, G, D, page)
    q, k, v = _randn(g, B, T, H, D, dtype=BF16), _randn(g, B, T, G, D, dtype=BF16), _randn(g, B, T, G, D, dtype=BF16)
    words, sees = _random_tree(g, B, T) if tree else (None, _chain(B, T))
    out, lse = fgmp.tree_attention(q, k, v, made.cache, tree=words)
    _compare_attention(out, lse, q, made, k, v, sees, [T] * B, D ** -0.5, H // G)


@pytest.mark.parametrize("H,D,T", [(8, 128, 1), (16, 128, 9), (2, 128, 64), (16, 64, 2), (20, 64, 17), (4, 256, 2), (8, 256, 5)])
def test_ranges_of_a_long_cache_of_8_bits_join(H, D, T):
    g = _gen(6)
    for n in (127, 129, 1000, 4097, 20011):
        made = Made8(g, [n], 1, D, 64)
        q, k, v = _randn(g, 1, T, H, D, dtype=BF16) * 2, _randn(g, 1, T, 1, D, dtype=BF16), _randn(g, 1, T, 1, D, dtype=BF16)
        for hint in (0, 1, 300):
            out, lse = fgmp.tree_attention(q, k, v, made.cache, max_length=hint)
            rows = sorted({0, T // 2, T - 1})
            heads = [0, H - 1]
            for t in rows:
                _compare_row(out, lse, q, made, k, v, t, heads, D)
            again, lse2 = fgmp.tree_attention(q, k, v, made.cache, max_length=hint)
            assert torch.equal(out, again) and torch.equal(lse, lse2)
    _say("ranges8", H, D, T)


def _compare_row(out, lse, q, made, k, v, t, heads, D):
    """One token of a chain over one sequence and key head."""
    n = made.lens[0]
    kh, vh = torch.cat([made.keys[0][:, 0], k[0, : t + 1, 0]]).cpu(), torch.cat([made.values[0][:, 0], v[0, : t + 1, 0]]).cpu()
    for h in heads:
        want, want_lse, size, mean = layer._attention(q[0, t, h].cpu(), kh, vh, D ** -0.5)
        e_w = (D + 6) * U32 * size + 4 * U32 * (1 + abs(want_lse)) + (n / 4 + 40) * U32
        tol = (2 * e_w + 2.1 * layer.U16) * mean + layer.U16 * want.abs()
        off = (out[0, t, h].cpu().double() - want).abs()
        assert bool((off <= tol).all()), (n, t, h, float((off / tol).max()))
        assert abs(float(lse[0, t, h]) - want_lse) <= e_w + 4 * U32 * abs(want_lse)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("H,G,D", [(4, 2, 64), (3, 1, 128), (10, 2, 128), (12, 1, 64), (4, 2, 256)])
def test_hidden_tokens_reach_no_row_over_8_bits(H, G, D, bad):
    g = _gen(3)
    T = 21
    made = Made8(g, [77], G, D, 16)
    q, k, v = _randn(g, 1, T, H, D, dtype=BF16), _randn(g, 1, T, G, D, dtype=BF16), _randn(g, 1, T, G, D, dtype=BF16)
    words, sees = _random_tree(g, 1, T)
    seen_by = [t for t in range(T) if 9 in sees[0][t]]
    others = [t for t in range(T) if t not in seen_by]
    plain, plain_lse = fgmp.tree_attention(q, k, v, made.cache, tree=words)
    kb, vb = k.clone(), v.clone()
    vb[0, 9, :, ::3] = bad
    out, lse = fgmp.tree_attention(q, k, vb, made.cache, tree=words)
    assert not bool(torch.isfinite(out[0, seen_by][..., ::3]).any())
    assert torch.equal(out[0, seen_by][..., 1::3], plain[0, seen_by][..., 1::3]) and torch.equal(lse, plain_lse)
    assert torch.equal(out[0, others], plain[0, others])
    kb[0, 9] = bad
    out, lse = fgmp.tree_attention(q, kb, vb, made.cache, tree=words)
    assert torch.equal(out[0, others], plain[0, others]) and torch.equal(lse[0, others], plain_lse[0, others])


@pytest.mark.parametrize("H,G,D,T,n", [(4, 2, 64, 1, 200), (4, 2, 128, 3, 200), (4, 2, 128, 1, 3000), (40, 2, 128, 3, 200), (4, 2, 256, 2, 200), (12, 2, 64, 9, 500)])
def test_a_code_that_is_no_number_reaches_what_the_formula_says(H, G, D, T, n):
    """NaN in a key: nothing but NaN for its head.  NaN in a value: in that element alone."""
    g = _gen(14)
    made = Made8(g, [n], G, D, 0)
    q = _randn(g, 1, T, H, D, dtype=BF16)
    plain, plain_lse = fgmp.tree_attention(q, None, None, made.cache)
    made.v[0, n - 2, 1, 5] = 0x7F
    out, lse = fgmp.tree_attention(q, None, None, made.cache)
    per = H // G
    bad = torch.zeros(1, T, H, D, dtype=torch.bool, device=DEV)
    bad[:, :, per:, 5] = True
    assert torch.equal(torch.isnan(out), bad) and torch.equal(out[~bad], plain[~bad]) and torch.equal(lse, plain_lse)
    made.k[0, 3, 0, 1] = 0xFF
    out, lse = fgmp.tree_attention(q, None, None, made.cache)
    assert bool(torch.isnan(out[:, :, :per]).all()) and bool(torch.isnan(lse[:, :, :per]).all())
    assert torch.equal(lse[:, :, per:], plain_lse[:, :, per:])


def test_rotations_past_32_bits():
    """Vectors more than 4 GiB behind their pointers, read and written."""
    g = _gen(9)
    step = 9 << 27
    wide = torch.empty(3 * step, dtype=F32, device=DEV).as_strided((1, 3, 2, 64), (3 * step, step, 64, 1))
    q = _randn(g, 1, 3, 2, 64)
    wide.copy_(q)
    f = (10000.0 ** (-torch.arange(32, device=DEV) / 32)).float()
    want, _, _ = fgmp.rotate_heads(q, positions=_i32([[7, 8, 9]]), inv_freq=f, dtype=F32)
    got, _, _ = fgmp.rotate_heads(wide, positions=_i32([[7, 8, 9]]), inv_freq=f, dtype=F32)
    assert torch.equal(got, want)
    fgmp.rotate_heads(q, positions=_i32([[7, 8, 9]]), inv_freq=f, q_out=wide)
    assert torch.equal(wide, want)


def test_offsets_of_8_bits_past_32_bits():
    """Codes and scales that lie more than 4 GiB behind their pointers: one token, many rows, append, read."""
    g = _gen(7)
    D, G, page, n = 128, 2, 64, 150
    pages = (5 << 30) // (page * G * D)
    k, v = (torch.empty(pages, page, G, D, dtype=torch.uint8, device=DEV) for _ in range(2))
    far = (5 << 30) // pages // 16 * 16
    ks, vs = (torch.empty(pages * far, dtype=torch.uint8, device=DEV).as_strided((pages, G, page), (far, page, 1)) for _ in range(2))
    table = [pages - 1, 0, pages - 7, pages - 3]
    made = Made8(g, [n], G, D, 0)
    for j, at in enumerate(table[:3]):
        m = min(page, n - page * j)
        k[at, :m], v[at, :m] = made.k[0, page * j:page * j + m], made.v[0, page * j:page * j + m]
        ks[at, :, :m], vs[at, :, :m] = made.ks[0, :, page * j:page * j + m], made.vs[0, :, page * j:page * j + m]
    cache = fgmp.QuantCache(k.view(E4M3), v.view(E4M3), ks, vs, _i32([n]), _i32([table]))
    for T in (1, 2, 40):
        _say("offsets8", T)
        q = _randn(g, 1, T, 4, D, dtype=BF16)
        out, lse = fgmp.tree_attention(q, None, None, cache)
        _compare_attention(out, lse, q, made, None, None, None, [T], D ** -0.5, 2)
    new = _randn(g, 1, 60, G, D)
    cache.lengths = fgmp.cache_append(new, -new, cache)
    got_k, got_v = fgmp.cache_read(cache, tokens=n + 60, dtype=F32)
    assert torch.equal(got_k[0, :n], made.keys[0].float()) and torch.equal(got_v[0, :n], made.values[0].float())
    assert torch.equal(got_k[0, n:], -got_v[0, n:])
    code, scale = _quantized(new[0])
    assert torch.equal(got_k[0, n:].cpu(), code.view(E4M3).float() * torch.pow(2.0, scale.float() - 127)[..., None])


# ---- verification ----

def _verified(target, tokens, u, draft, parents, counts):
    """By the definition, in 64 bits on the CPU: rows, accepted, and the token behind with the sums around its draw."""
    target, tokens, u = target.double().cpu().nan_to_num(0.0).clamp(min=0), tokens.tolist(), u.double().cpu().nan_to_num(0.0).clamp(0, 1)
    draft = None if draft is None else draft.double().cpu().nan_to_num(0.0).clamp(min=0)
    B, N, V = target.shape
    rows, accepted, behind = [], [], []
    for b in range(B):
        count = max(0, min(N, counts[b]))
        if count == 0:
            rows.append([-1] * N), accepted.append(0), behind.append(-1)
            continue
        up = list(range(-1, N - 1)) if parents is None else parents[b].tolist()
        path, out = [0], []
        for t in range(1, count):
            r, x = path[-1], tokens[b][t]
            if up[t] != r or up[t] >= t or x in out:
                continue
            p = float(target[b, r, x]) if 0 <= x < V else 0.0
            q = (float(draft[b, t - 1, x]) if 0 <= x < V else 1.0) if draft is not None else 1.0 - sum(max(0.0, float(target[b, r, y])) for y in out if 0 <= y < V)
            if float(u[b, t]) * q < p:
                path, out = path + [t], []
            else:
                out.append(x)
        w = target[b, path[-1]].clone()
        if out and draft is not None:
            w -= draft[b, path[-1]]
        elif out:
            w[[y for y in out if 0 <= y < V]] = 0.0
        w = torch.where(w > 0, w, 0.0)
        if float(w.sum()) == 0.0:
            w = torch.where(target[b, path[-1]] > 0, target[b, path[-1]], 0.0)
        rows.append(path + [-1] * (N - len(path))), accepted.append(len(path))
        sums = w.cumsum(0)
        if float(sums[-1]) == 0.0:
            behind.append(-1)
        else:
            at = int(torch.searchsorted(sums, u[b, 0] * sums[-1], right=True))
            behind.append(at if at < V else int(w.nonzero().max()))
    return rows, accepted, behind


def _distributions(g, *shape, spread=3.0):
    return torch.softmax(torch.randn(*shape, generator=g) * spread, -1)


VERIFY = [
    # batch, tokens, vocab, kind, dtype, counts
    (1, 1, 1, "given", F32, None),
    (3, 5, 2, "chain", F32, [5, 0, 1]),
    (2, 8, 63, "tree", F32, None),
    (5, 9, 1023, "tree", BF16, [9, 4, 1, 0, 7]),
    (4, 6, 1024, "chain", F32, [6, 6, 2, 99]),
    (4, 6, 1025, "given", F32, None),
    (2, 33, 5003, "tree", F32, [33, 17]),
    (16, 8, 32000, "chain", BF16, None),
    (3, 25, 32001, "tree", F32, None),
    (2, 70, 4097, "given", BF16, [70, -3]),
    (1, 300, 700, "tree", F32, None),
    (1, 2, 300001, "chain", F32, None),
    (1100, 3, 100, "chain", F32, None),
    (600, 2, 9000, "chain", BF16, None),        # (more segments than a sequence's workgroups have waves)
    (300, 3, 20001, "given", F32, None),
]


@pytest.mark.parametrize("B,N,V,kind,dtype,counts", VERIFY)
def test_verification_against_its_definition(B, N, V, kind, dtype, counts):
    _say("verify", B, N, V, kind, dtype, counts)
    g = _gen(B + N + V)
    wide = torch.zeros(B, N, V + 3, dtype=dtype, device=DEV)     # (rows that start at any element)
    target = wide[..., 1:V + 1]
    seen = set()
    for trial in range(3):
        logits = torch.randn(B, N, V, generator=g) * 3.0
        target.copy_(torch.softmax(logits, -1))
        u = torch.rand(B, N, generator=g)
        if trial == 2:
            u[:, 0] = torch.where(torch.rand(B, generator=g) < 0.5, 0.0, 1.0 - 2.0 ** -24)
        draft, parents = None, None
        if kind == "chain":
            draft = torch.softmax(logits[:, :-1] * 0.9 + torch.randn(B, N - 1, V, generator=g) * (0.3 + trial), -1).to(dtype).to(DEV)
            tokens = torch.cat([torch.zeros(B, 1, dtype=torch.int64), torch.multinomial(draft.float().cpu().view(-1, V), 1).view(B, N - 1)], 1)
        else:
            if kind == "tree":
                parents = (torch.arange(N) - torch.randint(1, 4, (B, N), generator=g)).clamp(min=0)
                parents[:, 0] = 77          # (not read)
                if N > 6:
                    parents[0, 5], parents[0, 6] = 6, -1      # behind itself, none: never reached
            likely = logits.topk(min(V, 4), -1).indices
            up = (torch.arange(N) - 1).clamp(min=0).expand(B, N) if parents is None else parents.clamp(0, N - 1)
            tokens = likely[torch.arange(B)[:, None], up, torch.randint(0, likely.shape[-1], (B, N), generator=g)]
            if N > 3:
                tokens[0, 3] = V + 5        # no such token
                tokens[-1, 2] = -1
        tokens[:, 0] = -9                   # (not read)
        given = dict(draft=draft, parents=None if parents is None else parents.int().to(DEV), counts=None if counts is None else _i32(counts))
        rows, accepted, behind = fgmp.verify_drafts(target, tokens.int().to(DEV), u.to(DEV), **given)
        want = _verified(target, tokens, u, draft, parents, [N] * B if counts is None else counts)
        assert rows.tolist() == want[0] and accepted.tolist() == want[1] and behind.tolist() == want[2], trial
        seen |= set(want[1])
    _say("kept", sorted(seen))


def test_a_workspace_serves_one_verification_after_another():
    g = _gen(31)
    ws = fgmp.new_workspace(fgmp.verify_drafts_workspace_bytes(4, 6, 20000), DEV)
    for V, B in ((20000, 4), (1000, 2), (19999, 4), (3, 1)):
        target, u = _distributions(g, B, 6, V).to(DEV), torch.rand(B, 6, generator=g)
        tokens = torch.randint(0, V, (B, 6), generator=g)
        got = fgmp.verify_drafts(target, tokens.int().to(DEV), u.to(DEV), workspace=ws)
        assert [x.tolist() for x in got] == list(_verified(target, tokens, u, None, None, [6] * B))
        assert not bool(ws[:fgmp.WORKSPACE_CONTROL_BYTES].any())


@pytest.mark.parametrize("N", [1, 2, 63, 64, 65, 200])
@pytest.mark.parametrize("kind", ["chain", "given", "path", "children"])
def test_everything_is_kept_or_refused(N, kind):
    """Around the most tokens that a wave walks over by itself.  Of one token with N - 1 children all but the last are refused."""
    _say("verify all", N, kind)
    g = _gen(N)
    V = 777
    target = _distributions(g, 2, N, V)
    tokens = target.roll(1, 1).argmax(-1)
    u = torch.zeros(2, N)
    draft = parents = None
    if kind == "chain":
        draft = _distributions(g, 2, N - 1, V).to(DEV)
    elif kind == "path":
        parents = (torch.arange(N) - 1).expand(2, N)
    elif kind == "children":
        parents = torch.zeros(2, N, dtype=torch.int64)
        tokens = torch.arange(N).expand(2, N)
        target[:, 0] = torch.rand(2, V, generator=g) + 0.5
        target[:, 0] /= target[:, 0].sum(-1, keepdim=True)
        u[:] = 1.0 - 2.0 ** -24
        u[:, -1] = 0.0
    u[:, 0] = 0.6
    got = fgmp.verify_drafts(target.to(DEV), tokens.int().to(DEV), u.to(DEV), draft=draft, parents=None if parents is None else parents.int().contiguous().to(DEV))
    assert [x.tolist() for x in got] == list(_verified(target, tokens, u, draft, parents, [N] * 2))
    assert got[1].tolist() == [min(N, 2) if kind == "children" else N] * 2


@pytest.mark.parametrize("N", [4, 70])
@pytest.mark.parametrize("bad", [math.nan, -2.0])
def test_what_is_no_probability_counts_as_zero(N, bad):
    """In the drafted distributions too: such a token is kept where the target has it, never where the target has 0, and takes nothing from w."""
    g = _gen(int(N))
    B, V = 64, 1500
    target, draft = _distributions(g, B, N, V), _distributions(g, B, N - 1, V)
    target[torch.rand(B, N, V, generator=g) < 0.3] = bad
    target[torch.rand(B, N, V, generator=g) < 0.3] = 0.0
    draft[torch.rand(B, N - 1, V, generator=g) < 0.5] = bad
    tokens = torch.randint(0, V, (B, N), generator=g)
    tokens[::7, 1] = -1
    tokens[3::7, 1] = V
    u = torch.rand(B, N, generator=g) * 1.4 - 0.2
    u[5::9] = math.nan
    for given in (None, draft):
        got = fgmp.verify_drafts(target.to(DEV), tokens.int().to(DEV), u.to(DEV), draft=None if given is None else given.to(DEV))
        assert [x.tolist() for x in got] == list(_verified(target, tokens, u, given, None, [N] * B)), given is None
        parents = torch.zeros(B, N, dtype=torch.int64)
    got = fgmp.verify_drafts(target.to(DEV), tokens.int().to(DEV), u.to(DEV), parents=parents.int().to(DEV))
    assert [x.tolist() for x in got] == list(_verified(target, tokens, u, None, parents, [N] * B))


def test_rows_of_which_nothing_is_left():
    """A draft that covers the target: drawn from the target itself.  A row of zeros, of NaN, of negative numbers: no token."""
    V = 3000
    target = torch.zeros(4, 2, V, device=DEV)
    target[0, :, 17], target[0, :, 2999] = 0.25, 0.5
    target[1] = math.nan
    target[2] = -1.0
    target[3, :, 5], target[3, :, 6] = 1.0, math.nan
    draft = target[:, :1].clone()
    draft[0, 0, 17], draft[0, 0, 3] = 0.5, 0.5
    draft[0, 0, 2999] = 0.5
    tokens = _i32([[0, 17], [0, 1], [0, 1], [0, 7]])
    for u0, want in ((0.0, [17, -1, -1, 5]), (0.3, [17, -1, -1, 5]), (0.34, [2999, -1, -1, 5]), (0.999, [2999, -1, -1, 5])):
        u = torch.tensor([[u0, 0.9]] * 4, device=DEV)
        rows, accepted, behind = fgmp.verify_drafts(target, tokens, u, draft=draft)
        assert behind.tolist() == want and accepted.tolist() == [1] * 4 and rows.tolist() == [[0, -1]] * 4, u0
    # numbers outside of 0 .. 1 are taken as the nearest
    for u0, want in ((-1.0, 17), (2.0, 2999), (math.nan, 17)):
        _, _, behind = fgmp.verify_drafts(target, tokens, torch.tensor([[u0, 0.0]] * 4, device=DEV))
        assert int(behind[0]) == want, u0


@pytest.mark.parametrize("kind", ["chain", "tree"])
def test_first_tokens_are_distributed_as_the_target(kind):
    """What a verification gives first -- a kept drafted token, or the one behind -- has the target's distribution, whatever was drafted: counts of 16384
    sequences within five standard deviations."""
    g = _gen(5)
    B, V, N = 16384, 7, 3
    p, q = _distributions(g, V, spread=1.0), _distributions(g, V, spread=1.0)
    target = p.expand(B, N, V).contiguous().to(DEV)
    u = torch.rand(B, N, generator=g).to(DEV)
    if kind == "chain":
        tokens = torch.multinomial(q.expand(B, V), N, replacement=True, generator=g).int().to(DEV)
        rows, accepted, behind = fgmp.verify_drafts(target, tokens, u, draft=q.expand(B, N - 1, V).contiguous().to(DEV))
    else:
        tokens = torch.tensor([0, 2, 5], dtype=torch.int32).expand(B, N).contiguous().to(DEV)
        rows, accepted, behind = fgmp.verify_drafts(target, tokens, u, parents=torch.tensor([0, 0, 0], dtype=torch.int32).expand(B, N).contiguous().to(DEV))
    kept = tokens.gather(1, rows[:, 1:2].clamp(min=0).long())[:, 0]
    first = torch.where(accepted > 1, kept, behind)
    seen = torch.bincount(first.cpu().long(), minlength=V).double()
    assert bool(((seen - B * p.double()).abs() <= 5 * (B * p.double() * (1 - p.double())).sqrt() + 1).all()), (seen / B, p)


def test_probabilities_past_32_bits():
    """Rows more than 4 GiB behind their pointer."""
    g = _gen(8)
    V, step = 5000, 3 << 29
    buffer = torch.zeros(2 * step + V, dtype=F32, device=DEV)
    target = buffer.as_strided((1, 3, V), (1, step, 1))
    target.copy_(_distributions(g, 1, 3, V))
    tokens, u = torch.zeros(1, 3, dtype=torch.int64), torch.tensor([[0.77, 0.0, 0.0]])
    tokens[0, 1:] = target[0, :2].argmax(-1).cpu()
    got = fgmp.verify_drafts(target, tokens.int().to(DEV), u.to(DEV))
    assert [x.tolist() for x in got] == list(_verified(target, tokens, u, None, None, [3])) and got[1].tolist() == [3]


# ---- a step of all of them: streams, graphs ----

def _step(g):
    B, T, H, G, D, V = 2, 5, 8, 2, 64, 3001
    made = Made8(g, [700, 333], G, D, 16, room=8)
    st = {"made": made, "qkv": _randn(g, B, T, H + 2 * G, D), "w": 1.0 + 0.1 * _randn(g, D), "f": (10000.0 ** (-torch.arange(32, device=DEV) / 32)).float(),
          "positions": _i32([[700 + i for i in range(T)], [333 + i for i in range(T)]]), "target": _distributions(g, B, T, V).to(DEV),
          "draft": _distributions(g, B, T - 1, V).to(DEV), "u": torch.rand(B, T, generator=g).to(DEV) * 0.5}
    st["tokens"] = torch.cat([torch.zeros(B, 1, dtype=torch.int64), st["target"][:, :-1].argmax(-1).cpu()], 1).int().to(DEV)
    st["q"], st["k"], st["v"] = (torch.empty(B, T, n, D, dtype=BF16, device=DEV) for n in (H, G, G))
    st["out"], st["lse"] = torch.empty_like(st["q"]), torch.empty(B, T, H, device=DEV)
    st["ws"] = fgmp.new_workspace(fgmp.tree_attention_workspace_bytes(B, T, H, G, D, made.slots), DEV)
    st["ws2"] = fgmp.new_workspace(fgmp.verify_drafts_workspace_bytes(B, T, V), DEV)
    st["rows"], st["accepted"], st["next"], st["after"] = _i32([[0] * T] * B), _i32([0, 0]), _i32([0, 0]), _i32([0, 0])
    st["longer"] = fgmp.QuantCache(made.k.view(E4M3), made.v.view(E4M3), made.ks, made.vs, st["after"], made.cache.page_table)
    st["read"] = [torch.zeros(B, 40, G, D, dtype=BF16, device=DEV) for _ in range(2)]
    return st


def _run_step(st):
    q, k, v = st["qkv"].split([8, 2, 2], 2)
    fgmp.rotate_heads(q, k, v, st["positions"], st["f"], None, st["w"], st["w"], q_out=st["q"], k_out=st["k"], v_out=st["v"])
    fgmp.tree_attention(st["q"], st["k"], st["v"], st["made"].cache, scale=0.125, out=st["out"], lse=st["lse"], workspace=st["ws"])
    fgmp.verify_drafts(st["target"], st["tokens"], st["u"], draft=st["draft"], rows=st["rows"], accepted=st["accepted"], next_tokens=st["next"], workspace=st["ws2"])
    fgmp.cache_append(st["k"], st["v"], st["made"].cache, rows=st["rows"], counts=st["accepted"], lengths_out=st["after"])
    fgmp.cache_read(st["longer"], first=320, k_out=st["read"][0], v_out=st["read"][1])
    return [st[n] for n in ("q", "k", "v", "out", "lse", "rows", "accepted", "next", "after")] + st["read"] + [st["made"].k, st["made"].v, st["made"].ks, st["made"].vs]


def _bits(ts):
    return [t.clone().view(torch.uint8) for t in ts]


def test_a_step_on_another_stream_and_in_a_graph():
    st = _step(_gen(20))
    want = _bits(_run_step(st))
    torch.cuda.synchronize()
    assert st["accepted"].tolist() != [1, 1]               # (something was kept)
    side = torch.cuda.Stream()
    st = _step(_gen(20))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _bits(_run_step(st))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # two graphs that share their workspaces, replayed in turn, with other work and other inputs between
    states = [_step(_gen(20)), _step(_gen(22))]
    for n in ("ws", "ws2"):
        states[1][n] = states[0][n]
    firsts = [[t.clone() for t in (s["made"].k, s["made"].v, s["made"].ks, s["made"].vs)] for s in states]
    graphs, outs = [], []
    torch.cuda.synchronize()
    for s in states:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(_run_step(s))
        graphs.append(graph)

    def put_back(i):
        s = states[i]
        for t, f in zip((s["made"].k, s["made"].v, s["made"].ks, s["made"].vs), firsts[i]):
            t.copy_(f)

    for replay in range(6):
        i = replay % 2
        _say("replay", replay)
        put_back(i)
        for t in outs[i][:-4]:
            t.zero_()
        if replay >= 2:
            states[i]["u"].copy_(torch.rand(2, 5, generator=_gen(replay)))
            states[i]["qkv"].mul_(1.01)
        graphs[i].replay()
        torch.cuda.synchronize()
        got = _bits(outs[i])
        put_back(i)
        eager = _bits(_run_step(states[i]))
        assert all(torch.equal(a, b) for a, b in zip(got, eager)), replay
        if replay == 0:
            assert all(torch.equal(a, b) for a, b in zip(got, want))
