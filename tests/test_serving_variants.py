"""The kernels' other forms on the GPU, against the same definitions with the same bounds: rotations of two tokens to a workgroup, verification of many
tokens over long segments, appends of several tokens to a workgroup with elements of every kind anywhere."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import test_serving_ops as ops  # noqa: E402
from paper_2504_14152_amd import fgmp  # noqa: E402
from test_serving_ops import BF16, DEV, F32, _distributions, _gen, _i32, _say, _vectors, _verified  # noqa: E402

pytestmark = pytest.mark.gpu

# As many tokens as go two to a workgroup: every number of lanes that a vector takes, filled and not, both norms and none, several axes, both kinds of pairs, part of a vector
# rotated and nothing of it, every pair of types; odd numbers of tokens, whose last workgroup has one.
ROTATE_MANY = [
    (BF16, BF16, 2, 513, 5, 1, 128, 48, 3, "layer", True, 131072),
    (F32, F32, 1, 1025, 3, 2, 256, 128, 1, "rms", False, 7),
    (F32, BF16, 3, 343, 2, 1, 80, 40, 1, "rms", False, 0),
    (BF16, F32, 1, 1031, 1, 1, 512, 256, 2, "layer", False, -5),
    (F32, BF16, 1, 1024, 40, 8, 128, 64, 1, "rms", True, (1 << 29) - 3),
    (BF16, BF16, 1, 1027, 2, 1, 192, 96, 1, "rms", False, 1000003),
    (F32, F32, 5, 205, 3, 1, 64, 0, 1, "rms", False, 0),
    (F32, BF16, 2, 601, 1, 1, 8, 4, 1, "layer", True, 3),
    (BF16, BF16, 1024, 2, 1, 1, 64, 32, 1, "rms", False, 9),
    (F32, BF16, 401, 3, 2, 1, 96, 20, 2, "layer", False, 9),
    (BF16, F32, 1, 1033, 3, 3, 256, 64, 2, "none", True, 40),
]


@pytest.mark.parametrize("row", ROTATE_MANY, ids=str)
def test_rotated_heads_two_tokens_to_a_workgroup(row):
    assert row[2] * row[3] >= 1024 and row[3] >= 2
    ops.test_rotated_heads_against_their_formula(*row)


# ---- verification over long segments ----

def _long(B, V):
    """Whether a verification's segments are the long ones."""
    return B * -(-V // 512) > 8192


def _same(got, target, tokens, u, draft, parents, counts):
    """Sequence by sequence: their distributions may be one in memory."""
    rows, accepted, behind = (x.tolist() for x in got)
    for b in range(tokens.shape[0]):
        one = slice(b, b + 1)
        want = _verified(target[one], tokens[one], u[one], None if draft is None else draft[one], None if parents is None else parents[one], counts[one])
        assert ([rows[b]], [accepted[b]], [behind[b]]) == want, b


@pytest.mark.parametrize("B,N,V,kind,dtype", [(300, 70, 15001, "tree", BF16), (300, 9, 20001, "tree", F32), (300, 65, 15001, "chain", F32), (280, 64, 16000, "children", BF16),
                                              (290, 300, 14999, "children", F32), (300, 66, 15001, "given", BF16)])
def test_verification_over_long_segments(B, N, V, kind, dtype):
    """All sequences share their distributions (a batch stride of zero), not their tokens and numbers."""
    assert _long(B, V)
    _say("verify long", B, N, V, kind, dtype)
    g = _gen(N + V)
    logits = torch.randn(1, N, V, generator=g) * 3.0
    target = torch.softmax(logits, -1).to(dtype).expand(B, N, V)
    u = torch.rand(B, N, generator=g)
    draft = parents = None
    if kind == "chain":
        draft = torch.softmax(logits[:, :-1] * 0.9 + torch.randn(1, N - 1, V, generator=g) * 0.4, -1).to(dtype).expand(B, N - 1, V)
        tokens = torch.cat([torch.zeros(B, 1, dtype=torch.int64), torch.multinomial(draft[0].float(), B, replacement=True, generator=g).t()], 1)
    else:
        if kind == "tree":
            parents = (torch.arange(N) - torch.randint(1, 4, (B, N), generator=g)).clamp(min=0)
        elif kind == "children":           # (of few tokens, most of the first one: refused tokens all over the vocabulary)
            parents = torch.where(torch.rand(B, N, generator=g) < 0.9, 0, torch.randint(0, 8, (B, N), generator=g).minimum((torch.arange(N) - 1).clamp(min=0)))
            u[: B // 2] = 1.0 - 2.0 ** -24
            u[:, 0] = torch.rand(B, generator=g)
        up = (torch.arange(N) - 1).clamp(min=0).expand(B, N) if parents is None else parents
        likely = logits[0].topk(min(V, 4 if kind != "children" else N), -1).indices
        tokens = likely[up, torch.randint(0, likely.shape[-1], (B, N), generator=g)]
        tokens[0, 3], tokens[-1, 2] = V + 5, -1
    counts = torch.randint(0, N + 1, (B,), generator=g)
    counts[::3] = N

    def shared(x):
        return None if x is None else x[:1].to(DEV).expand(x.shape)

    given = dict(draft=shared(draft), parents=None if parents is None else parents.int().contiguous().to(DEV), counts=counts.int().to(DEV))
    got = fgmp.verify_drafts(shared(target), tokens.int().to(DEV), u.to(DEV), **given)
    _same(got, target, tokens, u, draft, parents, counts.tolist())
    again = fgmp.verify_drafts(shared(target), tokens.int().to(DEV), u.to(DEV), **given)
    assert all(torch.equal(x, y) for x, y in zip(got, again))


@pytest.mark.parametrize("N", [2, 70])
def test_rows_of_which_nothing_is_left_over_long_segments(N):
    B, V = 600, 9000
    assert _long(B, V)
    g = _gen(N)
    target = torch.zeros(1, N, V)
    target[0, :, 17], target[0, :, 5000], target[0, :, 8999] = 0.25, 0.25, 0.5
    draft = torch.zeros(1, N - 1, V)
    draft[0, :, 17], draft[0, :, 5000], draft[0, :, 8999], draft[0, :, 1023] = 0.25, 0.25, 0.5, 0.5
    tokens, u = torch.full((B, N), 1023), torch.rand(B, N, generator=g)
    got = fgmp.verify_drafts(target.to(DEV).expand(B, N, V), tokens.int().to(DEV), u.to(DEV), draft=draft.to(DEV).expand(B, N - 1, V))
    _same(got, target.expand(B, N, V), tokens, u, draft.expand(B, N - 1, V), None, [N] * B)
    assert set(got[2].tolist()) == {17, 5000, 8999} and got[1].tolist() == [1] * B
    nothing = torch.zeros(1, N, V, device=DEV).expand(B, N, V)
    assert fgmp.verify_drafts(nothing, tokens.int().to(DEV), u.to(DEV), draft=draft.to(DEV).expand(B, N - 1, V))[2].tolist() == [-1] * B


# ---- appends ----

@pytest.mark.parametrize("source", [BF16, F32])
@pytest.mark.parametrize("G,D,T,lens", [(1, 64, 9001, [0, 77]), (1, 128, 4099, [3, 0, 50]), (3, 256, 811, [47, 1]), (8, 128, 301, [5, 0, 16, 31]), (5, 64, 1301, [31, 0, 1])])
def test_append_of_many_tokens_of_every_kind(source, G, D, T, lens):
    """Vectors that are not finite, zeros, the scale's ends and halves between codes in any place of a workgroup's, its last tokens' too."""
    _say("append8 kinds", source, G, D, T, lens)
    g = _gen(T + D)
    B = len(lens)
    made = ops.Made8(g, lens, G, D, 0, room=T)
    kinds = _vectors(g, 64, D, dtype=source)
    inputs = []
    for _ in range(2):
        x = _vectors(g, B, T, G, D, dtype=source)
        place = torch.rand(B, T, G, generator=g) < 0.3
        place[:, -8:] = True
        inputs.append(torch.where(place.to(DEV)[..., None], kinds[torch.randint(0, 11, (B, T, G), generator=g).to(DEV)], x))
    want = [x.cpu() for x in (made.k, made.v, made.ks, made.vs)]
    lengths = fgmp.cache_append(*inputs, made.cache)
    for x, c, s in ((inputs[0], want[0], want[2]), (inputs[1], want[1], want[3])):
        code, scale = ops._quantized(x)
        for b in range(B):
            m = min(T, made.slots - lens[b])
            c[b, lens[b]:lens[b] + m], s[b, :, lens[b]:lens[b] + m] = code[b, :m], scale[b, :m].t()
    assert ops._is_code(made.k, want[0]) and ops._is_code(made.v, want[1])
    assert torch.equal(made.ks.cpu(), want[2]) and torch.equal(made.vs.cpu(), want[3])
    assert lengths.tolist() == [min(n + T, made.slots) for n in lens]
