"""What a transformer layer does between this library's products when it serves: attention of drafted tokens
over a cache, the upkeep of that cache, and the norms around a block.

  attend   drafted tokens -- a single one, a chain, or a tree of candidates -- attend to a paged cache of keys and
           values and to their drafted ancestors
  weights  the attention weight that the accepted tokens give to each cached one, added to what it had
  append   keys and values of the accepted tokens into their slots of the cache
  evict    a cache cut to its budget: first and last tokens are kept, then those with the most attention weight;
           kept entries from behind the budget move into the places that became free
  norm     y = a x + b act(gate) * norm(o), h = norm(y): residual stream and next block's input

The plain forms are elementary torch operations in 32 bits, rounded once at the end; `exact` restates each
operator in 64 bits, one sequence and head at a time.
"""
from __future__ import annotations

import math

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f32": 4}


def _attend(name, batch, tokens, heads, kv_heads, dim, length, page, dtype="bf16", ragged=False, tree=False):
    return {"name": name, "op": "attend", "batch": batch, "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "length": length, "page": page, "dtype": dtype, "ragged": ragged, "tree": tree}


def _weights(name, batch, tokens, accepted, heads, kv_heads, dim, length, page, dtype="bf16", ragged=False):
    return {"name": name, "op": "weights", "batch": batch, "tokens": tokens, "accepted": accepted, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "length": length, "page": page, "dtype": dtype, "ragged": ragged}


def _append(name, batch, tokens, kv_heads, dim, length, page, dtype="bf16", source="f32", ragged=False):
    return {"name": name, "op": "append", "batch": batch, "tokens": tokens, "kv_heads": kv_heads, "dim": dim, "length": length,
            "page": page, "dtype": dtype, "source": source, "ragged": ragged}


def _evict(name, batch, kv_heads, dim, length, budget, sinks, recent, page, dtype="bf16", ragged=False):
    return {"name": name, "op": "evict", "batch": batch, "kv_heads": kv_heads, "dim": dim, "length": length, "budget": budget,
            "sinks": sinks, "recent": recent, "page": page, "dtype": dtype, "ragged": ragged}


def _norm(name, rows, width, stream="bf16", block="f32", out="bf16", kind="rms", gate="none", act="none", bias=False):
    return {"name": name, "op": "norm", "rows": rows, "width": width, "stream": stream, "block": block, "out": out,
            "kind": kind, "gate": gate, "act": act, "bias": bias}


def listed():
    return [
        # one token of one conversation that has just begun, a head of its own for each query head: latency
        _attend("attend_token_short", 1, 1, 32, 32, 128, 517, 0),
        # eight conversations of different lengths, each verifying a tree of drafted tokens
        _attend("attend_tree_ragged", 8, 25, 64, 8, 128, 4999, 64, ragged=True, tree=True),
        # one token after a very long document, for two requests: all cache, hardly any arithmetic
        _attend("attend_token_long", 2, 1, 64, 8, 128, 131071, 256),
        # drafted chains of a small model in 32 bits, pages of 16
        _attend("attend_chain_f32", 4, 5, 16, 16, 64, 2047, 16, dtype="f32", ragged=True),
        # what one decoded token per sequence adds to the weights of a small batch's caches
        _weights("weights_token", 8, 1, 1, 32, 8, 128, 1055, 16, ragged=True),
        # a few accepted tokens out of a tree each, over long caches
        _weights("weights_accepted_long", 4, 32, 6, 64, 8, 128, 65537, 64, ragged=True),
        # a decode step of a well-filled batch: up to four accepted tokens of each sequence's tree
        _append("append_accepted", 32, 16, 8, 128, 2011, 64, ragged=True),
        # a prompt's keys and values as a product leaves them, into an empty cache
        _append("append_prompt", 1, 4099, 32, 128, 0, 128),
        # a cache that has grown a few tokens over its budget
        _evict("evict_step", 8, 8, 128, 1031, 1024, 4, 256, 64),
        # prompts cut to an eighth, heads choosing for themselves
        _evict("evict_prompt", 2, 32, 128, 16381, 2048, 16, 512, 64, ragged=True),
        # the residual stream of a single token: latency
        _norm("norm_token", 1, 4096),
        # the quantizer benchmark's activations: gated branch, norms on both sides
        _norm("norm_prompt", 16384, 8192, block="bf16", gate="full", act="sigmoid"),
    ]


def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    op = rng.choices(["attend", "weights", "append", "evict", "norm"], [5, 2, 2, 2, 3])[0]
    dtype = rng.choices(["bf16", "f32"], [4, 1])[0]
    if op == "norm":
        width = _log_int(rng, 64, 16384, 16)
        gate = rng.choice(["none", "channel", "group", "full"])
        kind = rng.choices(["rms", "layer"], [3, 1])[0]
        return _unnamed(_norm("", _log_int(rng, 1, 16384 * 8192 // (2 * width)), width, rng.choice(["bf16", "f32"]), rng.choice(["bf16", "f32"]),
                              dtype, kind, gate, rng.choice(["none", "sigmoid", "silu"]) if gate != "none" else "none",
                              kind == "layer" and rng.random() < 0.5))
    heads, kv_heads = rng.choice([(32, 32), (32, 8), (64, 8), (16, 16), (8, 1), (24, 4), (20, 20)])
    dim = rng.choices([64, 128, 256], [2, 5, 1])[0]
    page = rng.choice([0, 16, 64, 256])
    batch, ragged = _log_int(rng, 1, 32), rng.random() < 0.6
    # slots of all sequences together, so that the caches hold at most half of the largest listed ones' bytes
    slots = 131072 * 8 * 128 * 2 // (kv_heads * dim * _SIZE[dtype])
    if op == "attend":
        length = _log_int(rng, 1, min(131072, slots // batch))
        tokens = _log_int(rng, 1, max(1, min(64, (1 << 27) // (batch * heads * (length + 64)))))
        return _unnamed(_attend("", batch, tokens, heads, kv_heads, dim, length, page, dtype, ragged, rng.random() < 0.5))
    if op == "weights":
        accepted = _log_int(rng, 1, 8)
        length = _log_int(rng, 16, min(65536, slots // batch, (1 << 27) // (batch * heads * accepted)))
        return _unnamed(_weights("", batch, accepted + _log_int(rng, 1, 24), accepted, heads, kv_heads, dim, length, page, dtype, ragged))
    if op == "append":
        length = _log_int(rng, 1, 4096)
        tokens = _log_int(rng, 1, max(1, min(4096, slots // (8 * batch))))
        return _unnamed(_append("", batch, tokens, kv_heads, dim, length, page, dtype, rng.choice(["bf16", "f32"]), ragged))
    length = _log_int(rng, 64, min(32768, max(64, slots // (2 * batch))))
    budget = _log_int(rng, 48, length)
    return _unnamed(_evict("", batch, kv_heads, dim, length, budget, rng.choice([0, 4, 16]), rng.choice([0, budget // 8, budget // 3]),
                           page, dtype, ragged))


def _unnamed(case):
    del case["name"]
    return case


# ---- inputs ----

def _lengths(case):
    """Cached tokens of each sequence: all the same, or falling from the longest to about half of it."""
    n, B = case["length"], case["batch"]
    return [n * (2 * B - b) // (2 * B) if case["ragged"] else n for b in range(B)]


def _counts(case):
    """Drafted (attend) or accepted (weights, append) tokens of each sequence."""
    B = case["batch"]
    if case["op"] == "weights":
        return [max(1, case["accepted"] - b % case["accepted"]) if case["ragged"] else case["accepted"] for b in range(B)]
    if case["op"] == "append" and case["ragged"]:
        return [min(case["tokens"], (3 * b + 4) % 5) for b in range(B)]
    return [max(1, case["tokens"] * (2 * B - b) // (2 * B)) if case["ragged"] else case["tokens"] for b in range(B)]


def _generator(seed, part):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + part)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _queries(g, case):
    """Queries whose logits spread over a few units, as those of a trained model do."""
    return (_randn(g, case["batch"], case["tokens"], case["heads"], case["dim"]) * 2.0).to(_TORCH[case["dtype"]])


def _pages(g, pages, page, case):
    """Keys or values: a common direction and what tells tokens apart."""
    common = _randn(g, case["kv_heads"], case["dim"]) * 0.5
    x = torch.randn(pages, page, case["kv_heads"], case["dim"], generator=g, device="cuda", dtype=_TORCH[case["dtype"]])
    return x.add_(common.to(x.dtype))


def _cache(case, seed, room):
    """Keys, values, page table and lengths of a cache that has `room` for more tokens than it holds; where there
    are no pages, one row of slots for each sequence."""
    g = _generator(seed, 1)
    B, page = case["batch"], case["page"]
    most = case["length"] + room
    table = None
    if page:
        each = -(-most // page)
        pages = B * each + 3
        table = torch.randperm(pages, generator=g, device="cuda")[: B * each].view(B, each).int()
    else:
        pages, page = B, -(-most // 64) * 64
    return {"k": _pages(g, pages, page, case), "v": _pages(g, pages, page, case), "table": table, "lengths": _int32(_lengths(case)),
            "slots": page * (1 if table is None else table.shape[1])}


def prepare(case, seed):
    op = case["op"]
    st = {"case": case, "op": op}
    g = _generator(seed, 2)
    if op == "norm":
        M, K = case["rows"], case["width"]
        st["x"] = (_randn(g, M, K) * 3.0).to(_TORCH[case["stream"]])
        st["o"] = (_randn(g, M, K) + 0.25).to(_TORCH[case["block"]])
        st["gate_rows"] = {"none": 0, "channel": M, "group": max(1, min(M, 64)), "full": 1}[case["gate"]]
        st["gate"] = _randn(g, -(-M // st["gate_rows"]), K).to(_TORCH[case["block"]]) if st["gate_rows"] else None
        st["w"] = [1.0 + 0.1 * _randn(g, K) for _ in range(2)]
        st["b"] = [0.1 * _randn(g, K) if case["bias"] else None for _ in range(2)]
        st["y"] = torch.empty_like(st["x"])
        st["h"] = torch.empty(M, K, device="cuda", dtype=_TORCH[case["out"]])
    else:
        room = {"attend": 0, "weights": 0, "evict": 0, "append": case.get("tokens", 0)}[op]
        st.update(_cache(case, seed, room))
        B, H = case["batch"], case["kv_heads"]
    if op in ("attend", "append"):
        kind = _TORCH[case.get("source", case["dtype"])]
        st["new_k"] = _randn(g, B, case["tokens"], H, case["dim"]).to(kind)
        st["new_v"] = _randn(g, B, case["tokens"], H, case["dim"]).to(kind)
        st["counts"] = _int32(_counts(case))
    if op == "attend":
        T = case["tokens"]
        st["q"] = _queries(g, case)
        st["scale"] = 1.0 / math.sqrt(case["dim"])
        st["tree"] = None
        if case["tree"]:
            # every token's parent is one of the three before it, or the last cached token; a bit for each
            # ancestor and for the token itself
            back = torch.randint(1, 4, (B, T), generator=g, device="cuda").cpu()
            sees = torch.eye(T, dtype=torch.bool).repeat(B, 1, 1)
            for t in range(1, T):
                parent = t - back[:, t]
                sees[:, t] |= sees[torch.arange(B), parent.clamp(min=0)] & (parent >= 0)[:, None]
            words = torch.zeros(B, T, -(-T // 64) * 64, dtype=torch.int64)
            words[:, :, :T] = sees
            st["tree"] = (words.view(B, T, -1, 64) << torch.arange(64)).sum(-1).cuda()
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty(B, T, case["heads"], device="cuda")
    if op == "weights":
        st["q"] = _queries(g, case)
        st["scale"] = 1.0 / math.sqrt(case["dim"])
        order = torch.rand(B, case["tokens"], generator=g, device="cuda").argsort(-1)[:, : case["accepted"]]
        st["rows"] = order.sort(-1).values.int()
        st["counts"] = _int32(_counts(case))
        st["have"] = _randn(g, B, H, st["slots"]).square()
        st["out"] = torch.zeros(B, H, st["slots"], device="cuda")
        logits, seen = _accepted_logits(st)
        st["lse"] = torch.zeros(B, case["tokens"], case["heads"], device="cuda")
        norm = torch.logsumexp(logits.masked_fill(~seen, -math.inf), -1).transpose(1, 2)
        st["lse"].scatter_(1, st["rows"].long()[:, :, None].expand(-1, -1, case["heads"]), norm.reshape(B, -1, case["heads"]))
    if op == "append":
        st["rows"] = torch.rand(B, case["tokens"], generator=g, device="cuda").argsort(-1).int() if case["ragged"] else None
        if st["rows"] is not None:
            st["rows"] = torch.where(torch.arange(case["tokens"], device="cuda") < st["counts"][:, None], st["rows"], -1)
        st["positions"] = st["lengths"][:, None] + torch.arange(case["tokens"], device="cuda", dtype=torch.int32)
        st["slot_positions"] = torch.zeros(B, H, st["slots"], dtype=torch.int32, device="cuda")
        st["slot_weights"] = torch.ones(B, H, st["slots"], device="cuda")
        st["lengths_out"] = torch.empty_like(st["lengths"])
    if op == "evict":
        # tokens whose weight is a few hundred times another's, the newest ones without any yet
        w = torch.exp(1.5 * _randn(g, B, H, st["slots"]))
        st["weights"] = torch.where(torch.arange(st["slots"], device="cuda") < (st["lengths"] - 3)[:, None, None], w, 0.0)
        # an eighth more tokens have been seen than are held, different ones in each head
        gone = torch.rand(B, H, st["slots"], generator=g, device="cuda") < 0.125
        st["positions"] = (torch.arange(st["slots"], device="cuda") + gone.long().cumsum(-1)).int()
        last = (st["lengths"].long() - 1)[:, None, None].expand(B, H, 1)
        st["seen"] = (st["positions"].gather(-1, last.clamp(min=0)).amax((1, 2)) + 1).int()
        st["weights_out"] = torch.zeros_like(st["weights"])
        st["positions_out"] = torch.zeros_like(st["positions"])
        st["lengths_out"] = torch.empty_like(st["lengths"])
    if own and op != "norm":
        # what a serving program keeps beside its tensors: the cache's handle and the workspace
        from paper_2504_14152_amd import fgmp
        st["cache"] = fgmp.Cache(st["k"], st["v"], st["lengths"], st["table"])
        size = 0
        if op == "attend":
            size = fgmp.tree_attention_workspace_bytes(B, case["tokens"], case["heads"], H, case["dim"], st["slots"])
        if op == "evict":
            size = fgmp.cache_evict_workspace_bytes(B, H, st["slots"], case["budget"])
        st["workspace"] = fgmp.new_workspace(size, "cuda")
    return st


# ---- the plain forms ----

def _gathered(st, pages):
    """Slots of the longest sequence's length for every sequence, in 32 bits: batch x heads x slots x dim."""
    most, page = st["case"]["length"], st["k"].shape[1]
    if st["table"] is None:
        return pages[:, :most].float().transpose(1, 2)
    slot = torch.arange(most, device="cuda")
    return pages[st["table"].long()[:, slot // page], slot % page].float().transpose(1, 2)


def _grouped(q, kv_heads):
    """batch x tokens x heads x dim -> batch x kv heads x (tokens, heads of the group) x dim, in 32 bits."""
    B, T, H, D = q.shape
    return q.float().view(B, T, kv_heads, H // kv_heads, D).transpose(1, 2).reshape(B, kv_heads, T * H // kv_heads, D)


def _accepted_logits(st):
    """Logits of the accepted tokens over the cache, and which slots each sees: batch x kv heads x accepted x
    heads of the group x slots."""
    case = st["case"]
    B, H, A, G = case["batch"], case["kv_heads"], case["accepted"], case["heads"] // case["kv_heads"]
    rows = st["rows"].long()[:, :, None, None].expand(-1, -1, case["heads"], case["dim"])
    logits = torch.matmul(_grouped(st["q"].gather(1, rows), H), _gathered(st, st["k"]).transpose(2, 3)) * st["scale"]
    i = torch.arange(A, device="cuda")
    ends = (st["lengths"] - st["counts"])[:, None] + i + 1
    seen = torch.arange(case["length"], device="cuda") < torch.where(i < st["counts"][:, None], ends, 0)[:, :, None]
    return logits.view(B, H, A, G, -1), seen[:, None, :, None, :]


def _plain_attend(st):
    case = st["case"]
    B, T, H, D = st["q"].shape
    q = _grouped(st["q"], case["kv_heads"])
    k = torch.cat([_gathered(st, st["k"]), st["new_k"].float().transpose(1, 2)], 2)
    v = torch.cat([_gathered(st, st["v"]), st["new_v"].float().transpose(1, 2)], 2)
    t = torch.arange(T, device="cuda")
    if st["tree"] is None:
        sees = (t[None, :] <= t[:, None]).expand(B, T, T)
    else:
        sees = (st["tree"][:, :, t // 64] >> (t % 64)) & 1 == 1
    drafted = t < st["counts"][:, None]
    sees = sees & drafted[:, None, :]
    cached = (torch.arange(case["length"], device="cuda") < st["lengths"][:, None])[:, None, :].expand(B, T, -1)
    seen = (torch.cat([cached, sees], -1) & drafted[:, :, None])[:, None, :, None, :]
    logits = (torch.matmul(q, k.transpose(2, 3)) * st["scale"]).view(B, case["kv_heads"], T, H // case["kv_heads"], -1)
    logits = torch.where(seen, logits, -math.inf)
    most = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - torch.where(most == -math.inf, 0.0, most))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, case["kv_heads"], -1, p.shape[-1]), v).view(B, case["kv_heads"], T, -1, D)
    out = out / torch.where(total == 0, 1.0, total)
    lse = (most + torch.log(total)).squeeze(-1)
    return out.transpose(1, 2).reshape(B, T, H, D).to(st["q"].dtype), lse.transpose(1, 2).reshape(B, T, H)


def _plain_weights(st):
    case = st["case"]
    logits, seen = _accepted_logits(st)
    B, H, A, G, n = logits.shape
    lse = st["lse"].gather(1, st["rows"].long()[:, :, None].expand(-1, -1, case["heads"]))
    lse = lse.view(B, A, H, G).transpose(1, 2)[..., None]
    p = torch.where(seen, torch.exp(logits - lse), 0.0).sum((2, 3))
    held = torch.arange(n, device="cuda") < st["lengths"][:, None, None]
    out = st["out"]
    out[:, :, :n] = torch.where(held, st["have"][:, :, :n] + p, out[:, :, :n])
    return out


def _plain_append(st):
    T, page = st["case"]["tokens"], st["k"].shape[1]
    i = torch.arange(T, device="cuda")
    taken = i < st["counts"][:, None]
    slot = (st["lengths"][:, None] + i)[taken].long()
    b = torch.arange(taken.shape[0], device="cuda")[:, None].expand_as(taken)[taken]
    row = (i.expand_as(taken) if st["rows"] is None else st["rows"].long())[taken]
    at = b if st["table"] is None else st["table"].long()[b, slot // page]
    st["k"][at, slot % page] = st["new_k"][b, row].to(st["k"].dtype)
    st["v"][at, slot % page] = st["new_v"][b, row].to(st["v"].dtype)
    st["slot_positions"][b, :, slot] = st["positions"][b, row][:, None]
    st["slot_weights"][b, :, slot] = 0.0
    return st["k"], st["v"], st["slot_positions"], st["slot_weights"], st["lengths"] + st["counts"]


def _plain_evict(st):
    case, page = st["case"], st["k"].shape[1]
    n, budget = st["weights"].shape[-1], case["budget"]
    slot = torch.arange(n, device="cuda")
    held = slot < st["lengths"][:, None, None]
    pos = st["positions"]
    fixed = (pos < case["sinks"]) | (pos >= (st["seen"] - case["recent"])[:, None, None])
    rank = torch.where(held, torch.where(fixed, math.inf, st["weights"]), -math.inf)
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices
    keep = torch.zeros_like(held.expand_as(rank)).scatter_(-1, order[..., :budget], True) & held
    left = torch.clamp(st["lengths"], max=budget)
    over = (st["lengths"] > budget)[:, None, None]
    b, h, to = torch.nonzero(held & ~keep & (slot < budget) & over, as_tuple=True)
    _, _, fro = torch.nonzero(keep & (slot >= budget) & over, as_tuple=True)
    if st["table"] is None:
        source, target = b, b
    else:
        source, target = st["table"].long()[b, fro // page], st["table"].long()[b, to // page]
    st["k"][target, to % page, h] = st["k"][source, fro % page, h]
    st["v"][target, to % page, h] = st["v"][source, fro % page, h]
    stays = slot < left[:, None, None]
    w = torch.where(stays, st["weights"], st["weights_out"])
    p = torch.where(stays, pos, st["positions_out"])
    w[b, h, to] = st["weights"][b, h, fro]
    p[b, h, to] = pos[b, h, fro]
    return st["k"], st["v"], w, p, left


def _plain_normed(x, w, b, kind):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5) * w
    return x if b is None else x + b


def _plain_norm(st):
    case = st["case"]
    u = _plain_normed(st["o"].float(), st["w"][0], st["b"][0], case["kind"])
    if st["gate"] is not None:
        gate = st["gate"].float()
        if case["act"] == "sigmoid":
            gate = 1.0 / (1.0 + torch.exp(-gate))
        elif case["act"] == "silu":
            gate = gate / (1.0 + torch.exp(-gate))
        u = u * gate.repeat_interleave(st["gate_rows"], 0)[: case["rows"]]
    y = 0.9375 * st["x"].float() + 0.5 * u
    return y.to(st["x"].dtype), _plain_normed(y, st["w"][1], st["b"][1], case["kind"]).to(st["h"].dtype)


_PLAIN = {"attend": _plain_attend, "weights": _plain_weights, "append": _plain_append, "evict": _plain_evict, "norm": _plain_norm}


def run(st):
    if not own:
        return _PLAIN[st["op"]](st)
    from paper_2504_14152_amd import fgmp
    op, case = st["op"], st["case"]
    if op == "attend":
        return fgmp.tree_attention(st["q"], st["new_k"], st["new_v"], st["cache"], tree=st["tree"], counts=st["counts"], scale=st["scale"],
                                   max_length=case["length"], out=st["out"], lse=st["lse"], workspace=st["workspace"])
    if op == "weights":
        return fgmp.attention_weights(st["q"], st["lse"], st["cache"], st["have"], rows=st["rows"], counts=st["counts"], scale=st["scale"],
                                      max_length=case["length"], out=st["out"])
    if op == "append":
        lengths = fgmp.cache_append(st["new_k"], st["new_v"], st["cache"], rows=st["rows"], counts=st["counts"], positions=st["positions"],
                                    slot_positions=st["slot_positions"], slot_weights=st["slot_weights"], lengths_out=st["lengths_out"])
        return st["k"], st["v"], st["slot_positions"], st["slot_weights"], lengths
    if op == "evict":
        w, p, lengths = fgmp.cache_evict(st["cache"], st["weights"], st["positions"], st["seen"], case["budget"], sinks=case["sinks"],
                                         recent=case["recent"], weights_out=st["weights_out"], positions_out=st["positions_out"],
                                         lengths_out=st["lengths_out"], workspace=st["workspace"])
        return st["k"], st["v"], w, p, lengths
    return fgmp.block_norm(st["x"], st["o"], post_weight=st["w"][0], post_bias=st["b"][0], pre_weight=st["w"][1], pre_bias=st["b"][1],
                           gate=st["gate"], gate_act=case["act"], gate_rows=st["gate_rows"], kind=case["kind"], eps=1e-5,
                           residual_scale=0.9375, branch_scale=0.5, out=st["y"], h=st["h"])


# ---- what a pass cannot do without ----

def work(case):
    op = case["op"]
    if op == "norm":
        M, K = case["rows"], case["width"]
        gate_rows = {"none": 0, "channel": 1, "group": -(-M // max(1, min(M, 64))), "full": M}[case["gate"]]
        size = M * (2 * _SIZE[case["stream"]] + _SIZE[case["block"]] + _SIZE[case["out"]]) + gate_rows * _SIZE[case["block"]]
        return {"bytes": float(K) * (size + 8 + 8 * case["bias"]), "flops": 16.0 * M * K}
    entry = case["kv_heads"] * case["dim"] * _SIZE[case["dtype"]]
    lengths = _lengths(case)
    if op == "attend":
        counts = _counts(case)
        drafted = sum(counts)
        size = 2.0 * entry * (sum(lengths) + drafted) + drafted * case["heads"] * (2 * case["dim"] * _SIZE[case["dtype"]] + 4)
        pairs = sum(c * n + (0 if case["tree"] else c * (c + 1) // 2) for c, n in zip(counts, lengths))
        return {"bytes": size, "flops": 4.0 * case["dim"] * case["heads"] * pairs}
    if op == "weights":
        counts = _counts(case)
        size = entry * sum(lengths) + 8.0 * case["kv_heads"] * sum(lengths) + sum(counts) * case["heads"] * (case["dim"] * _SIZE[case["dtype"]] + 4)
        return {"bytes": float(size), "flops": 2.0 * case["dim"] * case["heads"] * sum(c * n for c, n in zip(counts, lengths))}
    if op == "append":
        rows = sum(_counts(case))
        source = case["kv_heads"] * case["dim"] * _SIZE[case["source"]]
        return {"bytes": rows * (2.0 * (entry + source) + 8.0 * case["kv_heads"] + 4) + 12.0 * case["batch"], "flops": 0.0}
    # every head's weights and positions are read; what is kept is written, and entries move that are kept from
    # behind the budget: as many, to a good estimate, as there would be if all slots were kept alike
    size = 0.0
    for n in lengths:
        keep = min(n, case["budget"])
        moved = (n - keep) * keep / max(1, n)
        size += case["kv_heads"] * (8.0 * n + 8.0 * keep + moved * 4 * case["dim"] * _SIZE[case["dtype"]])
    return {"bytes": size, "flops": 4.0 * case["kv_heads"] * sum(lengths)}


# ---- the same in 64 bits, from the definitions ----

def _sequence(st, pages, b, n):
    """The first n slots of sequence b: n x heads x dim."""
    page = pages.shape[1]
    if st["table"] is None:
        return pages[b, :n].double()
    each = st["table"][b].long()[: -(-n // page)]
    return pages[each].reshape(-1, *pages.shape[2:])[:n].double()


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        x, o = st["x"].double(), st["o"].double()

        def normed(z, i):
            if case["kind"] == "layer":
                z = z - z.sum(-1, keepdim=True) / case["width"]
            z = z / (z.pow(2).sum(-1, keepdim=True) / case["width"] + 1e-5).sqrt() * st["w"][i].double()
            return z if st["b"][i] is None else z + st["b"][i].double()

        u = normed(o, 0)
        if st["gate"] is not None:
            gate = st["gate"].double()[torch.arange(case["rows"], device="cuda") // st["gate_rows"]]
            u = u * {"none": gate, "sigmoid": torch.sigmoid(gate), "silu": gate * torch.sigmoid(gate)}[case["act"]]
        y = 0.9375 * x + 0.5 * u
        return y, normed(y, 1)
    lengths = _lengths(case)
    B, H, D = case["batch"], case["kv_heads"], case["dim"]
    if op in ("attend", "weights"):
        counts, group = _counts(case), case["heads"] // H
    if op == "attend":
        out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.full(out.shape[:3], -math.inf, dtype=torch.float64, device="cuda")
        words = None if st["tree"] is None else st["tree"].cpu().tolist()
        for b in range(B):
            n, c = lengths[b], counts[b]
            k = torch.cat([_sequence(st, st["k"], b, n), st["new_k"][b, :c].double()])
            v = torch.cat([_sequence(st, st["v"], b, n), st["new_v"][b, :c].double()])
            hidden = torch.zeros(c, n + c, dtype=torch.bool)
            for t in range(c):
                for j in range(c):
                    hidden[t, n + j] = j > t if words is None else not (words[b][t][j // 64] >> (j % 64)) & 1
            hidden = hidden.cuda()
            for h in range(case["heads"]):
                s = torch.matmul(st["q"][b, :c, h].double(), k[:, h // group].t().contiguous()) * st["scale"]
                s[hidden] = -math.inf
                lse[b, :c, h] = torch.logsumexp(s, -1)
                out[b, :c, h] = torch.matmul(torch.softmax(s, -1), v[:, h // group].contiguous())
        return out, lse
    if op == "weights":
        out = st["out"].double()
        rows = st["rows"].cpu().tolist()
        for b in range(B):
            n, c = lengths[b], counts[b]
            k = _sequence(st, st["k"], b, n)
            out[b, :, :n] = st["have"][b, :, :n].double()
            for i in range(c):
                end, q = n - c + i + 1, st["q"][b, rows[b][i]].double()
                for h in range(case["heads"]):
                    s = torch.matmul(k[:end, h // group], q[h]) * st["scale"]
                    out[b, h // group, :end] += torch.exp(s - st["lse"][b, rows[b][i], h].double())
        return out
    if op == "append":
        # whole values and copies: one row after the other
        counts, rows = _counts(case), None if st["rows"] is None else st["rows"].cpu().tolist()
        table, page = None if st["table"] is None else st["table"].cpu().tolist(), st["k"].shape[1]
        k, v = st["k"], st["v"]
        for b in range(B):
            for i in range(counts[b]):
                slot, row = lengths[b] + i, i if rows is None else rows[b][i]
                at = b if table is None else table[b][slot // page]
                k[at, slot % page] = st["new_k"][b, row].to(k.dtype)
                v[at, slot % page] = st["new_v"][b, row].to(v.dtype)
                st["slot_positions"][b, :, slot] = st["positions"][b, row]
                st["slot_weights"][b, :, slot] = 0.0
        return k.double(), v.double(), st["slot_positions"], st["slot_weights"].double(), _int32([n + c for n, c in zip(lengths, counts)])
    table, page = None if st["table"] is None else st["table"].long().cpu(), st["k"].shape[1]
    weights, positions, seen = st["weights"].cpu(), st["positions"].cpu(), st["seen"].tolist()
    budget = case["budget"]
    w_out, p_out, kept = st["weights_out"].cpu(), st["positions_out"].cpu(), []
    for b in range(B):
        n = lengths[b]
        kept.append(min(n, budget))
        for h in range(H):
            w, p = weights[b, h, :n].tolist(), positions[b, h, :n].tolist()
            first = [i for i in range(n) if p[i] < case["sinks"] or p[i] >= seen[b] - case["recent"]]
            inside = set(first)
            others = sorted((i for i in range(n) if i not in inside), key=lambda i: -w[i])
            keep = set((first + others)[:budget]) if n > budget else set(range(n))
            holes = [i for i in range(kept[b]) if i not in keep]
            movers = sorted(i for i in keep if i >= kept[b])
            now = list(range(kept[b]))
            for to, fro in zip(holes, movers):
                now[to] = fro
            now = torch.tensor(now, dtype=torch.long)
            w_out[b, h, : kept[b]] = weights[b, h, now]
            p_out[b, h, : kept[b]] = positions[b, h, now]
            if holes:
                to, fro = torch.tensor(holes), torch.tensor(movers)
                target, source = (torch.full_like(to, b),) * 2 if table is None else (table[b, to // page], table[b, fro // page])
                to, fro, target, source = (to % page).cuda(), (fro % page).cuda(), target.cuda(), source.cuda()
                st["k"][target, to, h] = st["k"][source, fro, h]
                st["v"][target, to, h] = st["v"][source, fro, h]
    return st["k"].double(), st["v"].double(), w_out.cuda().double(), p_out.cuda(), _int32(kept)
