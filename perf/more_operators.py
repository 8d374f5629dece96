"""What the token tree's operators for long and shared texts are measured on: attention of many sequences over a prefix that
they share, appending with norms of queries and keys, the weight that context tokens receive from attention, and the
eviction of those that receive little.

`run` computes an operator in elementary torch operations where `own` is false, and calls the framework where it is true."""
import math

import torch

own = False

# ------------------------------------------------------------------------------------------------ cases
# An arena of 32 * words slots per sequence; `rows` hypotheses per sequence; `ctx` the longest context of the batch, the
# others down to (1 - ragged) of it.  `groups` prefixes, the longest of `prefix` tokens, each shared by sequences that stand
# next to one another; the last `outside` sequences have none.  `closed`: some hypotheses are finished.


def _shared(name, B, rows, heads, kv_heads, dim, groups, prefix, ctx, ragged, page, words, dtype="bf16", hnd=False, outside=0, closed=False):
    return dict(name=name, op="shared", B=B, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, groups=groups, prefix=prefix, ctx=ctx,
                ragged=ragged, page=page, words=words, dtype=dtype, hnd=hnd, outside=outside, closed=closed)


def _append(name, B, rows, heads, kv_heads, dim, rot, pairs, page, words, ctx, dtype="bf16", hnd=False):
    return dict(name=name, op="append", B=B, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, rot=rot, pairs=pairs, page=page,
                words=words, ctx=ctx, dtype=dtype, hnd=hnd)


def _weigh(name, B, rows, heads, kv_heads, dim, ctx, ragged, page, decay, dtype="bf16", hnd=False, closed=False):
    return dict(name=name, op="weigh", B=B, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, ctx=ctx, ragged=ragged, page=page,
                words=0, decay=decay, dtype=dtype, hnd=hnd, closed=closed)


def _evict(name, B, layers, kv_heads, dim, ctx, ragged, keep, recent, page, dtype="bf16", hnd=False):
    return dict(name=name, op="evict", B=B, layers=layers, kv_heads=kv_heads, dim=dim, ctx=ctx, ragged=ragged, keep=keep, recent=recent,
                page=page, words=0, dtype=dtype, hnd=hnd)


def listed():
    return [
        # two sentences, a beam of 5, a short instruction before both: what a call costs when there is next to nothing to do
        _shared("shared_small", 2, 5, 16, 16, 64, 1, 50, 10, 0.3, 16, 1),
        # translation at serving size: 256 sentences, a beam of 20, hidden size 1024; an instruction with a few examples, 509
        # tokens, before sources of 30 to 120
        _shared("shared_serving", 256, 20, 16, 16, 64, 1, 509, 120, 0.75, 16, 8),
        # beams of 20 on 64 sentences after a document of 6007 tokens, four query heads to a key head, heads outside tokens
        # within a page, some hypotheses finished
        _shared("shared_document", 64, 20, 32, 8, 128, 1, 6007, 300, 0.5, 64, 8, "bf16", True, 0, True),
        # eight conversations, one token each, about a text of 100003 tokens: the cache is read once and nothing else counts
        _shared("shared_few_rows", 8, 1, 32, 4, 128, 1, 100003, 200, 0.4, 64, 1),
        # the framework's fp32 side: beams of 20 on 16 sentences, three prefixes, two sentences without one
        _shared("shared_fp32", 16, 20, 16, 16, 64, 3, 700, 100, 0.5, 16, 8, "f32", False, 2),
        # one step's tokens: a beam of 20 on 16 sentences, queries and keys normed and rotated, keys and values into their slots
        _append("norm_step", 16, 20, 32, 8, 128, 128, False, 16, 8, 500),
        # prompts of 2039 tokens come in at once
        _append("norm_prompt", 8, 2039, 32, 8, 128, 128, False, 64, 8, 2039),
        # a step's weights: beams of 20 on 16 prompts of up to 4100 tokens, four query heads to a key head
        _weigh("weigh_beam", 16, 20, 32, 8, 128, 4100, 0.5, 64, 1.0, "bf16", True, True),
        # four long documents, one token each: the keys are read once
        _weigh("weigh_long", 4, 1, 32, 4, 128, 131071, 0.1, 64, 1.0),
        # fp32, older weights count less
        _weigh("weigh_fp32", 8, 5, 16, 16, 64, 1000, 0.5, 16, 0.9, "f32"),
        # one layer, sources somewhat longer than what is kept
        _evict("evict_layer", 4, 1, 8, 64, 300, 0.2, 256, 32, 16),
        # a quarter is kept of documents of up to 32768 tokens, four layers at once
        _evict("evict_documents", 4, 4, 8, 128, 32768, 0.3, 8192, 1024, 64),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(16, 16, 64), (32, 8, 128), (8, 8, 64), (32, 4, 128), (12, 4, 80), (6, 6, 96), (40, 8, 128), (8, 1, 128), (14, 2, 64)]
_PAGES = [1, 5, 16, 16, 24, 32, 64, 128]


def draw(rng):
    while True:
        op = rng.choice(["shared", "shared", "append", "weigh", "evict"])
        heads, kv_heads, dim = rng.choice(_HEADS)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        hnd, page, closed = rng.random() < 0.5, rng.choice(_PAGES), rng.random() < 0.3
        B, rows, ragged = _spread(rng, 1, 256), _spread(rng, 1, 64), round(rng.random(), 2)
        if op == "shared":
            words = max(rng.choice([1, 2, 3, 8]), (rows + 31) // 32)
            case = _shared("", B, rows, heads, kv_heads, dim, min(B, _spread(rng, 1, 16)), _spread(rng, 1, 100003), _spread(rng, 1, 500),
                           ragged, page, words, dtype, hnd, rng.choice([0, 0, B // 5]), closed)
            w = work(case)
            if w["bytes"] > 6e8 or w["flops"] > (1.2e11 if dtype == "bf16" else 1e10) or B * rows * heads * (32 * words + case["ctx"]) > 1.3e8:
                continue
            if max(_members(case)) * case["groups"] * rows * heads * case["prefix"] > 2.4e8:
                continue
        elif op == "append":
            rows = _spread(rng, 1, 2039)
            rot = dim if rng.random() < 0.7 else dim // 2
            case = _append("", B, rows, heads, kv_heads, dim, rot, rng.random() < 0.4, page, rng.choice([1, 2, 8, 13]), rows + rng.randint(0, 300),
                           dtype, hnd)
            if work(case)["bytes"] > 4e8:
                continue
        elif op == "weigh":
            case = _weigh("", B, rows, heads, kv_heads, dim, _spread(rng, 1, 131071), ragged, page, rng.choice([1.0, 1.0, 0.9]), dtype, hnd, closed)
            w = work(case)
            if w["bytes"] > 5.5e8 or w["flops"] > (3e10 if dtype == "bf16" else 3e9) or B * rows * heads * case["ctx"] > 1.3e8:
                continue
        else:
            ctx = _spread(rng, 2, 32768)
            keep = max(1, int(ctx * rng.uniform(0.1, 0.95)))
            case = _evict("", _spread(rng, 1, 64), rng.randint(1, 8), kv_heads, dim, ctx, ragged, keep, int(keep * rng.uniform(0.0, 0.6)), page, dtype, hnd)
            if work(case)["bytes"] > 1.0e9 or case["B"] * case["layers"] * kv_heads * dim * (ctx + keep + 2 * page) > 6e8:
                continue
        del case["name"]
        return case


# ------------------------------------------------------------------------------------------------ sizes
def _es(case):
    return 2 if case["dtype"] == "bf16" else 4


def _ragged(most, ragged, n):
    """Lengths spread over [most (1 - ragged), most] without regard to the seed, the first the longest."""
    return [max(0, int(most * (1.0 - ragged * ((i * 0.6180339887) % 1.0)))) for i in range(n)]


def _lens(case):
    return _ragged(case["ctx"], case["ragged"], case["B"])


def _prefixes(case):
    return _ragged(case["prefix"], case["ragged"], case["groups"])


def _first(case):
    """Prefix g stands before sequences first[g] .. first[g + 1] - 1; later prefixes before more of them."""
    n, groups = case["B"] - case["outside"], case["groups"]
    return [int(n * (g / groups) ** 1.3 + 1e-9) for g in range(groups)] + [n]


def _members(case):
    first = _first(case)
    return [b - a for a, b in zip(first, first[1:])]


def _places(case):
    return 32 * case["words"] + case["ctx"]


def work(case):
    op, B = case["op"], case["B"]
    if op == "evict":
        lens = _lens(case)
        moved = sum(min(n, case["keep"]) for n in lens) * case["layers"] * case["kv_heads"]
        looked = sum(lens) * case["layers"] * case["kv_heads"]
        return {"bytes": 4 * moved * case["dim"] * _es(case) + 4 * (2 * looked + moved), "flops": 0}
    es, H, K, D, n = _es(case), case["heads"], case["kv_heads"], case["dim"], case["rows"]
    if op == "shared":
        own_tokens = sum(_lens(case)) + B          # of the tree, at least one token
        before = _prefixes(case)
        seen = own_tokens + sum(a * b for a, b in zip(before, _members(case)))
        return {"bytes": (own_tokens + sum(before)) * 2 * K * D * es + 2 * B * n * H * D * es + B * n * (4 * case["words"] + 4 * H),
                "flops": 4 * n * H * D * seen}
    if op == "append":
        N = B * n
        return {"bytes": 2 * N * (H + 2 * K) * D * es + min(N, case["ctx"] + 1) * case["rot"] * 4 + 8 * D,
                "flops": N * (H + K) * (3 * case["rot"] + 4 * D)}
    tokens = sum(_lens(case))
    return {"bytes": tokens * K * (D * es + 8) + B * n * H * (D * es + 4), "flops": 2 * n * H * D * tokens}


# ------------------------------------------------------------------------------------------------ plain forms
def _unpack(masks):
    """[..., W] words to [..., 32 W] bits."""
    return ((masks.unsqueeze(-1) >> torch.arange(32, device=masks.device, dtype=torch.int32)) & 1).flatten(-2).bool()


def _pack(bits):
    w = (bits.unflatten(-1, (-1, 32)).long() << torch.arange(32, device=bits.device)).sum(-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).int()


def _rows_of(table, place, page):
    """The cache's rows (page * rows to a page + row in it) of places [B, P] of the sequences."""
    return torch.gather(table.long(), 1, place // page) * page + place % page


def _softmax_parts(x, v):
    """Scores [.., R, P] (-inf where nothing is seen) and values [.., P, D]: (largest, sum of exponentials, their product)."""
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top.masked_fill(top == -math.inf, 0.0))
    return top, e.sum(-1, keepdim=True), e @ v


def _plain_shared(s):
    q, table, page, first = s["q"], s["table"], s["page"], s["first"]
    B, n, H, D = q.shape
    K, A = s["k"].shape[2], 32 * s["masks"].shape[2]
    qg = q.float().view(B, n, K, H // K, D).permute(0, 2, 1, 3, 4).reshape(B, K, -1, D)          # [B, K, n G, D]
    # what is a sequence's own
    place = torch.arange(table.shape[1] * page, device=q.device).expand(B, -1)
    at = _rows_of(table, place, page)
    k = s["k"][at // page, at % page].float().permute(0, 2, 3, 1)
    v = s["v"][at // page, at % page].float().permute(0, 2, 1, 3)
    bits = _unpack(s["masks"])
    is_open = bits.any(-1, keepdim=True)
    ctx = (place[:, None, A:] - A < s["ctx_len"][:, None, None]) & is_open
    seen = torch.cat([bits, ctx], -1)[:, None, :, None].expand(B, K, n, H // K, place.shape[1]).reshape(B, K, -1, place.shape[1])
    m0, l0, o0 = _softmax_parts((qg @ k * s["scale"]).masked_fill_(~seen, -math.inf), v)
    # the prefixes, each once for all of its sequences
    groups, most = first.shape[0] - 1, s["most"]
    member = first[:-1, None] + torch.arange(most, device=q.device)
    there = member < first[1:, None]
    member = member.clamp(max=B - 1)
    pplace = torch.arange(s["ptable"].shape[1] * page, device=q.device).expand(groups, -1)
    at = _rows_of(s["ptable"], pplace, page)
    k = s["k"][at // page, at % page].float().permute(0, 2, 3, 1)
    v = s["v"][at // page, at % page].float().permute(0, 2, 1, 3)
    qp = qg[member].transpose(1, 2).reshape(groups, K, -1, D)
    x = (qp @ k).mul_(s["scale"]).masked_fill_((pplace >= s["plen"][:, None])[:, None, None], -math.inf)
    back = lambda t: t.view(groups, K, most, -1, t.shape[-1]).transpose(1, 2)[there]  # noqa: E731
    m1, l1, o1 = (back(t) for t in _softmax_parts(x, v))
    put = lambda fill, t: torch.full((B,) + t.shape[1:], fill, device=q.device).index_put_((member[there],), t)  # noqa: E731
    m1, l1, o1 = put(-math.inf, m1), put(0.0, l1), put(0.0, o1)
    m = torch.maximum(m0, m1)
    ref = m.masked_fill(m == -math.inf, 0.0)
    w0, w1 = torch.exp(m0 - ref), torch.exp(m1 - ref)
    total = w0 * l0 + w1 * l1
    o = (w0 * o0 + w1 * o1) / total.masked_fill(total == 0, 1.0)
    lse = torch.log(total) + ref
    o, lse = (t.view(B, K, n, H // K, -1).permute(0, 2, 1, 3, 4).reshape(B, n, H, -1) for t in (o, lse))
    o = o.masked_fill(~is_open[..., None], 0.0).to(q.dtype)
    return o, lse[..., 0].masked_fill(~is_open, -math.inf)


def _rotate(x, cos, sin, rot, pairs):
    """x [N, heads, D] in fp32, cos / sin [N, 1, rot / 2]."""
    y = x.clone()
    if pairs:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
    return y


def _plain_append(s):
    page, B = s["page"], s["table"].shape[0]
    position = (s["position"].view(B, -1) + s["offset"][:, None]).flatten().long()
    cos, sin = s["cos"][position][:, None], s["sin"][position][:, None]

    def normed(x, w):
        x = x.float()
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + s["eps"]) * w
        return _rotate(x, cos, sin, s["rot"], s["pairs"]).to(s["q"].dtype)
    q, k = normed(s["q"], s["q_weight"]), normed(s["new_k"], s["k_weight"])
    at = _rows_of(s["table"], s["place"].view(B, -1).long(), page).flatten()
    s["k"][at // page, at % page] = k
    s["v"][at // page, at % page] = s["new_v"]
    return q, s["k"], s["v"]


def _plain_weigh(s):
    q, page = s["q"], s["page"]
    B, n, H, D = q.shape
    K, P = s["k"].shape[2], s["weight"].shape[2]
    place = torch.arange(P, device=q.device).expand(B, P)
    at = _rows_of(s["table"], place, page)
    k = s["k"][at // page, at % page].float().permute(0, 2, 3, 1)
    by_head = lambda t: t.float().view(B, n, K, H // K, -1).permute(0, 2, 1, 3, 4).reshape(B, K, n * (H // K), -1)  # noqa: E731
    lse = by_head(s["lse"][..., None])
    p = torch.exp((by_head(q) @ k) * s["scale"] - lse).masked_fill_(lse == -math.inf, 0.0)
    valid = (place < s["ctx_len"][:, None])[:, None]
    s["out"].copy_(torch.where(valid, s["weight"] * s["decay"] + p.sum(2), s["out"]))
    return s["out"]


def _plain_evict(s):
    weight, keep, recent, page = s["weight"], s["keep"], s["recent"], s["page"]
    layers, B, K, P = weight.shape
    dev = weight.device
    L = s["ctx_len"][None, :, None, None].long()
    place = torch.arange(P, device=dev)
    key = torch.where(place >= L - min(recent, keep), math.inf, weight).masked_fill(place >= L, -math.inf)
    best = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :keep]
    n = min(keep, P)
    valid = (torch.arange(n, device=dev) < L).expand(layers, B, K, n)
    best = torch.where(valid, best, P).sort(-1).values
    kept = torch.where(valid, best, -1)
    new_len = s["ctx_len"].clamp(max=keep)
    # rows of the old and of the new pages
    src, dst = best.clamp(max=P - 1), torch.arange(n, device=dev).expand_as(best)
    b = torch.arange(B, device=dev)[None, :, None, None].expand_as(best)
    l = torch.arange(layers, device=dev)[:, None, None, None].expand_as(best)
    h = torch.arange(K, device=dev)[None, None, :, None].expand_as(best)
    b, l, h, src, dst = (t[valid] for t in (b, l, h, src, dst))
    from_page, to_page = s["table"].long()[b, src // page], s["table_out"].long()[b, dst // page]
    for c in (s["k"], s["v"]):
        c[l, to_page, dst % page, h] = c[l, from_page, src % page, h]
    moved = torch.gather(weight, 3, best.clamp(max=P - 1))
    out = s["weight_out"]
    out.copy_(torch.where(place < L, 0.0, out))
    out[..., :n] = torch.where(valid, moved, out[..., :n])
    wide = torch.full((layers, B, K, keep), -1, dtype=torch.int32, device=dev)
    wide[..., :n] = kept.int()
    return {"k": s["k"], "v": s["v"], "weight": out, "kept": wide, "ctx_len": new_len, "dropped": s["ctx_len"] - new_len}


# ------------------------------------------------------------------------------------------------ states
def _torch_dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _cache(case, gen, pages, layers=None):
    """Keys and values [pages, page, kv heads, dim]."""
    shape = (pages, case["kv_heads"], case["page"], case["dim"]) if case["hnd"] else (pages, case["page"], case["kv_heads"], case["dim"])
    if layers is not None:
        shape = (layers,) + shape
    k, v = (torch.randn(shape, generator=gen, device="cuda", dtype=_torch_dtype(case)) for _ in range(2))
    return (k.transpose(-3, -2), v.transpose(-3, -2)) if case["hnd"] else (k, v)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen, op, B, page = torch.Generator(device="cuda").manual_seed(seed), case["op"], case["B"], case["page"]
    per = -(-_places(case) // page)
    K, D, dt = case["kv_heads"], case["dim"], _torch_dtype(case)
    s = {"op": op, "page": page}
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda", dtype=dt)  # noqa: E731
    uniform = lambda *shape: torch.rand(shape, generator=gen, device="cuda")  # noqa: E731
    if op != "append":
        s["ctx_len"] = _ints(_lens(case))
    if op == "evict":
        layers, keep, cap = case["layers"], case["keep"], per * page
        per_out = -(-keep // page)
        pages = B * (per + per_out)
        s["k"], s["v"] = _cache(case, gen, pages, layers)
        order = torch.randperm(pages, generator=gen, device="cuda").int()
        s["table"], fresh = order[:B * per].view(B, per), order[B * per:].view(B, per_out)
        # what is kept goes to fresh pages, and the old ones are free
        s["table_out"] = torch.cat([fresh, s["table"][:, per_out:]], 1).contiguous() if per_out < per else fresh[:, :per].contiguous()
        # few tokens receive much, many next to nothing, some nothing at all
        w = uniform(layers, B, K, cap)
        s["weight"] = (-torch.log(w.clamp(min=1e-7))).pow(3) * (uniform(layers, B, K, cap) > 0.2)
        s["weight_out"] = torch.zeros_like(s["weight"])
        s.update(keep=keep, recent=case["recent"])
    else:
        n, H = case["rows"], case["heads"]
        pre = -(-case["prefix"] // page) if op == "shared" else 0
        pages = B * per + case.get("groups", 0) * pre
        s["k"], s["v"] = _cache(case, gen, pages)
        order = torch.randperm(pages, generator=gen, device="cuda").int()
        s["table"] = order[:B * per].view(B, per)
    if op == "shared":
        groups, W = case["groups"], case["words"]
        s["ptable"] = order[B * per:].view(groups, pre)
        s["first"], s["plen"], s["most"] = _ints(_first(case)), _ints(_prefixes(case)), max(_members(case))
        # a row sees its own slot and some of the others in use
        slot = torch.arange(32 * W, device="cuda")
        bits = (uniform(B, n, 32 * W) < 0.5) & (slot < min(32 * W, 2 * n)) | (slot == torch.arange(n, device="cuda")[:, None])
        if case["closed"]:
            bits &= uniform(B, n, 1) > 0.1
        s.update(masks=_pack(bits), q=normal(B, n, H, D) * 1.5, scale=D ** -0.5, top=_ints([min(32 * W, 2 * n)] * B),
                 lse=torch.zeros(B, n, H, device="cuda"))
    elif op == "append":
        N, A = B * n, 32 * case["words"]
        s.update(q=normal(N, H, D) * 2.0, new_k=normal(N, K, D) * 3.0, new_v=normal(N, K, D), rot=case["rot"], pairs=case["pairs"], eps=1e-6)
        s["q_weight"], s["k_weight"] = 1.0 + 0.1 * normal(D).float(), 1.0 + 0.1 * normal(D).float()
        s["offset"] = torch.randint(0, 300, (B,), generator=gen, device="cuda", dtype=torch.int32)
        angle = torch.arange(case["ctx"] + 301, device="cuda")[:, None] * 10000.0 ** (-torch.arange(case["rot"] // 2, device="cuda") * 2.0 / case["rot"])
        s["cos"], s["sin"] = angle.cos().float().contiguous(), angle.sin().float().contiguous()
        i = torch.arange(n, device="cuda").expand(B, -1)
        if n <= A and n <= 64:       # a step: the rows' new tokens, into the arena
            place = uniform(B, A).argsort(1)[:, :n]
            position = torch.randint(0, case["ctx"] + 1, (B, 1), generator=gen, device="cuda").expand(B, n)
        else:                        # a prompt, into the context
            place, position = A + i, i
        s["place"], s["position"] = place.flatten().int(), position.flatten().int()
    elif op == "weigh":
        cap = per * page
        s.update(q=normal(B, n, H, D) * 1.5, scale=D ** -0.5, decay=case["decay"])
        s["weight"], s["out"] = uniform(B, K, cap).pow(4) * 5.0, torch.zeros(B, K, cap, device="cuda")
        # rows whose scores are normal have a log-sum-exp of about this
        s["lse"] = torch.log(s["ctx_len"].clamp(min=1).float())[:, None, None] + 1.1 + 0.2 * torch.randn(B, n, H, generator=gen, device="cuda")
        if case["closed"]:
            s["lse"].masked_fill_(uniform(B, n, 1) < 0.1, -math.inf)
    if own:
        import paper_1804_06609_b200 as dba
        s["tree"] = dba.TokenTree(B, min(case.get("rows", 1), 64), case.get("heads", K), K, D, page, per, case["words"],
                                  dtype=dba.BF16 if dt == torch.bfloat16 else dba.F32, prefixes=case.get("groups", 0))
    return s


def run(s):
    op = s["op"]
    if own:
        t = s["tree"]
        if op == "shared":
            out = t.attend_shared(s["q"], s["k"], s["v"], s["table"], s["ctx_len"], (s["first"], s["plen"], s["ptable"]), masks=s["masks"],
                                  top=s["top"], scale=s["scale"], lse=s["lse"])
            return out, s["lse"]
        if op == "append":
            q = t.append(s["new_k"], s["new_v"], s["k"], s["v"], s["table"], s["place"], s["position"], rotary=(s["cos"], s["sin"]),
                         pairs=s["pairs"], q=s["q"], norm=(s["q_weight"], s["k_weight"], s["eps"]), offset=s["offset"])
            return q, s["k"], s["v"]
        if op == "weigh":
            return t.weigh(s["q"], s["k"], s["table"], s["ctx_len"], s["lse"], weight=s["weight"], decay=s["decay"], scale=s["scale"], out=s["out"])
        got = t.evict(s["k"], s["v"], s["table"], s["ctx_len"], s["weight"], s["keep"], recent=s["recent"], table_out=s["table_out"],
                      weight_out=s["weight_out"])
        return {"k": s["k"], "v": s["v"], **got}
    if op == "shared":
        return _plain_shared(s)
    if op == "append":
        return _plain_append(s)
    return _plain_weigh(s) if op == "weigh" else _plain_evict(s)


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_shared(case, s):
    q, page, A, first = s["q"].double(), s["page"], 32 * s["masks"].shape[2], _first(case)
    B, n, H, D = q.shape
    K, group = s["k"].shape[2], H // s["k"].shape[2]
    out, lse = torch.zeros_like(q), torch.full((B, n, H), -math.inf, dtype=torch.float64, device="cuda")
    masks = s["masks"].cpu().tolist()
    for b in range(B):
        rows = torch.tensor([[(w[j // 32] >> (j % 32)) & 1 for j in range(A)] for w in masks[b]], dtype=torch.bool, device="cuda")
        opened = rows.any(1)
        place = torch.cat([torch.arange(A, device="cuda"), torch.arange(A, A + int(s["ctx_len"][b]), device="cuda")])
        pages, inside = s["table"][b].long()[place // page], place % page
        for g in range(len(first) - 1):
            if first[g] <= b < first[g + 1]:
                before = torch.arange(int(s["plen"][g]), device="cuda")
                pages, inside = torch.cat([pages, s["ptable"][g].long()[before // page]]), torch.cat([inside, before % page])
        can = torch.cat([rows, opened[:, None].expand(n, len(pages) - A)], 1)
        k, v = s["k"][pages, inside].double().permute(1, 2, 0), s["v"][pages, inside].double().transpose(0, 1)       # [K, D, P], [K, P, D]
        x = (q[b].view(n, K, group, D).permute(1, 0, 2, 3).reshape(K, n * group, D) @ k).view(K, n, group, -1) * s["scale"]
        x = x.masked_fill(~can[None, :, None], -math.inf)
        z = torch.logsumexp(x, -1, keepdim=True)
        p = torch.exp(x - torch.where(opened[None, :, None, None], z, 0.0)).view(K, n * group, -1)
        out[b] = (p @ v).view(K, n, group, D).permute(1, 0, 2, 3).reshape(n, H, D)
        lse[b] = z[..., 0].permute(1, 0, 2).reshape(n, H)
    return out, lse


def _exact_append(case, s):
    half = case["rot"] // 2
    position = (s["position"] + s["offset"].repeat_interleave(case["rows"])).long()
    angle = torch.complex(s["cos"].double()[position], s["sin"].double()[position])[:, None]

    def turn(x, w):
        x = x.double()
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + s["eps"]) * w.double()
        z = x[..., :2 * half]
        z = torch.complex(z[..., 0::2], z[..., 1::2]) if case["pairs"] else torch.complex(z[..., :half], z[..., half:])
        z = z * angle
        turned = torch.stack([z.real, z.imag], -1).flatten(-2) if case["pairs"] else torch.cat([z.real, z.imag], -1)
        return torch.cat([turned, x[..., 2 * half:]], -1)
    place = s["place"].long()
    seq = torch.arange(len(place), device="cuda") // case["rows"]
    pages, inside = s["table"].long()[seq, place // s["page"]], place % s["page"]
    k, v = s["k"].double(), s["v"].double()
    k[pages, inside], v[pages, inside] = turn(s["new_k"], s["k_weight"]), s["new_v"].double()
    return turn(s["q"], s["q_weight"]), k, v


def _exact_weigh(case, s):
    q, page = s["q"].double(), s["page"]
    B, n, H, D = q.shape
    K, group = s["k"].shape[2], H // s["k"].shape[2]
    out = s["out"].double()
    for b in range(B):
        L = int(s["ctx_len"][b])
        place = torch.arange(L, device="cuda")
        k = s["k"][s["table"][b].long()[place // page], place % page].double().permute(1, 2, 0)
        x = q[b].view(n, K, group, D).permute(1, 0, 2, 3).reshape(K, n * group, D) @ k * s["scale"]
        z = s["lse"][b].double().view(n, K, group).permute(1, 0, 2).reshape(K, -1, 1)
        p = torch.where(z == -math.inf, 0.0, torch.exp(x - torch.where(z == -math.inf, 0.0, z)))
        out[b, :, :L] = s["weight"][b, :, :L].double() * s["decay"] + p.sum(1)
    return out


def _exact_evict(case, s):
    k, v, out = s["k"].double(), s["v"].double(), s["weight_out"].double()
    page, keep = s["page"], case["keep"]
    new_k, new_v = k.clone(), v.clone()
    for b, L in enumerate(_lens(case)):
        r, n = min(case["recent"], keep, L), min(L, keep)
        out[:, b, :, :L] = 0.0
        for layer in range(case["layers"]):
            for h in range(case["kv_heads"]):
                w = s["weight"][layer, b, h, :L].double()
                if L > keep:
                    old = w[:L - r]
                    # the (keep - r)-th largest, everything above it, and the first ones at it
                    best = torch.zeros(0, dtype=torch.long, device="cuda")
                    if keep > r:
                        bar = torch.sort(old).values[L - r - (keep - r)]
                        above = (old > bar).nonzero().flatten()
                        best = torch.cat([above, (old == bar).nonzero().flatten()[:keep - r - len(above)]]).sort().values
                    index = torch.cat([best, torch.arange(L - r, L, device="cuda")])
                else:
                    index = torch.arange(L, device="cuda")
                to = torch.arange(n, device="cuda")
                a, z = s["table"][b].long()[index // page], s["table_out"][b].long()[to // page]
                new_k[layer, z, to % page, h], new_v[layer, z, to % page, h] = k[layer, a, index % page, h], v[layer, a, index % page, h]
                out[layer, b, h, :n] = w[index]
    return {"k": new_k, "v": new_v, "weight": out, "kept": None, "ctx_len": None, "dropped": None}


def exact(case, seed):
    if case["op"] == "shared" and work(case)["flops"] > 2e11 or case["op"] == "evict" and case["B"] * case["layers"] * case["kv_heads"] > 4000:
        return None
    s = prepare(case, seed)
    return {"shared": _exact_shared, "append": _exact_append, "weigh": _exact_weigh, "evict": _exact_evict}[case["op"]](case, s)
