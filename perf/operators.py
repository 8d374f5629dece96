"""What the token-tree operators are measured on: attention over the paged cache and the arena, appending to it, the
re-ordering of the tree after a step of the beam, and the copying of settled tokens into the context.

`run` computes an operator in elementary torch operations where `own` is false, and calls the framework where it is true."""
import math

import torch

own = False

# ------------------------------------------------------------------------------------------------ cases
# An arena of 32 * words slots per sequence; `rows` hypotheses or drafted tokens per sequence; `ctx` the longest
# context of the batch, the others down to (1 - ragged) of it; `steps` steps of a beam before the measured call (0: one
# drafted tree instead, each token's parent drawn among the earlier ones).


def _attend(name, B, rows, heads, kv_heads, dim, ctx, ragged, page, words, steps, dtype="bf16", hnd=False):
    return dict(name=name, op="attend", B=B, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, ctx=ctx, ragged=ragged,
                page=page, words=words, steps=steps, dtype=dtype, hnd=hnd)


def _append(name, B, rows, heads, kv_heads, dim, rot, pairs, page, words, ctx, dtype="bf16", hnd=False):
    return dict(name=name, op="append", B=B, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, rot=rot, pairs=pairs,
                page=page, words=words, ctx=ctx, dtype=dtype, hnd=hnd)


def _advance(name, B, rows, words, steps, draft=False):
    return dict(name=name, op="advance", B=B, rows=rows, words=words, steps=steps, draft=draft)


def _commit(name, B, layers, kv_heads, dim, most, page, words, ctx, dtype="bf16", hnd=False):
    return dict(name=name, op="commit", B=B, layers=layers, kv_heads=kv_heads, dim=dim, most=most, page=page, words=words,
                ctx=ctx, dtype=dtype, hnd=hnd)


def listed():
    return [
        # one sentence, one hypothesis, its first tokens: what a call costs when there is next to nothing to do
        _attend("attend_one_token", 1, 1, 16, 16, 64, 37, 0.0, 16, 1, 1),
        # translation at serving size: 256 sentences, a beam of 20, hidden size 1024; sources of 30 to 120 tokens
        _attend("attend_serving_beam", 256, 20, 16, 16, 64, 120, 0.75, 16, 8, 40),
        # a beam over prompts of up to 4100 tokens, four query heads to a key head, heads outside tokens within a page
        _attend("attend_grouped_beam", 16, 20, 32, 8, 128, 4100, 0.5, 64, 8, 30, "bf16", True),
        # a tree of 61 drafted tokens to verify in one pass over 8189 tokens of context
        _attend("attend_drafted_tree", 8, 61, 32, 8, 128, 8189, 0.3, 16, 2, 0),
        # four long documents, one token each: the cache is read once and nothing else counts
        _attend("attend_long_context", 4, 1, 32, 4, 128, 131071, 0.1, 64, 1, 1),
        # the framework's fp32 side: beams of 20 on 16 sentences
        _attend("attend_fp32_beam", 16, 20, 16, 16, 64, 1000, 0.5, 16, 8, 30, "f32"),
        # one step's tokens: a beam of 20 on 16 sentences, queries and keys rotated, keys and values into their slots
        _append("append_step", 16, 20, 32, 8, 128, 128, False, 16, 8, 500),
        # prompts of 2039 tokens come in at once
        _append("append_prompt", 8, 2039, 32, 8, 128, 128, False, 64, 8, 2039),
        # the tree after one step: the smallest workload, and the serving one
        _advance("advance_tiny", 1, 5, 2, 12),
        _advance("advance_serving", 256, 20, 16, 40),
        # settled tokens of one step into the context of every layer
        _commit("commit_step", 16, 32, 8, 128, 2, 64, 8, 500),
        _commit("commit_serving", 64, 6, 16, 64, 9, 16, 8, 120),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(16, 16, 64), (32, 8, 128), (8, 8, 64), (32, 4, 128), (12, 4, 80), (6, 6, 96), (40, 8, 128), (8, 1, 128), (14, 2, 64)]
_PAGES = [1, 5, 16, 16, 24, 32, 64, 128]


def draw(rng):
    while True:
        op = rng.choice(["attend", "attend", "attend", "append", "advance", "commit"])
        heads, kv_heads, dim = rng.choice(_HEADS)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        hnd, page, words = rng.random() < 0.5, rng.choice(_PAGES), rng.choice([1, 2, 3, 8, 13])
        B, rows = _spread(rng, 1, 256), _spread(rng, 1, 64)
        if op == "attend":
            steps = rng.choice([0, rng.randint(1, 40)])
            words = max(words, (rows * (2 if steps else 1) + 31) // 32)
            case = _attend("", B, rows, heads, kv_heads, dim, _spread(rng, 1, 131071), round(rng.random(), 2), page, words,
                           steps, dtype, hnd)
            w = work(case)
            if w["bytes"] > 1.0e9 or w["flops"] > (6e10 if dtype == "bf16" else 5e9) or B * rows * heads * (32 * words + case["ctx"]) > 1.3e8:
                continue
        elif op == "append":
            rows = _spread(rng, 1, 2039)
            rot = dim if rng.random() < 0.7 else dim // 2
            case = _append("", B, rows, heads, kv_heads, dim, rot, rng.random() < 0.4, page, words, rows + rng.randint(0, 300),
                           dtype, hnd)
            if work(case)["bytes"] > 6e8:
                continue
        elif op == "advance":
            case = _advance("", B, rows, rng.choice([2, 3, 8, 16, 31]), rng.randint(1, 40), rng.random() < 0.3)
            if case["draft"] and rows > 32 * case["words"]:
                continue
        else:
            case = _commit("", B, rng.randint(1, 32), kv_heads, dim, rng.randint(1, 12), page, words, _spread(rng, 12, 500),
                           dtype, hnd)
            if B * case["layers"] * kv_heads * dim * (32 * words + case["ctx"] + page) > 4e8:
                continue
        del case["name"]
        return case


# ------------------------------------------------------------------------------------------------ sizes
def _es(case):
    return 2 if case["dtype"] == "bf16" else 4


def _lens(case):
    """Context lengths: spread over [ctx (1 - ragged), ctx] without regard to the seed, the first the longest."""
    return [max(0, int(case["ctx"] * (1.0 - case.get("ragged", 0.0) * ((b * 0.6180339887) % 1.0)))) for b in range(case["B"])]


def _counts(case):
    """Settled tokens of each sequence of a commit: 0 to most."""
    return [min((b * 7 + case["most"]) % (case["most"] + 1), 32 * case["words"], case["ctx"]) for b in range(case["B"])]


def _capacity(case):
    places = 32 * case["words"] + case["ctx"]
    return (places + case["page"] - 1) // case["page"]


def work(case):
    op, B = case["op"], case["B"]
    if op == "attend":
        es, H, K, D, n = _es(case), case["heads"], case["kv_heads"], case["dim"], case["rows"]
        tokens = sum(_lens(case)) + B          # of the tree, at least one token
        return {"bytes": tokens * 2 * K * D * es + 2 * B * n * H * D * es + B * n * case["words"] * 4,
                "flops": 4 * n * H * D * tokens}
    if op == "append":
        N = B * case["rows"]
        return {"bytes": 2 * N * (case["heads"] + 2 * case["kv_heads"]) * case["dim"] * _es(case) + min(N, case["ctx"] + 1) * case["rot"] * 4,
                "flops": 3 * N * (case["heads"] + case["kv_heads"]) * case["rot"]}
    if op == "advance":
        n, W = case["rows"], case["words"]
        return {"bytes": B * (2 * n * W * 4 + 5 * n * 4 + 3 * 32 * W * 4), "flops": 4 * B * n * W}
    return {"bytes": 4 * sum(_counts(case)) * case["layers"] * case["kv_heads"] * case["dim"] * _es(case), "flops": 0}


# ------------------------------------------------------------------------------------------------ plain forms
def _unpack(masks):
    """[..., W] words to [..., 32 W] bits."""
    bits = (masks.unsqueeze(-1) >> torch.arange(32, device=masks.device, dtype=torch.int32)) & 1
    return bits.flatten(-2).bool()


def _pack(bits):
    w = bits.unflatten(-1, (-1, 32)).long() << torch.arange(32, device=bits.device)
    s = w.sum(-1)
    return torch.where(s >= 1 << 31, s - (1 << 32), s).int()


def _rows_of(table, place, page):
    """The cache's rows (page * rows to a page + row in it) of places [B, P] of the sequences."""
    return torch.gather(table.long(), 1, place // page) * page + place % page


def _plain_attend(s):
    q, table, page = s["q"], s["table"], s["page"]
    B, n, H, D = q.shape
    K, arena, P = s["k"].shape[2], 32 * s["masks"].shape[2], table.shape[1] * page
    place = torch.arange(P, device=q.device).expand(B, P)
    at = _rows_of(table, place, page)
    k = s["k"][at // page, at % page].float().permute(0, 2, 3, 1)            # [B, K, D, P]
    v = s["v"][at // page, at % page].float().permute(0, 2, 1, 3)            # [B, K, P, D]
    bits = _unpack(s["masks"])                                              # [B, n, arena]
    ctx = (place[:, None, arena:] - arena < s["ctx_len"][:, None, None]) & bits.any(-1, keepdim=True)
    seen = torch.cat([bits, ctx], -1)[:, None, :, None]                       # [B, 1, n, 1, P]
    qg = q.float().view(B, n, K, H // K, D).permute(0, 2, 1, 3, 4)            # [B, K, n, G, D]
    x = (qg.reshape(B, K, -1, D) @ k).view(B, K, n, H // K, P) * s["scale"]
    x = x.masked_fill(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top.masked_fill(top == -math.inf, 0.0))
    total = e.sum(-1, keepdim=True)
    v = v.masked_fill(~seen.any(2).any(2)[..., None], 0.0)
    o = (e.reshape(B, K, -1, P) @ v).view(B, K, n, H // K, D) / total.masked_fill(total == 0, 1.0)
    return o.permute(0, 2, 1, 3, 4).reshape(B, n, H, D).to(q.dtype)


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
    page = s["page"]
    cos, sin = s["cos"][s["position"].long()][:, None], s["sin"][s["position"].long()][:, None]
    q = _rotate(s["q"].float(), cos, sin, s["rot"], s["pairs"]).to(s["q"].dtype)
    k = _rotate(s["new_k"].float(), cos, sin, s["rot"], s["pairs"]).to(s["q"].dtype)
    B = s["table"].shape[0]
    at = _rows_of(s["table"], s["place"].view(B, -1).long(), page).flatten()
    s["k"][at // page, at % page] = k
    s["v"][at // page, at % page] = s["new_v"]
    return q, s["k"], s["v"]


def _plain_advance(masks, slot_pos, ctx_len, backptr, score, token, eos):
    """The tree after a step: rows' masks, new slots and positions, context lengths, and the list of settled slots."""
    B, n_in, W = masks.shape
    n, A = backptr.shape[1], 32 * W
    dev = masks.device
    bits = _unpack(masks)
    is_open = backptr >= 0
    if score is not None:
        is_open = is_open & (score > -math.inf) & (token != eos)
    # rows that extend rows of this call: their ancestors in it by squaring the parent relation (n <= 64)
    anc = (backptr[..., None] - n_in == torch.arange(n, device=dev)).float()
    hop = torch.eye(n, device=dev) + anc
    for _ in range(6):
        hop = ((hop @ hop) > 0).float()
    anc = hop - torch.eye(n, device=dev)
    is_open = is_open & ~((anc > 0) & ~is_open[:, None]).any(-1)
    root = torch.where(backptr < n_in, backptr, -1).long()
    root = torch.where(hop > 0, root[:, None], -1).amax(-1)
    base = torch.gather(bits, 1, root.clamp(0, n_in - 1)[..., None].expand(B, n, A)) & is_open[..., None]
    used = base.any(1)
    settled = (base | ~is_open[..., None]).all(1) & is_open.any(1, keepdim=True)
    # the j-th open row takes the j-th lowest free slot
    order = torch.argsort(used.to(torch.int32), dim=1, stable=True)
    free = (~used).sum(1, keepdim=True)
    place = is_open.int().cumsum(1) - 1
    has = is_open & (place < free)
    slot = torch.where(has, torch.gather(order, 1, place.clamp(0, A - 1).long()), -1)
    position = torch.where(is_open, ctx_len[:, None] + base.sum(-1) + anc.sum(-1).int(), -1)
    own_bit = (slot[..., None] == torch.arange(A, device=dev)) & has[..., None]
    chain = (anc @ own_bit.float()) > 0
    out = (base & ~settled[:, None]) | own_bit | (chain & is_open[..., None])
    pos2 = _put(slot_pos, slot, position, has)
    key = torch.where(settled, slot_pos.long() * A + torch.arange(A, device=dev), 1 << 60)
    src = torch.argsort(key, dim=1)
    count = settled.sum(1).int()
    src = torch.where(torch.arange(A, device=dev) < count[:, None], src, -1).int()
    seen = out.any(1)
    top = (seen * torch.arange(1, A + 1, device=dev)).amax(1).int()
    return {"masks": _pack(out), "slot": slot.int(), "position": position.int(), "slot_pos": pos2.int(),
            "ctx_len": ctx_len + count, "top": top, "commit_src": src, "commit_n": count}


def _put(slot_pos, slot, position, has):
    """slot_pos with the new slots' positions (slots are distinct; rows without one write past the end)."""
    wide = torch.cat([slot_pos, slot_pos.new_zeros(slot_pos.shape[0], 1)], 1)
    wide.scatter_(1, torch.where(has, slot, slot_pos.shape[1]).long(), position.to(slot_pos.dtype))
    return wide[:, :-1]


def _plain_commit(s):
    src, count, page = s["commit_src"], s["commit_n"], s["page"]
    B, A = src.shape
    i = torch.arange(s["most"], device=src.device)
    live = i < count[:, None]
    a = _rows_of(s["table"], src[:, :s["most"]].clamp(min=0).long(), page)[live]
    b = _rows_of(s["table"], ((A + s["ctx_len"] - count)[:, None] + i) * live, page)[live]
    s["k"][:, b // page, b % page] = s["k"][:, a // page, a % page]
    s["v"][:, b // page, b % page] = s["v"][:, a // page, a % page]
    return s["k"], s["v"]


# ------------------------------------------------------------------------------------------------ states
def _torch_dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _cache(case, gen, layers=None):
    """Keys and values [pages, page, kv heads, dim] and the sequences' tables: their pages lie anywhere."""
    per = _capacity(case)
    pages = case["B"] * per
    shape = (pages, case["kv_heads"], case["page"], case["dim"]) if case["hnd"] else (pages, case["page"], case["kv_heads"], case["dim"])
    if layers is not None:
        shape = (layers,) + shape
    k = torch.randn(shape, generator=gen, device="cuda", dtype=_torch_dtype(case))
    v = torch.randn(shape, generator=gen, device="cuda", dtype=_torch_dtype(case))
    if case["hnd"]:
        k, v = k.transpose(-3, -2), v.transpose(-3, -2)
    table = torch.randperm(pages, generator=gen, device="cuda").int().view(case["B"], per)
    return k, v, table


def _parents(B, n, gen, n_in):
    """Back-pointers of a beam's step: better hypotheses have more children."""
    u = torch.rand(B, n, generator=gen, device="cuda")
    return (u * u * n_in).long().clamp(max=n_in - 1).sort(1).values.int()


def _drafted(B, n, gen, n_in):
    """A drafted tree: the first token extends row 0, each other one an earlier token of the same call."""
    i = torch.arange(n, device="cuda")
    u = torch.rand(B, n, generator=gen, device="cuda")
    p = (u * i).long().clamp(min=0)
    return torch.where(i == 0, torch.zeros_like(p), n_in + torch.minimum(p, (i - 1).clamp(min=0))).int()


def _tree(case, gen, steps, ctx_len):
    """A beam's tree after some steps: the first step's rows all extend the sequence's start."""
    B, n, W = case["B"], case["rows"], case["words"]
    t = {"masks": torch.zeros(B, n, W, dtype=torch.int32, device="cuda"),
         "slot_pos": torch.zeros(B, 32 * W, dtype=torch.int32, device="cuda"), "ctx_len": ctx_len}
    for _ in range(steps):
        t = _plain_advance(t["masks"], t["slot_pos"], t["ctx_len"], _parents(B, n, gen, n), None, None, -1)
    return t


def prepare(case, seed):
    gen, op, B = _generator(seed), case["op"], case["B"]
    s = {"op": op}
    if op == "advance":
        n, W = case["rows"], case["words"]
        t = _tree(case, gen, case["steps"], torch.tensor([20 + b % 50 for b in range(B)], dtype=torch.int32, device="cuda"))
        s.update(masks=t["masks"], slot_pos=t["slot_pos"], ctx_len=t["ctx_len"], backptr=_parents(B, n, gen, n), eos=2)
        if case["draft"]:
            s.update(backptr=_drafted(B, n, gen, n), score=None, token=None)
        else:       # towards the end of a sentence some hypotheses are finished, and late slots may be empty
            s["token"] = torch.randint(4, 1000, (B, n), generator=gen, device="cuda", dtype=torch.int32)
            s["token"][torch.rand(B, n, generator=gen, device="cuda") < 0.15] = 2
            s["score"] = -torch.rand(B, n, generator=gen, device="cuda").cumsum(1)
            s["score"][torch.rand(B, n, generator=gen, device="cuda") < 0.02] = -math.inf
        shape = dict(n=n, heads=1, kv_heads=1, dim=8, page=16, pages=(32 * W + 200) // 16 + 1, words=W, dtype=torch.float32)
    else:
        s["page"] = case["page"]
        s["k"], s["v"], s["table"] = _cache(case, gen, case.get("layers"))
        A = 32 * case["words"]
        shape = dict(n=case.get("rows", 1), heads=case.get("heads", case["kv_heads"]), kv_heads=case["kv_heads"], dim=case["dim"],
                     page=case["page"], pages=s["table"].shape[1], words=case["words"], dtype=_torch_dtype(case))
        if op == "attend":
            n, H, D = case["rows"], case["heads"], case["dim"]
            ctx = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")
            t = _tree(case, gen, case["steps"], ctx)
            if case["steps"] == 0:
                t = _plain_advance(t["masks"], t["slot_pos"], ctx, _drafted(B, n, gen, n), None, None, -1)
            s.update(masks=t["masks"], top=t["top"], ctx_len=ctx, scale=D ** -0.5,
                     q=torch.randn(B, n, H, D, generator=gen, device="cuda", dtype=_torch_dtype(case)) * 1.5)
        elif op == "append":
            N, D = B * case["rows"], case["dim"]
            draw_ = lambda heads: torch.randn(N, heads, D, generator=gen, device="cuda", dtype=_torch_dtype(case))  # noqa: E731
            s.update(q=draw_(case["heads"]), new_k=draw_(case["kv_heads"]), new_v=draw_(case["kv_heads"]), rot=case["rot"], pairs=case["pairs"])
            angle = torch.arange(case["ctx"] + 1, device="cuda")[:, None] * 10000.0 ** (-torch.arange(case["rot"] // 2, device="cuda") * 2.0 / case["rot"])
            s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
            i = torch.arange(case["rows"], device="cuda").expand(B, -1)
            if case["rows"] <= A and case["rows"] <= 64:       # a step: the rows' new tokens, into the arena
                place = torch.rand(B, A, generator=gen, device="cuda").argsort(1)[:, :case["rows"]]
                position = torch.randint(0, case["ctx"] + 1, (B, 1), generator=gen, device="cuda").expand(B, case["rows"])
            else:                                             # a prompt, into the context
                place, position = A + i, i
            s["place"], s["position"] = place.flatten().int(), position.flatten().int()
        else:
            count = _counts(case)
            src = torch.rand(B, A, generator=gen, device="cuda").argsort(1).int()
            s["commit_n"] = torch.tensor(count, dtype=torch.int32, device="cuda")
            s["commit_src"] = torch.where(torch.arange(A, device="cuda") < s["commit_n"][:, None], src, -1).int()
            s["ctx_len"] = torch.full((B,), case["ctx"], dtype=torch.int32, device="cuda")
            s["most"] = max(count)
    if own:
        import paper_1804_06609_b200 as dba
        n = min(shape["n"], 64)
        s["tree"] = dba.TokenTree(B, n, shape["heads"], shape["kv_heads"], shape["dim"], shape["page"], shape["pages"], shape["words"],
                                  dtype=dba.BF16 if shape["dtype"] == torch.bfloat16 else dba.F32)
    return s


def run(s):
    op = s["op"]
    if own:
        t = s["tree"]
        if op == "attend":
            return t.attend(s["q"], s["k"], s["v"], s["table"], s["ctx_len"], masks=s["masks"], top=s["top"], scale=s["scale"])
        if op == "append":
            q = t.append(s["new_k"], s["new_v"], s["k"], s["v"], s["table"], s["place"], s["position"], rotary=(s["cos"], s["sin"]),
                         pairs=s["pairs"], q=s["q"])
            return q, s["k"], s["v"]
        if op == "advance":
            return t.advance(s["backptr"], s["masks"], s["slot_pos"], s["ctx_len"], score=s["score"], token=s["token"], eos=s["eos"])
        t.commit(s["k"], s["v"], s["table"], s["ctx_len"], s["commit_src"], s["commit_n"])
        return s["k"], s["v"]
    if op == "attend":
        return _plain_attend(s)
    if op == "append":
        return _plain_append(s)
    if op == "advance":
        return _plain_advance(s["masks"], s["slot_pos"], s["ctx_len"], s["backptr"], s["score"], s["token"], s["eos"])
    return _plain_commit(s)


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attend":
        q, page, A = s["q"].double(), s["page"], 32 * s["masks"].shape[2]
        B, n, H, D = q.shape
        group = H // s["k"].shape[2]
        out = torch.zeros_like(q)
        for b in range(B):
            length, words = int(s["ctx_len"][b]), s["masks"][b].cpu().tolist()
            rows = [[(w[j // 32] >> (j % 32)) & 1 for j in range(A)] for w in words]
            seen = torch.tensor(rows, dtype=torch.bool, device="cuda")
            live = seen.any(0).nonzero().flatten()
            place = torch.cat([live, torch.arange(A, A + length, device="cuda")])
            pages, inside = s["table"][b].long()[place // page], place % page
            can = torch.cat([seen[:, live], seen.any(1, keepdim=True).expand(n, length)], 1)
            for h in range(s["k"].shape[2]):
                k, v = s["k"][pages, inside, h].double(), s["v"][pages, inside, h].double()
                x = torch.einsum("ngd,pd->ngp", q[b, :, h * group:(h + 1) * group], k) * s["scale"]
                p = torch.softmax(x.masked_fill(~can[:, None], -math.inf), -1).nan_to_num(0.0)
                out[b, :, h * group:(h + 1) * group] = torch.einsum("ngp,pd->ngd", p, v)
        return out
    if case["op"] == "append":
        half = case["rot"] // 2
        angle_cos, angle_sin = s["cos"].double()[s["position"].long()], s["sin"].double()[s["position"].long()]

        def turn(x):
            x = x.double()
            z = x[..., :2 * half]
            z = torch.complex(z[..., 0::2], z[..., 1::2]) if case["pairs"] else torch.complex(z[..., :half], z[..., half:])
            z = z * torch.complex(angle_cos, angle_sin)[:, None]
            turned = torch.stack([z.real, z.imag], -1).flatten(-2) if case["pairs"] else torch.cat([z.real, z.imag], -1)
            return torch.cat([turned, x[..., 2 * half:]], -1)
        place = s["place"].long()
        seq = torch.arange(len(place), device="cuda") // case["rows"]
        pages, inside = s["table"].long()[seq, place // s["page"]], place % s["page"]
        k, v = s["k"].double(), s["v"].double()
        k[pages, inside], v[pages, inside] = turn(s["new_k"]), s["new_v"].double()
        return turn(s["q"]), k, v
    if case["op"] == "advance":
        return None           # whole numbers throughout
    k, v, page, A = s["k"].double(), s["v"].double(), s["page"], s["commit_src"].shape[1]
    for b, count in enumerate(s["commit_n"].tolist()):
        for i, src in enumerate(s["commit_src"][b, :count].tolist()):
            dst = A + case["ctx"] - count + i
            a, z = (s["table"][b, p // page].item() for p in (src, dst))
            for x in (k, v):
                x[:, z, dst % page] = x[:, a, src % page]
    return k, v
