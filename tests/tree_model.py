"""Plain models of the token tree, in 64 bits and one sequence, row and slot at a time: what the tests compare with."""
import numpy as np
import torch


def bits_of(words):
    """int32 words [W] -> list of set bits."""
    return [32 * w + j for w, x in enumerate(np.asarray(words, np.int32).view(np.uint32).tolist()) for j in range(32) if x >> j & 1]


def words_of(bits, W):
    out = np.zeros(W, np.uint32)
    for b in bits:
        out[b >> 5] |= np.uint32(1) << np.uint32(b & 31)
    return out.view(np.int32)


def attend(q, k, v, table, ctx_len, masks, scale, page_size, W, num_pages):
    """(out, lse, spread, reach) in float64 on the CPU; k, v [pages, page_size, K, D].  spread [B, n, H, D] = sum p |v| and
    reach [B, n, H] = the largest scale * sum |q||k| over what the row sees: what an error bound is made of."""
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    B, n, H, D = q.shape
    K = k.shape[2]
    out, spread = torch.zeros_like(q), torch.zeros_like(q)
    lse, reach = torch.full((B, n, H), -np.inf, dtype=torch.float64), torch.zeros(B, n, H, dtype=torch.float64)
    A = 32 * W
    table = table.cpu().numpy()
    cap = table.shape[1] * page_size - A
    for b in range(B):
        ctx = min(max(int(ctx_len[b]), 0), cap)
        for i in range(n):
            places = list(range(A, A + ctx))
            if masks is not None:
                own = bits_of(masks[b, i].cpu().numpy())
                places = own + places if own else []
            at = [(int(table[b, p // page_size]), p % page_size) for p in places]
            at = [(pg, r) for pg, r in at if 0 <= pg < num_pages]
            if not at:
                continue
            pg, r = torch.tensor([x[0] for x in at]), torch.tensor([x[1] for x in at])
            for h in range(H):
                kk, vv = k[pg, r, h // (H // K)], v[pg, r, h // (H // K)]
                s = (kk @ q[b, i, h]) * scale
                p = torch.softmax(s, 0)
                out[b, i, h] = p @ vv
                spread[b, i, h] = p @ vv.abs()
                lse[b, i, h] = torch.logsumexp(s, 0)
                reach[b, i, h] = (kk.abs() @ q[b, i, h].abs()).max() * abs(scale)
    return out, lse, spread, reach


def attend_tolerance(out, spread, reach, D, seen, dtype):
    """Bound on |computed - exact|.  fp32: a score is a sum of D products (each partial sum rounded: D 2^-24 of sum |q||k|),
    its error e moves a probability by a factor of at most exp(2 e); exponentials and the sums over `seen` places
    add (seen + 16) 2^-23.  bf16: the same, and the probabilities and the output are rounded to 8 bits (2^-8 of each)."""
    e = reach * (D + 4) * 2.0 ** -24
    rel = (2 * e + (seen + 16) * 2.0 ** -23)[..., None] * spread
    return rel * 1.1 + 1e-30 if dtype == torch.float32 else rel * 1.1 + 2.0 ** -8 * (spread + out.abs()) * 1.02 + 1e-30


def advance(masks, slot_pos, ctx_len, backptr, score, token, eos, capacity):
    """One sequence.  masks: list of sets; returns a dict and the flags (arena_full, no_room)."""
    n_in, n, A = len(masks), len(backptr), len(slot_pos)
    slot_pos = list(slot_pos)
    is_open, past, chain = [False] * n, [set() for _ in range(n)], [[] for _ in range(n)]
    for j, bp in enumerate(backptr):
        ok = 0 <= bp < n_in + j
        if score is not None and not score[j] > -np.inf:
            ok = False
        if token is not None and token[j] == eos:
            ok = False
        if ok and bp >= n_in:
            up = bp - n_in
            ok = is_open[up]
            if ok:
                past[j], chain[j] = past[up], chain[up] + [up]
        elif ok:
            past[j] = set(masks[bp])
        is_open[j] = ok
    opens = [j for j in range(n) if is_open[j]]
    used = set().union(*[past[j] for j in opens]) if opens else set()
    settled = set.intersection(*[past[j] for j in opens]) if opens else set()
    no_room = bool(settled) and (ctx_len < 0 or ctx_len + len(settled) > capacity)
    if no_room:
        settled = set()
    free = [s for s in range(A) if s not in used]
    slot, position, out = [-1] * n, [-1] * n, [set() for _ in range(n)]
    for r, j in enumerate(opens):
        if r < len(free):
            slot[j] = free[r]
        position[j] = ctx_len + len(past[j]) + len(chain[j])
    order = sorted(settled, key=lambda s: (slot_pos[s], s))
    for j in opens:
        if slot[j] >= 0:
            slot_pos[slot[j]] = position[j]
        out[j] = (past[j] - settled) | {slot[c] for c in chain[j] + [j] if slot[c] >= 0}
    top = max((s + 1 for o in out for s in o), default=0)
    return dict(masks=out, slot=slot, position=position, slot_pos=slot_pos, ctx_len=ctx_len + len(settled), top=top,
                commit_src=order), (len(opens) > len(free), no_room)


def rotate(x, cos, sin, pairs):
    """x [N, heads, D] float64; cos, sin [N, rot / 2] float64."""
    y = x.clone()
    half = cos.shape[1]
    for d in range(half):
        a, b = (2 * d, 2 * d + 1) if pairs else (d, d + half)
        c, s = cos[:, None, d], sin[:, None, d]
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y
