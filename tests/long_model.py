"""Plain models of the token tree's operators for long and shared texts, in 64 bits on the CPU."""
import math

import torch

from tests import tree_model as M


def rows_at(table, b, places, page_size, num_pages):
    """(page, row) of the places that have a page."""
    at = [(int(table[b][p // page_size]), p % page_size) for p in places]
    return [x for x in at if 0 <= x[0] < num_pages]


def attend_shared(q, k, v, table, ctx_len, masks, scale, page_size, W, first, length, ptable):
    """As tree_model.attend with a prefix before some sequences: (out, lse, spread, reach, seen, own lse)."""
    num_pages = k.shape[0]
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    B, n, H, D = q.shape
    K = k.shape[2]
    G = H // K
    out, spread = torch.zeros_like(q), torch.zeros_like(q)
    lse, reach = torch.full((B, n, H), -math.inf, dtype=torch.float64), torch.zeros(B, n, H, dtype=torch.float64)
    seen, A, cap = torch.zeros(B, n, H, dtype=torch.float64), 32 * W, table.shape[1] * page_size - 32 * W
    table, ptable = table.cpu().tolist(), ptable.cpu().tolist()
    for b in range(B):
        before = []
        for g in range(len(length)):
            if first[g] <= b < first[g + 1]:
                before = rows_at(ptable, g, range(length[g]), page_size, num_pages)
        ctx = rows_at(table, b, range(A, A + min(max(int(ctx_len[b]), 0), cap)), page_size, num_pages)
        for i in range(n):
            at = before + ctx
            if masks is not None:
                own = M.bits_of(masks[b, i].cpu().numpy())
                at = rows_at(table, b, own, page_size, num_pages) + at if own else []
            if not at:
                continue
            pg, r = torch.tensor([x[0] for x in at]), torch.tensor([x[1] for x in at])
            kk, vv = k[pg, r].permute(1, 0, 2), v[pg, r].permute(1, 0, 2)                 # [K, P, D]
            qq = q[b, i].view(K, G, D)
            s = torch.einsum("kgd,kpd->kgp", qq, kk) * scale
            p = torch.softmax(s, -1)
            out[b, i], spread[b, i] = torch.einsum("kgp,kpd->kgd", p, vv).reshape(H, D), torch.einsum("kgp,kpd->kgd", p, vv.abs()).reshape(H, D)
            lse[b, i] = torch.logsumexp(s, -1).reshape(H)
            reach[b, i] = torch.einsum("kgd,kpd->kgp", qq.abs(), kk.abs()).amax(-1).reshape(H) * abs(scale)
            seen[b, i] = len(at)
    return out, lse, spread, reach, seen


def shared_tolerance(out, lse, spread, reach, seen, D, dtype):
    """Bounds on |computed - exact| of outputs and of log-sum-exps.  As tree_model.attend_tolerance, and what joining adds: the two parts'
    log-sum-exps are rounded (natural, to powers of two and back: 2^-23 of their size each, so as much relative in the weights), four more
    operations for a weight; bf16: the own part is rounded once more, half a unit of its share."""
    e = reach * (D + 4) * 2.0 ** -24
    size = lse.abs().nan_to_num(0, 0, 0) + reach + 8
    rel = 2 * e + (seen + 24) * 2.0 ** -23 + size * 2.0 ** -22
    tol = rel[..., None] * spread * 1.1 + 1e-30
    if dtype != torch.float32:
        tol = tol + 2.0 ** -8 * (2 * spread + out.abs()) * 1.02
    return tol, e + (seen + 40) * 2.0 ** -23 + size * 2.0 ** -22


def norm(x, weight, eps):
    x = x.double()
    return x if weight is None else x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * weight.double()


def weigh(q, k, table, ctx_len, lse, weight, decay, scale, page_size, W):
    """(new weights, bound): weights [B, K, P] of the context places, in 64 bits; places from ctx_len on are as in `weight`."""
    num_pages = k.shape[0]
    q, k, lse = q.double().cpu(), k.double().cpu(), lse.double().cpu()
    B, n, H, D = q.shape
    K = k.shape[2]
    G, A = H // K, 32 * W
    out = weight.double().cpu().clone()
    bound = torch.zeros_like(out)
    table = table.cpu().tolist()
    for b in range(B):
        L = min(max(int(ctx_len[b]), 0), len(table[b]) * page_size - A)
        if not L:
            continue
        places = [(int(table[b][p // page_size]), p % page_size) for p in range(A, A + L)]
        ok = torch.tensor([0 <= x[0] < num_pages for x in places])
        pg, r = torch.tensor([x[0] if 0 <= x[0] < num_pages else 0 for x in places]), torch.tensor([x[1] for x in places])
        kk = k[pg, r].permute(1, 0, 2)
        qq, z = q[b].view(n, K, G, D), lse[b].view(n, K, G)
        live = z > -math.inf
        qq = torch.where(live[..., None], qq, 0.0)
        s = torch.einsum("nkgd,kpd->nkgp", qq, kk) * scale
        p = torch.where(live[..., None], torch.exp(s - torch.where(live, z, 0.0)[..., None]), 0.0)
        p = torch.where(ok, p, 0.0)
        reach = torch.einsum("nkgd,kpd->nkgp", qq.abs(), kk.abs()) * abs(scale)
        # a score's D products, the rounding of lse and of the difference, the exponential
        err = 1.1 * p * (reach * (D + 4) * 2.0 ** -24 + (reach + z.abs().nan_to_num(0, 0, 0)[..., None] + 8) * 2.0 ** -22)
        bound[b, :, :L] = err.sum((0, 2)) + (out[b, :, :L].abs() * abs(decay) + p.sum((0, 2))) * (n * G + 4) * 2.0 ** -23
        out[b, :, :L] = out[b, :, :L] * decay + p.sum((0, 2))
    return out, bound + 1e-30


def keep(weight, keep, recent):
    """Which of a row of weights stay (a list of indices in order)."""
    w = [float(x) for x in weight]
    L = len(w)
    if L <= keep:
        return list(range(L))
    old = L - min(recent, keep)
    order = sorted(range(old), key=lambda i: (1, 0, i) if math.isnan(w[i]) else (0, -w[i], i))
    return sorted(order[:keep - (L - old)]) + list(range(old, L))
