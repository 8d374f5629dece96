#!/usr/bin/env python
"""Lexically constrained beam search of a small random decoder whose keys and values live in a token tree.

    python examples/constrained_decode.py [--B 4] [--k 8] [--steps 24] [--shared 20] [--norm] [--keep 16] [--check]

One pass over a step is the loop a serving program runs:
    DbaStepper.step      the step over the logits: back-pointers, tokens, scores        (dba_step)
    TokenTree.advance    the tree after it: masks, slots and positions of the new tokens (dba_tree_advance)
    TokenTree.commit     tokens all open hypotheses share into the paged context         (dba_tree_commit)
    per layer            keys, values and queries rotated and stored, attention           (dba_tree_append, dba_tree_attend)
The prompt goes in as a chain of drafted tokens: row i extends row i - 1 of the same call, and the step after it accepts the
chain by advancing from its last row.
    --shared n   n tokens before every sentence, in the cache once: a tree of one sequence takes them in and settles them, and the sentences
                 read them as a prefix (dba_tree_attend_shared), their positions counting on from it (dba_tree_append_norm's offset)
    --norm       a decoder that norms queries and keys per head (dba_tree_append_norm)
    --keep n     contexts are thinned to n tokens after every step: the attention that tokens receive is added up (dba_tree_weigh), and those
                 that receive least go (dba_tree_evict)
The weights are random, so the text means nothing; with --check every open
hypothesis' logits are computed again from its whole text without a cache (with --keep every token sees there what was left for it when it came, by
layer and key head, and the weights that tokens have received are added up again)."""
from __future__ import annotations

import argparse
import math
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

PAD, BOS, EOS = 0, 1, 2


class Decoder:
    """Pre-norm transformer decoder: rotary positions, grouped key heads, two matrices to a feed-forward block."""

    def __init__(self, V, layers, heads, kv_heads, dim, seed, dtype, device="cuda", positions=512, norm=False):
        import torch
        self.torch, self.heads, self.kv_heads, self.dim, self.dtype, self.width = torch, heads, kv_heads, dim, dtype, heads * dim
        g = torch.Generator(device=device).manual_seed(seed)
        r = lambda *s: (torch.randn(*s, generator=g, device=device) / math.sqrt(s[0])).to(dtype)  # noqa: E731
        d = self.width
        self.embed, self.unembed = r(V, d) * math.sqrt(V) * 0.5, r(d, V) * 3
        self.layers = [dict(qkv=r(d, (heads + 2 * kv_heads) * dim), o=r(d, d), up=r(d, 2 * d), down=r(2 * d, d)) for _ in range(layers)]
        for w in self.layers:
            w["norm"] = tuple(1 + 0.2 * torch.randn(dim, generator=g, device=device) for _ in range(2)) + (1e-5,) if norm else None
        angle = torch.arange(positions, device=device)[:, None] * 10000.0 ** (-torch.arange(dim // 2, device=device) * 2.0 / dim)
        self.rotary = (angle.cos().float().contiguous(), angle.sin().float().contiguous())

    def _norm(self, x):
        y = x.float()
        return (y * (y.square().mean(-1, keepdim=True) + 1e-5).rsqrt()).to(self.dtype)

    def _qkv(self, w, x):
        y = (self._norm(x) @ w["qkv"]).view(x.shape[0], -1, self.dim)
        return y[:, :self.heads], y[:, self.heads:self.heads + self.kv_heads], y[:, self.heads + self.kv_heads:]

    def _after(self, w, x, attended):
        x = x + attended.reshape(x.shape[0], self.width) @ w["o"]
        return x + self.torch.nn.functional.silu(self._norm(x) @ w["up"]) @ w["down"]

    def step(self, tree, cache, table, tokens, nx, prefix=None, offset=None, weights=None):
        """Logits [B * n, V] of the tree's newest tokens [B, n]; their keys and values go into the cache.  prefix, offset: what stands before
        the sequences, and how many tokens their positions count on from.  weights: of the context tokens, by layer, added to."""
        B, n = tokens.shape
        k, v = cache
        x = self.embed[tokens.flatten().long()]
        place, position = nx["slot"].flatten(), nx["position"].flatten()
        for i, w in enumerate(self.layers):
            q, new_k, new_v = self._qkv(w, x)
            q = tree.append(new_k, new_v, k[i], v[i], table, place, position, rotary=self.rotary, q=q, norm=w["norm"], offset=offset).view(B, n, self.heads, self.dim)
            lse = None if weights is None else self.torch.empty(B, n, self.heads, dtype=self.torch.float32, device=q.device)
            args = (q, k[i], v[i], table, nx["ctx_len"])
            o = tree.attend(*args, nx["masks"], nx["top"], lse=lse) if prefix is None else tree.attend_shared(*args, prefix, nx["masks"], nx["top"], lse=lse)
            if weights is not None:
                tree.weigh(q, k[i], table, nx["ctx_len"], lse, weight=weights[i])
            x = self._after(w, x, o)
        return self._norm(x) @ self.unembed

    def whole_text(self, text, seen=None):
        """Logits after the last token of `text` (a list), computed without a cache, and its attention by layer, [heads, tokens].  seen: by layer, [kv_heads,
        tokens, tokens]: whether a token sees another (None: all up to itself)."""
        torch, n, half = self.torch, len(text), self.dim // 2
        x = self.embed[torch.tensor(text, device=self.embed.device)]
        cos, sin = self.rotary[0][:n, None], self.rotary[1][:n, None]

        def turn(y):
            y = y.float()
            a, b = y[..., :half], y[..., half:]
            return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(self.dtype)
        causal = torch.ones(n, n, dtype=torch.bool, device=x.device).tril()
        attention = []
        for i, w in enumerate(self.layers):
            q, k, v = self._qkv(w, x)
            if w["norm"] is not None:
                root = lambda y, c: y.float() * (y.float().square().mean(-1, keepdim=True) + w["norm"][2]).rsqrt() * c  # noqa: E731
                q, k = root(q, w["norm"][0]), root(k, w["norm"][1])
            q, k = turn(q).float(), turn(k).float()
            k, v = (y.repeat_interleave(self.heads // self.kv_heads, 1).float() for y in (k, v))
            sees = causal if seen is None else seen[i].repeat_interleave(self.heads // self.kv_heads, 0)
            p = (torch.einsum("ihd,jhd->hij", q, k) * self.dim ** -0.5).masked_fill(~sees, -math.inf).softmax(-1)
            attention.append(p[:, -1])
            x = self._after(w, x, torch.einsum("hij,jhd->ihd", p, v).to(self.dtype))
        return (self._norm(x) @ self.unembed)[-1], attention


class Check:
    """The hypotheses' texts, what each of their tokens has seen, and what settled tokens have received: kept beside a decoding, without a cache."""

    def __init__(self, model, texts, k, before):
        self.model, self.k, self.worst, self.worst_weight = model, k, 0.0, 0.0
        self.settled = [before for _ in texts]             # tokens of a sequence that are no longer in the tree, those before all sentences among them
        each = lambda x: [[[list(x) for _ in range(model.kv_heads)] for _ in texts] for _ in model.layers]  # noqa: E731
        self.before, self.context, self.received = before, each(()), each(())       # by layer, sequence and key head: context places' tokens, and their weights
        # a text, and by token, layer and key head what it has seen (None: all before it)
        self.lines = [[(text, [None] * len(text))] * k for text in texts]

    def step(self, nx, backptr, tokens, offset):
        """The texts after a step, and what has settled by it."""
        self.open = (nx["position"] >= 0).tolist()
        position, n, new = nx["position"].tolist(), nx["commit_n"].tolist(), []
        for b, count in enumerate(n):
            for layer in range(len(self.model.layers)):
                for h in range(self.model.kv_heads):
                    self.context[layer][b][h] += range(self.settled[b], self.settled[b] + count)
                    self.received[layer][b][h] += [0.0] * count
            self.settled[b] += count
            new.append([])
            for j in range(self.k):
                text, seen = self.lines[b][backptr[b][j]]
                if not self.open[b][j]:
                    new[b].append(([], []))
                    continue
                text = text + [tokens[b][j]]
                assert position[b][j] + offset[b] == len(text) - 1
                own = list(range(self.settled[b], len(text)))
                sees = [[list(range(self.before)) + at[b][h] + own for h in range(self.model.kv_heads)] for at in self.context]
                new[b].append((text, seen + [sees]))
        self.lines = new

    def logits(self, logits, weights):
        """The step's logits [B, k, V] and, where contexts are thinned, the weights by layer, against those of whole texts."""
        torch, K = self.model.torch, self.model.kv_heads
        for b, lines in enumerate(self.lines):
            for j, (text, rows) in enumerate(lines):
                if not self.open[b][j]:
                    continue
                seen = None
                if weights is not None:
                    seen = torch.ones(len(self.model.layers), K, len(text), len(text), dtype=torch.bool).tril()
                    for i, row in enumerate(rows):
                        for layer, h in [] if row is None else [(x, h) for x in range(len(row)) for h in range(K)]:
                            seen[layer, h, i] = False
                            seen[layer, h, i, row[layer][h]] = True
                    seen = seen.to(logits.device)
                want, attention = self.model.whole_text(text, seen)
                self.worst = max(self.worst, float((logits[b, j].float() - want.float()).abs().max()))
                for layer, p in enumerate(attention if weights is not None else []):
                    p = p.view(K, -1, len(text)).sum(1).tolist()
                    for h in range(K):
                        self.received[layer][b][h] = [x + p[h][at] for x, at in zip(self.received[layer][b][h], self.context[layer][b][h])]
        if weights is not None:
            got = weights.tolist()
            for layer, by_sequence in enumerate(self.received):
                for b, by_head in enumerate(by_sequence):
                    for h, row in enumerate(by_head):
                        self.worst_weight = max([self.worst_weight] + [abs(x - y) / (1 + y) for x, y in zip(got[layer][b][h], row)])

    def evicted(self, kept):
        """kept [layers, B, kv_heads, keep]: the context places that stay."""
        for layer, by_sequence in enumerate(kept.tolist()):
            for b, by_head in enumerate(by_sequence):
                for h, places in enumerate(by_head):
                    for rows in (self.context, self.received):
                        rows[layer][b][h] = [rows[layer][b][h][p] for p in places if p >= 0]


def take_in(dba, model, cache, pages, tokens, page_size, heads, kv_heads, dim, code):
    """The tokens that stand before all sentences, through a tree of one sequence: a chain, settled and committed.  Returns the prefix' pages."""
    import torch
    n, words = len(tokens), (len(tokens) + 32) // 32
    while 32 * words % page_size:          # the context begins with a page
        words += 1
    tree = dba.TokenTree(1, n, heads, kv_heads, dim, page_size, pages.numel(), words, dtype=code)
    z = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    table, slot_pos = pages.view(1, -1), z(1, 32 * words)
    nx = tree.advance(torch.arange(n, dtype=torch.int32, device="cuda").view(1, n), z(1, 1, words), slot_pos, z(1))
    model.step(tree, cache, table, torch.tensor([tokens], dtype=torch.int32, device="cuda"), nx)
    nx = tree.advance(torch.tensor([[n - 1]], dtype=torch.int32, device="cuda"), nx["masks"], slot_pos, nx["ctx_len"])       # all of the chain settles
    tree.commit(*cache, table, nx["ctx_len"], nx["commit_src"], nx["commit_n"])
    if tree.status():
        raise RuntimeError("token tree: the prefix did not settle")
    return table[:, 32 * words // page_size:].contiguous()


def decode(B=4, k=8, steps=24, prompt=12, V=997, layers=2, heads=8, kv_heads=2, dim=64, page_size=16, words=8, dtype="bf16", seed=0, check=False,
           shared=0, norm=False, keep=0):
    """Returns (tokens, lengths, scores, flags) of dba_finalize, the largest difference of a logit from the one computed without
    a cache (check) and what fell on the way: settled and evicted tokens, the highest slot, the largest difference of a token's weight (over 1 + weight)."""
    import torch
    import paper_1804_06609_b200 as dba
    g = torch.Generator().manual_seed(seed)
    code, tdt = (dba.BF16, torch.bfloat16) if dtype == "bf16" else (dba.F32, torch.float32)
    model = Decoder(V, layers, heads, kv_heads, dim, seed, tdt, norm=norm)
    constraints = [[[int(torch.randint(4, V, (1,), generator=g)) for _ in range(1 + b % 2)] for _ in range(b % 3)] for b in range(B)]
    texts = torch.cat([torch.full((B, 1), BOS), torch.randint(4, V, (B, prompt - 1), generator=g)], 1).int().cuda()
    per = (32 * words + prompt + steps) // page_size + 1
    rows = max(k, prompt)
    tree = dba.TokenTree(B, rows, heads, kv_heads, dim, page_size, per, words, dtype=code, prefixes=1 if shared else 0)
    stepper = dba.DbaStepper(B, k, V, steps, constraints=constraints, dtype=code, pad=PAD, bos=BOS, eos=EOS)
    before, more = torch.randint(4, V, (shared,), generator=g).tolist(), -(-(2 * shared + 33 + 32 * page_size) // page_size) if shared else 0
    shape = (layers, B * per + more, page_size, kv_heads, dim)
    cache = tuple(torch.empty(shape, dtype=tdt, device="cuda") for _ in range(2))
    table = torch.arange(B * per, dtype=torch.int32, device="cuda").view(B, per)
    prefix = offset = weights = None
    if shared:
        pages = take_in(dba, model, cache, torch.arange(B * per, B * per + more, dtype=torch.int32, device="cuda"), before, page_size, heads, kv_heads, dim, code)
        ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        prefix = (ints(0, B), ints(shared), pages)
    if shared or keep:
        offset = torch.full((B,), shared, dtype=torch.int32, device="cuda")
    if keep:
        weights = torch.zeros(layers, B, kv_heads, per * page_size - 32 * words, device="cuda")
    slot_pos = torch.zeros(B, 32 * words, dtype=torch.int32, device="cuda")

    # the prompt: a chain from the sequence's start
    chain = torch.arange(prompt, dtype=torch.int32, device="cuda").expand(B, prompt).contiguous()       # row i extends new row i - 1
    nx = tree.advance(chain, torch.zeros(B, 1, words, dtype=torch.int32, device="cuda"), slot_pos, torch.zeros(B, dtype=torch.int32, device="cuda"))
    chain_logits = model.step(tree, cache, table, texts, nx, prefix, offset).view(B, prompt, V)
    logits = torch.zeros(B, k, V, dtype=tdt, device="cuda")
    logits[:, 0] = chain_logits[:, -1]                       # the beam's one live hypothesis
    settled, top, evicted = 0, 0, 0
    checked = Check(model, [before + t for t in texts.tolist()], k, shared) if check else None
    for step in range(steps):
        out = stepper.step(logits.view(B * k, V).contiguous())
        backptr = out["backptr"].view(B, k)
        if step == 0:
            backptr = torch.where(backptr >= 0, backptr + (prompt - 1), backptr)      # slot 0 of the beam is the chain's last row
        nx = tree.advance(backptr, nx["masks"], slot_pos, nx["ctx_len"], score=out["score"], token=out["token"], eos=EOS)
        tree.commit(*cache, table, nx["ctx_len"], nx["commit_src"], nx["commit_n"])
        tokens = out["token"].view(B, k)
        logits = model.step(tree, cache, table, tokens, nx, prefix, offset, weights).view(B, k, V)
        if check:
            checked.step(nx, out["backptr"].view(B, k).tolist(), tokens.tolist(), [0] * B if offset is None else offset.tolist())
            checked.logits(logits, weights)
            settled, top = settled + int(nx["commit_n"].sum()), max(top, int(nx["top"].max()))
        if keep:             # (the last quarter stays whatever it receives)
            got = tree.evict(*cache, table, nx["ctx_len"], weights, keep, recent=(keep + 3) // 4, slot_pos=slot_pos)
            nx["ctx_len"] = got["ctx_len"]
            offset += got["dropped"]
            evicted += int(got["dropped"].sum())
            if check:
                checked.evicted(got["kept"])
    result = stepper.finalize()
    bits = tree.status()
    if bits:
        raise RuntimeError(f"token tree: status {bits}")
    worst, worst_weight = (checked.worst, checked.worst_weight) if check else (0.0, 0.0)
    return result, worst, dict(settled=settled, top=top, evicted=evicted, context=nx["ctx_len"].tolist(), constraints=constraints, worst_weight=worst_weight)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("B", 4), ("k", 8), ("steps", 24), ("prompt", 12)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    for name in ("shared", "keep"):
        ap.add_argument("--" + name, type=int, default=0)
    for name in ("check", "norm"):
        ap.add_argument("--" + name, action="store_true")
    a = ap.parse_args()
    (tokens, length, score, flags), worst, info = decode(a.B, a.k, a.steps, a.prompt, dtype=a.dtype, check=a.check, shared=a.shared, norm=a.norm, keep=a.keep)
    for b in range(a.B):
        print(f"sentence {b}: constraints {info['constraints'][b]}, {'completed' if flags[b] & 1 else 'not completed'}, score {score[b]:.3f}: {tokens[b, :length[b]].tolist()}")
    if a.keep:
        print(f"{info['evicted']} tokens evicted, contexts of {info['context']} tokens are left")
    if a.check:
        print(f"largest difference of a logit from the whole text's: {worst:.3g}; {info['settled']} tokens settled, highest slot {info['top']}"
              + (f"; of a token's weight: {info['worst_weight']:.3g}" if a.keep else ""))


if __name__ == "__main__":
    main()
