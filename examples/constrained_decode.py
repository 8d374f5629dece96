#!/usr/bin/env python
"""Lexically constrained beam search of a small random decoder whose keys and values live in a token tree.

    python examples/constrained_decode.py [--B 4] [--k 8] [--steps 24] [--check]

One pass over a step is the loop a serving program runs:
    DbaStepper.step      the step over the logits: back-pointers, tokens, scores        (dba_step)
    TokenTree.advance    the tree after it: masks, slots and positions of the new tokens (dba_tree_advance)
    TokenTree.commit     tokens all open hypotheses share into the paged context         (dba_tree_commit)
    per layer            keys, values and queries rotated and stored, attention           (dba_tree_append, dba_tree_attend)
The prompt goes in as a chain of drafted tokens: row i extends row i - 1 of the same call, and the step after it accepts the
chain by advancing from its last row.  The weights are random, so the text means nothing; with --check every open
hypothesis' logits are computed again from its whole text without a cache."""
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

    def __init__(self, V, layers, heads, kv_heads, dim, seed, dtype, device="cuda", positions=512):
        import torch
        self.torch, self.heads, self.kv_heads, self.dim, self.dtype, self.width = torch, heads, kv_heads, dim, dtype, heads * dim
        g = torch.Generator(device=device).manual_seed(seed)
        r = lambda *s: (torch.randn(*s, generator=g, device=device) / math.sqrt(s[0])).to(dtype)  # noqa: E731
        d = self.width
        self.embed, self.unembed = r(V, d) * math.sqrt(V) * 0.5, r(d, V) * 3
        self.layers = [dict(qkv=r(d, (heads + 2 * kv_heads) * dim), o=r(d, d), up=r(d, 2 * d), down=r(2 * d, d)) for _ in range(layers)]
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

    def step(self, tree, cache, table, tokens, nx):
        """Logits [B * n, V] of the tree's newest tokens [B, n]; their keys and values go into the cache."""
        B, n = tokens.shape
        k, v = cache
        x = self.embed[tokens.flatten().long()]
        place, position = nx["slot"].flatten(), nx["position"].flatten()
        for i, w in enumerate(self.layers):
            q, new_k, new_v = self._qkv(w, x)
            q = tree.append(new_k, new_v, k[i], v[i], table, place, position, rotary=self.rotary, q=q)
            x = self._after(w, x, tree.attend(q.view(B, n, self.heads, self.dim), k[i], v[i], table, nx["ctx_len"], nx["masks"], nx["top"]))
        return self._norm(x) @ self.unembed

    def whole_text(self, text):
        """Logits after the last token of `text` (a list), computed without a cache."""
        torch, n, half = self.torch, len(text), self.dim // 2
        x = self.embed[torch.tensor(text, device=self.embed.device)]
        cos, sin = self.rotary[0][:n, None], self.rotary[1][:n, None]

        def turn(y):
            y = y.float()
            a, b = y[..., :half], y[..., half:]
            return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(self.dtype)
        causal = torch.ones(n, n, dtype=torch.bool, device=x.device).tril()
        for w in self.layers:
            q, k, v = self._qkv(w, x)
            q, k = turn(q).float(), turn(k).float()
            k, v = (y.repeat_interleave(self.heads // self.kv_heads, 1).float() for y in (k, v))
            s = torch.einsum("ihd,jhd->hij", q, k) * self.dim ** -0.5
            x = self._after(w, x, torch.einsum("hij,jhd->ihd", s.masked_fill(~causal, -math.inf).softmax(-1), v).to(self.dtype))
        return (self._norm(x) @ self.unembed)[-1]


def decode(B=4, k=8, steps=24, prompt=12, V=997, layers=2, heads=8, kv_heads=2, dim=64, page_size=16, words=8, dtype="bf16", seed=0, check=False):
    """Returns (tokens, lengths, scores, flags) of dba_finalize, the largest difference of a logit from the one computed without
    a cache (check) and what fell on the way: settled tokens, the highest slot."""
    import torch
    import paper_1804_06609_b200 as dba
    g = torch.Generator().manual_seed(seed)
    code, tdt = (dba.BF16, torch.bfloat16) if dtype == "bf16" else (dba.F32, torch.float32)
    model = Decoder(V, layers, heads, kv_heads, dim, seed, tdt)
    constraints = [[[int(torch.randint(4, V, (1,), generator=g)) for _ in range(1 + b % 2)] for _ in range(b % 3)] for b in range(B)]
    texts = torch.cat([torch.full((B, 1), BOS), torch.randint(4, V, (B, prompt - 1), generator=g)], 1).int().cuda()
    per = (32 * words + prompt + steps) // page_size + 1
    rows = max(k, prompt)
    tree = dba.TokenTree(B, rows, heads, kv_heads, dim, page_size, per, words, dtype=code)
    stepper = dba.DbaStepper(B, k, V, steps, constraints=constraints, dtype=code, pad=PAD, bos=BOS, eos=EOS)
    shape = (layers, B * per, page_size, kv_heads, dim)
    cache = tuple(torch.empty(shape, dtype=tdt, device="cuda") for _ in range(2))
    table = torch.arange(B * per, dtype=torch.int32, device="cuda").view(B, per)
    slot_pos = torch.zeros(B, 32 * words, dtype=torch.int32, device="cuda")

    # the prompt: a chain from the sequence's start
    chain = torch.arange(prompt, dtype=torch.int32, device="cuda").expand(B, prompt).contiguous()       # row i extends new row i - 1
    nx = tree.advance(chain, torch.zeros(B, 1, words, dtype=torch.int32, device="cuda"), slot_pos, torch.zeros(B, dtype=torch.int32, device="cuda"))
    chain_logits = model.step(tree, cache, table, texts, nx).view(B, prompt, V)
    logits = torch.zeros(B, k, V, dtype=tdt, device="cuda")
    logits[:, 0] = chain_logits[:, -1]                       # the beam's one live hypothesis
    worst, settled, top, lines = 0.0, 0, 0, [[t] for t in texts.tolist()]
    for step in range(steps):
        out = stepper.step(logits.view(B * k, V).contiguous())
        backptr = out["backptr"].view(B, k)
        if step == 0:
            backptr = torch.where(backptr >= 0, backptr + (prompt - 1), backptr)      # slot 0 of the beam is the chain's last row
        nx = tree.advance(backptr, nx["masks"], slot_pos, nx["ctx_len"], score=out["score"], token=out["token"], eos=EOS)
        tree.commit(*cache, table, nx["ctx_len"], nx["commit_src"], nx["commit_n"])
        tokens = out["token"].view(B, k)
        logits = model.step(tree, cache, table, tokens, nx).view(B, k, V)
        if check:
            bp, tk, opened = out["backptr"].view(B, k).tolist(), tokens.tolist(), (nx["position"] >= 0).tolist()
            lines = [[lines[b][bp[b][j]] + [tk[b][j]] if opened[b][j] else [] for j in range(k)] for b in range(B)]
            for b in range(B):
                for j in range(k):
                    if opened[b][j]:
                        assert int(nx["position"][b, j]) == len(lines[b][j]) - 1
                        worst = max(worst, float((logits[b, j].float() - model.whole_text(lines[b][j]).float()).abs().max()))
            settled, top = settled + int(nx["commit_n"].sum()), max(top, int(nx["top"].max()))
    result = stepper.finalize()
    bits = tree.status()
    if bits:
        raise RuntimeError(f"token tree: status {bits}")
    return result, worst, dict(settled=settled, top=top, constraints=constraints)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("B", 4), ("k", 8), ("steps", 24), ("prompt", 12)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args()
    (tokens, length, score, flags), worst, info = decode(a.B, a.k, a.steps, a.prompt, dtype=a.dtype, check=a.check)
    for b in range(a.B):
        print(f"sentence {b}: constraints {info['constraints'][b]}, {'completed' if flags[b] & 1 else 'not completed'}, score {score[b]:.3f}: {tokens[b, :length[b]].tolist()}")
    if a.check:
        print(f"largest difference of a logit from the whole text's: {worst:.3g}; {info['settled']} tokens settled, highest slot {info['top']}")


if __name__ == "__main__":
    main()
