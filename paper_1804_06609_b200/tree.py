"""Binding of the token tree over a paged cache (dba_tree_* in include/dba.h): attention of a beam's hypotheses, or of
drafted tokens, over a paged cache; appending to it; the tree after a step.  Argument marshalling only, as in binding.py."""
from __future__ import annotations

import ctypes as C
import math

from .binding import BF16, F32, _check, lib

TREE_TIMEOUT, TREE_BAD_PAGE, TREE_ARENA_FULL, TREE_NO_ROOM, TREE_BAD_INDEX = 1, 2, 4, 8, 16


class TreeConfig(C.Structure):
    _fields_ = [(f, C.c_int32) for f in ("B", "rows", "heads", "kv_heads", "head_dim", "page_size", "max_pages", "words", "dtype")]


class KvCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("num_pages", C.c_int32), ("layers", C.c_int32), ("page_stride", C.c_int64),
                ("token_stride", C.c_int64), ("head_stride", C.c_int64), ("layer_stride", C.c_int64)]


class TreeTokens(C.Structure):
    _fields_ = [("N", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p), ("k_token_stride", C.c_int64), ("k_head_stride", C.c_int64),
                ("v_token_stride", C.c_int64), ("v_head_stride", C.c_int64), ("q", C.c_void_p), ("q_out", C.c_void_p),
                ("q_token_stride", C.c_int64), ("q_head_stride", C.c_int64), ("qo_token_stride", C.c_int64), ("qo_head_stride", C.c_int64),
                ("place", C.c_void_p), ("seq", C.c_void_p), ("position", C.c_void_p), ("cos", C.c_void_p), ("sin", C.c_void_p),
                ("positions", C.c_int32), ("rot_dim", C.c_int32), ("pairs", C.c_int32)]


class TreeQuery(C.Structure):
    _fields_ = [("rows", C.c_int32), ("q", C.c_void_p), ("q_seq_stride", C.c_int64), ("q_row_stride", C.c_int64), ("q_head_stride", C.c_int64),
                ("out", C.c_void_p), ("out_seq_stride", C.c_int64), ("out_row_stride", C.c_int64), ("out_head_stride", C.c_int64),
                ("lse", C.c_void_p), ("scale", C.c_float)]


class TreeNext(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in ("masks", "slot", "position", "ctx_len", "top", "commit_src", "commit_n")]


class TreePrefix(C.Structure):
    _fields_ = [("groups", C.c_int32), ("max_pages", C.c_int32), ("first", C.c_void_p), ("len", C.c_void_p), ("table", C.c_void_p), ("table_stride", C.c_int64)]


class TreeNorm(C.Structure):
    _fields_ = [("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("eps", C.c_float), ("offset", C.c_void_p)]


class TreeEvicted(C.Structure):
    _fields_ = [("weight", C.c_void_p), ("weight_out", C.c_void_p), ("layer_stride", C.c_int64), ("seq_stride", C.c_int64), ("head_stride", C.c_int64),
                ("keep", C.c_int32), ("recent", C.c_int32), ("to_table", C.c_void_p), ("to_table_stride", C.c_int64), ("kept", C.c_void_p),
                ("ctx_len_out", C.c_void_p), ("dropped", C.c_void_p), ("slot_pos", C.c_void_p), ("slot_pos_stride", C.c_int64)]


def _rows_apart(shape, strides, places):
    """Whether rows of so many places, the strides apart, have none in common.  (A stride of 0 is refused by the call.)"""
    span, dims = places, sorted((s, n) for s, n in zip(strides, shape) if n > 1 and s)
    for s, n in dims:
        if s < span:
            break
        span += s * (n - 1)
    else:
        return True
    at = [0]                                             # (not one within the other: rows may still lie between one another's)
    for s, n in dims:
        at = [a + s * i for a in at for i in range(n)]
    at.sort()
    return all(b - a >= places for a, b in zip(at, at[1:]))


class TokenTree:
    """Owns a dba_tree handle and its workspace.  Caches, tables, masks and lengths are the caller's tensors:
    k, v [pages, page_size, kv_heads, head_dim] (any strides with a unit inner one; both alike; commit and evict: a leading layer
    dimension), table [B, max_pages] int32, masks [B, rows, words] int32, ctx_len [B] int32.

    prefixes: the most prefixes a call of attend_shared may have; 0: none, and the handle holds no scratch for it.

    Calls are short (a few microseconds of work each at the smallest sizes), so the argument structures are made once and
    filled in by each call; calls on one handle must not overlap."""

    def __init__(self, B, rows, heads, kv_heads, head_dim, page_size, max_pages, words, dtype=BF16, device="cuda:0", stream=None, prefixes=0):
        import torch
        self.torch = torch
        self.prefixes = prefixes
        self.B, self.rows, self.heads, self.kv_heads, self.head_dim = B, rows, heads, kv_heads, head_dim
        self.page_size, self.max_pages, self.words, self.dtype = page_size, max_pages, words, dtype
        self.torch_dtype = torch.float32 if dtype == F32 else torch.bfloat16
        self.device = torch.device(device)
        self._dev = self.device.index if self.device.index is not None else torch.cuda.current_device()
        self._i32t, self._f32t = torch.int32, torch.float32
        cfg = TreeConfig(B, rows, heads, kv_heads, head_dim, page_size, max_pages, words, dtype)
        L = lib()
        with torch.cuda.device(self.device):
            n = C.c_size_t()
            _check(L.dba_tree_workspace_bytes(C.byref(cfg), C.byref(n)), "dba_tree_workspace_bytes")
            self.workspace_bytes = n.value
            self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
            with torch.cuda.stream(self.stream):     # what the handle owns belongs to its stream
                self.workspace = torch.empty(n.value + 256, dtype=torch.uint8, device=self.device)
                h = C.c_void_p()
                base = (self.workspace.data_ptr() + 255) // 256 * 256
                _check(L.dba_tree_init(C.byref(cfg), base, n.value, self.stream.cuda_stream, C.byref(h)), "dba_tree_init")
                self._h = h
                self.out = torch.empty(B, rows, heads, head_dim, dtype=self.torch_dtype, device=self.device)
                self.q_out = torch.empty(B * rows, heads, head_dim, dtype=self.torch_dtype, device=self.device)
                self._next = [self.new_next(), self.new_next()] if words else []
                if prefixes:
                    _check(L.dba_tree_shared_bytes(h, C.byref(n)), "dba_tree_shared_bytes")
                    self._scratch_bytes = n.value
                    self.scratch = torch.empty(n.value + 256, dtype=torch.uint8, device=self.device)
                    self._scratch_at = (self.scratch.data_ptr() + 255) // 256 * 256
        self._prefix, self._norm, self._evict = TreePrefix(), TreeNorm(), TreeEvicted()
        self._prefix_ref, self._norm_ref, self._evict_ref = (C.byref(x) for x in (self._prefix, self._norm, self._evict))
        self._next = [(x, self._next_struct(x)) for x in self._next]
        self._turn = 0
        self._f_append, self._f_attend, self._f_advance, self._f_commit = L.dba_tree_append, L.dba_tree_attend, L.dba_tree_advance, L.dba_tree_commit
        self._kv, self._tok, self._query = KvCache(), TreeTokens(), TreeQuery()
        self._kv_ref, self._tok_ref, self._query_ref = (C.byref(x) for x in (self._kv, self._tok, self._query))
        self._shape_table, self._shape_page, self._shape_arena = (B, max_pages), (page_size, kv_heads, head_dim), (B, 32 * words)
        # the strides the structures hold: they are filled in again where a call's are others
        self._kv_last = self._tok_last = self._query_last = None
        self._no_stride = (0, 0, 1)

    NEXT = ("masks", "slot", "position", "ctx_len", "top", "commit_src", "commit_n")

    def new_next(self):
        """Tensors for the tree after a step (what advance returns)."""
        torch, B, n, W = self.torch, self.B, self.rows, self.words
        z = lambda *s: torch.zeros(s, dtype=torch.int32, device=self.device)  # noqa: E731
        return dict(masks=z(B, n, W), slot=z(B, n), position=z(B, n), ctx_len=z(B), top=z(B), commit_src=z(B, 32 * W), commit_n=z(B))

    def _next_struct(self, out):
        return TreeNext(*[out[f].data_ptr() if out.get(f) is not None else None for f in self.NEXT])

    def _next_views(self, out, n):
        """out with its tensors in the shapes that n rows are written in (the front of larger ones), each looked over."""
        B, W, dev, out = self.B, self.words, self._dev, dict(out)
        if out.get("masks") is None:
            raise ValueError("out: a dict with masks [B, rows, words] at least")
        for f in self.NEXT:
            t = out.get(f)
            if t is None:
                continue
            shape = (B, n, W) if f == "masks" else (B, n) if f in ("slot", "position") else (B, 32 * W) if f == "commit_src" else (B,)
            size = math.prod(shape)
            if t.dtype is not self._i32t or t.get_device() != dev or not t.is_contiguous() or t.numel() < size:
                raise ValueError(f"out: {f} int32 {shape}, contiguous, on the handle's device")
            if t.shape != shape:
                out[f] = t.view(-1)[:size].view(shape)
        return out

    # Checks are written out in the calls and look at no more than memory safety and the argument's meaning need.
    def _cache(self, k, v, layers):
        s, sh = k.stride(), k.shape
        if (s, sh, layers) != self._kv_last:
            if s[-1] != 1 or len(s) != 4 + layers or sh[-3:] != self._shape_page:
                raise ValueError("k and v: [pages, page_size, kv_heads, head_dim] with a unit inner stride (commit: layers in front)")
            c = self._kv
            c.num_pages, c.page_stride, c.token_stride, c.head_stride = sh[-4], s[-4], s[-3], s[-2]
            c.layers, c.layer_stride = (sh[0], s[0]) if layers else (1, 0)
            self._kv_last = (s, sh, layers)
        dt, dev = self.torch_dtype, self._dev
        if k.dtype is not dt or v.dtype is not dt or k.get_device() != dev or v.get_device() != dev or v.stride() != s or v.shape != sh:
            raise ValueError("k and v: alike, of the handle's type and on its device")
        self._kv.k, self._kv.v = k.data_ptr(), v.data_ptr()
        return self._kv_ref

    def _i32(self, t, numel, what):
        if t.dtype is not self._i32t or t.numel() != numel or t.get_device() != self._dev or not t.is_contiguous():
            raise ValueError(what)
        return t.data_ptr()

    def _table(self, table):
        if table.dtype is not self._i32t or table.get_device() != self._dev or table.shape != self._shape_table:
            raise ValueError(f"table: int32 {self._shape_table} on the handle's device")
        s = table.stride()
        if s[1] != 1:
            raise ValueError("table: rows of a unit stride")
        return s[0] if self.B > 1 else self.max_pages

    def append(self, new_k, new_v, k, v, table, place, position=None, rotary=None, pairs=False, q=None, seq=None, q_out=None, norm=None, offset=None):
        """new_k, new_v [N, kv_heads, head_dim] into the cache at `place` [N] of sequence `seq` [N] (None: N / B tokens to a
        sequence, in order), keys rotated by `position` [N] with rotary = (cos, sin) [positions, rot / 2] fp32.  Rotates
        q [N, heads, head_dim] too and returns it (q_out: where to; may be q; default: the handle's own buffer for up to
        B * rows tokens, overwritten by the next call, or a new tensor).
        norm = (q_weight, k_weight, eps), weights [head_dim] fp32 or None: every head's queries and keys are normed before the rotation
        (root mean square).  offset [B] int32: added to the positions of the sequence's tokens."""
        dt, dev, t, shape = self.torch_dtype, self._dev, self._tok, new_k.shape
        N, _, D = shape
        sk, sv = new_k.stride(), new_v.stride()
        if (new_k.dtype is not dt or new_v.dtype is not dt or new_k.get_device() != dev or new_v.get_device() != dev or new_v.shape != shape
                or shape[1] != self.kv_heads or D != self.head_dim or sk[2] != 1 or sv[2] != 1):
            raise ValueError("new_k, new_v: [N, kv_heads, head_dim] of the handle's type and on its device")
        t.N, t.k, t.v = N, new_k.data_ptr(), new_v.data_ptr()
        if q is not None:
            if q_out is None:
                q_out = self._q_out(N)
            sq, so, shape = q.stride(), q_out.stride(), q.shape
            if (q.dtype is not dt or q_out.dtype is not dt or q.get_device() != dev or q_out.get_device() != dev or q_out.shape != shape
                    or shape[0] != N or shape[1] != self.heads or shape[2] != D or sq[2] != 1 or so[2] != 1):
                raise ValueError("q, q_out: [N, heads, head_dim] of the handle's type and on its device")
            t.q, t.q_out = q.data_ptr(), q_out.data_ptr()
        else:
            sq = so = self._no_stride
            t.q = t.q_out = None
        if (sk, sv, sq, so) != self._tok_last:
            t.k_token_stride, t.k_head_stride, t.v_token_stride, t.v_head_stride = sk[0], sk[1], sv[0], sv[1]
            t.q_token_stride, t.q_head_stride, t.qo_token_stride, t.qo_head_stride = sq[0], sq[1], so[0], so[1]
            self._tok_last = (sk, sv, sq, so)
        t.place = self._i32(place, N, "place: int32 [N]")
        t.seq = None if seq is None else self._i32(seq, N, "seq: int32 [N]")
        if rotary is not None:
            cos, sin = rotary
            shape = cos.shape
            if (cos.dtype is not self._f32t or sin.dtype is not self._f32t or sin.shape != shape or not cos.is_contiguous() or not sin.is_contiguous()
                    or cos.get_device() != dev or sin.get_device() != dev):
                raise ValueError("rotary: cos, sin [positions, rot / 2] fp32")
            t.cos, t.sin, t.positions, t.rot_dim, t.pairs = cos.data_ptr(), sin.data_ptr(), shape[0], 2 * shape[1], int(pairs)
            t.position = None if position is None else self._i32(position, N, "position: int32 [N]")
        else:
            if position is not None:
                raise ValueError("positions need a rotary table")
            t.position = t.cos = t.sin = None
            t.positions = t.rot_dim = t.pairs = 0
        stride = self._table(table)
        if norm is None and offset is None:
            code = self._f_append(self._h, self._tok_ref, self._cache(k, v, 0), table.data_ptr(), stride)
            if code:
                _check(code, "dba_tree_append")
            return q_out
        nm = self._norm
        nm.q_weight, nm.k_weight, nm.eps = (self._weight(norm[0]), self._weight(norm[1]), norm[2]) if norm is not None else (None, None, 0.0)
        nm.offset = None if offset is None else self._i32(offset, self.B, "offset: int32 [B]")
        code = lib().dba_tree_append_norm(self._h, self._tok_ref, self._norm_ref, self._cache(k, v, 0), table.data_ptr(), stride)
        if code:
            _check(code, "dba_tree_append_norm")
        return q_out

    def _weight(self, w):
        if w is None:
            return None
        if w.dtype is not self._f32t or w.get_device() != self._dev or w.shape != (self.head_dim,) or not w.is_contiguous():
            raise ValueError("norm: (q_weight, k_weight, eps), weights [head_dim] fp32 on the handle's device or None")
        return w.data_ptr()

    def _q_out(self, N):
        if N <= self.B * self.rows:
            return self.q_out if N == self.B * self.rows else self.q_out[:N]
        torch = self.torch
        with torch.cuda.stream(self.stream):         # (the allocator gives freed memory out by stream)
            return torch.empty(N, self.heads, self.head_dim, dtype=self.torch_dtype, device=self.device)

    def attend(self, q, k, v, table, ctx_len, masks=None, top=None, scale=None, out=None, lse=None, _shared=None):
        """q [B, rows, heads, head_dim] (rows up to the handle's) over the context and the arena slots of `masks`; returns out
        (default: the handle's own buffer, overwritten by the next call)."""
        B, d, dt, dev, shape, sq = self.B, self._query, self.torch_dtype, self._dev, q.shape, q.stride()
        n = shape[1]
        if out is None:
            out = self.out if n == self.rows else self.out[:, :n]
        so = out.stride()
        if (q.dtype is not dt or out.dtype is not dt or q.get_device() != dev or out.get_device() != dev or out.shape != shape or shape[0] != B
                or shape[2] != self.heads or shape[3] != self.head_dim or sq[3] != 1 or so[3] != 1):
            raise ValueError("q, out: [B, rows, heads, head_dim] of the handle's type and on its device")
        if (n, sq, so) != self._query_last:
            d.rows, d.q_seq_stride, d.q_row_stride, d.q_head_stride = n, sq[0], sq[1], sq[2]
            d.out_seq_stride, d.out_row_stride, d.out_head_stride = so[0], so[1], so[2]
            self._query_last = (n, sq, so)
        if lse is None:
            d.lse = None
        else:
            if lse.dtype is not self._f32t or lse.get_device() != dev or lse.shape != (B, n, self.heads) or not lse.is_contiguous():
                raise ValueError("lse: [B, rows, heads] fp32")
            d.lse = lse.data_ptr()
        d.q, d.out, d.scale = q.data_ptr(), out.data_ptr(), self.head_dim ** -0.5 if scale is None else scale
        stride = self._table(table)
        code = (self._f_attend if _shared is None else _shared)(
            self._h, self._query_ref, self._cache(k, v, 0), table.data_ptr(), stride, self._i32(ctx_len, B, "ctx_len: int32 [B]"),
            None if masks is None else self._i32(masks, B * n * self.words, "masks: int32 [B, rows, words]"),
            None if top is None else self._i32(top, B, "top: int32 [B]"))
        if code:
            _check(code, "dba_tree_attend" if _shared is None else "dba_tree_attend_shared")
        return out

    def attend_shared(self, q, k, v, table, ctx_len, prefix, masks=None, top=None, scale=None, out=None, lse=None):
        """attend where the sequences also see a prefix that several of them share, gone through once for all: prefix = (first, length,
        table).  Prefix g, length[g] tokens at the places of table[g], stands before sequences first[g] .. first[g + 1] - 1:
        first int32 [groups + 1], length int32 [groups], table int32 [groups, pages], pages of the same cache.  See dba_tree_attend_shared."""
        first, length, ptable = prefix
        groups, dev, p = length.numel(), self._dev, self._prefix
        if not self.prefixes:
            raise ValueError("attend_shared: the handle was made without prefixes=")
        if groups < 1 or groups > self.prefixes:
            raise ValueError("prefix: between 1 and the handle's `prefixes` of them")
        if ptable.dtype is not self._i32t or ptable.get_device() != dev or ptable.dim() != 2 or ptable.shape[0] != groups or ptable.shape[1] < 1:
            raise ValueError("prefix table: int32 [groups, pages] on the handle's device")
        s = ptable.stride()
        if s[1] != 1 and ptable.shape[1] > 1:
            raise ValueError("prefix table: rows of a unit stride")
        p.groups, p.max_pages = groups, ptable.shape[1]
        p.first, p.len = self._i32(first, groups + 1, "prefix first: int32 [groups + 1]"), self._i32(length, groups, "prefix length: int32 [groups]")
        p.table, p.table_stride = ptable.data_ptr(), s[0] if groups > 1 else ptable.shape[1]
        return self.attend(q, k, v, table, ctx_len, masks, top, scale, out, lse, _shared=self._call_shared)

    def _call_shared(self, *args):
        return lib().dba_tree_attend_shared(*args, self._prefix_ref, self._scratch_at, self._scratch_bytes)

    def _slot_pos(self, slot_pos):
        s = slot_pos.stride()
        if slot_pos.dtype is not self._i32t or slot_pos.shape != self._shape_arena or s[1] != 1 or slot_pos.get_device() != self._dev:
            raise ValueError("slot_pos: int32 [B, 32 * words]")
        return s[0] if self.B > 1 else 32 * self.words

    def advance(self, backptr, masks, slot_pos, ctx_len, score=None, token=None, eos=-1, out=None):
        """The tree after a step: see dba_tree_advance.  backptr (and score, token: dba_step's outputs) [B, rows] or [B * rows];
        slot_pos [B, 32 * words] is updated in place.  Returns a dict of masks, slot, position, ctx_len, top, commit_src,
        commit_n (default: one of two sets of the handle's own tensors, in turn; out: a dict of such tensors, as new_next makes
        them or larger, all but masks optional) with slot_pos."""
        B, W, dev = self.B, self.words, self._dev
        if not W:
            raise ValueError("advance: the handle has no arena (words = 0)")
        size, rows_in = backptr.numel(), masks.shape[1]
        n = size // B
        if size != B * n or n > self.rows:
            raise ValueError("backptr: [B, rows], rows up to the handle's")
        at = masks.data_ptr()
        if out is None:
            own = self._next[self._turn][0]["masks"]
            if 0 <= at - own.data_ptr() < 4 * own.numel():         # (a part of it may be the old masks)
                self._turn = 1 - self._turn
            out, nx = self._next[self._turn]
            self._turn = 1 - self._turn
            if n != self.rows:
                out = self._next_views(out, n)
        else:
            out = self._next_views(out, n)
            nx = self._next_struct(out)
        s = self._slot_pos(slot_pos)
        if score is not None and (score.dtype is not self._f32t or score.numel() != size or not score.is_contiguous() or score.get_device() != dev):
            raise ValueError("score: fp32 [B, rows]")
        code = self._f_advance(self._h, rows_in, self._i32(masks, B * rows_in * W, "masks: int32 [B, rows, words]"), n,
                               self._i32(backptr, size, "backptr: int32 [B, rows]"), None if score is None else score.data_ptr(),
                               None if token is None else self._i32(token, size, "token: int32 [B, rows]"), eos,
                               slot_pos.data_ptr(), s, self._i32(ctx_len, B, "ctx_len: int32 [B]"), C.byref(nx))
        if code:
            _check(code, "dba_tree_advance")
        return {**out, "slot_pos": slot_pos}

    def commit(self, k, v, table, ctx_len, commit_src, commit_n):
        """Settled tokens (advance's commit_src, commit_n, ctx_len) to the end of the context in every layer of the cache."""
        B = self.B
        stride = self._table(table)
        code = self._f_commit(self._h, self._cache(k, v, int(k.dim() == 5)), table.data_ptr(), stride, self._i32(ctx_len, B, "ctx_len: int32 [B]"),
                              self._i32(commit_src, B * 32 * self.words, "commit_src: int32 [B, 32 * words]"), self._i32(commit_n, B, "commit_n: int32 [B]"))
        if code:
            _check(code, "dba_tree_commit")

    _rows_last = None          # strides, shape and leading dimensions of the weights last looked over

    # [B, kv_heads, places] (evict: layers in front) fp32 with a unit inner stride: at least the places a table leaves the context
    def _weights(self, w, lead, what):
        sh, s = w.shape, w.stride()
        good = w.dtype is self._f32t and w.get_device() == self._dev
        if not good or (s, sh, lead) != self._rows_last:
            places = self.max_pages * self.page_size - 32 * self.words
            if not good or len(sh) != len(lead) + 3 or sh[:-1] != (*lead, self.B, self.kv_heads) or sh[-1] < places or s[-1] != 1:
                raise ValueError(f"{what}: fp32 [{'layers, ' if lead else ''}B, kv_heads, context places], unit inner stride")
            if not _rows_apart(sh[:-1], s[:-1], places):
                raise ValueError(f"{what}: rows that do not overlap")
            self._rows_last = (s, sh, lead)
        return s

    def weigh(self, q, k, table, ctx_len, lse, weight=None, decay=1.0, scale=None, out=None):
        """The attention that context tokens receive from the rows of q [B, rows, heads, head_dim], whose log-sum-exps lse [B, rows, heads]
        attend (or attend_shared) has written:  out = decay * weight + sum of the probabilities, [B, kv_heads, context places] fp32,
        for places below ctx_len; the others are left as they are.  out: default weight itself, in place; weight None: zeros.  Returns out."""
        B, d, dev, shape, sq = self.B, self._query, self._dev, q.shape, q.stride()
        if out is None:
            out = weight
        if out is None:
            raise ValueError("weigh: weight or out")
        s = self._weights(out, (), "out")
        if weight is not None and weight is not out and self._weights(weight, (), "weight") != s:
            raise ValueError("weight and out: of the same strides")
        if (q.dtype is not self.torch_dtype or q.get_device() != dev or len(shape) != 4 or shape[0] != B or shape[2] != self.heads
                or shape[3] != self.head_dim or sq[3] != 1):
            raise ValueError("q: [B, rows, heads, head_dim] of the handle's type and on its device")
        if lse.dtype is not self._f32t or lse.get_device() != dev or lse.shape != shape[:3] or not lse.is_contiguous():
            raise ValueError("lse: [B, rows, heads] fp32")
        d.rows, d.q_seq_stride, d.q_row_stride, d.q_head_stride = shape[1], sq[0], sq[1], sq[2]
        d.q, d.scale = q.data_ptr(), self.head_dim ** -0.5 if scale is None else scale
        self._query_last = None
        code = lib().dba_tree_weigh(self._h, self._query_ref, lse.data_ptr(), self._cache(k, k, 0), table.data_ptr(), self._table(table),
                                    self._i32(ctx_len, B, "ctx_len: int32 [B]"), None if weight is None else weight.data_ptr(), out.data_ptr(), s[0], s[1], decay)
        if code:
            _check(code, "dba_tree_weigh")
        return out

    _evicted = _evicted_key = _evict_lens = None
    _evict_turn, _evict_own = 0, ()

    # Two sets in turn, as advance's, for every number of tokens to keep out of the same memory.  What a larger number outgrows is held on to: a recorded call
    # (CUDA graph) may go on writing there.
    def _evict_sets(self, layers, keep):
        torch, shape = self.torch, (*layers, self.B, self.kv_heads, keep)
        size, room = math.prod(shape), self._evict_own[-1].shape[1] if self._evict_own else 0
        with torch.cuda.stream(self.stream):             # (the allocator gives freed memory out by stream)
            if self._evict_lens is None:
                self._evict_lens = torch.empty(2, 2, self.B, dtype=self._i32t, device=self.device)
            if size > room:
                self._evict_own += (torch.empty(2, max(size, 2 * room), dtype=self._i32t, device=self.device),)
        return [(*self._evict_lens[i], self._evict_own[-1][i, :size].view(shape)) for i in (0, 1)]

    def evict(self, k, v, table, ctx_len, weight, keep, recent=0, table_out=None, weight_out=None, slot_pos=None):
        """Keeps `keep` tokens of every longer context: the last `recent` and, of the others, those of the largest weight, in their order,
        at the front.  weight [layers, B, kv_heads, context places] fp32 (without layers where k, v have none).  table_out, weight_out:
        where to; default the same, in place (arena slots go along where table_out has other pages for them).  slot_pos: advance's, of an open
        tree, lowered in place by what is dropped, so that its tokens go on settling in their order.  Returns a dict of ctx_len and dropped
        [B], kept [(layers,) B, kv_heads, keep] (the old context places, -1 beyond) and weight (weight_out); the first three are one of two
        sets of the handle's own tensors, in turn.  See dba_tree_evict."""
        B, layers = self.B, k.shape[:-4]
        if len(layers) > 1:
            raise ValueError("k and v: [pages, page_size, kv_heads, head_dim], or layers in front")
        if keep < 1 or not 0 <= recent <= keep:
            raise ValueError("evict: 0 <= recent <= keep, keep >= 1")
        table_out = table if table_out is None else table_out
        weight_out = weight if weight_out is None else weight_out
        s = self._weights(weight, tuple(layers), "weight")
        if weight_out is not weight and self._weights(weight_out, tuple(layers), "weight_out") != s:
            raise ValueError("weight and weight_out: of the same strides")
        cache, n = self._cache(k, v, len(layers)), self._i32(ctx_len, B, "ctx_len: int32 [B]")
        stride, stride_out = self._table(table), self._table(table_out)
        key = (*layers, keep)
        if key != self._evicted_key:
            self._evicted, self._evicted_key = self._evict_sets(layers, keep), key
        e = self._evict
        if slot_pos is not None or e.slot_pos:
            e.slot_pos, e.slot_pos_stride = (None, 0) if slot_pos is None else (slot_pos.data_ptr(), self._slot_pos(slot_pos))
        new_len, dropped, kept = self._evicted[self._evict_turn]
        self._evict_turn = 1 - self._evict_turn
        e.weight, e.weight_out, e.layer_stride, e.seq_stride, e.head_stride = weight.data_ptr(), weight_out.data_ptr(), s[0] if layers else 0, s[-3], s[-2]
        e.keep, e.recent, e.to_table, e.to_table_stride = keep, recent, table_out.data_ptr(), stride_out
        e.kept, e.ctx_len_out, e.dropped = kept.data_ptr(), new_len.data_ptr(), dropped.data_ptr()
        code = lib().dba_tree_evict(self._h, cache, table.data_ptr(), stride, n, self._evict_ref)
        if code:
            _check(code, "dba_tree_evict")
        return {"ctx_len": new_len, "dropped": dropped, "kept": kept, "weight": weight_out}

    def status(self):
        """TREE_* bits since the last call.  Waits for the handle's stream."""
        bits = C.c_uint32()
        _check(lib().dba_tree_status(self._h, C.byref(bits)), "dba_tree_status")
        return bits.value

    def test_hook(self, wait_clocks=0, drop_item=-1):
        _check(lib().dba_tree_test_hook(self._h, wait_clocks, drop_item), "dba_tree_test_hook")

    def launch_count(self):
        return int(lib().dba_tree_launch_count(self._h))

    def close(self):
        if getattr(self, "_h", None):
            lib().dba_tree_destroy(self._h)
            self._h = None

    def __del__(self):
        self.close()
