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


class TokenTree:
    """Owns a dba_tree handle and its workspace.  Caches, tables, masks and lengths are the caller's tensors:
    k, v [pages, page_size, kv_heads, head_dim] (any strides with a unit inner one; both alike; commit: a leading layer
    dimension), table [B, max_pages] int32, masks [B, rows, words] int32, ctx_len [B] int32.

    Calls are short (a few microseconds of work each at the smallest sizes), so the argument structures are made once and
    filled in by each call; calls on one handle must not overlap."""

    def __init__(self, B, rows, heads, kv_heads, head_dim, page_size, max_pages, words, dtype=BF16, device="cuda:0", stream=None):
        import torch
        self.torch = torch
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

    def append(self, new_k, new_v, k, v, table, place, position=None, rotary=None, pairs=False, q=None, seq=None, q_out=None):
        """new_k, new_v [N, kv_heads, head_dim] into the cache at `place` [N] of sequence `seq` [N] (None: N / B tokens to a
        sequence, in order), keys rotated by `position` [N] with rotary = (cos, sin) [positions, rot / 2] fp32.  Rotates
        q [N, heads, head_dim] too and returns it (q_out: where to; may be q; default: the handle's own buffer for up to
        B * rows tokens, overwritten by the next call, or a new tensor)."""
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
        code = self._f_append(self._h, self._tok_ref, self._cache(k, v, 0), table.data_ptr(), stride)
        if code:
            _check(code, "dba_tree_append")
        return q_out

    def _q_out(self, N):
        if N <= self.B * self.rows:
            return self.q_out if N == self.B * self.rows else self.q_out[:N]
        torch = self.torch
        with torch.cuda.stream(self.stream):         # (the allocator gives freed memory out by stream)
            return torch.empty(N, self.heads, self.head_dim, dtype=self.torch_dtype, device=self.device)

    def attend(self, q, k, v, table, ctx_len, masks=None, top=None, scale=None, out=None, lse=None):
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
        code = self._f_attend(self._h, self._query_ref, self._cache(k, v, 0), table.data_ptr(), stride, self._i32(ctx_len, B, "ctx_len: int32 [B]"),
                              None if masks is None else self._i32(masks, B * n * self.words, "masks: int32 [B, rows, words]"),
                              None if top is None else self._i32(top, B, "top: int32 [B]"))
        if code:
            _check(code, "dba_tree_attend")
        return out

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
        s = slot_pos.stride()
        if slot_pos.dtype is not self._i32t or slot_pos.shape != self._shape_arena or s[1] != 1 or slot_pos.get_device() != dev:
            raise ValueError("slot_pos: int32 [B, 32 * words]")
        if score is not None and (score.dtype is not self._f32t or score.numel() != size or not score.is_contiguous() or score.get_device() != dev):
            raise ValueError("score: fp32 [B, rows]")
        code = self._f_advance(self._h, rows_in, self._i32(masks, B * rows_in * W, "masks: int32 [B, rows, words]"), n,
                               self._i32(backptr, size, "backptr: int32 [B, rows]"), None if score is None else score.data_ptr(),
                               None if token is None else self._i32(token, size, "token: int32 [B, rows]"), eos,
                               slot_pos.data_ptr(), s[0] if B > 1 else 32 * W, self._i32(ctx_len, B, "ctx_len: int32 [B]"), C.byref(nx))
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
