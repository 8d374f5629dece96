"""Binding of the token tree over a paged cache (dba_tree_* in include/dba.h): attention of a beam's hypotheses, or of
drafted tokens, over a paged cache; appending to it; the tree after a step.  Argument marshalling only, as in binding.py."""
from __future__ import annotations

import ctypes as C

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


def _ptr(t):
    return None if t is None else t.data_ptr()


class TokenTree:
    """Owns a dba_tree handle and its workspace.  Caches, tables, masks and lengths are the caller's tensors:
    k, v [pages, page_size, kv_heads, head_dim] (any strides with a unit inner one; both alike; commit: a leading layer
    dimension), table [B, max_pages] int32, masks [B, rows, words] int32, ctx_len [B] int32."""

    def __init__(self, B, rows, heads, kv_heads, head_dim, page_size, max_pages, words, dtype=BF16, device="cuda:0", stream=None):
        import torch
        self.torch = torch
        self.B, self.rows, self.heads, self.kv_heads, self.head_dim = B, rows, heads, kv_heads, head_dim
        self.page_size, self.max_pages, self.words, self.dtype = page_size, max_pages, words, dtype
        self.torch_dtype = torch.float32 if dtype == F32 else torch.bfloat16
        self.device = torch.device(device)
        cfg = TreeConfig(B, rows, heads, kv_heads, head_dim, page_size, max_pages, words, dtype)
        with torch.cuda.device(self.device):
            n = C.c_size_t()
            _check(lib().dba_tree_workspace_bytes(C.byref(cfg), C.byref(n)), "dba_tree_workspace_bytes")
            self.workspace_bytes = n.value
            self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
            with torch.cuda.stream(self.stream):     # what the handle owns belongs to its stream
                self.workspace = torch.empty(n.value + 256, dtype=torch.uint8, device=self.device)
                h = C.c_void_p()
                base = (self.workspace.data_ptr() + 255) // 256 * 256
                _check(lib().dba_tree_init(C.byref(cfg), base, n.value, self.stream.cuda_stream, C.byref(h)), "dba_tree_init")
                self._h = h
                self.out = torch.empty(B, rows, heads, head_dim, dtype=self.torch_dtype, device=self.device)
                self._next = [self.new_next(), self.new_next()] if words else None
        self._turn = 0

    def new_next(self):
        """Tensors for the tree after a step (what advance returns)."""
        torch, B, n, W = self.torch, self.B, self.rows, self.words
        z = lambda *s: torch.zeros(s, dtype=torch.int32, device=self.device)  # noqa: E731
        return dict(masks=z(B, n, W), slot=z(B, n), position=z(B, n), ctx_len=z(B), top=z(B), commit_src=z(B, 32 * W), commit_n=z(B))

    def _empty(self, *shape):
        """A tensor that belongs to the handle's stream (the allocator gives freed memory out by stream)."""
        torch = self.torch
        if torch.cuda.current_stream(self.device) == self.stream:
            return torch.empty(shape, dtype=self.torch_dtype, device=self.device)
        with torch.cuda.stream(self.stream):
            return torch.empty(shape, dtype=self.torch_dtype, device=self.device)

    def _cache(self, k, v, layers):
        assert k.is_cuda and k.dtype == v.dtype == self.torch_dtype and k.shape == v.shape and k.stride() == v.stride()
        assert k.stride(-1) == 1 and k.dim() == (5 if layers else 4)
        assert k.shape[-3:] == (self.page_size, self.kv_heads, self.head_dim)
        s = k.stride()
        return KvCache(k.data_ptr(), v.data_ptr(), k.shape[-4], k.shape[0] if layers else 1, s[-4], s[-3], s[-2], s[0] if layers else 0)

    def _i32(self, t, shape):
        assert t is None or (t.is_cuda and t.dtype == self.torch.int32 and tuple(t.shape) == shape and t.is_contiguous()), (shape,)
        return _ptr(t)

    def _table(self, table):
        assert table.is_cuda and table.dtype == self.torch.int32 and table.shape == (self.B, self.max_pages) and table.stride(1) == 1
        return table.data_ptr(), (table.stride(0) if self.B > 1 else self.max_pages)

    def append(self, new_k, new_v, k, v, table, place, position=None, rotary=None, pairs=False, q=None, seq=None, q_out=None):
        """new_k, new_v [N, kv_heads, head_dim] into the cache at `place` [N] of sequence `seq` [N] (None: N / B tokens to a
        sequence, in order), keys rotated by `position` [N] with rotary = (cos, sin) [positions, rot / 2] fp32.  Rotates
        q [N, heads, head_dim] too and returns it (q_out: where to; may be q)."""
        torch, N = self.torch, new_k.shape[0]
        assert new_k.is_cuda and new_k.dtype == new_v.dtype == self.torch_dtype and new_k.stride(2) == new_v.stride(2) == 1
        assert new_k.shape == new_v.shape == (N, self.kv_heads, self.head_dim)
        t = TreeTokens(N, new_k.data_ptr(), new_v.data_ptr(), new_k.stride(0), new_k.stride(1), new_v.stride(0), new_v.stride(1))
        if q is not None:
            assert q.is_cuda and q.dtype == self.torch_dtype and q.shape == (N, self.heads, self.head_dim) and q.stride(2) == 1
            if q_out is None:
                q_out = self._empty(N, self.heads, self.head_dim)
            assert q_out.is_cuda and q_out.dtype == self.torch_dtype and q_out.shape == q.shape and q_out.stride(2) == 1
            t.q, t.q_out = q.data_ptr(), q_out.data_ptr()
            t.q_token_stride, t.q_head_stride, t.qo_token_stride, t.qo_head_stride = q.stride(0), q.stride(1), q_out.stride(0), q_out.stride(1)
        t.place, t.seq, t.position = self._i32(place, (N,)), self._i32(seq, (N,)), self._i32(position, (N,))
        if rotary is not None:
            cos, sin = rotary
            assert cos.is_cuda and cos.dtype == sin.dtype == torch.float32 and cos.shape == sin.shape and cos.is_contiguous() and sin.is_contiguous()
            t.cos, t.sin, t.positions, t.rot_dim, t.pairs = cos.data_ptr(), sin.data_ptr(), cos.shape[0], 2 * cos.shape[1], int(pairs)
        else:
            assert position is None, "positions need a rotary table"
        tp, ts = self._table(table)
        _check(lib().dba_tree_append(self._h, C.byref(t), C.byref(self._cache(k, v, False)), tp, ts), "dba_tree_append")
        return q_out

    def attend(self, q, k, v, table, ctx_len, masks=None, top=None, scale=None, out=None, lse=None):
        """q [B, rows, heads, head_dim] (rows up to the handle's) over the context and the arena slots of `masks`; returns out
        (default: the handle's own buffer, overwritten by the next call)."""
        torch, n = self.torch, q.shape[1]
        assert q.is_cuda and q.dtype == self.torch_dtype and q.shape == (self.B, n, self.heads, self.head_dim) and q.stride(3) == 1
        if out is None:
            assert n <= self.rows
            out = self.out if n == self.rows else self.out[:, :n]
        assert out.is_cuda and out.dtype == self.torch_dtype and out.shape == q.shape and out.stride(3) == 1
        if lse is not None:
            assert lse.is_cuda and lse.dtype == torch.float32 and lse.shape == (self.B, n, self.heads) and lse.is_contiguous()
        sq, so = q.stride(), out.stride()
        d = TreeQuery(n, q.data_ptr(), sq[0], sq[1], sq[2], out.data_ptr(), so[0], so[1], so[2], _ptr(lse),
                      self.head_dim ** -0.5 if scale is None else scale)
        tp, ts = self._table(table)
        _check(lib().dba_tree_attend(self._h, C.byref(d), C.byref(self._cache(k, v, False)), tp, ts, self._i32(ctx_len, (self.B,)),
                                     self._i32(masks, (self.B, n, self.words)), self._i32(top, (self.B,))), "dba_tree_attend")
        return out

    def advance(self, backptr, masks, slot_pos, ctx_len, score=None, token=None, eos=-1, out=None):
        """The tree after a step: see dba_tree_advance.  backptr (and score, token: dba_step's outputs) [B, rows] or [B * rows];
        slot_pos [B, 32 * words] is updated in place.  Returns a dict of masks, slot, position, ctx_len, top, commit_src,
        commit_n (default: one of two sets of the handle's own tensors, in turn) with slot_pos."""
        n = backptr.numel() // self.B
        assert backptr.numel() == self.B * n and n <= self.rows and masks.dim() == 3
        if out is None:
            out = self._next[self._turn]
            if out["masks"].data_ptr() == masks.data_ptr():
                out = self._next[1 - self._turn]
            self._turn = 1 - self._turn
        if n != out["slot"].shape[1]:                       # fewer rows than the handle's: the front of its tensors
            out = dict(out)
            out["masks"] = out["masks"].view(-1)[:self.B * n * self.words].view(self.B, n, self.words)
            for f in ("slot", "position"):
                out[f] = out[f].view(-1)[:self.B * n].view(self.B, n)
        nx = TreeNext(*[_ptr(out.get(f)) for f in ("masks", "slot", "position", "ctx_len", "top", "commit_src", "commit_n")])
        assert slot_pos.is_cuda and slot_pos.dtype == self.torch.int32 and slot_pos.shape == (self.B, 32 * self.words) and slot_pos.stride(1) == 1
        for t, dt in ((backptr, self.torch.int32), (score, self.torch.float32), (token, self.torch.int32)):
            assert t is None or (t.is_cuda and t.dtype == dt and t.numel() == self.B * n and t.is_contiguous())
        _check(lib().dba_tree_advance(self._h, masks.shape[1], self._i32(masks, (self.B, masks.shape[1], self.words)), n, backptr.data_ptr(),
                                      _ptr(score), _ptr(token), eos, slot_pos.data_ptr(),
                                      slot_pos.stride(0) if self.B > 1 else 32 * self.words, self._i32(ctx_len, (self.B,)), C.byref(nx)), "dba_tree_advance")
        return {**out, "slot_pos": slot_pos}

    def commit(self, k, v, table, ctx_len, commit_src, commit_n):
        """Settled tokens (advance's commit_src, commit_n, ctx_len) to the end of the context in every layer of the cache."""
        tp, ts = self._table(table)
        _check(lib().dba_tree_commit(self._h, C.byref(self._cache(k, v, k.dim() == 5)), tp, ts, self._i32(ctx_len, (self.B,)),
                                     self._i32(commit_src, (self.B, 32 * self.words)), self._i32(commit_n, (self.B,))), "dba_tree_commit")

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
