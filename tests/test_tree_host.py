"""What the token tree refuses on the host, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest

from paper_1804_06609_b200 import binding, tree

INVALID, UNSUPPORTED = 1, 2


def _config(**kw):
    d = dict(B=2, rows=4, heads=8, kv_heads=2, head_dim=64, page_size=16, max_pages=8, words=2, dtype=1)
    d.update(kw)
    return tree.TreeConfig(*[d[f] for f, _ in tree.TreeConfig._fields_])


@pytest.mark.parametrize("change,code", [
    (dict(B=0), INVALID), (dict(rows=0), INVALID), (dict(heads=0), INVALID), (dict(kv_heads=0), INVALID), (dict(head_dim=0), INVALID),
    (dict(page_size=0), INVALID), (dict(max_pages=0), INVALID), (dict(words=-1), INVALID), (dict(dtype=2), INVALID),
    (dict(heads=7), INVALID), (dict(words=5), INVALID),              # 160 slots do not fit 128 places
    (dict(rows=65), UNSUPPORTED), (dict(words=129, max_pages=1000), UNSUPPORTED), (dict(head_dim=264), UNSUPPORTED),
    (dict(head_dim=60), UNSUPPORTED), (dict(head_dim=6, dtype=0), UNSUPPORTED), (dict(max_pages=1 << 27), UNSUPPORTED),
    (dict(heads=8192, kv_heads=8192), UNSUPPORTED)])
def test_configurations_that_are_refused(change, code):
    n = C.c_size_t()
    L = binding.lib()
    assert L.dba_tree_workspace_bytes(C.byref(_config(**change)), C.byref(n)) == code
    h = C.c_void_p(1)
    assert L.dba_tree_init(C.byref(_config(**change)), 256, 1 << 30, None, C.byref(h)) == code and not h.value


def test_calls_without_a_handle_are_refused():
    L = binding.lib()
    n, bits = C.c_size_t(), C.c_uint32()
    assert L.dba_tree_workspace_bytes(None, C.byref(n)) == INVALID and L.dba_tree_workspace_bytes(C.byref(_config()), None) == INVALID
    assert L.dba_tree_init(C.byref(_config()), None, 0, None, C.byref(C.c_void_p())) == 6          # no workspace
    assert L.dba_tree_init(C.byref(_config()), 128, 0, None, C.byref(C.c_void_p())) == 6           # misaligned
    assert L.dba_tree_init(C.byref(_config()), 256, 0, None, None) == INVALID
    assert L.dba_tree_append(None, None, None, None, 0) == INVALID
    assert L.dba_tree_attend(None, None, None, None, 0, None, 0, None, None) == INVALID
    assert L.dba_tree_advance(None, 1, None, 1, None, None, None, 0, None, 0, None, None) == INVALID
    assert L.dba_tree_commit(None, None, None, 0, None, 0, None, None) == INVALID
    assert L.dba_tree_status(None, C.byref(bits)) == INVALID and L.dba_tree_test_hook(None, 0, -1) == INVALID
    assert L.dba_tree_launch_count(None) == 0
    L.dba_tree_destroy(None)


# The binding's own checks, on a handle without a device: calls that pass them are noted instead of made.
def _handle(B=2, rows=4, words=2, kv_heads=2, head_dim=64, page_size=16, max_pages=8):
    torch = pytest.importorskip("torch")
    t = object.__new__(tree.TokenTree)
    t.torch, t.B, t.rows, t.heads, t.kv_heads, t.head_dim, t.page_size, t.max_pages, t.words = torch, B, rows, 4, kv_heads, head_dim, page_size, max_pages, words
    t.device, t._dev, t.dtype, t.torch_dtype, t._i32t, t._f32t = torch.device("cpu"), -1, 1, torch.bfloat16, torch.int32, torch.float32
    t._h, t.calls = None, []
    note = lambda name: lambda *a: t.calls.append((name, a)) or 0  # noqa: E731
    t._f_append, t._f_attend, t._f_advance, t._f_commit = (note(x) for x in ("append", "attend", "advance", "commit"))
    t._next = [(x, t._next_struct(x)) for x in ([t.new_next(), t.new_next()] if words else [])]
    t._turn = 0
    t._kv, t._tok, t._query = tree.KvCache(), tree.TreeTokens(), tree.TreeQuery()
    t._kv_ref, t._tok_ref, t._query_ref = (C.byref(x) for x in (t._kv, t._tok, t._query))
    t._shape_table, t._shape_page, t._shape_arena = (B, max_pages), (page_size, kv_heads, head_dim), (B, 32 * words)
    t._kv_last = t._tok_last = t._query_last = None
    t._no_stride = (0, 0, 1)
    t.out = torch.zeros(B, rows, t.heads, head_dim, dtype=torch.bfloat16)
    return t


def _advance(t, out, rows=None):
    torch, n = t.torch, t.rows if rows is None else rows
    return t.advance(torch.zeros(t.B, n, dtype=torch.int32), torch.zeros(t.B, t.rows, t.words, dtype=torch.int32),
                     torch.zeros(t.B, 32 * t.words, dtype=torch.int32), torch.zeros(t.B, dtype=torch.int32), out=out)


def test_advance_takes_outputs_that_hold_its_results():
    t = _handle()
    out = t.new_next()
    got = _advance(t, out)
    assert all(got[f].data_ptr() == out[f].data_ptr() and got[f].shape == out[f].shape for f in t.NEXT) and len(t.calls) == 1
    got = _advance(t, out, rows=3)                                    # fewer rows: the front of the tensors
    assert got["masks"].shape == (2, 3, 2) and got["slot"].shape == got["position"].shape == (2, 3) and got["masks"].is_contiguous()
    got = _advance(t, dict(masks=out["masks"]))                       # what is not wanted is left out, or None
    assert set(got) == {"masks", "slot_pos"}
    assert _advance(t, dict(out, top=None, slot=None))["top"] is None and len(t.calls) == 4
    for larger in (_handle(B=3), _handle(rows=6), _handle(words=3)):
        got = _advance(t, larger.new_next())
        assert all(got[f].shape == out[f].shape and got[f].is_contiguous() for f in t.NEXT)


@pytest.mark.parametrize("change", [
    lambda t, o: _handle(B=1).new_next(), lambda t, o: _handle(words=1).new_next(), lambda t, o: _handle(rows=3).new_next(),
    lambda t, o: setattr(t, "_dev", 0) or o, lambda t, o: {f: x for f, x in o.items() if f != "masks"}, lambda t, o: dict(o, masks=None),
    *[(lambda t, o, f=f: dict(o, **{f: o[f].long()})) for f in tree.TokenTree.NEXT],
    *[(lambda t, o, f=f: dict(o, **{f: o[f].flatten()[:-1]})) for f in tree.TokenTree.NEXT],
    *[(lambda t, o, f=f: dict(o, **{f: o[f].repeat_interleave(2, -1)[..., ::2]})) for f in tree.TokenTree.NEXT]])
def test_advance_refuses_outputs_that_do_not_hold_its_results(change):
    t = _handle()
    with pytest.raises(ValueError, match="out:"):
        _advance(t, change(t, t.new_next()))
    assert not t.calls


def test_a_cache_with_layers_is_refused_whatever_was_called_before():
    t = _handle()
    torch = t.torch
    k, v = (torch.zeros(3, 16, 16, 2, 64, dtype=torch.bfloat16) for _ in range(2))
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    table, ctx = i32(2, 8), i32(2)
    new, q = torch.zeros(8, 2, 64, dtype=torch.bfloat16), torch.zeros(2, 4, 4, 64, dtype=torch.bfloat16)
    for _ in range(2):
        for call in (lambda: t.append(new, new, k, v, table, i32(8)), lambda: t.attend(q, k, v, table, ctx)):
            with pytest.raises(ValueError):
                call()
        assert not t.calls
        t.commit(k, v, table, ctx, i32(2, 64), i32(2))
        assert t._kv.layers == 3 and t._kv.layer_stride == 16 * 16 * 2 * 64 and t._kv.num_pages == 16 and len(t.calls) == 1
        t.calls.clear()
    t.attend(q, k[1], v[1], table, ctx)
    assert t._kv.layers == 1 and t._kv.k == k[1].data_ptr() and len(t.calls) == 1


def test_advance_from_a_part_of_its_own_masks_uses_the_other_set():
    t = _handle(B=1)
    torch, i32 = t.torch, lambda *s: t.torch.zeros(*s, dtype=t.torch.int32)  # noqa: E731
    masks, seen = i32(1, 4, 2), []
    for _ in range(5):
        got = t.advance(i32(1, 4), masks, i32(1, 64), i32(1))
        lo, hi = got["masks"].data_ptr(), got["masks"].data_ptr() + 4 * got["masks"].numel()
        assert masks.data_ptr() + 4 * masks.numel() <= lo or hi <= masks.data_ptr()
        masks = got["masks"][:, 2:]
        assert masks.is_contiguous()
        seen.append(lo)
    first = t.advance(i32(1, 4), i32(1, 4, 2), i32(1, 64), i32(1))["masks"]      # from others' masks: the sets in turn
    again = t.advance(i32(1, 4), i32(1, 4, 2), i32(1, 64), i32(1))["masks"]
    part = t.advance(i32(1, 4), first[:, 2:], i32(1, 64), i32(1))["masks"]        # its turn would be the set that is read
    assert first.data_ptr() != again.data_ptr() == part.data_ptr()


def test_a_handle_without_an_arena_refuses_the_tree():
    t = _handle(words=0)
    i32 = lambda *s: t.torch.zeros(*s, dtype=t.torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="arena"):
        t.advance(i32(2, 4), i32(2, 4, 0), i32(2, 0), i32(2))
    assert not t.calls
