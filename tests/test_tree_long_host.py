"""What the token tree's operators for long and shared texts refuse on the host (no GPU needed), and their plain models."""
import ctypes as C
import math

import pytest

from paper_1804_06609_b200 import binding, tree
from tests.test_tree_host import INVALID, _handle

torch = pytest.importorskip("torch")


def test_calls_without_a_handle_are_refused():
    L = binding.lib()
    n = C.c_size_t()
    assert L.dba_tree_shared_bytes(None, C.byref(n)) == INVALID
    assert L.dba_tree_attend_shared(None, None, None, None, 0, None, None, None, None, None, 0) == INVALID
    assert L.dba_tree_append_norm(None, None, None, None, None, 0) == INVALID
    assert L.dba_tree_weigh(None, None, None, None, None, 0, None, None, None, 0, 0, 1.0) == INVALID
    assert L.dba_tree_evict(None, None, None, 0, None, None) == INVALID


def _long_handle(**kw):
    t = _handle(**kw)
    t.prefixes, t._prefix, t._norm = 2, tree.TreePrefix(), tree.TreeNorm()
    t._prefix_ref, t._norm_ref = C.byref(t._prefix), C.byref(t._norm)
    t._query_last = t._kv_last = t._tok_last = None
    t._shape_table, t._shape_page = (t.B, t.max_pages), (t.page_size, t.kv_heads, t.head_dim)
    t._no_stride = (0, 0, 1)
    t._call_shared = lambda *a: t.calls.append(("shared", a)) or 0
    return t


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def _kv(t, pages=20, layers=None):
    shape = (pages, t.page_size, t.kv_heads, t.head_dim)
    return torch.zeros(shape if layers is None else (layers,) + shape, dtype=torch.bfloat16)


def test_prefixes_that_are_refused():
    t = _long_handle()
    q, k, table, n = torch.zeros(2, 4, 4, 64, dtype=torch.bfloat16), _kv(t), _i32(2, 8), _i32(2)
    out = torch.empty_like(q)
    call = lambda prefix: t.attend_shared(q, k, k, table, n, prefix, out=out)  # noqa: E731
    call((_i32(3), _i32(2), _i32(2, 5)))
    call((_i32(2), _i32(1), _i32(1, 5)))
    assert len(t.calls) == 2 and (t._prefix.groups, t._prefix.max_pages, t._prefix.table_stride) == (1, 5, 5)
    for bad in ((_i32(2), _i32(2), _i32(2, 5)), (_i32(4), _i32(3), _i32(3, 5)), (_i32(1), _i32(0), _i32(0, 5)), (_i32(3), _i32(2), _i32(1, 5)),
                (_i32(3).long(), _i32(2), _i32(2, 5)), (_i32(3), _i32(2).float(), _i32(2, 5)), (_i32(3), _i32(2), _i32(2, 5).long()),
                (_i32(3), _i32(2), _i32(5, 2).t()), (_i32(6)[::2], _i32(2), _i32(2, 5)), (_i32(3), _i32(2), _i32(2, 0)), (_i32(3), _i32(2), _i32(2, 5, 1))):
        with pytest.raises(ValueError):
            call(bad)
    t.prefixes = 0
    with pytest.raises(ValueError):
        call((_i32(3), _i32(2), _i32(2, 5)))
    assert len(t.calls) == 2


def test_norms_that_are_refused():
    t = _long_handle()
    N, k, table, place = 4, _kv(t), _i32(2, 8), _i32(4)
    new, w = torch.zeros(N, 2, 64, dtype=torch.bfloat16), torch.ones(64)
    for bad in ((w.bfloat16(), w, 1e-6), (w[:32], w, 1e-6), (w, torch.ones(128)[::2], 1e-6), (w, w[None], 1e-6)):
        with pytest.raises(ValueError):
            t.append(new, new, k, k, table, place, norm=bad)
    with pytest.raises(ValueError):
        t.append(new, new, k, k, table, place, norm=(w, w, 1e-6), offset=_i32(3))
    with pytest.raises(ValueError):
        t.append(new, new, k, k, table, place, offset=_i32(2).long())
    with pytest.raises(binding.DbaError):                            # (past the binding: there is no handle behind it)
        t.append(new, new, k, k, table, place, norm=(w, None, 1e-6), offset=_i32(2))


def test_weights_that_are_refused():
    t = _long_handle()
    q, k, table, n, lse = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16), _kv(t), _i32(2, 8), _i32(2), torch.zeros(2, 3, 4)
    w = torch.zeros(2, 2, 64)                                          # 8 pages of 16 less 64 slots
    bad = [dict(weight=None), dict(weight=w[..., :63]), dict(weight=w.double()), dict(weight=w[:1]), dict(weight=torch.zeros(2, 64, 2).transpose(1, 2)),
           dict(weight=w, out=torch.zeros(2, 2, 80)), dict(weight=w, q=q.float()), dict(weight=w, q=q[:1]), dict(weight=w, q=q[:, :, :2]),
           dict(weight=w, lse=lse[:, :2]), dict(weight=w, lse=lse.double()), dict(weight=w, n=_i32(3)), dict(weight=w, table=_i32(2, 7))]
    for kw in bad:
        a = dict(q=q, n=n, lse=lse, table=table, out=None)
        a.update(kw)
        with pytest.raises(ValueError):
            t.weigh(a["q"], k, a["table"], a["n"], a["lse"], weight=a["weight"], out=a["out"])
    with pytest.raises(binding.DbaError):
        t.weigh(q, k, table, n, lse, weight=w)


def test_evictions_that_are_refused():
    t = _long_handle()
    k, table, n = _kv(t, layers=3), _i32(2, 8), _i32(2)
    w = torch.zeros(3, 2, 2, 64)
    for kw in (dict(keep=0), dict(keep=5, recent=6), dict(keep=5, recent=-1), dict(weight=w[:2]), dict(weight=w[0]), dict(weight=w.bfloat16()),
               dict(weight_out=torch.zeros(3, 2, 2, 70)), dict(table_out=_i32(2, 7)), dict(table_out=table.long()), dict(k=_kv(t)), dict(n=_i32(1)),
               dict(k=_kv(t, layers=3)[None])):
        a = dict(k=k, n=n, weight=w, keep=10, recent=2, weight_out=None, table_out=None)
        a.update(kw)
        with pytest.raises(ValueError):
            t.evict(a["k"], a["k"], table, a["n"], a["weight"], a["keep"], recent=a["recent"], table_out=a["table_out"], weight_out=a["weight_out"])


def test_which_tokens_the_plain_model_keeps():
    from tests.long_model import keep
    assert keep([1, 2], 3, 0) == [0, 1] and keep([1.0, 3.0, 2.0, 0.0], 2, 0) == [1, 2]
    assert keep([1.0, 3.0, 2.0, 0.0], 2, 1) == [1, 3] and keep([1.0, 3.0, 2.0, 0.0], 2, 2) == [2, 3]
    assert keep([0.0, -0.0, 0.0, 0.0], 2, 0) == [0, 1]
    assert keep([math.nan, -math.inf, math.nan, 1.0], 3, 0) == [0, 1, 3]
