"""Evictions that keep different numbers of tokens on one handle, on the host (no GPU needed)."""
import pytest

from paper_1804_06609_b200 import tree
from tests.test_tree_long_host import _i32, _kv, _long_handle

torch = pytest.importorskip("torch")


def _handle(monkeypatch):
    """A handle whose evictions note the addresses they are given: (lengths, dropped, kept) each."""
    t, noted = _long_handle(), []
    t.stream, t._evict = None, tree.TreeEvicted()
    t._evict_ref = t._evict

    class Lib:
        @staticmethod
        def dba_tree_evict(*args):
            noted.append((args[-1].ctx_len_out, args[-1].dropped, args[-1].kept))
            return 0
    monkeypatch.setattr(tree, "lib", lambda: Lib)
    return t, noted


def _evict(t, keep, layers=3):
    shape = () if layers is None else (layers,)
    return t.evict(_kv(t, layers=layers), _kv(t, layers=layers), _i32(t.B, 8), _i32(t.B), torch.zeros(*shape, t.B, t.kv_heads, 64), keep)


def test_tensors_that_an_eviction_has_written_to_stay_the_handles(monkeypatch):
    """A recorded call (CUDA graph) goes on writing to them, so no later call may give them back."""
    t, noted = _handle(monkeypatch)
    for keep, layers in ((10, 3), (7, 3), (40, 3), (10, 3), (41, 2), (9, None), (300, 4), (40, 3), (10, 3)):
        got = _evict(t, keep, layers)
        assert got["kept"].shape == ((layers,) if layers else ()) + (t.B, t.kv_heads, keep) and got["kept"].is_contiguous()
        assert got["ctx_len"].shape == got["dropped"].shape == (t.B,)
        assert (got["ctx_len"].data_ptr(), got["dropped"].data_ptr(), got["kept"].data_ptr()) == noted[-1]
        del got
        # whatever lies at those addresses is still theirs: new tensors of any size get others
        new = [torch.empty(n, dtype=torch.int32) for n in (4, 8, 2 * 3 * 4 * 10, 2 * 3 * 4 * 7, 2 * 3 * 4 * 40)]
        mine = {a for call in noted for a in call}
        assert not any(x.data_ptr() <= a < x.data_ptr() + 4 * x.numel() for x in new for a in mine)


def test_evictions_of_one_kind_take_turns(monkeypatch):
    t, noted = _handle(monkeypatch)
    for _ in range(4):
        _evict(t, 12)
    assert noted[0] == noted[2] and noted[1] == noted[3] and not set(noted[0]) & set(noted[1])
    results = [_evict(t, keep) for keep in (12, 30)]       # one after the other: the first one's results are still there
    spans = [[(x.data_ptr(), x.data_ptr() + 4 * x.numel()) for x in (r["ctx_len"], r["dropped"], r["kept"])] for r in results]
    assert all(b <= c or d <= a for a, b in spans[0] for c, d in spans[1])


def test_many_numbers_to_keep_do_not_pile_up(monkeypatch):
    t, noted = _handle(monkeypatch)
    for keep in list(range(1, 300)) + list(range(300, 0, -1)):
        _evict(t, keep)
    assert len({call[2] for call in noted}) <= 24          # twice, for each doubling


def test_positions_that_an_eviction_refuses(monkeypatch):
    t, noted = _handle(monkeypatch)
    evict = lambda slot_pos: t.evict(_kv(t), _kv(t), _i32(2, 8), _i32(2), torch.zeros(2, 2, 64), 10, slot_pos=slot_pos)  # noqa: E731
    for bad in (_i32(2, 63), _i32(1, 64), _i32(2, 64).long(), _i32(64, 2).t(), _i32(128)):
        with pytest.raises(ValueError):
            evict(bad)
    assert not noted
    evict(_i32(2, 64))
    assert t._evict.slot_pos_stride == 64
    evict(_i32(2, 100)[:, :64])
    assert t._evict.slot_pos_stride == 100
    evict(None)
    assert t._evict.slot_pos is None and len(noted) == 3
