"""Weights whose rows overlap, on the host (no GPU needed)."""
import pytest

from paper_1804_06609_b200 import binding
from tests.test_tree_long_host import _i32, _kv, _long_handle

torch = pytest.importorskip("torch")


def _weigh(t, w, out=None):
    q, lse = torch.zeros(t.B, 3, 4, 64, dtype=torch.bfloat16), torch.zeros(t.B, 3, 4)
    t.weigh(q, _kv(t), _i32(t.B, 8), _i32(t.B), lse, weight=w, out=out)


def test_weights_whose_rows_overlap_are_refused():
    t, flat = _long_handle(), torch.zeros(4000)                       # 2 sequences, 2 key heads, 64 places
    for strides in ((1, 128, 1), (128, 1, 1), (64, 64, 1), (127, 64, 1), (128, 63, 1), (100, 60, 1)):
        w = flat.as_strided((2, 2, 64), strides)
        with pytest.raises(ValueError):
            _weigh(t, w)
        with pytest.raises(ValueError):
            _weigh(t, None, out=w)
        with pytest.raises(ValueError):
            t.evict(_kv(t), _kv(t), _i32(2, 8), _i32(2), w, 10)
    for strides in ((64, 128, 1), (128, 64, 1), (500, 70, 1), (70, 500, 1), (64, 1000, 1)):
        with pytest.raises(binding.DbaError):                         # (past the binding: there is no handle behind it)
            _weigh(t, flat.as_strided((2, 2, 64), strides))
    with pytest.raises(binding.DbaError):                             # places beyond the context's are nobody's: rows may share them
        _weigh(t, flat.as_strided((2, 2, 80), (128, 64, 1)))
    # rows that lie between one another's without touching
    t = _long_handle(B=3)
    w = flat.as_strided((3, 2, 64), (150, 225, 1))                    # 0, 150, 300 and 225, 375, 525
    with pytest.raises(binding.DbaError):
        _weigh(t, w)


def test_weights_of_layers_whose_rows_overlap_are_refused():
    t, flat = _long_handle(), torch.zeros(4000)
    k = _kv(t, layers=3)
    for strides in ((64, 128, 64, 1), (255, 128, 64, 1), (1, 128, 64, 1), (256, 128, 32, 1)):
        with pytest.raises(ValueError):
            t.evict(k, k, _i32(2, 8), _i32(2), flat.as_strided((3, 2, 2, 64), strides), 10)
