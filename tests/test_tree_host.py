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
