"""The largest numbers that the token tree's operators for long and shared texts take: texts of 2^31 - 2 tokens (on pages that stand in a table many times),
and as many to keep."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_tree_gpu import DT, _tree, dba                                          # noqa: E402,F401
from tests.test_tree_long_gpu import _i32                                               # noqa: E402

PS, PAGES = 1549411, 1386
N = PS * PAGES


@pytest.fixture(autouse=True)
def room(dba):
    assert N == 2 ** 31 - 2
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,D", [("bf16", 8), ("f32", 4)])
def test_a_prefix_of_the_largest_length(dba, dtype, D):
    tree = _tree(dba, 2, 1, 1, 1, D, PS, 1, 0, dtype, prefixes=1)
    k, v = torch.zeros(1, PS, 1, D, dtype=DT[dtype], device="cuda"), torch.ones(1, PS, 1, D, dtype=DT[dtype], device="cuda")
    q, lse = torch.ones(2, 1, 1, D, dtype=DT[dtype], device="cuda"), torch.zeros(2, 1, 1, device="cuda")
    prefix = (_i32([0, 2]), _i32([N]), torch.zeros(1, PAGES, dtype=torch.int32, device="cuda"))
    out = tree.attend_shared(q, k, v, torch.zeros(2, 1, dtype=torch.int32, device="cuda"), _i32([0, 3]), prefix, lse=lse)
    assert tree.status() == 0
    # all scores 0 and all values 1: sums of at most 2^31, a hundred or so pieces of them below 2^24, where fp32 counts exactly
    assert torch.allclose(out.float(), torch.ones_like(out.float()), rtol=2.0 ** -8 if dtype == "bf16" else 1e-4, atol=0)
    assert torch.allclose(lse, torch.full_like(lse, math.log(N)), rtol=0, atol=1e-4)


@pytest.mark.parametrize("dtype,D", [("bf16", 8), ("f32", 4)])
def test_weights_of_a_text_of_the_largest_length(dba, dtype, D):
    tree = _tree(dba, 1, 1, 1, 1, D, PS, PAGES, 0, dtype)
    k, w = torch.zeros(1, PS, 1, D, dtype=DT[dtype], device="cuda"), torch.full((1, 1, N), 4.0, device="cuda")
    q, lse = torch.ones(1, 1, 1, D, dtype=DT[dtype], device="cuda"), torch.zeros(1, 1, 1, device="cuda")
    tree.weigh(q, k, torch.zeros(1, PAGES, dtype=torch.int32, device="cuda"), _i32([N]), lse, weight=w, decay=0.5)
    assert tree.status() == 0 and float(w.min()) == 3.0 == float(w.max())


def test_an_eviction_from_a_text_of_the_largest_length(dba):
    tree = _tree(dba, 1, 1, 1, 1, 8, PS, PAGES, 0)
    k = torch.zeros(2, PS, 1, 8, dtype=torch.bfloat16, device="cuda")
    k[0] = (torch.arange(PS, device="cuda") % 251).bfloat16()[:, None, None]
    v = -k
    w = torch.zeros(1, 1, N, device="cuda")
    stay = [7, 1 << 30, N - 10, N - 3, N - 1]
    for p, x in zip(stay, (3.0, 2.0, 4.0, 5.0, 0.0)):
        w[0, 0, p] = x
    got = tree.evict(k, v, torch.zeros(1, PAGES, dtype=torch.int32, device="cuda"), _i32([N]), w, 5, recent=1, table_out=torch.ones(1, PAGES, dtype=torch.int32, device="cuda"))
    assert tree.status() == 0 and got["kept"].flatten().tolist() == stay and got["ctx_len"].tolist() == [5] and got["dropped"].tolist() == [N - 5]
    assert w[0, 0, :5].tolist() == [3.0, 2.0, 4.0, 5.0, 0.0] and float(w[0, 0, 5:].max()) == 0.0 == float(w[0, 0, 5:].min())
    want = torch.tensor([p % PS % 251 for p in stay], device="cuda").bfloat16()
    assert torch.equal(k[1, :5, 0], want[:, None].expand(5, 8)) and torch.equal(v[1, :5, 0], -want[:, None].expand(5, 8))
    assert (k[1, 5:] == 0).all()


def test_an_eviction_that_keeps_the_largest_number(dba):
    tree = _tree(dba, 1, 1, 1, 1, 8, 16, 8, 0)
    k = torch.randn(8, 16, 1, 8, device="cuda").bfloat16()
    old, w = k.clone(), torch.rand(1, 1, 128, device="cuda")
    before = w.clone()
    got = tree.evict(k, k.clone(), torch.arange(8, dtype=torch.int32, device="cuda")[None], _i32([100]), w, 2 ** 31 - 1, recent=2 ** 31 - 1)
    kept = got["kept"].flatten()
    assert tree.status() == 0 and kept[:100].tolist() == list(range(100)) and int(kept[100:].max()) == -1 == int(kept[100:].min())
    assert torch.equal(k, old) and torch.equal(w, before) and got["ctx_len"].tolist() == [100] and got["dropped"].tolist() == [0]
