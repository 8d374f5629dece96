"""Attention over shared prefixes where the two streams of a block have the same rows and tiles in turn: many short items in every order to a block,
so that a stage of the copies goes from one stream to the other."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_tree_gpu import dba                                                     # noqa: E402,F401
from tests.test_tree_long_gpu import _attend, _compare, _setup                          # noqa: E402


@pytest.mark.parametrize("D,ps", [(64, 16), (64, 5), (128, 64), (128, 7)])
@pytest.mark.parametrize("tiles", [(3,), (1, 3), (1, 2, 3, 4, 5)])
def test_items_of_few_tiles_one_after_another(dba, D, ps, tiles):
    groups, K, rows = 300, 3, 2
    rng = torch.Generator().manual_seed(len(tiles))
    length = [128 * (tiles[i % len(tiles)] - 1) + 1 + int(torch.randint(0, 128, (1,), generator=rng)) for i in range(groups)]
    s = _setup(dba, 7, groups, rows, 2 * K, K, D, [i % 20 for i in range(groups)], ps, 1, "bf16", list(range(groups + 1)), length)
    got, lse = _attend(s, 0.2)
    _compare(s, got, lse, 0.2)
    for _ in range(5):
        again, lse2 = _attend(s, 0.2, out=torch.empty_like(got))
        assert torch.equal(got, again) and torch.equal(lse, lse2)
    assert s["tree"].status() == 0


@pytest.mark.parametrize("D,ps", [(64, 16), (128, 64)])
def test_items_of_few_rows_among_items_of_many(dba, D, ps):
    """Blocks that go from items whose rows both streams have to items of 256 rows and back."""
    first, length, rng = [0], [], torch.Generator().manual_seed(1)
    for i in range(60):
        first.append(first[-1] + (1 + i % 9))
        length.append(1 + int(torch.randint(0, 640, (1,), generator=rng)))
    B = first[-1]
    s = _setup(dba, 8, B, 10, 8, 2, D, [i % 20 for i in range(B)], ps, 1, "bf16", first, length)
    got, lse = _attend(s, 0.2)
    _compare(s, got, lse, 0.2)
    for _ in range(5):
        again, lse2 = _attend(s, 0.2, out=torch.empty_like(got))
        assert torch.equal(got, again) and torch.equal(lse, lse2)
    assert s["tree"].status() == 0
