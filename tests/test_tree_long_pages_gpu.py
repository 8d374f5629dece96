"""Eviction of context tokens to tables whose pages differ from the own ones in the arena too."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests import long_model as L                                                       # noqa: E402
from tests.test_tree_gpu import DT, _cache, _tree, dba                                  # noqa: E402,F401
from tests.test_tree_long_gpu import _i32                                               # noqa: E402


def _arena(k, table, A, ps):
    """The arena's rows [layers, B, A, heads, D]."""
    p = torch.arange(A, device=k.device)
    return k[:, table.long()[:, p // ps], p % ps]


@pytest.mark.parametrize("dtype,D,ps,W,ctx,keep,changed", [
    ("bf16", 64, 64, 1, [200, 90, 20], 50, "all"), ("bf16", 64, 64, 1, [200, 90, 20], 50, "last"),       # the arena ends inside a page
    ("bf16", 128, 5, 2, [700, 0, 300], 290, "all"), ("bf16", 128, 5, 2, [700, 0, 300], 290, "some"),
    ("f32", 64, 16, 9, [100, 100, 31], 31, "all"), ("bf16", 64, 16, 2, [300, 3, 290], 280, "some"), ("bf16", 80, 7, 1, [100, 50, 20], 40, "last")])
def test_eviction_takes_arena_slots_along_where_their_pages_change(dba, dtype, D, ps, W, ctx, keep, changed):
    rng = torch.Generator().manual_seed(ps)
    layers, B, K, A = 2, len(ctx), 2, 32 * W
    per, first = -(-(A + max(ctx)) // ps), A // ps
    pages = 2 * B * per + 2
    k, v = (torch.randn(layers, pages, ps, K, D, generator=rng).to(DT[dtype]).cuda() for _ in range(2))
    order = torch.randperm(pages, generator=rng).int().cuda()
    table, out = order[:B * per].view(B, per), order[B * per:2 * B * per].view(B, per).clone()
    if changed == "last":                                       # of the arena's pages the one in which it ends
        out[:, :first] = table[:, :first]
    elif changed == "some":
        out[:, 1::2] = table[:, 1::2]
    tree = _tree(dba, B, 1, K, K, D, ps, per, W, dtype)
    w = torch.rand(layers, B, K, per * ps - A, generator=rng).cuda()
    old_k, old_v, old_w = k.clone(), v.clone(), w.clone()
    got = tree.evict(k, v, table, _i32(ctx), w, keep, recent=3, table_out=out)
    assert tree.status() == 0
    assert torch.equal(_arena(k, out, A, ps), _arena(old_k, table, A, ps)) and torch.equal(_arena(v, out, A, ps), _arena(old_v, table, A, ps))
    for layer in range(layers):
        for b in range(B):
            for h in range(K):
                stay = L.keep(old_w[layer, b, h, :ctx[b]].tolist(), keep, 3)
                assert got["kept"][layer, b, h].tolist() == stay + [-1] * (keep - len(stay))
                src, dst = (torch.tensor(x, device="cuda", dtype=torch.long) + A for x in (stay, range(len(stay))))
                for x, old in ((k, old_k), (v, old_v)):
                    assert torch.equal(x[layer, out[b].long()[dst // ps], dst % ps, h], old[layer, table[b].long()[src // ps], src % ps, h])
    # pages that neither table names are as they were
    rest = order[2 * B * per:].long()
    assert torch.equal(k[:, rest], old_k[:, rest]) and torch.equal(v[:, rest], old_v[:, rest])


def test_arena_pages_outside_the_cache_are_nobodys_concern(dba):
    """Whether slots are in use is not known to an eviction: those without a page are neither copied nor reported."""
    rng = torch.Generator().manual_seed(1)
    k, v, table = _cache(rng, 2, 8, 16, 2, 64, "bf16", spare=20)
    tree = _tree(dba, 2, 1, 2, 2, 64, 16, 8, 1)
    out = table.clone()
    table[0, 0], out[0, 0], out[1, 0], out[1, 1] = -1, 5, -1, 1 << 30
    old = k.clone()
    tree.evict(k, v, table, _i32([20, 90]), torch.rand(2, 2, 96, generator=rng).cuda(), 90, table_out=out)
    assert tree.status() == 0 and torch.equal(k, old)


def test_a_recorded_eviction_goes_on_where_later_ones_keep_other_numbers(dba):
    rng = torch.Generator().manual_seed(3)
    side = torch.cuda.Stream()
    k, v, table = _cache(rng, 2, 8, 16, 2, 64, "bf16")
    tree = _tree(dba, 2, 1, 2, 2, 64, 16, 8, 0, stream=side)
    n, w, out_w = _i32([128, 100]), torch.rand(2, 2, 128, generator=rng).cuda(), torch.zeros(2, 2, 128, device="cuda")
    out = table.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        tree.evict(k.clone(), v.clone(), table, n, w, 50, recent=5, table_out=out, weight_out=out_w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = tree.evict(k, v, table, n, w, 50, recent=5, table_out=out, weight_out=out_w)
    others = []
    with torch.cuda.stream(side):
        for keep in (10, 70, 127, 50):
            tree.evict(k.clone(), v.clone(), table, n, w, keep, table_out=out, weight_out=out_w)
            others += [torch.full((size,), 12345, dtype=torch.int32, device="cuda") for size in (2, 4, 2 * 2 * 2 * 10, 2 * 2 * 2 * 50, 2 * 2 * 2 * 70)]
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert all((x == 12345).all() for x in others)
    assert got["ctx_len"].tolist() == [50, 50] and got["dropped"].tolist() == [78, 50]
    for b, c in enumerate((128, 100)):
        for h in range(2):
            assert got["kept"][b, h].tolist() == L.keep(w[b, h, :c].tolist(), 50, 5)


@pytest.mark.parametrize("ps,keep", [(16, 12), (5, 3)])
def test_tokens_that_settle_after_an_eviction_come_in_order(dba, ps, keep):
    """An open tree's positions count the context before them: an eviction lowers them, or its later tokens would settle before its earlier ones."""
    rng = torch.Generator().manual_seed(1)
    B, W, A = 2, 1, 32
    per = -(-(A + 60) // ps)
    k, v, table = _cache(rng, B, per, ps, 1, 64, "bf16")
    tree = _tree(dba, B, 2, 1, 1, 64, ps, per, W)
    w, slot_pos = torch.rand(B, 1, per * ps - A, generator=rng).cuda(), torch.zeros(B, A, dtype=torch.int32, device="cuda")
    nx = tree.advance(_i32([[0, 0], [0, 0]]), torch.zeros(B, 1, W, dtype=torch.int32, device="cuda"), slot_pos, _i32([24, 2]))
    first = nx["slot"].clone()
    nx = {key: x.clone() for key, x in nx.items() if key != "slot_pos"}
    before = slot_pos.clone()
    got = tree.evict(k, v, table, nx["ctx_len"], w, keep, slot_pos=slot_pos)
    assert got["dropped"].tolist() == [24 - keep, 0] and torch.equal(slot_pos, before - got["dropped"][:, None])
    nx = tree.advance(_i32([[0, 1], [0, 1]]), nx["masks"], slot_pos, got["ctx_len"].clone())
    assert nx["commit_n"].tolist() == [0, 0] and nx["position"].tolist() == [[keep + 1] * 2, [3, 3]]
    second = nx["slot"].clone()
    lengths = nx["ctx_len"].clone()
    nx = tree.advance(_i32([[1, 1], [1, 1]]), nx["masks"].clone(), slot_pos, lengths)
    assert nx["commit_n"].tolist() == [2, 2]
    assert nx["commit_src"][:, :2].tolist() == [[int(first[b, 1]), int(second[b, 1])] for b in range(B)]
    assert tree.status() == 0
