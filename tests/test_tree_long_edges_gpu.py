"""The token tree's operators for long and shared texts where ordinary calls seldom go: waits that run out, scores that grow, many small sequences,
caches of more than 2^31 elements, long rows of weights; and a run of all of them together."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests import long_model as L                                                       # noqa: E402
from tests import tree_model as M                                                       # noqa: E402
from tests.test_tree_gpu import DT, _cache, _tree, dba                                  # noqa: E402,F401
from tests.test_tree_long_gpu import _attend, _compare, _i32, _setup                    # noqa: E402


@pytest.mark.parametrize("D,ps,length", [(64, 16, 300), (128, 16, 40), (128, 5, 300), (64, 64, 64), (64, 7, 5)])
def test_a_wait_that_runs_out_in_attention_over_a_shared_prefix(dba, D, ps, length):
    s = _setup(dba, 1, 4, 6, 4, 2, D, [20, 3, 0, 40], ps, 1, "bf16", [0, 4], [length], closed=0.0, more_pages=0)
    want, want_lse = (x.clone() for x in _attend(s, 0.2))
    s["tree"].test_hook(wait_clocks=2_000_000, drop_item=0)
    got, lse = _attend(s, 0.2)
    assert torch.isnan(got).all() and torch.isnan(lse).all()
    assert s["tree"].status() & dba.TREE_TIMEOUT
    s["tree"].test_hook()
    got, lse = _attend(s, 0.2)
    assert torch.equal(got, want) and torch.equal(lse, want_lse) and s["tree"].status() == 0


@pytest.mark.parametrize("D,ps", [(64, 16), (128, 5)])
def test_a_wait_that_runs_out_while_weighing(dba, D, ps):
    rng = torch.Generator().manual_seed(1)
    k, v, table = _cache(rng, 3, -(-300 // ps), ps, 2, D, "bf16")
    tree = _tree(dba, 3, 4, 4, 2, D, ps, table.shape[1], 0)
    q, lse = torch.randn(3, 4, 4, D, generator=rng).bfloat16().cuda(), torch.full((3, 4, 4), 5.0, device="cuda")
    ctx, w = _i32([300, 10, 129]), torch.zeros(3, 2, table.shape[1] * ps, device="cuda")
    want = tree.weigh(q, k, table, ctx, lse, out=w).clone()
    tree.test_hook(wait_clocks=2_000_000, drop_item=0)
    tree.weigh(q, k, table, ctx, lse, out=w)
    assert tree.status() == dba.TREE_TIMEOUT
    assert all(torch.isnan(w[b, :, :c]).all() and (w[b, :, c:] == 0).all() for b, c in enumerate((300, 10, 129)))
    tree.test_hook()
    assert torch.equal(tree.weigh(q, k, table, ctx, lse, out=w), want) and tree.status() == 0


@pytest.mark.parametrize("dtype,D,ps", [("bf16", 64, 16), ("bf16", 128, 32), ("bf16", 128, 5), ("f32", 64, 16)])
@pytest.mark.parametrize("rows,grow", [(20, 0.05), (3, 0.3), (20, -0.3)])
def test_shared_scores_that_grow_along_the_prefix(dba, dtype, D, ps, rows, grow):
    """A row's maximum rises again and again (or never does), by much more than what leaves its reference where it is."""
    B, H, K, n = 6, 4, 1, 700
    s = _setup(dba, 2, B, rows, H, K, D, [5, 0, 9, 1, 1, 40], ps, 1, dtype, [0, B], [n])
    u = torch.zeros(D)
    u[::2] = 1.0
    s["q"] = (s["q"].cpu() * 0.1 + u).to(DT[dtype]).cuda()
    for p in range(n):
        page, row = int(s["ptable"][0, p // ps]), p % ps
        s["k"][page, row] = (s["k"][page, row].float() * 0.3 + (u * (p * grow) / (D / 2)).cuda()).to(DT[dtype])
    got, lse = _attend(s, 1.0)
    _compare(s, got, lse, 1.0)


def test_shared_many_prefixes_of_few_rows(dba):
    B, groups = 40, 25
    rng = torch.Generator().manual_seed(1)
    cut = sorted(torch.randint(0, B + 1, (groups - 1,), generator=rng).tolist())
    lengths = torch.randint(0, 400, (groups,), generator=rng).tolist()
    for D, ps in ((64, 16), (128, 24), (64, 3)):
        s = _setup(dba, 3, B, 3, 6, 3, D, torch.randint(0, 30, (B,), generator=rng).tolist(), ps, 1, "bf16", [0] + cut + [B - 2], lengths)
        got, lse = _attend(s, 0.2)
        _compare(s, got, lse, 0.2)
        again, _ = _attend(s, 0.2, out=torch.empty_like(got))
        assert torch.equal(got, again)


@pytest.mark.parametrize("D,ps", [(64, 16), (128, 8), (64, 3)])
@pytest.mark.parametrize("rows,heads", [(1, 3), (9, 6), (50, 24)])          # 1, 18 and 400 queries to a key head
def test_weights_of_many_small_sequences(dba, D, ps, rows, heads):
    rng = torch.Generator().manual_seed(rows)
    B, K = 45, 3
    ctx = torch.randint(0, 300, (B,), generator=rng).tolist()
    ctx[3], ctx[7], ctx[11] = 128, 256, 1
    per = -(-300 // ps)
    k, v, table = _cache(rng, B, per, ps, K, D, "bf16")
    tree = _tree(dba, B, rows, heads, K, D, ps, per, 0)
    q = torch.randn(B, rows, heads, D, generator=rng).bfloat16().cuda()
    lse = (4.5 + 0.3 * torch.randn(B, rows, heads, generator=rng)).cuda()
    lse[torch.rand(B, rows, heads, generator=rng).cuda() < 0.1] = -math.inf
    w = torch.rand(B, K, per * ps, generator=rng).cuda()
    want, bound = L.weigh(q, k, table, ctx, lse, w, 0.5, 0.1, ps, 0)
    for _ in range(3):
        out = torch.zeros_like(w)
        tree.weigh(q, k, table, _i32(ctx), lse, weight=w, decay=0.5, scale=0.1, out=out)
        for b in range(B):
            assert ((out[b, :, :ctx[b]].double().cpu() - want[b, :, :ctx[b]]).abs() <= bound[b, :, :ctx[b]]).all()
            assert (out[b, :, ctx[b]:] == 0).all()
    assert tree.status() == 0


@pytest.mark.parametrize("ps", [16, 5])
def test_offsets_beyond_two_to_the_31(dba, ps):
    """The same pages at the front of a small cache and at the end of one of more than 2^31 elements: the same bits."""
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 30 GB")
    K, D, B, pre, per = 8, 128, 3, -(-300 // ps), -(-(32 + 200) // ps)
    used = B * per + pre + B * per
    pages = (1 << 31) // (ps * K * D) + used + 1
    rng = torch.Generator(device="cuda").manual_seed(1)
    small = [torch.randn(used, ps, K, D, generator=rng, device="cuda").bfloat16() for _ in range(2)]
    ctx, masks = _i32([200, 0, 150]), torch.tensor([[[7], [1], [0]]] * B, dtype=torch.int32, device="cuda")
    q = torch.randn(B, 3, 16, D, generator=rng, device="cuda").bfloat16()
    weight = torch.rand(B, K, per * ps - 32, generator=rng, device="cuda")
    answers = []
    for far in (False, True):
        first = pages - used if far else 0
        if far:
            k, v = (torch.zeros(pages, ps, K, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            k[first:], v[first:] = small
        else:
            k, v = (x.clone() for x in small)
        ids = torch.randperm(used, generator=torch.Generator().manual_seed(2)).int().cuda() + first
        table, ptable, table_out = ids[:B * per].view(B, per).contiguous(), ids[B * per:B * per + pre].view(1, pre), ids[B * per + pre:].view(B, per).contiguous()
        table_out[:, :-(-32 // ps)] = table[:, :-(-32 // ps)]              # (the arena stays where it is)
        tree = _tree(dba, B, 3, 16, K, D, ps, per, 1, prefixes=1)
        lse, w = torch.zeros(B, 3, 16, device="cuda"), weight.clone()
        out = tree.attend_shared(q, k, v, table, ctx, (_i32([0, B]), _i32([300]), ptable), masks=masks, lse=lse).clone()
        tree.weigh(q, k, table, ctx, lse, weight=w)
        got = tree.evict(k, v, table, ctx, w, 77, recent=10, table_out=table_out)
        kept = [k[first:].clone(), v[first:].clone()] if far else [k, v]
        assert tree.status() == 0
        answers.append([out, lse, w, got["kept"], got["ctx_len"]] + kept)
        del k, v
        torch.cuda.empty_cache()
    assert all(torch.equal(a, b) for a, b in zip(*answers))


@pytest.mark.parametrize("n,keep,recent", [(60000, 30001, 500), (9000, 17, 0), (49153, 49152, 49152), (3000, 1500, 7)])
@pytest.mark.parametrize("weights", ["any", "ties", "nothing"])
def test_eviction_from_long_rows(dba, n, keep, recent, weights):
    rng = torch.Generator().manual_seed(n)
    ps, D = 64, 8
    per = -(-n // ps)
    k, v, table = _cache(rng, 1, per, ps, 2, D, "bf16")
    tree = _tree(dba, 1, 1, 2, 2, D, ps, per, 0)
    w = torch.rand(1, 2, per * ps, generator=rng).pow(3)
    if weights == "ties":
        w = (w * 50).floor() / 50
    elif weights == "nothing":
        w.zero_()
    old = [k.clone(), v.clone()]
    got = tree.evict(k, v, table, _i32([n]), w.cuda(), keep, recent=recent)
    for h in range(2):
        stay = L.keep(w[0, h, :n].tolist(), keep, recent)
        assert got["kept"][0, h].tolist() == stay
        src, dst = torch.tensor(stay, device="cuda"), torch.arange(keep, device="cuda")
        for x, o in zip((k, v), old):
            assert torch.equal(x[table[0].long()[dst // ps], dst % ps, h], o[table[0].long()[src // ps], src % ps, h])
    assert tree.status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_run_of_them_together(dba, dtype):
    """Prompts after a prefix, with norms: appended, attended, weighed, thinned, and a next token on what is left; every stage against its model."""
    rng = torch.Generator().manual_seed(4)
    B, H, K, D, ps, W, P = 3, 8, 2, 64, 16, 1, 75
    scale, keep, recent, A = D ** -0.5, 20, 4, 32
    lens = [40, 17, 33]
    per, pre = -(-(A + 48) // ps), -(-P // ps)
    shape = (B * per + pre, ps, K, D)
    k, v = (torch.zeros(shape, dtype=DT[dtype], device="cuda") for _ in range(2))
    table, ptable = torch.arange(B * per).int().view(B, per).cuda(), torch.arange(B * per, B * per + pre).int().view(1, pre).cuda()
    angle = torch.arange(200)[:, None] * 0.7 ** torch.arange(D // 2)
    rotary = tuple(x.float().contiguous().cuda() for x in (angle.cos(), angle.sin()))
    qw, kw = (1 + 0.3 * torch.randn(D, generator=rng)).cuda(), (1 + 0.3 * torch.randn(D, generator=rng)).cuda()
    norm = (qw, kw, 1e-5)
    draw = lambda n, h: torch.randn(n, h, D, generator=rng).to(DT[dtype]).cuda()  # noqa: E731

    # the prefix, at its own places: a tree of one sequence without an arena
    one = _tree(dba, 1, 4, H, K, D, ps, pre, 0, dtype)
    one.append(draw(P, K), draw(P, K), k, v, ptable, torch.arange(P).int().cuda(), torch.arange(P).int().cuda(), rotary=rotary, norm=norm)
    tree = _tree(dba, B, 1, H, K, D, ps, per, W, dtype, prefixes=1)
    seq = torch.cat([torch.full((n,), b) for b, n in enumerate(lens)]).int().cuda()
    place = torch.cat([A + torch.arange(n) for n in lens]).int().cuda()
    position, offset = place - A, _i32([P] * B)
    new_k, new_v = draw(sum(lens), K), draw(sum(lens), K)
    tree.append(new_k, new_v, k, v, table, place, position, rotary=rotary, norm=norm, offset=offset, seq=seq)
    at = (position.cpu() + P).long()
    want = M.rotate(L.norm(new_k.cpu(), kw.cpu(), 1e-5), rotary[0].cpu().double()[at], rotary[1].cpu().double()[at], False)
    stored = k[table[seq.long(), (place // ps).long()].long(), (place % ps).long()].cpu().double()
    assert ((stored - want).abs() <= 3 * (1 + want.abs()) * (torch.finfo(DT[dtype]).eps / 2 + 2.0 ** -19)).all()

    prefix, ctx, weight = (_i32([0, B]), _i32([P]), ptable), _i32(lens), torch.zeros(B, K, per * ps - A, device="cuda")
    masks = torch.zeros(B, 1, W, dtype=torch.int32, device="cuda")
    for step in range(3):
        # a token of each sequence, in slot `step` of the arena; what went before it there is seen too
        masks |= 1 << step
        slots, now = _i32([step] * B), ctx + step
        q = tree.append(draw(B, K), draw(B, K), k, v, table, slots, now, rotary=rotary, norm=norm, offset=offset, q=draw(B, H)).view(B, 1, H, D)
        lse = torch.zeros(B, 1, H, device="cuda")
        out = tree.attend_shared(q, k, v, table, ctx, prefix, masks=masks, lse=lse)
        s = dict(q=q, k=k, v=v, table=table, ctx=ctx.tolist(), masks=masks.cpu(), ps=ps, W=W, D=D, dtype=dtype, first=[0, B], length=[P], ptable=ptable)
        _compare(s, out, lse, scale)
        before = weight.clone()
        tree.weigh(q, k, table, ctx, lse, weight=weight)
        want, bound = L.weigh(q, k, table, ctx.tolist(), lse, before, 1.0, scale, ps, W)
        assert ((weight.double().cpu() - want).abs() <= bound).all()
        old_k, old_w, was = k.clone(), weight.clone(), ctx.tolist()
        got = tree.evict(k, v, table, ctx, weight, keep, recent=recent)
        for b in range(B):
            for h in range(K):
                stay = L.keep(old_w[b, h, :was[b]].tolist(), keep, recent)
                src, dst = A + torch.tensor(stay, device="cuda"), A + torch.arange(len(stay), device="cuda")
                assert torch.equal(k[table[b].long()[dst // ps], dst % ps, h], old_k[table[b].long()[src // ps], src % ps, h])
        offset += got["dropped"]
        ctx = got["ctx_len"]
        assert (ctx + offset).tolist() == [n + P for n in lens] and max(ctx.tolist()) == keep
    assert tree.status() == 0 and one.status() == 0
