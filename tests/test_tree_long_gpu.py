"""The token tree's operators for long and shared texts on the GPU, against plain 64-bit models (tests/long_model.py)."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests import long_model as L                                     # noqa: E402
from tests import tree_model as M                                     # noqa: E402
from tests.test_tree_gpu import DT, _cache, _masks, _top, _tree, dba  # noqa: E402,F401


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------------ attention over shared prefixes
def _setup(dba, seed, B, n, H, K, D, ctx, ps, W, dtype, first, length, hnd=False, density=0.3, closed=0.1, qscale=1.0, more_pages=1):
    rng = torch.Generator().manual_seed(seed)
    A = 32 * W
    per = -(-(A + max(ctx + [1])) // ps)
    pre = -(-max(length + [1]) // ps) + more_pages
    groups = len(length)
    pages = B * per + groups * pre + 3
    shape = (pages, K, ps, D) if hnd else (pages, ps, K, D)
    k, v = (torch.randn(shape, generator=rng).to(DT[dtype]).cuda() for _ in range(2))
    if hnd:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    order = torch.randperm(pages, generator=rng).int()
    table, ptable = order[:B * per].view(B, per).cuda(), order[B * per:B * per + groups * pre].view(groups, pre).cuda()
    masks = _masks(rng, B, n, W, density, closed) if W else None
    q = (torch.randn(B, n, H, D, generator=rng) * qscale).to(DT[dtype]).cuda()
    tree = _tree(dba, B, n, H, K, D, ps, per, W, dtype, prefixes=max(groups, 1))
    return dict(tree=tree, q=q, k=k, v=v, table=table, ptable=ptable, masks=masks, ctx=ctx, first=first, length=length, ps=ps, W=W, D=D, dtype=dtype)


def _attend(s, scale, lse=True, top=None, out=None):
    B, n, H, _ = s["q"].shape
    lse = torch.full((B, n, H), 7.0, device="cuda") if lse else None
    masks = None if s["masks"] is None else s["masks"].cuda()
    out = s["tree"].attend_shared(s["q"], s["k"], s["v"], s["table"], _i32(s["ctx"]), (_i32(s["first"]), _i32(s["length"]), s["ptable"]), masks=masks,
                                  top=top, scale=scale, lse=lse, out=out)
    return out, lse


def _compare(s, got, lse, scale, first=None):
    want = L.attend_shared(s["q"], s["k"], s["v"], s["table"], s["ctx"], s["masks"], scale, s["ps"], s["W"], first or s["first"], s["length"], s["ptable"])
    out, wlse, spread, reach, seen = want
    tol, ltol = L.shared_tolerance(out, wlse, spread, reach, seen, s["D"], DT[s["dtype"]])
    assert not torch.isnan(got).any()
    err = (got.double().cpu() - out).abs()
    assert (err <= tol).all(), f"worst {float((err / tol).max()):.3f} of the bound"
    if lse is not None:
        lse = lse.double().cpu()
        assert torch.equal(torch.isinf(lse), torch.isinf(wlse))
        live = ~torch.isinf(wlse)
        assert ((lse - wlse).abs()[live] <= ltol[live]).all()


SHARED = [  # B, n, H, K, D, context lengths, page size, words, dtype, first, prefix lengths, heads outside tokens
    (1, 1, 1, 1, 64, [0], 16, 1, "bf16", [0, 1], [1], False),
    (2, 5, 16, 16, 64, [10, 3], 16, 1, "bf16", [0, 2], [50], False),
    (3, 20, 8, 2, 128, [30, 0, 127], 64, 2, "bf16", [0, 3], [129], True),
    (6, 20, 4, 1, 64, [5, 40, 0, 9, 1, 12], 16, 1, "bf16", [0, 2, 2, 5], [300, 77, 128], False),      # a prefix without sequences, a sequence without one
    (5, 3, 6, 6, 96, [4, 4, 4, 4, 4], 24, 1, "bf16", [1, 3, 5], [0, 257], True),                      # an empty prefix
    (8, 1, 8, 1, 128, [20] * 8, 64, 1, "bf16", [0, 8], [3001], False),                                 # few rows, a long prefix
    (9, 16, 8, 2, 80, [33] * 9, 5, 1, "bf16", [0, 9], [640], False),                                   # 576 rows: whole blocks and a rest of 64
    (3, 43, 3, 1, 64, [8, 0, 70], 1, 2, "bf16", [0, 1, 3], [255, 256], False),                         # 129 and 258 rows
    (2, 64, 16, 2, 128, [100, 200], 128, 2, "bf16", [0, 2], [1024], True),                             # 1024 rows
    (4, 2, 4, 2, 8, [6, 0, 1, 2], 16, 1, "bf16", [0, 4], [70], False),
    (4, 2, 4, 2, 72, [6, 0, 1, 2], 7, 1, "bf16", [0, 4], [135], False),
    (3, 7, 8, 2, 256, [20, 1, 0], 16, 1, "bf16", [0, 3], [200], False),
    (2, 5, 8, 8, 64, [10, 3], 16, 1, "f32", [0, 2], [50], False),
    (3, 20, 8, 2, 128, [30, 0, 127], 16, 2, "f32", [0, 1, 3], [333, 64], True),
    (4, 1, 4, 1, 68, [20] * 4, 16, 1, "f32", [0, 4], [2000], False),
    (2, 9, 4, 1, 256, [20, 4], 16, 1, "f32", [0, 2], [150], False),
    (4, 6, 4, 4, 4, [3, 3, 3, 3], 16, 0, "f32", [0, 4], [20], False),                                   # no arena
    (4, 6, 4, 4, 64, [3, 0, 0, 3], 16, 0, "bf16", [0, 3], [20], False),                                 # no arena, nothing of its own
]


@pytest.mark.parametrize("case", range(len(SHARED)))
def test_attention_over_shared_prefixes(dba, case):
    B, n, H, K, D, ctx, ps, W, dtype, first, length, hnd = SHARED[case]
    s = _setup(dba, case, B, n, H, K, D, ctx, ps, W, dtype, first, length, hnd)
    got, lse = _attend(s, D ** -0.5)
    _compare(s, got, lse, D ** -0.5)
    assert s["tree"].status() == 0
    # the same call again, and without the log-sum-exps: the same bits
    again, _ = _attend(s, D ** -0.5, lse=False, out=torch.empty_like(got))
    assert torch.equal(got, again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale,qscale", [(1.0, 6.0), (-0.3, 2.0), (0.0, 1.0)])
def test_shared_scores_far_apart_of_either_sign_and_alike(dba, dtype, scale, qscale):
    s = _setup(dba, 5, 4, 10, 8, 2, 64, [100, 0, 3, 50], 16, 1, dtype, [0, 3], [700], qscale=qscale)
    got, lse = _attend(s, scale)
    _compare(s, got, lse, scale)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64), ("bf16", 160)])
def test_shared_rows_that_are_closed_hold_anything(dba, dtype, D):
    s = _setup(dba, 6, 5, 6, 4, 2, D, [9, 0, 30, 2, 2], 16, 1, dtype, [0, 2, 4], [40, 200], closed=0.5)
    closed = torch.tensor([[not M.bits_of(s["masks"][b, i].numpy()) for i in range(6)] for b in range(5)], device="cuda")
    assert closed.any() and not closed.all()
    clean = s["q"].clone()
    s["q"][closed] = math.nan
    got, lse = _attend(s, 0.2)
    assert (got[closed] == 0).all() and (lse[closed] == -math.inf).all()
    s["q"] = clean
    _compare(s, got, lse, 0.2)


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f32", 64)])
def test_shared_what_is_behind_the_prefix_is_not_read(dba, dtype, D):
    s = _setup(dba, 7, 3, 4, 4, 4, D, [9, 0, 30], 16, 1, dtype, [0, 3], [75])
    for p in range(75, s["ptable"].shape[1] * 16):
        page, row = int(s["ptable"][0, p // 16]), p % 16
        s["k"][page, row], s["v"][page, row] = math.nan, math.inf
    s["ptable"][0, -1] = 1 << 30                                   # an entry that no token needs
    got, lse = _attend(s, 0.2)
    _compare(s, got, lse, 0.2)
    assert s["tree"].status() == 0


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f32", 64), ("bf16", 128)])
def test_shared_pages_outside_the_cache_count_as_absent(dba, dtype, D):
    s = _setup(dba, 8, 3, 4, 4, 2, D, [9, 0, 30], 16, 1, dtype, [0, 1, 3], [200, 170])
    s["ptable"][0, 2], s["ptable"][1, 0], s["ptable"][1, 5] = -1, s["k"].shape[0], 1 << 30
    got, lse = _attend(s, 0.2)
    _compare(s, got, lse, 0.2)
    assert s["tree"].status() == dba.TREE_BAD_PAGE


def test_shared_prefixes_out_of_range_are_reported(dba):
    s = _setup(dba, 9, 4, 2, 4, 2, 64, [9, 0, 30, 1], 16, 1, "bf16", [0, 2, 4], [20, 30])
    for first, length in (([0, 5, 4], [20, 30]), ([-1, 2, 4], [20, 30]), ([0, 3, 2], [20, 30]), ([0, 2, 4], [20, 1 << 20]), ([0, 2, 4], [-5, 30])):
        s["first"], s["length"] = first, length
        _attend(s, 0.2)
        assert s["tree"].status() == dba.TREE_BAD_INDEX
    s["first"], s["length"] = [0, 2, 4], [20, 30]
    got, lse = _attend(s, 0.2)
    _compare(s, got, lse, 0.2)
    assert s["tree"].status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_shared_fewer_rows_strided_queries_and_outputs_on_another_stream(dba, dtype):
    rng = torch.Generator().manual_seed(3)
    B, H, K, D = 4, 8, 2, 64
    side = torch.cuda.Stream()
    s = _setup(dba, 10, B, 5, H, K, D, [9, 0, 30, 4], 16, 1, dtype, [0, 4], [333])
    s["tree"] = _tree(dba, B, 12, H, K, D, 16, s["table"].shape[1], 1, dtype, prefixes=3, stream=side)
    wide = torch.randn(B, 5, H, 3 * D, generator=rng).to(DT[dtype]).cuda()
    s["q"] = wide[..., D:2 * D]
    out = torch.zeros(B, H, 5, 2 * D, dtype=DT[dtype], device="cuda").transpose(1, 2)[..., :D]
    torch.cuda.synchronize()
    got, lse = _attend(s, 0.2, out=out)
    side.synchronize()
    _compare(s, got, lse, 0.2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_shared_calls_recorded_in_a_graph(dba, dtype):
    s = _setup(dba, 11, 6, 4, 8, 2, 64, [9, 0, 30, 4, 1, 2], 16, 1, dtype, [0, 6], [500])
    side = torch.cuda.Stream()
    s["tree"] = _tree(dba, 6, 4, 8, 2, 64, 16, s["table"].shape[1], 1, dtype, prefixes=1, stream=side)
    ctx, first, length, masks = _i32(s["ctx"]), _i32(s["first"]), _i32(s["length"]), s["masks"].cuda()
    lse = torch.zeros(6, 4, 8, device="cuda")
    call = lambda: s["tree"].attend_shared(s["q"], s["k"], s["v"], s["table"], ctx, (first, length, s["ptable"]), masks=masks, scale=0.2, lse=lse)  # noqa: E731
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = call()
    for length_now, ctx_now in ([500], s["ctx"]), ([37], [1, 2, 3, 4, 5, 6]):
        s["length"], s["ctx"] = length_now, ctx_now
        length.copy_(_i32(length_now)); ctx.copy_(_i32(ctx_now))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        _compare(s, out, lse, 0.2)


def test_shared_agrees_with_a_context_of_its_own(dba):
    """Each sequence with the prefix at the front of its own context: the same attention."""
    s = _setup(dba, 12, 4, 20, 8, 2, 128, [40, 0, 9, 17], 16, 1, "bf16", [0, 4], [400])
    got, lse = _attend(s, 0.1)
    A, ps, B = 32, 16, 4
    per = -(-(A + 440) // ps)
    k, v = (torch.zeros(B * per, ps, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.arange(B * per, device="cuda").int().view(B, per)
    for b in range(B):
        at = [(int(s["table"][b, p // ps]), p % ps) for p in range(A)] + [(int(s["ptable"][0, p // ps]), p % ps) for p in range(400)] + \
             [(int(s["table"][b, (A + p) // ps]), (A + p) % ps) for p in range(s["ctx"][b])]
        for i, (page, row) in enumerate(at):
            k[int(table[b, i // ps]), i % ps], v[int(table[b, i // ps]), i % ps] = s["k"][page, row], s["v"][page, row]
    tree = _tree(dba, B, 20, 8, 2, 128, ps, per, 1)
    lse2 = torch.zeros_like(lse)
    want = tree.attend(s["q"], k, v, table, _i32([400 + c for c in s["ctx"]]), masks=s["masks"].cuda(), scale=0.1, lse=lse2)
    assert torch.allclose(lse, lse2, atol=2e-5)
    # each side: probabilities and result rounded, and the own part here; values up to 4
    assert (got.float() - want.float()).abs().max() < 4 * 5 * 2.0 ** -8


# ------------------------------------------------------------------------------------------------ append with norms
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype,D,rot", [("bf16", 64, 64), ("bf16", 128, 128), ("bf16", 128, 64), ("bf16", 80, 80), ("bf16", 96, 32), ("bf16", 8, 2), ("bf16", 72, 34),
                                         ("bf16", 256, 256), ("bf16", 256, 250), ("bf16", 256, 252), ("f32", 64, 64), ("f32", 128, 96), ("f32", 4, 4), ("f32", 256, 256),
                                         ("f32", 256, 126), ("f32", 12, 6), ("f32", 132, 132)])
def test_append_with_norms(dba, dtype, D, rot, pairs):
    rng = torch.Generator().manual_seed(D + rot)
    B, H, K, ps, W, N = 3, 6, 2, 7, 1, 12
    per = -(-(32 + 20) // ps)
    k, v, table = _cache(rng, B, per, ps, K, D, dtype)
    tree = _tree(dba, B, 4, H, K, D, ps, per, W, dtype)
    q, new_k, new_v = ((torch.randn(N, heads, D, generator=rng) * 3).to(DT[dtype]).cuda() for heads in (H, K, K))
    place = torch.stack([torch.randperm(50, generator=rng)[:4] for _ in range(B)]).flatten().int()
    place[5] = -1
    position = torch.randint(0, 90, (N,), generator=rng).int()
    position[2] = -1
    offset = [0, 9, 5]
    angle = torch.arange(100)[:, None] * 0.3 ** torch.arange(rot // 2)
    cos, sin = angle.cos().float().contiguous().cuda(), angle.sin().float().contiguous().cuda()
    qw, kw = (1 + 0.3 * torch.randn(D, generator=rng)).cuda(), (1 + 0.3 * torch.randn(D, generator=rng)).cuda()
    old_k, old_v = k.clone(), v.clone()
    q_out = tree.append(new_k, new_v, k, v, table, place.cuda(), position.cuda(), rotary=(cos, sin), pairs=pairs, q=q, norm=(qw, kw, 1e-5), offset=_i32(offset))
    assert tree.status() == 0
    at = torch.where(position >= 0, position + torch.tensor(offset).repeat_interleave(4), -1).long()
    c, z = cos.cpu().double()[at.clamp(min=0)], sin.cpu().double()[at.clamp(min=0)]
    c[at < 0], z[at < 0] = 1.0, 0.0
    for x, w, got in ((q, qw, q_out), (new_k, kw, None)):
        y = L.norm(x.cpu(), w.cpu(), 1e-5)
        want = M.rotate(y, c, z, pairs)
        size = M.rotate(y.abs(), c.abs(), -z.abs(), pairs).abs() + M.rotate(y.abs(), c.abs(), z.abs(), pairs).abs()
        tol = size * (D / 2 + 16) * 2.0 ** -24 + want.abs() * torch.finfo(DT[dtype]).eps / 2 * 1.01 + 1e-30
        if got is None:
            want_k, tol_k = want, tol
        else:
            assert ((got.cpu().double() - want).abs() <= tol).all()
    stored = torch.zeros(k.shape[:2], dtype=torch.bool)
    for t in range(N):
        p = int(place[t])
        if p < 0:
            continue
        page, row = int(table[t // 4, p // ps]), p % ps
        stored[page, row] = True
        assert ((k[page, row].cpu().double() - want_k[t]).abs() <= tol_k[t]).all()
        assert torch.equal(v[page, row], new_v[t])
    assert torch.equal(k.cpu()[~stored], old_k.cpu()[~stored]) and torch.equal(v.cpu()[~stored], old_v.cpu()[~stored])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_with_norms_of_one_side_in_place_and_without_a_rotation(dba, dtype):
    rng = torch.Generator().manual_seed(2)
    B, H, K, D, N = 2, 5, 1, 64, 2050                            # more tokens than a step's, one key head
    k, v, table = _cache(rng, B, 80, 16, K, D, dtype)
    tree = _tree(dba, B, 4, H, K, D, 16, 80, 1, dtype)
    q, new_k, new_v = (torch.randn(N, heads, D, generator=rng).to(DT[dtype]).cuda() for heads in (H, K, K))
    clean = q.clone()
    w = (1 + 0.3 * torch.randn(D, generator=rng)).cuda()
    place = (32 + torch.arange(N) % (N // 2)).int().cuda()
    got = tree.append(new_k, new_v, k, v, table, place, q=q, q_out=q, norm=(w, None, 0.0))
    assert got is q and tree.status() == 0
    want = L.norm(clean.cpu(), w.cpu(), 0.0)
    assert ((got.cpu().double() - want).abs() <= want.abs() * ((D / 2 + 8) * 2.0 ** -24 + torch.finfo(DT[dtype]).eps / 2 * 1.01) + 1e-30).all()
    at = table[(torch.arange(N) // (N // 2)).cuda(), (place // 16).long()].long()
    assert torch.equal(k[at, (place % 16).long()], new_k) and torch.equal(v[at, (place % 16).long()], new_v)
    # an offset alone: dba_tree_append at other positions
    cos, sin = torch.rand(50, 32, generator=rng).cuda(), torch.rand(50, 32, generator=rng).cuda()
    position, offset = torch.randint(0, 20, (N,), generator=rng).int().cuda(), _i32([7, 29])
    a = tree.append(new_k, new_v, k, v, table, place, position, rotary=(cos, sin), q=clean, offset=offset)
    k1 = k.clone()
    b = tree.append(new_k, new_v, k, v, table, place, position + offset.repeat_interleave(N // 2), rotary=(cos, sin), q=clean)
    assert torch.equal(a, b) and torch.equal(k, k1)


def test_append_with_norms_reports_positions_and_places_out_of_range(dba):
    rng = torch.Generator().manual_seed(2)
    k, v, table = _cache(rng, 2, 8, 16, 1, 64, "bf16")
    tree = _tree(dba, 2, 4, 2, 1, 64, 16, 8, 1)
    q, new_k, new_v = (torch.randn(4, heads, 64, generator=rng).bfloat16().cuda() for heads in (2, 1, 1))
    cos, sin, w = torch.rand(20, 32).cuda(), torch.rand(20, 32).cuda(), torch.ones(64).cuda()
    call = lambda place, position, offset, seq=None: tree.append(new_k, new_v, k, v, table, _i32(place), _i32(position), rotary=(cos, sin), q=q,  # noqa: E731
                                                                norm=(w, w, 1e-6), offset=_i32(offset), seq=None if seq is None else _i32(seq))
    for bad in (([0, 1, 2, 3], [0, 1, 2, 3], [0, 17]), ([0, 1, 2, 3], [0, 1, 2, 3], [-1, 0]), ([0, 1, 2, 128], [0, 1, 2, 3], [0, 0]),
                ([0, 1, 2, 3], [0, 1, 2, 3], [(1 << 31) - 1, 0]), ([0, 1, 2, 3], [0, 1, 2, 3], [0, 0], [0, 1, 2, 1]), ([0, 1, 2, 3], [0, 1, 2, 20], [0, 0])):
        call(*bad)
        assert tree.status() == dba.TREE_BAD_INDEX
    call([0, 1, 2, 3], [0, 1, -1, 3], [16, 16])
    assert tree.status() == 0


# ------------------------------------------------------------------------------------------------ weights of context tokens
WEIGH = [  # B, n, H, K, D, context lengths, page size, words, dtype, decay, heads outside tokens
    (1, 1, 1, 1, 64, [1], 16, 0, "bf16", 1.0, False),
    (2, 5, 16, 16, 64, [37, 0], 16, 2, "bf16", 1.0, False),
    (3, 20, 8, 2, 128, [128, 129, 127], 64, 1, "bf16", 0.9, True),
    (2, 1, 8, 1, 128, [1000, 513], 16, 1, "bf16", 1.0, False),
    (2, 64, 16, 2, 64, [130, 70], 5, 1, "bf16", 1.0, True),                     # 512 rows
    (1, 33, 8, 1, 80, [300], 24, 1, "bf16", 0.5, False),                         # 264 rows
    (3, 7, 6, 6, 96, [40, 1, 260], 1, 0, "bf16", 1.0, False),
    (2, 3, 4, 2, 8, [40, 1], 16, 0, "bf16", 1.0, False),
    (2, 3, 4, 2, 256, [70, 1], 16, 0, "bf16", 1.0, False),
    (2, 5, 8, 8, 64, [37, 100], 16, 1, "f32", 1.0, False),
    (2, 20, 8, 2, 128, [130, 65], 16, 1, "f32", 0.9, True),
    (2, 3, 4, 1, 256, [70, 33], 16, 0, "f32", 1.0, False),
    (2, 3, 4, 1, 4, [70, 33], 16, 0, "f32", 0.0, False),
]


@pytest.mark.parametrize("case", range(len(WEIGH)))
def test_weights_of_context_tokens(dba, case):
    B, n, H, K, D, ctx, ps, W, dtype, decay, hnd = WEIGH[case]
    rng = torch.Generator().manual_seed(case)
    per = -(-(32 * W + max(ctx)) // ps)
    k, v, table = _cache(rng, B, per, ps, K, D, dtype, hnd)
    tree = _tree(dba, B, n, H, K, D, ps, per, W, dtype)
    q = torch.randn(B, n, H, D, generator=rng).to(DT[dtype]).cuda()
    lse = (math.log(max(ctx)) + 0.5 + 0.3 * torch.randn(B, n, H, generator=rng)).cuda()
    closed = torch.rand(B, n, generator=rng).cuda() < 0.2
    lse[closed] = -math.inf
    q[closed] = math.nan                                        # whatever its query holds
    cap = per * ps - 32 * W
    weight = torch.rand(B, K, cap + 3, generator=rng).cuda()
    out = torch.full_like(weight, 5.0)
    got = tree.weigh(q, k, table, _i32(ctx), lse, weight=weight, decay=decay, scale=0.2, out=out)
    assert got is out and tree.status() == 0
    want, bound = L.weigh(torch.where(closed[..., None, None], 0.0, q.float()), k, table, ctx, lse, weight, decay, 0.2, ps, W)
    for b in range(B):
        c = ctx[b]
        assert ((got[b, :, :c].double().cpu() - want[b, :, :c]).abs() <= bound[b, :, :c]).all()
        assert (got[b, :, c:] == 5.0).all()
    # in place, and from nothing
    first = got.clone()
    tree.weigh(q, k, table, _i32(ctx), lse, weight=weight, decay=decay, scale=0.2)
    new = torch.zeros_like(weight)
    tree.weigh(q, k, table, _i32(ctx), lse, scale=0.2, out=new)
    want0, bound0 = L.weigh(torch.where(closed[..., None, None], 0.0, q.float()), k, table, ctx, lse, torch.zeros_like(weight), 1.0, 0.2, ps, W)
    for b in range(B):
        assert torch.equal(weight[b, :, :ctx[b]], first[b, :, :ctx[b]])
        assert ((new[b, :, :ctx[b]].double().cpu() - want0[b, :, :ctx[b]]).abs() <= bound0[b, :, :ctx[b]]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weights_sum_to_the_rows_that_attended(dba, dtype):
    """After attend over a context alone, the weights of a (sequence, key head) add up to its rows and heads."""
    rng = torch.Generator().manual_seed(1)
    B, n, H, K, D, ctx = 3, 6, 8, 2, 64, [200, 1, 77]
    k, v, table = _cache(rng, B, 13, 16, K, D, dtype)
    tree = _tree(dba, B, n, H, K, D, 16, 13, 0, dtype)
    q = torch.randn(B, n, H, D, generator=rng).to(DT[dtype]).cuda()
    lse, w = torch.zeros(B, n, H, device="cuda"), torch.zeros(B, K, 208, device="cuda")
    tree.attend(q, k, v, table, _i32(ctx), lse=lse)
    tree.weigh(q, k, table, _i32(ctx), lse, out=w)
    assert (w.sum(-1) - n * H // K).abs().max() < 1e-3             # 24 rows, each 1 within 200 roundings of 2^-22 and the scores' errors


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f32", 64), ("bf16", 136)])
def test_weights_pages_outside_the_cache_receive_nothing(dba, dtype, D):
    rng = torch.Generator().manual_seed(1)
    k, v, table = _cache(rng, 2, 4, 16, 2, D, dtype)
    tree = _tree(dba, 2, 2, 4, 2, D, 16, 4, 0, dtype)
    table[0, 1], table[1, 0] = -1, 1 << 30
    q, lse = torch.randn(2, 2, 4, D, generator=rng).to(DT[dtype]).cuda(), torch.ones(2, 2, 4, device="cuda") * 3
    w = torch.ones(2, 2, 64, device="cuda")
    tree.weigh(q, k, table, _i32([60, 20]), lse, weight=w, decay=0.5)
    assert tree.status() == dba.TREE_BAD_PAGE
    assert (w[0, :, 16:32] == 0.5).all() and (w[1, :, :16] == 0.5).all()
    want, bound = L.weigh(q, k, table, [60, 20], lse, torch.ones(2, 2, 64), 0.5, D ** -0.5, 16, 0)
    assert ((w.double().cpu() - want).abs() <= bound)[:, :, :20].all()


# ------------------------------------------------------------------------------------------------ eviction
EVICT = [  # B, layers, K, D, context lengths, page size, words, keep, recent, dtype, heads outside tokens, where to
    (1, 1, 1, 64, [2], 16, 0, 1, 0, "bf16", False, "fresh"),
    (1, 1, 1, 64, [2], 16, 0, 1, 1, "bf16", False, "place"),
    (3, 2, 4, 64, [300, 256, 10], 16, 1, 256, 32, "bf16", False, "fresh"),
    (3, 2, 4, 64, [300, 256, 10], 16, 1, 256, 32, "bf16", False, "place"),
    (2, 1, 2, 128, [1300, 700], 5, 1, 513, 100, "bf16", True, "place"),          # the arena ends inside a page
    (2, 1, 2, 128, [1300, 700], 5, 1, 513, 100, "bf16", True, "mixed"),
    (2, 3, 2, 80, [2000, 1000], 64, 0, 700, 0, "bf16", False, "fresh"),
    (2, 3, 2, 80, [2000, 1000], 64, 0, 700, 700, "bf16", False, "place"),        # the last ones alone
    (2, 1, 3, 4, [700, 3], 1, 0, 100, 7, "f32", True, "fresh"),
    (2, 2, 1, 256, [120, 119], 24, 2, 119, 5, "f32", False, "place"),
    (4, 1, 2, 64, [0, 5, 40, 41], 16, 0, 40, 3, "f32", False, "place"),
]


def _evict_case(case, weights):
    B, layers, K, D, ctx, ps, W, keep, recent, dtype, hnd, where = EVICT[case]
    rng = torch.Generator().manual_seed(case)
    A = 32 * W
    per = -(-(A + max(ctx)) // ps)
    pages = 2 * B * per + 3
    shape = (layers, pages, K, ps, D) if hnd else (layers, pages, ps, K, D)
    k, v = (torch.randn(shape, generator=rng).to(DT[dtype]) for _ in range(2))
    if hnd:
        k, v = k.transpose(2, 3), v.transpose(2, 3)
    order = torch.randperm(pages, generator=rng).int()
    table = order[:B * per].view(B, per).clone()
    table_out = table.clone()
    if where != "place":      # the arena's pages stay (the one in which it ends too: "mixed"), the context's are others
        keep_pages = -(-A // ps)
        table_out[:, keep_pages:] = order[B * per:2 * B * per].view(B, per)[:, keep_pages:]
    cap = per * ps - A
    w = torch.rand(layers, B, K, cap + 2, generator=rng).pow(4)
    if weights == "ties":
        w = (w * 4).round() / 4
    elif weights == "odd":    # zeros of either sign, infinities, NaN, negative ones
        kind = torch.randint(0, 8, w.shape, generator=rng)
        for i, x in enumerate((0.0, -0.0, math.inf, -math.inf, math.nan, -1.5)):
            w[kind == i] = x
    elif weights == "alike":
        w.fill_(0.25)
    return B, layers, K, D, ctx, ps, W, keep, recent, dtype, where, per, k, v, table, table_out, w


@pytest.mark.parametrize("weights", ["any", "ties", "odd", "alike"])
@pytest.mark.parametrize("case", range(len(EVICT)))
def test_eviction(dba, case, weights):
    B, layers, K, D, ctx, ps, W, keep, recent, dtype, where, per, k, v, table, table_out, w = _evict_case(case, weights)
    A = 32 * W
    tree = _tree(dba, B, 1, K, K, D, ps, per, W, dtype)
    gk, gv, gw, n = k.cuda(), v.cuda(), w.cuda(), _i32(ctx)
    lone = layers == 1                                            # a cache without layers too
    one = lambda t: t[0] if lone else t                           # noqa: E731
    t0 = table.cuda()
    got = tree.evict(one(gk), one(gv), t0, n, one(gw), keep, recent=recent, table_out=None if where == "place" else table_out.cuda())
    assert tree.status() == 0
    kept = got["kept"][None] if lone else got["kept"]
    assert got["ctx_len"].tolist() == [min(c, keep) for c in ctx] and got["dropped"].tolist() == [c - min(c, keep) for c in ctx]
    want_k, want_v, want_w = k.clone(), v.clone(), w.clone()
    for layer in range(layers):
        for b in range(B):
            for h in range(K):
                stay = L.keep(w[layer, b, h, :ctx[b]].tolist(), keep, recent)
                assert kept[layer, b, h].tolist() == stay + [-1] * (keep - len(stay))
                want_w[layer, b, h, :ctx[b]] = 0.0
                want_w[layer, b, h, :len(stay)] = w[layer, b, h, torch.tensor(stay, dtype=torch.long)]
                if stay:
                    src, dst = torch.tensor(stay) + A, torch.arange(len(stay)) + A
                    a, z = table[b].long()[src // ps], table_out[b].long()[dst // ps]
                    want_k[layer, z, dst % ps, h], want_v[layer, z, dst % ps, h] = k[layer, a, src % ps, h], v[layer, a, src % ps, h]
    assert torch.equal(gk.cpu(), want_k) and torch.equal(gv.cpu(), want_v)
    assert torch.equal(gw.cpu().view(torch.int32), want_w.view(torch.int32))
    assert torch.equal(n.cpu(), torch.tensor(ctx, dtype=torch.int32))


def test_eviction_into_other_weights_and_pages_outside_the_cache(dba):
    B, layers, K, D, ctx, ps, W, keep, recent, dtype, where, per, k, v, table, table_out, w = _evict_case(2, "any")
    tree = _tree(dba, B, 1, K, K, D, ps, per, W, dtype)
    gk, gv, gw, out = k.cuda(), v.cuda(), w.cuda(), torch.full_like(w, 9.0).cuda()
    bad = table_out.cuda()
    bad[0, 3], bad[1, 4] = -1, 1 << 30
    got = tree.evict(gk, gv, table.cuda(), _i32(ctx), gw, keep, recent=recent, table_out=bad, weight_out=out)
    assert tree.status() == dba.TREE_BAD_PAGE and got["weight"] is out
    assert torch.equal(gw.cpu(), w)
    for b in range(B):
        assert (out[:, b, :, ctx[b]:] == 9.0).all() and (out[:, b, :, min(ctx[b], keep):ctx[b]] == 0.0).all()
    # pages that no row went to are as they were
    used = torch.zeros(k.shape[1], dtype=torch.bool)
    used[table_out[:, 2:].flatten().long()] = True
    assert torch.equal(gk.cpu()[:, ~used], k[:, ~used])


def test_a_captured_eviction_follows_the_lengths(dba):
    rng = torch.Generator().manual_seed(1)
    k, v, table = _cache(rng, 2, 8, 16, 2, 64, "bf16")
    side = torch.cuda.Stream()
    tree = _tree(dba, 2, 1, 2, 2, 64, 16, 8, 0, stream=side)
    n, w = _i32([128, 100]), torch.rand(2, 2, 128, generator=rng).cuda()
    out_table = table.clone()
    out_w = torch.zeros_like(w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = tree.evict(k, v, table, n, w, 50, recent=5, table_out=out_table, weight_out=out_w)
    for lens in ([128, 100], [60, 40]):
        w.copy_(torch.rand(2, 2, 128, generator=rng))
        n.copy_(_i32(lens))
        torch.cuda.synchronize()
        before = k.clone()
        graph.replay()
        torch.cuda.synchronize()
        assert got["ctx_len"].tolist() == [min(x, 50) for x in lens]
        for b in range(2):
            for h in range(2):
                stay = L.keep(w[b, h, :lens[b]].tolist(), 50, 5)
                src, dst = torch.tensor(stay, device="cuda"), torch.arange(len(stay), device="cuda")
                assert torch.equal(k[table[b].long()[dst // 16], dst % 16, h], before[table[b].long()[src // 16], src % 16, h])
