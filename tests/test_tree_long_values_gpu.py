"""Values that are not finite, and zeros of either sign, in the token tree's operators for long and shared texts."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests import long_model as L                                                       # noqa: E402
from tests import tree_model as M                                                       # noqa: E402
from tests.test_tree_gpu import DT, _cache, _tree, dba                                  # noqa: E402,F401
from tests.test_tree_long_gpu import _attend, _i32, _setup                              # noqa: E402

# the places of a tile's columns: eight neighbours at its front, in its second half, in the next tile and in the last one
PLACES = [*range(8), *range(70, 78), *range(130, 138), *range(292, 300)]


@pytest.mark.parametrize("kind", ["nan", "+inf", "-inf"])
@pytest.mark.parametrize("dtype,D,ps,rows,G", [("bf16", 64, 16, 3, 2), ("bf16", 64, 5, 3, 2), ("bf16", 64, 16, 50, 4), ("bf16", 128, 32, 3, 2), ("bf16", 128, 32, 50, 4),
                                               ("bf16", 128, 7, 50, 4), ("bf16", 256, 16, 3, 2), ("f32", 64, 16, 3, 2), ("f32", 128, 16, 20, 4)])
def test_prefix_keys_that_are_not_finite(dba, dtype, D, ps, rows, G, kind):
    """A score of NaN or +inf makes NaN of its row's output and log-sum-exp, wherever in a prefix the key stands; one of -inf is a key that is not seen."""
    B, K = len(PLACES), 2
    s = _setup(dba, 3, B, rows, K * G, K, D, [(7 * i) % 40 for i in range(B)], ps, 2, dtype, list(range(B + 1)), [300] * B)
    q = s["q"].float()
    q[..., 3] = (q[..., 3].abs() + 0.5) * (-1 if kind == "-inf" else 1)
    s["q"] = q.to(DT[dtype])
    plain = s["k"].clone()                                      # (-inf: a score so far below the others that its exponential is 0)
    for g, p in enumerate(PLACES):
        page, row = int(s["ptable"][g, p // ps]), p % ps
        s["k"][page, row, 1, 3] = math.nan if kind == "nan" else math.inf
        plain[page, row, 1, 3] = 4096.0
    got, lse = _attend(s, 0.2)
    assert s["tree"].status() == 0
    got, lse = got.double().cpu().view(B, rows, K, G, D), lse.double().cpu().view(B, rows, K, G)
    want = L.attend_shared(s["q"], plain, s["v"], s["table"], s["ctx"], s["masks"], 0.2, ps, 2, s["first"], s["length"], s["ptable"])
    tol, ltol = L.shared_tolerance(*want, D, DT[dtype])
    closed = torch.isinf(want[1]).view(B, rows, K, G)
    if kind != "-inf":                                          # the second key head's open rows
        spoilt = ~closed
        spoilt[:, :, 0] = False
        assert torch.isnan(got[spoilt]).all() and torch.isnan(lse[spoilt]).all()
    else:
        spoilt = torch.zeros_like(closed)
    out, wlse = want[0].view(got.shape), want[1].view(lse.shape)
    assert ((got - out).abs() <= tol.view(got.shape))[~spoilt].all()
    assert torch.equal(torch.isinf(lse[~spoilt]), closed[~spoilt]) and ((lse - wlse).abs() <= ltol.view(lse.shape))[~spoilt & ~closed].all()


@pytest.mark.parametrize("kind", [math.nan, math.inf])
@pytest.mark.parametrize("dtype,D,rows", [("bf16", 64, 3), ("bf16", 128, 50), ("f32", 64, 3)])
def test_prefix_keys_that_are_not_finite_where_several_blocks_have_a_row(dba, dtype, D, rows, kind):
    B, K, G, ps, n = 4, 1, 4, 16, 3001
    s = _setup(dba, 4, B, rows, K * G, K, D, [30] * B, ps, 2, dtype, [0, B], [n], closed=0.0)
    s["q"][..., 3] = s["q"][..., 3].abs() + 0.5
    clean = s["k"].clone()
    for p in range(1500, 1508):
        s["k"].copy_(clean)
        s["k"][int(s["ptable"][0, p // ps]), p % ps, 0, 3] = kind
        got, lse = _attend(s, 0.2)
        assert torch.isnan(got).all() and torch.isnan(lse).all()
    s["k"].copy_(clean)
    got, lse = _attend(s, 0.2)
    assert torch.isfinite(got).all() and torch.isfinite(lse).all()

# ------------------------------------------------------------------------------------------------ append
def _bits(x):
    return x.contiguous().view(torch.int32 if x.dtype == torch.float32 else torch.int16)


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("H,K", [(4, 2), (45, 15), (7, 1)])
@pytest.mark.parametrize("dtype,D,rot", [("bf16", 64, 32), ("bf16", 128, 64), ("bf16", 72, 34), ("bf16", 8, 2), ("bf16", 256, 252), ("f32", 64, 32), ("f32", 12, 6), ("f32", 256, 126)])
def test_dimensions_that_are_not_rotated_keep_to_themselves(dba, dtype, D, rot, H, K, pairs):
    """Without norms they are copies, as dba_tree_append's; with norms no dimension's value is another's."""
    rng = torch.Generator().manual_seed(D + rot)
    B, ps, N = 2, 16, 40
    k, v, table = _cache(rng, B, 8, ps, K, D, dtype)
    tree = _tree(dba, B, 4, H, K, D, ps, 8, 1, dtype)
    q, new_k, new_v = (torch.randn(N, heads, D, generator=rng) for heads in (H, K, K))
    position = torch.arange(N, dtype=torch.int32) % 20
    position[::5] = -1                                          # these have no rotation at all
    for x in (q, new_k):
        for t in range(N):
            lo = 0 if t % 5 == 0 else rot
            for j, y in enumerate((math.inf, -math.inf, math.nan, -0.0)):
                x[t, :, lo + (7 * t + 3 * j) % (D - lo)] = y
    q, new_k, new_v = (x.to(DT[dtype]).cuda() for x in (q, new_k, new_v))
    cos, sin = torch.rand(50, rot // 2, generator=rng).cuda(), torch.rand(50, rot // 2, generator=rng).cuda()
    place, offset = (32 + torch.arange(N) % (N // 2)).int().cuda(), _i32([7, 29])
    at = table[(torch.arange(N) // (N // 2)).cuda(), (place // ps).long()].long(), (place % ps).long()
    moved = torch.where(position >= 0, position + offset.cpu().repeat_interleave(N // 2), position).int().cuda()
    call = lambda pos, **kw: (tree.append(new_k, new_v, k, v, table, place, pos, rotary=(cos, sin), pairs=pairs, q=q, q_out=torch.empty_like(q), **kw), k[at])  # noqa: E731
    want = call(moved)
    for got in (call(position.cuda(), offset=offset), call(moved, norm=(None, None, 0.0))):
        assert all(torch.equal(_bits(a), _bits(b)) for a, b in zip(got, want))
    # one side normed: the other one as before
    w = (1 + 0.3 * torch.randn(D, generator=rng)).cuda()
    assert torch.equal(_bits(call(moved, norm=(w, None, 1e-5))[1]), _bits(want[1])) and torch.equal(_bits(call(moved, norm=(None, w, 1e-5))[0]), _bits(want[0]))
    # normed: an infinite value takes the others of its head to zero, and is NaN itself
    q = torch.randn(N, H, D, generator=rng)
    q[::5, :, 1], q[1::5, :, D - 1] = math.inf, -math.inf
    q = q.to(DT[dtype]).cuda()
    got = call(moved, norm=(w, w, 1e-5))[0].cpu()
    for first, d, lo in ((0, 1, 0), (1, D - 1, rot)):
        others = [i for i in range(lo, D) if i != d]
        assert torch.isnan(got[first::5, :, d]).all() and (got[first::5][:, :, others] == 0).all()
    assert tree.status() == 0


def test_an_offset_alone_reports_positions_out_of_range(dba):
    rng = torch.Generator().manual_seed(2)
    k, v, table = _cache(rng, 2, 8, 16, 1, 64, "bf16")
    tree = _tree(dba, 2, 4, 2, 1, 64, 16, 8, 1)
    q, new_k, new_v = (torch.randn(4, heads, 64, generator=rng).bfloat16().cuda() for heads in (2, 1, 1))
    cos, sin = torch.rand(20, 32).cuda(), torch.rand(20, 32).cuda()
    call = lambda position, offset: tree.append(new_k, new_v, k, v, table, _i32([0, 1, 2, 3]), _i32(position), rotary=(cos, sin), q=q, offset=_i32(offset))  # noqa: E731
    for position, offset in (([0, 1, 2, 3], [0, 17]), ([0, 1, 2, 3], [-1, 0]), ([0, 1, 2, 3], [(1 << 31) - 1, 0]), ([0, 1, 2, (1 << 31) - 1], [0, 1]), ([0, 1, 2, 20], [0, 0])):
        call(position, offset)
        assert tree.status() == dba.TREE_BAD_INDEX
    call([0, 1, -1, 3], [18, 16])
    assert tree.status() == 0


@pytest.mark.parametrize("dtype,D,rot,N", [("bf16", 128, 128, 24), ("bf16", 64, 32, 2050), ("f32", 128, 96, 24), ("f32", 64, 64, 2050), ("bf16", 256, 250, 24)])
def test_heads_whose_squares_sum_to_about_the_largest_number(dba, dtype, D, rot, N):
    """Whether a head's sum of squares is finite is found twice: no head may be left out between the two."""
    rng = torch.Generator().manual_seed(N + D)
    B, H, K, ps = 2, 6, 2, 16
    per = -(-(32 + N) // ps)
    k, v, table = _cache(rng, B, per, ps, K, D, dtype)
    tree = _tree(dba, B, 4, H, K, D, ps, per, 1, dtype)
    # sums within some roundings of 2^128, on either side
    q, new_k, new_v = (torch.randn(N, heads, D, generator=rng) for heads in (H, K, K))
    q = q / q.square().sum(-1, keepdim=True).sqrt() * 2.0 ** 64 * (1 + (torch.rand(N, H, 1, generator=rng) - 0.5) * 2.0 ** -6)
    q, new_k, new_v = (x.to(DT[dtype]).cuda() for x in (q, new_k, new_v))
    cos, sin, w = torch.rand(N, rot // 2, generator=rng).cuda(), torch.rand(N, rot // 2, generator=rng).cuda(), torch.ones(D).cuda()
    place, position = (32 + torch.arange(N) % (N // 2)).int().cuda(), (torch.arange(N) % (N // 2)).int().cuda()
    out = torch.full_like(q, math.nan)
    tree.append(new_k, new_v, k, v, table, place, position, rotary=(cos, sin), q=q, q_out=out, norm=(w, w, 1e-5))
    assert torch.isfinite(out).all()                            # (a sum of infinity is a root's inverse of 0)
    zero = (out == 0).all(-1)
    c, z = cos[position.long()].cpu().double(), sin[position.long()].cpu().double()
    want = M.rotate(L.norm(q.cpu(), w.cpu(), 1e-5), c, z, False)
    assert zero.any() and not zero.all()
    err = (out.cpu().double() - want).abs()[~zero.cpu()]
    assert (err <= 12 * ((D / 2 + 16) * 2.0 ** -24 + torch.finfo(DT[dtype]).eps / 2)).all()       # (a normed value is at most sqrt(D), 11.4 turned 16)
