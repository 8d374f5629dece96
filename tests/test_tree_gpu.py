"""The token tree over a paged cache on the GPU, against plain 64-bit models (tests/tree_model.py)."""
import ctypes as C
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests import tree_model as M                                     # noqa: E402

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def dba():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_1804_06609_b200 as pkg
    pkg.lib()
    return pkg


def _tree(dba, B, n, H, K, D, ps, pages, W, dtype="bf16", **kw):
    return dba.TokenTree(B, n, H, K, D, ps, pages, W, dtype=dba.F32 if dtype == "f32" else dba.BF16, **kw)


def _cache(rng, B, per, ps, K, D, dtype, hnd=False, spare=3, fill=None):
    """k, v [pages, ps, K, D] with a few pages nobody uses, and the tables."""
    pages = B * per + spare
    shape = (pages, K, ps, D) if hnd else (pages, ps, K, D)
    k, v = (torch.randn(shape, generator=rng).to(DT[dtype]) for _ in range(2))
    if hnd:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    table = torch.randperm(pages, generator=rng)[:B * per].int().view(B, per)
    return k.cuda(), v.cuda(), table.cuda()


def _masks(rng, B, n, W, density, closed=0.1):
    A = 32 * W
    m = torch.zeros(B, n, W, dtype=torch.int32)
    for b in range(B):
        for i in range(n):
            if torch.rand(1, generator=rng).item() >= closed:
                bits = torch.nonzero(torch.rand(A, generator=rng) < density).flatten().tolist() + [int(torch.randint(0, A, (1,), generator=rng))]
                m[b, i] = torch.from_numpy(M.words_of(set(bits), W))
    return m


def _top(masks):
    return torch.tensor([max([s + 1 for i in range(masks.shape[1]) for s in M.bits_of(masks[b, i].numpy())], default=0) for b in range(masks.shape[0])],
                        dtype=torch.int32)


def _check(got, lse, want, D, seen, dtype):
    out, wlse, spread, reach = want
    tol = M.attend_tolerance(out, spread, reach, D, seen, DT[dtype])
    err = (got.double().cpu() - out).abs()
    assert not torch.isnan(got).any()
    assert (err <= tol).all(), f"worst {float((err / tol).max()):.3f} of the bound at {np.unravel_index(int((err / tol).argmax()), err.shape)}"
    if lse is not None:
        lse = lse.double().cpu()
        assert torch.equal(torch.isinf(lse), torch.isinf(wlse))
        live = ~torch.isinf(wlse)
        # the score's error plus that of the sum (relative, so absolute in the logarithm) and the rounding of the result
        bound = reach * (D + 4) * 2.0 ** -24 + (seen + 32) * 2.0 ** -23 + wlse.abs().nan_to_num(0, 0, 0) * 2.0 ** -22
        assert ((lse - wlse).abs()[live] <= bound[live]).all()


SHAPES = [  # B, n, H, K, D, context lengths, page size, words, density, dtype, heads outside tokens
    (1, 1, 1, 1, 64, [0], 16, 1, 0.0, "bf16", False),
    (1, 1, 16, 16, 64, [1], 16, 1, 0.0, "bf16", False),
    (2, 5, 16, 16, 64, [37, 0], 16, 2, 0.3, "bf16", False),
    (3, 20, 8, 2, 128, [128, 129, 127], 64, 4, 0.2, "bf16", True),
    (2, 20, 32, 8, 128, [700, 1], 16, 3, 0.5, "bf16", False),
    (1, 61, 8, 1, 128, [300], 16, 2, 0.2, "bf16", False),
    (2, 64, 8, 2, 64, [65, 500], 5, 5, 0.1, "bf16", True),
    (4, 3, 12, 4, 80, [10, 100, 257, 33], 24, 1, 0.2, "bf16", False),
    (2, 7, 6, 6, 96, [1000, 3], 1, 2, 0.1, "bf16", False),
    (2, 2, 4, 2, 8, [40, 200], 16, 1, 0.3, "bf16", False),
    (1, 9, 40, 8, 128, [1500], 128, 13, 0.02, "bf16", False),
    (2, 4, 4, 2, 192, [90, 300], 32, 2, 0.2, "bf16", True),
    (1, 3, 2, 1, 256, [129], 16, 1, 0.2, "bf16", False),
    (5, 1, 8, 8, 128, [4096, 1, 0, 777, 2048], 64, 1, 0.0, "bf16", False),
    (1, 4, 8, 8, 64, [20000], 16, 1, 0.2, "bf16", False),
    (1, 1, 1, 1, 64, [0], 16, 1, 0.0, "f32", False),
    (2, 5, 16, 16, 64, [37, 0], 16, 2, 0.3, "f32", False),
    (3, 20, 8, 2, 128, [128, 129, 500], 64, 4, 0.2, "f32", True),
    (2, 33, 6, 2, 44, [65, 400], 5, 3, 0.1, "f32", False),
    (1, 3, 2, 1, 256, [129], 16, 1, 0.2, "f32", False),
    (1, 2, 8, 1, 4, [3000], 16, 1, 0.2, "f32", False),
]


@pytest.mark.parametrize("B,n,H,K,D,ctx,ps,W,density,dtype,hnd", SHAPES)
def test_attend_matches_the_model(dba, B, n, H, K, D, ctx, ps, W, density, dtype, hnd):
    rng = torch.Generator().manual_seed(B * 1000 + n * 10 + D)
    per = (32 * W + max(ctx) + ps - 1) // ps
    k, v, table = _cache(rng, B, per, ps, K, D, dtype, hnd)
    q = (torch.randn(B, n, H, D, generator=rng) * 1.5).to(DT[dtype]).cuda()
    masks = _masks(rng, B, n, W, density)
    t = _tree(dba, B, n, H, K, D, ps, per, W, dtype)
    c = torch.tensor(ctx, dtype=torch.int32)
    lse = torch.full((B, n, H), 7.0, device="cuda")
    want = M.attend(q, k, v, table, c, masks, D ** -0.5, ps, W, k.shape[0])
    seen = max(ctx) + 32 * W
    got = t.attend(q, k, v, table, c.cuda(), masks.cuda(), _top(masks).cuda(), lse=lse).clone()
    _check(got, lse, want, D, seen, dtype)
    # the whole arena looked at, and another scale
    want = M.attend(q, k, v, table, c, masks, 0.3, ps, W, k.shape[0])
    _check(t.attend(q, k, v, table, c.cuda(), masks.cuda(), scale=0.3, lse=lse), lse, want, D, seen, dtype)
    # no masks: the context alone, seen by every row
    want = M.attend(q, k, v, table, c, None, D ** -0.5, ps, W, k.shape[0])
    _check(t.attend(q, k, v, table, c.cuda(), lse=lse), lse, want, D, seen, dtype)
    assert t.status() == 0


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("bf16", 192), ("f32", 128)])
def test_places_no_row_sees_may_hold_anything(dba, dtype, D):
    """Dead slots, the rest of the last page, the pages of nobody: NaN and infinities there must not show."""
    B, n, H, K, ps, W, ctx = 3, 6, 8, 4, 24, 3, [50, 0, 131]
    rng = torch.Generator().manual_seed(3)
    per = (32 * W + max(ctx)) // ps + 2
    k, v, table = _cache(rng, B, per, ps, K, D, dtype)
    masks = _masks(rng, B, n, W, 0.1)
    masks[1] = 0                                                      # a sequence whose rows are all closed
    c = torch.tensor(ctx, dtype=torch.int32)
    q = torch.randn(B, n, H, D, generator=rng).to(DT[dtype]).cuda()
    seen = torch.zeros(k.shape[0], ps, dtype=torch.bool)
    for b in range(B):
        live = set().union(*[set(M.bits_of(masks[b, i].numpy())) for i in range(n)]) | set(range(32 * W, 32 * W + ctx[b]))
        for p in live:
            seen[int(table[b, p // ps]), p % ps] = True
    want = M.attend(q, k, v, table, c, masks, D ** -0.5, ps, W, k.shape[0])
    for bad in (math.nan, math.inf, -math.inf, torch.finfo(DT[dtype]).max):
        k2 = torch.where(seen[..., None, None].cuda(), k, torch.full_like(k, bad))
        v2 = torch.where(seen[..., None, None].cuda(), v, torch.full_like(v, bad))
        t = _tree(dba, B, n, H, K, D, ps, per, W, dtype)
        for top in (None, _top(masks).cuda()):
            got = t.attend(q, k2, v2, table, c.cuda(), masks.cuda(), top)
            _check(got, None, want, D, 200, dtype)
            assert (got[1] == 0).all()


@pytest.mark.parametrize("dtype,D,n", [("bf16", 64, 5), ("bf16", 128, 20), ("f32", 64, 5)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_value_that_is_not_finite_reaches_only_the_rows_that_see_it(dba, dtype, D, n, bad):
    B, H, K, ps, W, ctx = 2, 8, 2, 16, 2, [150, 20]
    rng = torch.Generator().manual_seed(4)
    per = (32 * W + max(ctx)) // ps + 1
    k, v, table = _cache(rng, B, per, ps, K, D, dtype)
    masks = torch.zeros(B, n, W, dtype=torch.int32)
    for b in range(B):
        for i in range(n):
            masks[b, i] = torch.from_numpy(M.words_of({i, 30 + i % 3}, W))
    c = torch.tensor(ctx, dtype=torch.int32)
    q = torch.randn(B, n, H, D, generator=rng).to(DT[dtype]).cuda()
    want = M.attend(q, k, v, table, c, masks, D ** -0.5, ps, W, k.shape[0])
    v2 = v.clone()
    v2[int(table[0, 1 // ps]), 1 % ps, 1, 3] = bad                     # slot 1 of sequence 0, key head 1, dimension 3: row 1 alone
    t = _tree(dba, B, n, H, K, D, ps, per, W, dtype)
    got = t.attend(q, k, v2, table, c.cuda(), masks.cuda()).cpu()
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[0, 1, H // K:, 3] = True
    assert not torch.isfinite(got[hit].float()).any() and torch.isfinite(got[~hit].float()).all()
    out, _, spread, reach = want
    err = (got.double() - out).abs()
    assert (err <= M.attend_tolerance(out, spread, reach, D, 300, DT[dtype]))[~hit].all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_takes_strided_arguments_and_fewer_rows(dba, dtype):
    B, n, H, K, D, ps, W, ctx = 2, 6, 8, 2, 64, 16, 1, [70, 33]
    rng = torch.Generator().manual_seed(5)
    per = (32 * W + max(ctx)) // ps + 1
    pages = B * per
    big = torch.randn(pages, ps, 2, K, D + 16, generator=rng).to(DT[dtype]).cuda()     # keys and values side by side, wider rows
    k, v = big[:, :, 0, :, :D], big[:, :, 1, :, :D]
    table = torch.full((B, per + 5), -9, dtype=torch.int32)
    table[:, :per] = torch.randperm(pages, generator=rng).int().view(B, per)
    table = table.cuda()[:, :per]
    wide = torch.randn(B, H, n, 3, D, generator=rng).to(DT[dtype]).cuda()
    q = wide[:, :, :, 1].transpose(1, 2)
    out = torch.zeros(n, B, H, 2 * D, dtype=DT[dtype], device="cuda")
    masks = _masks(rng, B, n, W, 0.3, closed=0.0)
    c = torch.tensor(ctx, dtype=torch.int32)
    want = M.attend(q, k, v, table, c, masks, D ** -0.5, ps, W, pages)
    t = _tree(dba, B, 9, H, K, D, ps, per, W, dtype)
    view = out.transpose(0, 1)[..., :D]
    got = t.attend(q, k, v, table, c.cuda(), masks.cuda(), out=view)
    _check(got, None, want, D, 200, dtype)
    assert (out[..., D:] == 0).all()
    _check(t.attend(q, k, v, table, c.cuda(), masks.cuda()), None, want, D, 200, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_cache_longer_than_32_bit_offsets(dba, dtype):
    """Pages at element offsets past 2^31 (and byte offsets past 2^32)."""
    B, n, H, K, D, ps, W, ctx = 1, 2, 4, 2, 64, 16, 1, [100]
    rng = torch.Generator().manual_seed(6)
    per = (32 + 100) // ps + 1
    page_elems, stride = ps * K * D, 1 << 28
    room = torch.empty((per + 1) * stride + 4 * page_elems, dtype=DT[dtype], device="cuda")
    k = room.as_strided((per + 2, ps, K, D), (stride, K * D, D, 1))
    v = room.as_strided((per + 2, ps, K, D), (stride, K * D, D, 1), 2 * page_elems)
    table = torch.arange(per, dtype=torch.int32).flip(0).add(1).view(1, per).cuda()      # pages 1 .. per
    for p in range(1, per + 1):
        k[p].copy_(torch.randn(ps, K, D, generator=rng)); v[p].copy_(torch.randn(ps, K, D, generator=rng))
    assert per * stride > 1 << 31
    masks = _masks(rng, B, n, W, 0.3, closed=0.0)
    q = torch.randn(B, n, H, D, generator=rng).to(DT[dtype]).cuda()
    c = torch.tensor(ctx, dtype=torch.int32)
    t = _tree(dba, B, n, H, K, D, ps, per, W, dtype)
    # one more token at the end of the last page's rows, through the operator
    nk, nv = (torch.randn(2, K, D, generator=rng).to(DT[dtype]).cuda() for _ in range(2))
    place = torch.tensor([32 + 99, 3], dtype=torch.int32)
    t.append(nk, nv, k, v, table, place.cuda())
    for i, p in enumerate(place.tolist()):
        assert torch.equal(k[int(table[0, p // ps]), p % ps], nk[i]) and torch.equal(v[int(table[0, p // ps]), p % ps], nv[i])
    small_k, small_v = (torch.stack([x[p] if 1 <= p <= per else torch.zeros_like(x[1]) for p in range(per + 2)]) for x in (k, v))
    want = M.attend(q, small_k, small_v, table, c, masks, D ** -0.5, ps, W, per + 2)
    _check(t.attend(q, k, v, table, c.cuda(), masks.cuda()), None, want, D, 200, dtype)
    # a settled token across pages
    src, count = torch.full((1, 32), -1, dtype=torch.int32), torch.tensor([1], dtype=torch.int32)
    src[0, 0] = 3
    t.commit(k, v, table, torch.tensor([50], dtype=torch.int32).cuda(), src.cuda(), count.cuda())
    at = 32 + 49
    assert torch.equal(k[int(table[0, at // ps]), at % ps], nk[1]) and torch.equal(v[int(table[0, at // ps]), at % ps], nv[1])
    assert t.status() == 0


def test_pages_outside_the_cache_are_reported_and_not_read(dba):
    B, n, H, K, D, ps, W, ctx = 2, 3, 4, 2, 64, 16, 1, [200, 90]
    rng = torch.Generator().manual_seed(7)
    per = (32 + 200) // ps + 1
    for dtype in ("bf16", "f32"):
        k, v, table = _cache(rng, B, per, ps, K, D, dtype)
        table[0, 5] = k.shape[0]; table[1, 3] = -1
        masks = _masks(rng, B, n, W, 0.3, closed=0.0)
        q = torch.randn(B, n, H, D, generator=rng).to(DT[dtype]).cuda()
        c = torch.tensor(ctx, dtype=torch.int32)
        want = M.attend(q, k, v, table, c, masks, D ** -0.5, ps, W, k.shape[0])
        t = _tree(dba, B, n, H, K, D, ps, per, W, dtype)
        _check(t.attend(q, k, v, table, c.cuda(), masks.cuda()), None, want, D, 300, dtype)
        assert t.status() == dba.TREE_BAD_PAGE and t.status() == 0
        # lengths beyond the table are cut to it
        c2 = torch.tensor([1 << 30, -5], dtype=torch.int32)
        want = M.attend(q, k, v, table, c2, masks, D ** -0.5, ps, W, k.shape[0])
        _check(t.attend(q, k, v, table, c2.cuda(), masks.cuda()), None, want, D, 300, dtype)
        t.status()
        nk = torch.randn(4, K, D, generator=rng).to(DT[dtype]).cuda()
        before = k.clone()
        place = torch.tensor([5 * ps, per * ps, -1, 2], dtype=torch.int32).cuda()
        t.append(nk, nk, k, v, table, place, seq=torch.tensor([0, 1, 0, 2], dtype=torch.int32).cuda())
        assert torch.equal(before, k) and t.status() == dba.TREE_BAD_PAGE | dba.TREE_BAD_INDEX


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_equal_calls_give_equal_bits_and_nothing_is_kept(dba, dtype):
    """Long and short contexts in one batch (work split over many blocks), then another batch through the same handle."""
    B, n, H, K, D, ps, W = 4, 3, 8, 2, 128, 16, 1
    ctx = [3000, 0, 17, 1200]
    rng = torch.Generator().manual_seed(8)
    per = (32 + max(ctx)) // ps + 1
    k, v, table = _cache(rng, B, per, ps, K, D, dtype)
    masks = _masks(rng, B, n, W, 0.3).cuda()
    q = torch.randn(B, n, H, D, generator=rng).to(DT[dtype]).cuda()
    t = _tree(dba, B, n, H, K, D, ps, per, W, dtype)
    a, b = (torch.tensor(x, dtype=torch.int32).cuda() for x in (ctx, ctx[::-1]))
    first, other = t.attend(q, k, v, table, a, masks).clone(), t.attend(q, k, v, table, b, masks).clone()
    for _ in range(5):
        assert torch.equal(t.attend(q, k, v, table, a, masks), first)
        assert torch.equal(t.attend(q, k, v, table, b, masks), other)


def test_a_handle_works_on_its_own_stream(dba):
    B, n, H, K, D, ps, W = 2, 4, 8, 2, 128, 16, 1
    rng = torch.Generator().manual_seed(9)
    k, v, table = _cache(rng, B, 40, ps, K, D, "bf16")
    masks = _masks(rng, B, n, W, 0.3).cuda()
    q = torch.randn(B, n, H, D, generator=rng).to(torch.bfloat16).cuda()
    c = torch.tensor([500, 77], dtype=torch.int32).cuda()
    want = _tree(dba, B, n, H, K, D, ps, 40, W).attend(q, k, v, table, c, masks).clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    t = _tree(dba, B, n, H, K, D, ps, 40, W, stream=side)
    with torch.cuda.stream(side):
        q2 = torch.zeros_like(q)
        torch.cuda._sleep(20_000_000)
        q2.copy_(q)                                   # late: the call must come after it
    got = t.attend(q2, k, v, table, c, masks)
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("D,drop", [(64, 0), (128, 0), (128, 3)])
def test_a_wait_that_runs_out_is_reported(dba, D, drop):
    """The tensor-core kernel's waits are bounded: with one tile's hand-over withheld and a 1 ms limit the call ends, its
    outputs are NaN, the status says why, and the next call is right."""
    B, n, H, K, ps, W = 2, 3, 4, 2, 16, 1
    rng = torch.Generator().manual_seed(13)
    per = (32 + 40000) // ps + 1
    k, v, table = _cache(rng, B, per, ps, K, D, "bf16")
    masks = _masks(rng, B, n, W, 0.3, closed=0.0).cuda()
    q = torch.randn(B, n, H, D, generator=rng).to(torch.bfloat16).cuda()
    c = torch.tensor([40000, 39000], dtype=torch.int32).cuda()          # some four tiles for every block
    t = _tree(dba, B, n, H, K, D, ps, per, W)
    lse = torch.zeros(B, n, H, device="cuda")
    want = t.attend(q, k, v, table, c, masks, lse=lse).clone()
    assert t.status() == 0 and torch.isfinite(want.float()).all()
    t.test_hook(wait_clocks=2_000_000, drop_item=drop)
    got = t.attend(q, k, v, table, c, masks, lse=lse)
    assert t.status() == dba.TREE_TIMEOUT and torch.isnan(got.float()).all() and torch.isnan(lse).all()
    t.test_hook()
    assert torch.equal(t.attend(q, k, v, table, c, masks, lse=lse), want) and torch.isfinite(lse).all() and t.status() == 0


@pytest.mark.parametrize("n,H,K,D", [(3, 4, 2, 64), (20, 8, 2, 128), (5, 8, 8, 64)])
def test_a_wait_that_runs_out_on_short_tables(dba, n, H, K, D):
    """Items of a few tiles stay whole and no second kernel follows: the blocks that give up undo their own items."""
    B, ps, W = 40, 16, 1
    rng = torch.Generator().manual_seed(14)
    per = (32 + 150) // ps + 1
    k, v, table = _cache(rng, B, per, ps, K, D, "bf16")
    masks = _masks(rng, B, n, W, 0.3, closed=0.0).cuda()
    q = torch.randn(B, n, H, D, generator=rng).to(torch.bfloat16).cuda()
    c = torch.full((B,), 150, dtype=torch.int32).cuda()
    t = _tree(dba, B, n, H, K, D, ps, per, W)
    lse = torch.zeros(B, n, H, device="cuda")
    want = t.attend(q, k, v, table, c, masks, lse=lse).clone()
    launches = t.launch_count()
    assert t.status() == 0 and torch.isfinite(want.float()).all()
    t.test_hook(wait_clocks=2_000_000, drop_item=1)
    got = t.attend(q, k, v, table, c, masks, lse=lse)
    assert t.launch_count() == launches + 1
    assert t.status() == dba.TREE_TIMEOUT and torch.isnan(got.float()).all() and torch.isnan(lse).all()
    t.test_hook()
    assert torch.equal(t.attend(q, k, v, table, c, masks, lse=lse), want) and torch.isfinite(lse).all() and t.status() == 0


# ------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("N,H,K,D,rot,pairs,dtype,hnd,inplace", [
    (1, 1, 1, 64, 64, False, "bf16", False, False), (10, 8, 2, 128, 128, False, "bf16", False, True), (40, 8, 2, 128, 64, True, "bf16", True, False),
    (6, 12, 4, 80, 40, False, "bf16", False, False), (6, 6, 6, 96, 36, True, "bf16", True, True), (4, 2, 2, 8, 6, False, "bf16", False, False),
    (10, 4, 4, 44, 44, False, "f32", False, False), (12, 8, 2, 64, 32, True, "f32", True, True), (2, 3, 1, 256, 2, False, "f32", False, False),
    (8, 4, 2, 64, 0, False, "bf16", False, False)])
def test_append_matches_the_model(dba, N, H, K, D, rot, pairs, dtype, hnd, inplace):
    rng = torch.Generator().manual_seed(N + D + rot)
    B, ps, W, per = 2, 5, 1, 30
    if N % B:
        B = 1
    k, v, table = _cache(rng, B, per, ps, K, D, dtype, hnd)
    wide = torch.randn(N, H + 2 * K + 1, D, generator=rng).to(DT[dtype]).cuda()          # queries, keys and values in one tensor
    q, nk, nv = wide[:, :H], wide[:, H:H + K], wide[:, H + K:H + 2 * K]
    places = torch.stack([torch.randperm(32 * W + 100, generator=rng)[:N // B] for _ in range(B)]).flatten().int()
    pos = torch.randint(0, 50, (N,), generator=rng).int()
    if N > 2:
        places[1], pos[2] = -1, -1                                                       # not stored; not rotated
    ang = torch.rand(50, max(rot // 2, 1), generator=rng, dtype=torch.float64) * 6.3
    cos, sin = ang.cos().float(), ang.sin().float()
    for shuffled in (False, True):
        kk, vv, qq = k.clone(memory_format=torch.preserve_format), v.clone(memory_format=torch.preserve_format), wide.clone()[:, :H]
        if hnd:
            assert kk.stride() == k.stride()
        order = torch.randperm(N, generator=rng) if shuffled else torch.arange(N)
        seq = (torch.arange(N) // (N // B)).int()
        args = dict(seq=seq[order].cuda() if shuffled else None, q=qq[order.cuda()] if shuffled else qq)
        if rot:
            args.update(position=pos[order].cuda(), rotary=(cos.cuda(), sin.cuda()), pairs=pairs)
        if inplace:
            args["q_out"] = args["q"]
        src_q = args["q"].double().cpu().clone()
        t = _tree(dba, B, 4, H, K, D, ps, per, W, dtype)
        got = t.append(nk[order.cuda()] if shuffled else nk, nv[order.cuda()] if shuffled else nv, kk, vv, table, places[order].cuda(), **args)
        turn = lambda x, o: torch.where((pos[o] < 0)[:, None, None], x, M.rotate(x, cos.double()[pos[o].clamp(min=0).long()], sin.double()[pos[o].clamp(min=0).long()], pairs)) if rot else x  # noqa: E731
        want_q = turn(src_q, order)
        want_k, want_v = k.double().cpu(), v.double().cpu()
        tk = turn(nk.double().cpu(), torch.arange(N))
        for i in range(N):
            p = int(places[i])
            if p >= 0:
                b = int(seq[i])
                want_k[int(table[b, p // ps]), p % ps] = tk[i]
                want_v[int(table[b, p // ps]), p % ps] = nv[i].double().cpu()
        # two products and a sum in fp32 (3 roundings of terms no larger than |a| + |b| <= 2 max), then one to the type
        u = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8
        for x, w in ((got, want_q), (kk, want_k)):
            assert ((x.double().cpu() - w).abs() <= u * w.abs() * 1.01 + 4 * 2.0 ** -24 * 8.0).all()
        assert torch.equal(vv.double().cpu(), want_v)
        assert t.status() == 0


def test_append_reports_positions_outside_the_rotary_table(dba):
    rng = torch.Generator().manual_seed(1)
    k, v, table = _cache(rng, 1, 10, 16, 2, 64, "bf16")
    t = _tree(dba, 1, 4, 4, 2, 64, 16, 10, 1)
    nk = torch.randn(2, 2, 64, generator=rng).to(torch.bfloat16).cuda()
    cs = torch.rand(8, 32, generator=rng).cuda()
    t.append(nk, nk, k, v, table, torch.tensor([0, 1], dtype=torch.int32).cuda(), torch.tensor([8, 7], dtype=torch.int32).cuda(), (cs, cs))
    assert t.status() == dba.TREE_BAD_INDEX
    assert torch.equal(k[int(table[0, 0]), 0], nk[0])                   # not rotated
    empty = nk[:0]
    t.append(empty, empty, k, v, table, torch.empty(0, dtype=torch.int32, device="cuda"))
    assert t.status() == 0


# ------------------------------------------------------------------------------------------------ advance, commit
def _run_advance(dba, t, sets, slot_pos, ctx, back, score, token, eos, W, cap):
    B, n_in, n = len(sets), len(sets[0]), back.shape[1]
    masks = torch.from_numpy(np.stack([np.stack([M.words_of(r, W) for r in s]) for s in sets])).cuda()
    sp = torch.zeros(B, 32 * W + 1, dtype=torch.int32).cuda()[:, :-1]           # rows further apart than they are long
    sp.copy_(torch.tensor(slot_pos, dtype=torch.int32))
    f = lambda x, dt: None if x is None else torch.tensor(x, dtype=dt).cuda()  # noqa: E731
    got = t.advance(f(back, torch.int32), masks, sp, f(ctx, torch.int32), score=f(score, torch.float32), token=f(token, torch.int32), eos=eos)
    bits = t.status()
    full = room = False
    out = []
    for b in range(B):
        want, (fl, rm) = M.advance(sets[b], slot_pos[b], ctx[b], back[b].tolist(), None if score is None else score[b], None if token is None else token[b], eos, cap)
        full |= fl; room |= rm
        out.append(want)
        assert [set(M.bits_of(got["masks"][b, i].cpu().numpy())) for i in range(n)] == want["masks"]
        for key in ("slot", "position"):
            assert got[key][b].tolist() == want[key], key
        assert sp[b].tolist() == want["slot_pos"]
        assert int(got["ctx_len"][b]) == want["ctx_len"] and int(got["top"][b]) == want["top"]
        c = len(want["commit_src"])
        assert int(got["commit_n"][b]) == c and got["commit_src"][b].tolist() == want["commit_src"] + [-1] * (32 * W - c)
    assert bits == (dba.TREE_ARENA_FULL if full else 0) | (dba.TREE_NO_ROOM if room else 0)
    return out


@pytest.mark.parametrize("B,n,W,steps,skew", [(1, 1, 1, 8, 1), (1, 5, 2, 20, 2), (7, 20, 8, 30, 2), (3, 64, 31, 12, 1), (2, 64, 128, 6, 1), (4, 16, 1, 12, 1), (300, 3, 1, 6, 3)])
def test_advance_over_the_steps_of_a_beam(dba, B, n, W, steps, skew):
    """Arenas that fill up (n = 16 on 32 slots) and finished and empty hypotheses among the cases."""
    rng = np.random.default_rng(B + n + W)
    per = (32 * W + 25) // 16 + 1
    cap = per * 16 - 32 * W
    t = _tree(dba, B, n, 1, 1, 64, 16, per, W)
    sets, slot_pos, ctx = [[set() for _ in range(n)] for _ in range(B)], [[0] * (32 * W) for _ in range(B)], [int(x) for x in rng.integers(0, 6, B)]
    for step in range(steps):
        back = np.sort((rng.random((B, n)) ** skew * n).astype(np.int32), 1)
        score = -np.cumsum(rng.random((B, n)), 1).astype(np.float32)
        score[rng.random((B, n)) < 0.05] = -np.inf
        token = rng.integers(3, 9, (B, n)).astype(np.int32)
        token[rng.random((B, n)) < 0.1] = 2
        back[rng.random((B, n)) < 0.03] = -1
        give = step % 3
        if give == 2:
            token[0] = 2                                            # a sentence whose hypotheses are all finished
        out = _run_advance(dba, t, sets, slot_pos, ctx, back, score if give else None, token if give else None, 2, W, cap)
        sets, slot_pos, ctx = [o["masks"] for o in out], [o["slot_pos"] for o in out], [o["ctx_len"] for o in out]


@pytest.mark.parametrize("B,n,W", [(1, 2, 1), (5, 17, 1), (3, 64, 2), (2, 61, 9)])
def test_advance_with_trees_of_drafted_tokens(dba, B, n, W):
    """A tree is drafted, one of its rows accepted, the next tree drafted from there."""
    rng = np.random.default_rng(n)
    per = 32 * W + 60
    t = _tree(dba, B, n, 1, 1, 64, 1, per, W)
    sets, slot_pos, ctx = [[set()] for _ in range(B)], [[0] * (32 * W) for _ in range(B)], [4] * B
    for step in range(4):
        n_in = len(sets[0])
        back = np.zeros((B, n), np.int32)
        for b in range(B):
            back[b, 0] = rng.integers(0, n_in)
            for j in range(1, n):
                back[b, j] = n_in + rng.integers(max(0, j - 4), j)
            if n > 10:
                back[b, 7] = n_in + 7                               # extends itself: closed, and what extends it
                back[b, 9] = n_in + 7
                back[b, 5] = -3
        out = _run_advance(dba, t, sets, slot_pos, ctx, back, None, None, -1, W, per - 32 * W)
        sets, slot_pos, ctx = [o["masks"] for o in out], [o["slot_pos"] for o in out], [o["ctx_len"] for o in out]


@pytest.mark.parametrize("layers,B,K,D,ps,W,dtype,hnd", [(1, 1, 1, 64, 16, 1, "bf16", False), (3, 5, 4, 128, 5, 2, "bf16", True), (6, 3, 2, 44, 24, 1, "f32", False), (2, 40, 1, 8, 1, 1, "bf16", False)])
def test_commit_copies_settled_tokens_in_every_layer(dba, layers, B, K, D, ps, W, dtype, hnd):
    rng = torch.Generator().manual_seed(layers + B)
    A = 32 * W
    per = (A + 60 + ps - 1) // ps
    shape = (layers, B * per, K, ps, D) if hnd else (layers, B * per, ps, K, D)
    k, v = (torch.randn(shape, generator=rng).to(DT[dtype]).cuda() for _ in range(2))
    if hnd:
        k, v = k.transpose(2, 3), v.transpose(2, 3)
    table = torch.randperm(B * per, generator=rng).int().view(B, per).cuda()
    n = torch.randint(0, 12, (B,), generator=rng).int()
    ctx = (n + torch.randint(0, 40, (B,), generator=rng)).int()
    src = torch.full((B, A), -1, dtype=torch.int32)
    want_k, want_v = k.clone(), v.clone()
    for b in range(B):
        src[b, :n[b]] = torch.randperm(A, generator=rng)[:n[b]].int()
        for i in range(int(n[b])):
            s, d = int(src[b, i]), A + int(ctx[b]) - int(n[b]) + i
            for x, w in ((k, want_k), (v, want_v)):
                w[:, int(table[b, d // ps]), d % ps] = x[:, int(table[b, s // ps]), s % ps]
    t = _tree(dba, B, 4, K, K, D, ps, per, W, dtype)
    for _ in range(2):                                                # a second time changes nothing
        t.commit(k, v, table, ctx.cuda(), src.cuda(), n.cuda())
        assert torch.equal(k, want_k) and torch.equal(v, want_v) and t.status() == 0
    # a slot or a place outside its range is reported and nothing is written for it
    src[0, 0], n[0], ctx[0] = A, 2, 2
    src[0, 1] = 0
    t.commit(k, v, table, ctx.cuda(), src.cuda(), n.cuda())
    assert t.status() == dba.TREE_BAD_INDEX


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype,drafts", [("bf16", False), ("f32", False), ("bf16", True)])
def test_a_beam_over_the_cache_sees_what_each_hypothesis_would_alone(dba, dtype, drafts):
    """Steps of a beam with its cache in the tree, against every hypothesis' own list of keys and values."""
    B, n, H, K, D, ps, W, steps = 3, 6, 8, 2, 64, 16, 3, 14
    rng = torch.Generator().manual_seed(11)
    per = (32 * W + 60) // ps + 1
    k, v, table = _cache(rng, B, per, ps, K, D, dtype, fill=None)
    k.fill_(math.nan); v.fill_(math.nan)
    k, v = k[None], v[None]
    t = _tree(dba, B, n, H, K, D, ps, per, W, dtype)
    prompt = [9, 1, 20]
    own = [[[]] * n for _ in range(B)]                                # per row: list of (key, value) of its whole past
    for b in range(B):
        nk, nv = (torch.randn(prompt[b], K, D, generator=rng).to(DT[dtype]) for _ in range(2))
        t.append(nk.cuda(), nv.cuda(), k[0], v[0], table, (32 * W + torch.arange(prompt[b])).int().cuda(), seq=torch.full((prompt[b],), b, dtype=torch.int32).cuda())
        own[b] = [[(nk[i], nv[i]) for i in range(prompt[b])] for _ in range(n)]
    masks = torch.zeros(B, n, W, dtype=torch.int32, device="cuda")
    slot_pos = torch.zeros(B, 32 * W, dtype=torch.int32, device="cuda")
    ctx = torch.tensor(prompt, dtype=torch.int32, device="cuda")
    for step in range(steps):
        back = (torch.rand(B, n, generator=rng) ** 2 * n).int().sort(1).values
        for b in range(B):                                            # a step extends rows that are open
            alive = [i for i in range(n) if own[b][i] is not None]
            back[b] = torch.tensor([alive[int(x) % len(alive)] for x in back[b]])
        if drafts:
            back[:, 1:] = n + (torch.rand(B, n - 1, generator=rng) * torch.arange(1, n)).int()
        tok = torch.full((B, n), 5, dtype=torch.int32)
        tok[torch.rand(B, n, generator=rng) < 0.1] = 2
        tok[:, 0] = 5
        nx = t.advance(back.cuda(), masks, slot_pos, ctx, token=tok.cuda(), eos=2)
        t.commit(k, v, table, nx["ctx_len"], nx["commit_src"], nx["commit_n"])
        nk, nv = (torch.randn(B, n, K, D, generator=rng).to(DT[dtype]) for _ in range(2))
        q = torch.randn(B, n, H, D, generator=rng).to(DT[dtype])
        t.append(nk.view(B * n, K, D).cuda(), nv.view(B * n, K, D).cuda(), k[0], v[0], table, nx["slot"].view(-1))
        got = t.attend(q.cuda(), k[0], v[0], table, nx["ctx_len"], nx["masks"], nx["top"])
        new = [[None] * n for _ in range(B)]
        for b in range(B):
            for i in range(n):
                p = int(back[b, i])
                past = own[b][p] if p < n else new[b][p - n]
                new[b][i] = past + [(nk[b, i], nv[b, i])] if past is not None and tok[b, i] != 2 else None
                if new[b][i] is None:
                    assert (got[b, i] == 0).all() and int(nx["position"][b, i]) == -1
                    continue
                assert int(nx["position"][b, i]) == len(past)
                kk, vv = (torch.stack([x[j] for x in new[b][i]])[None] for j in (0, 1))
                want = M.attend(q[b:b + 1, i:i + 1], kk, vv, torch.zeros(1, 1, dtype=torch.int32), [kk.shape[1]], None, D ** -0.5, kk.shape[1], 0, 1)
                _check(got[b:b + 1, i:i + 1], None, want, D, 100, dtype)
        own = new
        masks, ctx = nx["masks"], nx["ctx_len"]
        assert t.status() == 0


def test_arguments_that_are_refused(dba):
    rng = torch.Generator().manual_seed(12)
    k, v, table = _cache(rng, 2, 10, 16, 2, 64, "bf16")
    t = _tree(dba, 2, 4, 8, 2, 64, 16, 10, 1)
    L, T = dba.lib(), __import__("paper_1804_06609_b200.tree", fromlist=["x"])
    q = torch.randn(2, 4, 8, 64, generator=rng).to(torch.bfloat16).cuda()
    out, ctx, masks = torch.empty_like(q), torch.zeros(2, dtype=torch.int32).cuda(), torch.zeros(2, 4, 1, dtype=torch.int32).cuda()
    query = lambda **kw: T.TreeQuery(**{**dict(rows=4, q=q.data_ptr(), q_seq_stride=2048, q_row_stride=512, q_head_stride=64, out=out.data_ptr(), out_seq_stride=2048, out_row_stride=512, out_head_stride=64, lse=None, scale=0.1), **kw})  # noqa: E731
    cache = lambda **kw: T.KvCache(**{**dict(k=k.data_ptr(), v=v.data_ptr(), num_pages=23, layers=1, page_stride=2048, token_stride=128, head_stride=64, layer_stride=0), **kw})  # noqa: E731
    attend = lambda qq, cc, tb=table.data_ptr(), ts=10, c=ctx.data_ptr(): L.dba_tree_attend(t._h, C.byref(qq), C.byref(cc), tb, ts, c, masks.data_ptr(), None)  # noqa: E731
    assert attend(query(), cache()) == 0
    for kw, code in ((dict(rows=0), 1), (dict(rows=5), 1), (dict(q=None), 1), (dict(out=None), 1), (dict(scale=math.nan), 1), (dict(q=q.data_ptr() + 2), 2), (dict(q_head_stride=63), 2), (dict(out_row_stride=3), 2)):
        assert attend(query(**kw), cache()) == code, kw
    for kw, code in ((dict(k=None), 1), (dict(num_pages=0), 1), (dict(layers=0), 1), (dict(page_stride=-8), 1), (dict(k=k.data_ptr() + 8), 2), (dict(token_stride=129), 2), (dict(head_stride=60), 2)):
        assert attend(query(), cache(**kw)) == code, kw
    assert attend(query(), cache(), tb=None) == 1 and attend(query(), cache(), ts=9) == 1 and attend(query(), cache(), c=None) == 1
    nk = torch.zeros(4, 2, 64, dtype=torch.bfloat16).cuda()
    place = torch.zeros(4, dtype=torch.int32).cuda()
    tok = lambda **kw: T.TreeTokens(**{**dict(N=4, k=nk.data_ptr(), v=nk.data_ptr(), k_token_stride=128, k_head_stride=64, v_token_stride=128, v_head_stride=64, place=place.data_ptr()), **kw})  # noqa: E731
    append = lambda x: L.dba_tree_append(t._h, C.byref(x), C.byref(cache()), table.data_ptr(), 10)  # noqa: E731
    for kw, code in ((dict(N=-1), 1), (dict(N=3), 1), (dict(k=None), 1), (dict(place=None), 1), (dict(q=q.data_ptr()), 1), (dict(rot_dim=66), 1), (dict(rot_dim=3), 1),
                     (dict(rot_dim=8, position=place.data_ptr()), 1), (dict(v=nk.data_ptr() + 2), 2), (dict(k_head_stride=4), 2)):
        assert append(tok(**kw)) == code, kw
    sp = torch.zeros(2, 32, dtype=torch.int32).cuda()
    m2, nx = torch.zeros_like(masks), T.TreeNext()
    adv = lambda ni=4, m=masks.data_ptr(), no=4, bp=place.data_ptr(), o=m2.data_ptr(), st=32: L.dba_tree_advance(t._h, ni, m, no, bp, None, None, 0, sp.data_ptr(), st, ctx.data_ptr(), C.byref(T.TreeNext(masks=o)))  # noqa: E731
    assert adv(st=31) == 1 and adv(ni=0) == 1 and adv(ni=5) == 1 and adv(no=5) == 1 and adv(m=None) == 1 and adv(bp=None) == 1 and adv(o=None) == 1 and adv(o=masks.data_ptr()) == 1
    t0 = _tree(dba, 2, 4, 8, 2, 64, 16, 10, 0)
    assert L.dba_tree_attend(t0._h, C.byref(query()), C.byref(cache()), table.data_ptr(), 10, ctx.data_ptr(), masks.data_ptr(), None) == 1
    assert L.dba_tree_commit(t0._h, C.byref(cache()), table.data_ptr(), 10, ctx.data_ptr(), ctx.data_ptr(), ctx.data_ptr()) == 1
    with pytest.raises(dba.DbaError):
        t.attend(q, k[..., :-1, :, :].new_zeros(23, 16, 2, 64).as_strided((23, 16, 2, 64), (2048, 128, 60, 1)), v.as_strided((23, 16, 2, 64), (2048, 128, 60, 1)), table, ctx, masks)
