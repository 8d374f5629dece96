"""The token tree's branches that ordinary calls seldom reach, against the plain 64-bit models (tests/tree_model.py)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests import tree_model as M                                     # noqa: E402
from tests.test_tree_gpu import DT, _cache, _check, _masks, _top, _tree  # noqa: E402


@pytest.fixture(scope="module")
def dba():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_1804_06609_b200 as pkg
    pkg.lib()
    return pkg


@pytest.mark.parametrize("n,H,K,D", [(5, 8, 8, 64), (40, 8, 8, 64), (20, 32, 8, 128), (4, 8, 4, 128), (4, 4, 2, 64)])
@pytest.mark.parametrize("W", [3, 8])
def test_items_that_end_in_arena_tiles_have_all_their_outputs(dba, n, H, K, D, W):
    """Without a context an item's last tiles are of the arena, whose values are looked over before their products: the last
    two products of an item follow each other at once, and its output must wait for both.  Every SM is kept busy
    by sequences that repeat three, so that each is compared with the model."""
    B, kinds, ps = 240, 3, 16
    rng = torch.Generator().manual_seed(20 + n + W)
    per = 2 * W + 1
    k, v, table = _cache(rng, kinds, per, ps, K, D, "bf16")
    masks = _masks(rng, kinds, n, W, 0.4, closed=0.0)
    q = torch.randn(kinds, n, H, D, generator=rng).to(torch.bfloat16)
    c = torch.zeros(kinds, dtype=torch.int32)
    want = M.attend(q, k, v, table, c, masks, D ** -0.5, ps, W, k.shape[0])
    t = _tree(dba, B, n, H, K, D, ps, per, W)
    many = lambda x: x.repeat(*([B // kinds] + [1] * (x.dim() - 1))).cuda()  # noqa: E731
    args = (many(q), k, v, many(table), many(c), many(masks))
    first = t.attend(*args).clone()
    _check(first[:kinds], None, want, D, 32 * W, "bf16")
    assert torch.equal(first, first[:kinds].repeat(B // kinds, 1, 1, 1))
    for _ in range(40):
        assert torch.equal(t.attend(*args), first)
    assert t.status() == 0


def test_a_failure_in_a_recorded_call_ends_with_it(dba):
    """A graph runs one recorded call again and again.  The withheld hand-over is the seventh of a block: with long contexts the
    call fails, with short ones no block comes that far and it must be right again."""
    B, n, H, K, D, ps, W = 2, 3, 4, 2, 64, 16, 1
    rng = torch.Generator().manual_seed(31)
    per = (32 + 60000) // ps + 1
    k, v, table = _cache(rng, B, per, ps, K, D, "bf16")
    masks = _masks(rng, B, n, W, 0.3, closed=0.0).cuda()
    q = torch.randn(B, n, H, D, generator=rng).to(torch.bfloat16).cuda()
    long, short = (torch.full((B,), x, dtype=torch.int32).cuda() for x in (60000, 2000))
    c, side = long.clone(), torch.cuda.Stream()
    lse = torch.zeros(B, n, H, device="cuda")
    torch.cuda.synchronize()
    t = _tree(dba, B, n, H, K, D, ps, per, W, stream=side)
    with torch.cuda.stream(side):
        want = t.attend(q, k, v, table, short, masks).clone()
    launches = t.launch_count()
    assert t.status() == 0 and torch.isfinite(want.float()).all()
    t.test_hook(wait_clocks=2_000_000, drop_item=6)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        t.attend(q, k, v, table, c, masks, lse=lse)
    assert t.launch_count() == launches + 2                           # cut, and joined by a second kernel
    for _ in range(2):
        with torch.cuda.stream(side):
            c.copy_(long)
            graph.replay()
        assert t.status() == dba.TREE_TIMEOUT and torch.isnan(t.out.float()).all() and torch.isnan(lse).all()
        with torch.cuda.stream(side):
            c.copy_(short)
            graph.replay()
        assert t.status() == 0 and torch.equal(t.out, want) and torch.isfinite(lse).all()
    del graph


def _rows_far_apart(t, T, query, k, v, table, ctx, masks, **kw):
    """dba_tree_attend with a cache of these strides; nothing is seen, so nothing of the cache is read."""
    import ctypes as C
    import paper_1804_06609_b200 as pkg
    c = T.KvCache(k=k.data_ptr(), v=v.data_ptr(), layers=1, head_stride=8, layer_stride=0, **kw)
    return pkg.lib().dba_tree_attend(t._h, C.byref(query), C.byref(c), table.data_ptr(), table.shape[1], ctx.data_ptr(), masks.data_ptr(), None)


@pytest.fixture
def far(dba):
    """A handle of rows of 16 bytes, two to a page, and a call to it that sees nothing."""
    from paper_1804_06609_b200 import tree as T
    t = _tree(dba, 1, 1, 1, 1, 8, 2, 16, 1)
    k, v = (torch.zeros(4, 2, 1, 8, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, out = (torch.zeros(1, 1, 1, 8, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table, ctx, masks = (torch.zeros(*s, dtype=torch.int32, device="cuda") for s in ((1, 16), (1,), (1, 1, 1)))
    query = T.TreeQuery(rows=1, q=q.data_ptr(), q_seq_stride=8, q_row_stride=8, q_head_stride=8, out=out.data_ptr(), out_seq_stride=8, out_row_stride=8,
                        out_head_stride=8, lse=None, scale=1.0)
    keep = (k, v, q, out, table, ctx, masks)
    return lambda pages, page16, token16, keep=keep: _rows_far_apart(t, T, query, k, v, table, ctx, masks, num_pages=pages, page_stride=8 * page16, token_stride=8 * token16)


def test_the_last_row_number_is_not_taken_for_none(dba, far):
    """Rows are counted in 16 bytes; the number 2^32 - 1 stands for a place without a row, so a layer must not have it."""
    assert far(65537, 65535, 65534) == 0                              # the last row's number: 65536 * 65535 + 65534 = 2^32 - 2
    assert far(65537, 65535, 65535) == 2                              # 2^32 - 1
    assert far(65537, 65535, 65536) == 2
    torch.cuda.synchronize()


def test_strides_whose_span_passes_64_bits_are_refused(dba, far):
    """16 pages at 2^60 elements end where 64 bits wrap around to 0."""
    assert far(17, 1 << 57, 1) == 2
    assert far(2, 1 << 59, 1) == 2 and far(2, 1, 1 << 59) == 2
    assert far((1 << 31) - 1, (1 << 32) - 2, (1 << 32) - 2) == 2
    torch.cuda.synchronize()


def test_advance_refuses_new_masks_over_the_old_ones(dba):
    import ctypes as C
    from paper_1804_06609_b200 import tree as T
    B, n, W = 3, 4, 2
    t = _tree(dba, B, n, 1, 1, 64, 16, 8, W)
    room = torch.zeros(4, B, n, W, dtype=torch.int32, device="cuda")
    back, pos, ctx = (torch.zeros(*s, dtype=torch.int32, device="cuda") for s in ((B, n), (B, 32 * W), (B,)))
    whole, at = 4 * B * n * W, room.data_ptr() + 4 * B * n * W
    adv = lambda to, ni=n, no=n: dba.lib().dba_tree_advance(t._h, ni, at, no, back.data_ptr(), None, None, 0, pos.data_ptr(), 32 * W, ctx.data_ptr(), C.byref(T.TreeNext(masks=to)))  # noqa: E731
    assert all(adv(at + by) == 1 for by in (0, 4, -4, whole - 4, 4 - whole))
    assert adv(at + whole) == 0 and adv(at - whole) == 0
    assert adv(at + whole - 4 * B * W, ni=n - 1) == 0 and adv(at - whole + 4 * B * W, no=n - 1) == 0       # fewer rows end earlier
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("bf16", 192), ("f32", 64)])
def test_pages_of_slots_no_row_sees_need_not_exist(dba, dtype, D):
    """A table whose arena pages are handed out as slots come into use: the others' entries are -1 and nobody looks at them."""
    B, n, H, K, ps, W = 2, 5, 8, 2, 16, 4
    rng = torch.Generator().manual_seed(51)
    per = (32 * W + 100) // ps + 1
    k, v, table = _cache(rng, B, per, ps, K, D, dtype)
    masks = torch.zeros(B, n, W, dtype=torch.int32)
    for b in range(B):
        for i in range(n):
            masks[b, i] = torch.from_numpy(M.words_of({i, 40 + i, 70, 100 + b}, W))       # of pages 0, 2, 4 and 6 of 8
    table[:, [1, 3, 5, 7]] = -1
    c = torch.tensor([100, 0], dtype=torch.int32)
    q = torch.randn(B, n, H, D, generator=rng).to(DT[dtype]).cuda()
    want = M.attend(q, k, v, table, c, masks, D ** -0.5, ps, W, k.shape[0])
    t = _tree(dba, B, n, H, K, D, ps, per, W, dtype)
    for top in (None, _top(masks).cuda()):
        _check(t.attend(q, k, v, table, c.cuda(), masks.cuda(), top), None, want, D, 300, dtype)
        assert t.status() == 0
    table[1, 4] = -1                                                  # slot 70: seen, and without a page
    want = M.attend(q, k, v, table, c, masks, D ** -0.5, ps, W, k.shape[0])
    _check(t.attend(q, k, v, table, c.cuda(), masks.cuda()), None, want, D, 300, dtype)
    assert t.status() == dba.TREE_BAD_PAGE


VARIANTS = [  # n, H, K, D, dtype: a case for each kernel a call can come to
    (5, 8, 8, 64, "bf16"), (40, 8, 8, 64, "bf16"), (20, 32, 8, 128, "bf16"), (4, 8, 4, 128, "bf16"), (4, 4, 2, 64, "bf16"), (6, 8, 2, 192, "bf16"),
    (4, 4, 2, 64, "f32"), (20, 8, 2, 128, "f32")]


@pytest.mark.parametrize("scale", [-0.2, 0.0])
@pytest.mark.parametrize("n,H,K,D,dtype", VARIANTS)
def test_scales_below_zero_and_of_zero(dba, n, H, K, D, dtype, scale):
    """The sign is the matrix instruction's, the size the softmax's; with a scale of zero every place counts alike."""
    B, ps, W, ctx = 2, 16, 2, [300, 9]
    rng = torch.Generator().manual_seed(61 + n + D)
    per = (32 * W + max(ctx)) // ps + 1
    k, v, table = _cache(rng, B, per, ps, K, D, dtype)
    masks = _masks(rng, B, n, W, 0.3)
    c = torch.tensor(ctx, dtype=torch.int32)
    q = (torch.randn(B, n, H, D, generator=rng) * 1.5).to(DT[dtype]).cuda()
    lse = torch.zeros(B, n, H, device="cuda")
    t = _tree(dba, B, n, H, K, D, ps, per, W, dtype)
    want = M.attend(q, k, v, table, c, masks, scale, ps, W, k.shape[0])
    _check(t.attend(q, k, v, table, c.cuda(), masks.cuda(), scale=scale, lse=lse), lse, want, D, 32 * W + 300, dtype)
    assert t.status() == 0


@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("n,H,K,D,dtype", VARIANTS)
def test_values_that_are_not_finite_in_every_kernel_and_in_cut_items(dba, n, H, K, D, dtype, cut):
    """inf seen by row 1, NaN by row 2, inf and -inf in tiles far apart by row 3: theirs alone, whether an item is one block's or is
    joined from pieces that begin inside its arena tiles."""
    B, ps, W, ctx = 2, 16, 40 if cut else 3, [1500, 30] if cut else [100, 0]
    A = 32 * W
    rng = torch.Generator().manual_seed(71 + n + D)
    per = (A + max(ctx)) // ps + 1
    k, v, table = _cache(rng, B, per, ps, K, D, dtype)
    slots = [2, A // 2 + 5, A - 7, 9]                                  # inf, NaN, -inf and inf
    masks = _masks(rng, B, n, W, 0.2, closed=0.0)
    for b in range(B):
        for i in range(n):
            own = set(M.bits_of(masks[b, i].numpy())) - set(slots) | {20}
            own |= {1: {slots[0]}, 2: {slots[1]}, 3: {slots[2], slots[3]}}.get(i, set())
            masks[b, i] = torch.from_numpy(M.words_of(own, W))
    c = torch.tensor(ctx, dtype=torch.int32)
    q = torch.randn(B, n, H, D, generator=rng).to(DT[dtype]).cuda()
    want = M.attend(q, k, v, table, c, masks, D ** -0.5, ps, W, k.shape[0])
    v2, h, last = v.clone(), K - 1, D - 1
    for slot, head, d, x in ((slots[0], h, 3, math.inf), (slots[1], 0, last, math.nan), (slots[2], h, 5, -math.inf), (slots[3], h, 5, math.inf)):
        v2[int(table[0, slot // ps]), slot % ps, head, d] = x           # of sequence 0 alone
    t = _tree(dba, B, n, H, K, D, ps, per, W, dtype)
    launches = t.launch_count()
    for top in (None, _top(masks).cuda()):
        got = t.attend(q, k, v2, table, c.cuda(), masks.cuda(), top).double().cpu()
        G, hit = H // K, torch.zeros(B, n, H, D, dtype=torch.bool)
        assert (got[0, 1, h * G:, 3] == math.inf).all() and torch.isnan(got[0, 2, :G, last]).all() and torch.isnan(got[0, 3, h * G:, 5]).all()
        hit[0, 1, h * G:, 3] = hit[0, 2, :G, last] = hit[0, 3, h * G:, 5] = True
        out, _, spread, reach = want
        tol = M.attend_tolerance(out, spread, reach, D, A + max(ctx), DT[dtype])
        assert torch.isfinite(got[~hit]).all() and ((got - out).abs() <= tol)[~hit].all()
    assert t.launch_count() == launches + (4 if cut else 2) and t.status() == 0


@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("n,H,K,D,dtype", [(1, 2, 2, 64, "bf16"), (2, 4, 4, 64, "bf16"), (1, 2, 1, 64, "f32")])
def test_more_sequences_than_a_block_has_threads(dba, n, H, K, D, dtype, cut):
    """The lengths are scanned by blocks of 128 to 256 threads: each has several sequences, and the last ones none."""
    B, ps, W = 1000, 16, 1
    rng = torch.Generator().manual_seed(81 + n)
    ctx = (torch.rand(B, generator=rng) ** 3 * 60).int()
    ctx[0], ctx[500], ctx[B - 1] = 0, 61, 60
    per = (32 + 61) // ps + 1
    long = per if not cut else 50                                     # a table that could hold more: its items may be cut
    k, v, table = _cache(rng, B, per, ps, K, D, dtype)
    wide = torch.full((B, long), -1, dtype=torch.int32)
    wide[:, :per] = table.cpu()
    masks = _masks(rng, B, n, W, 0.1)
    q = torch.randn(B, n, H, D, generator=rng).to(DT[dtype]).cuda()
    want = M.attend(q, k, v, table, ctx, masks, D ** -0.5, ps, W, k.shape[0])
    t = _tree(dba, B, n, H, K, D, ps, long, W, dtype)
    launches, lse = t.launch_count(), torch.zeros(B, n, H, device="cuda")
    _check(t.attend(q, k, v, wide.cuda(), ctx.cuda(), masks.cuda(), lse=lse), lse, want, D, 93, dtype)
    assert t.launch_count() == launches + (2 if cut else 1) and t.status() == 0


@pytest.mark.parametrize("dtype,hnd", [("bf16", False), ("f32", True)])
def test_commit_of_more_tokens_than_a_block_has_threads(dba, dtype, hnd):
    """A block looks 256 places up at a time."""
    B, layers, K, D, ps, W = 5, 3, 2, 64, 24, 17
    A, rng = 32 * W, torch.Generator().manual_seed(91)
    n = torch.tensor([257, A, 0, 256, 512], dtype=torch.int32)
    ctx = n + torch.tensor([5, 0, 3, 40, 1], dtype=torch.int32)
    per = (A + int(ctx.max())) // ps + 1
    shape = (layers, B * per, K, ps, D) if hnd else (layers, B * per, ps, K, D)
    k, v = (torch.randn(shape, generator=rng).to(DT[dtype]).cuda() for _ in range(2))
    if hnd:
        k, v = k.transpose(2, 3), v.transpose(2, 3)
    table = torch.randperm(B * per, generator=rng).int().view(B, per)
    src = torch.full((B, A), -1, dtype=torch.int32)
    want_k, want_v = k.clone(), v.clone()
    for b in range(B):
        m = int(n[b])
        src[b, :m] = torch.randperm(A, generator=rng)[:m].int()
        s, d = src[b, :m].long(), A + int(ctx[b]) - m + torch.arange(m)
        at, to = (table[b].long()[x // ps].cuda() for x in (s, d))
        for x, w in ((k, want_k), (v, want_v)):
            w[:, to, d.cuda() % ps] = x[:, at, s.cuda() % ps]
    t = _tree(dba, B, 4, K, K, D, ps, per, W, dtype)
    t.commit(k, v, table.cuda(), ctx.cuda(), src.cuda(), n.cuda())
    assert torch.equal(k, want_k) and torch.equal(v, want_v) and t.status() == 0


def test_advance_into_tensors_of_the_callers(dba):
    B, n, W, per = 3, 6, 2, 30
    rng = torch.Generator().manual_seed(95)
    t = _tree(dba, B, n, 1, 1, 64, 16, per, W)
    masks = _masks(rng, B, n, W, 0.1, closed=0.0).cuda()
    ctx = torch.tensor([4, 0, 9], dtype=torch.int32).cuda()
    for rows in (n, 4):
        back = (torch.rand(B, rows, generator=rng) * n).int().cuda()
        pos = [torch.arange(64, dtype=torch.int32).repeat(B, 1).cuda() for _ in range(2)]
        want = {f: x.clone() for f, x in t.advance(back, masks, pos[0], ctx).items()}
        room = {f: torch.full((x.numel() + 40,), -7, dtype=torch.int32, device="cuda") for f, x in t.new_next().items()}
        got = t.advance(back, masks, pos[1], ctx, out=room)
        assert set(got) == set(want) and all(torch.equal(got[f], want[f]) for f in want)
        assert all((room[f][want[f].numel():] == -7).all() and got[f].data_ptr() == room[f].data_ptr() for f in room)
    assert t.status() == 0
