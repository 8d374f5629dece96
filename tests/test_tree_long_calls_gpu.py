"""Calls of the token tree's operators for long and shared texts that their documentation allows and ordinary runs do not make: keys that are not
finite, two handles at work at once, calls without log-sum-exps, tables longer than what is kept; and what is refused."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests import long_model as L                                                       # noqa: E402
from tests.test_tree_gpu import DT, _cache, _tree, dba                                  # noqa: E402,F401
from tests.test_tree_long_gpu import _attend, _compare, _i32, _setup                    # noqa: E402


@pytest.mark.parametrize("dtype,D,ps,rows,G", [("bf16", 64, 16, 3, 6), ("bf16", 128, 5, 3, 6), ("bf16", 128, 8, 50, 6), ("bf16", 256, 16, 3, 6), ("bf16", 256, 16, 4, 2), ("f32", 64, 16, 3, 6),
                                               ("f32", 128, 7, 50, 6), ("f32", 64, 16, 2, 1), ("f32", 64, 5, 4, 2), ("f32", 128, 7, 7, 1), ("f32", 256, 16, 2, 3), ("f32", 40, 9, 5, 1)])
def test_weights_of_keys_that_are_not_finite(dba, dtype, D, ps, rows, G):
    """An infinite element of a key whose scores are -inf receives nothing, whatever rows that are closed or not there would make of it."""
    rng = torch.Generator().manual_seed(1)
    B, K, n = 2, 2, 150
    k, v, table = _cache(rng, B, -(-n // ps), ps, K, D, dtype)
    q = torch.randn(B, rows, K * G, D, generator=rng).to(DT[dtype])
    q[..., 3] = -q[..., 3].abs() - 0.5                                  # all see a key with +inf there from the other side
    lse = torch.full((B, rows, K * G), 3.0)
    lse[0, 1] = -math.inf
    lse[1] = -math.inf                                                  # a sequence that has ended
    q[0, 1] = math.nan
    want, bound = L.weigh(q, k, table, [n, n], lse, torch.full((B, K, table.shape[1] * ps), 2.0), 0.5, D ** -0.5, ps, 0)
    for p, x in ((7, math.inf), (140, math.inf)):
        for b in range(B):
            k[int(table[b, p // ps]), p % ps, :, 3] = x
    for p in (9, 141):                                                  # NaN: where nobody looks it is nothing
        k[int(table[1, p // ps]), p % ps] = math.nan
    tree = _tree(dba, B, rows, K * G, K, D, ps, table.shape[1], 0, dtype)
    w = torch.full((B, K, table.shape[1] * ps), 2.0, device="cuda")
    tree.weigh(q.cuda(), k, table, _i32([n, n]), lse.cuda(), weight=w, decay=0.5)
    w = w.double().cpu()
    plain = torch.ones(n, dtype=torch.bool)
    plain[[7, 140]] = False
    assert (w[0, :, 7] == 1.0).all() and (w[0, :, 140] == 1.0).all() and (w[1, :, :n] == 1.0).all()
    assert ((w - want).abs() <= bound)[0, :, :n][:, plain].all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_shared_calls_without_log_sum_exps_and_one_after_another(dba, dtype):
    s = _setup(dba, 3, 5, 4, 4, 2, 64, [20, 3, 0, 40, 9], 16, 1, dtype, [0, 2, 5], [300, 41])
    with_lse, lse = _attend(s, 0.2)
    with_lse = with_lse.clone()
    _compare(s, with_lse, lse, 0.2)
    outs = [torch.empty_like(s["q"]) for _ in range(3)]
    q = s["q"]
    for i, out in enumerate(outs):                                      # (the same scratch, nothing waited for)
        s["q"] = q * (1 - i)
        _attend(s, 0.2, lse=False, out=out)
    assert torch.equal(outs[0], with_lse)
    for i in (1, 2):
        s["q"] = q * (1 - i)
        _compare(s, outs[i], None, 0.2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_handles_on_two_streams_at_once(dba, dtype):
    runs = []
    for seed in (5, 6):
        s = _setup(dba, seed, 8, 20, 8, 2, 64, [30 * i for i in range(8)], 16, 2, dtype, [0, 8], [3000 + seed])
        side = torch.cuda.Stream()
        per = s["table"].shape[1]
        s["tree"] = _tree(dba, 8, 20, 8, 2, 64, 16, per, 2, dtype, prefixes=1, stream=side)
        w = torch.zeros(8, 2, per * 16 - 64, device="cuda")
        args = (_i32(s["ctx"]), (_i32(s["first"]), _i32(s["length"]), s["ptable"]), s["masks"].cuda(), torch.empty_like(s["q"]), torch.empty(8, 20, 8, device="cuda"))
        runs.append((s, side, w, args))

    def call(s, side, w, args):
        n, prefix, masks, out, lse = args
        with torch.cuda.stream(side):
            s["tree"].attend_shared(s["q"], s["k"], s["v"], s["table"], n, prefix, masks=masks, scale=0.1, out=out, lse=lse)
            s["tree"].weigh(s["q"], s["k"], s["table"], n, lse, weight=w, decay=0.5, scale=0.1)

    torch.cuda.synchronize()
    want = []
    for run in runs:
        call(*run)
        torch.cuda.synchronize()
        want.append([x.clone() for x in (run[3][3], run[3][4], run[2])])
        run[2].zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for run in runs:
            run[3][3].fill_(0)
            run[3][4].fill_(0)
            run[2].zero_()
        torch.cuda.synchronize()
        for run in runs:
            call(*run)
        torch.cuda.synchronize()
        for run, w in zip(runs, want):
            assert all(torch.equal(a, b) for a, b in zip((run[3][3], run[3][4], run[2]), w)) and run[0]["tree"].status() == 0


@pytest.mark.parametrize("keep,recent", [(500, 3), (64, 64), (65, 0), (1, 1)])
def test_eviction_again_and_again_in_place(dba, keep, recent):
    """Also with more to keep than the table holds: then nothing changes."""
    rng = torch.Generator().manual_seed(keep)
    k, v, table = _cache(rng, 2, 8, 16, 2, 64, "bf16")
    tree = _tree(dba, 2, 1, 2, 2, 64, 16, 8, 0)
    w, n = torch.rand(2, 2, 128, generator=rng).cuda(), [128, 70]
    for _ in range(3):
        before_k, before_w = k.clone(), w.clone()
        got = tree.evict(k, v, table, _i32(n), w, keep, recent=recent)
        assert got["ctx_len"].tolist() == [min(x, keep) for x in n] and got["dropped"].tolist() == [x - min(x, keep) for x in n]
        for b in range(2):
            for h in range(2):
                stay = L.keep(before_w[b, h, :n[b]].tolist(), keep, recent)
                assert got["kept"][b, h].tolist() == stay + [-1] * (keep - len(stay))
                src, dst = torch.tensor(stay, device="cuda"), torch.arange(len(stay), device="cuda")
                assert torch.equal(k[table[b].long()[dst // 16], dst % 16, h], before_k[table[b].long()[src // 16], src % 16, h])
                assert torch.equal(w[b, h, :len(stay)], before_w[b, h, src]) and (w[b, h, len(stay):n[b]] == 0).all()
        n = [min(x, keep) for x in n]
        grown = [min(128, x + 20) for x in n]                            # tokens come behind them
        for b in range(2):
            w[b, :, n[b]:grown[b]] = torch.rand(2, grown[b] - n[b], generator=rng).cuda()
        n = grown


def test_calls_that_are_refused(dba):
    s = _setup(dba, 1, 3, 2, 2, 2, 64, [20, 3, 9], 16, 1, "bf16", [0, 3], [30])
    with pytest.raises(RuntimeError):
        _attend(s, 0.2, out=s["q"])
    q, lse, table, n = s["q"], torch.zeros(3, 2, 2, device="cuda"), s["table"], _i32(s["ctx"])
    places = table.shape[1] * 16
    for w in (torch.zeros(1, 2, places, device="cuda").expand(3, 2, places), torch.zeros(3, 1, places, device="cuda").expand(3, 2, places)):
        with pytest.raises(RuntimeError):
            s["tree"].weigh(q, s["k"], table, n, lse, weight=w)
        with pytest.raises(RuntimeError):
            s["tree"].evict(s["k"], s["v"], table, n, w, 4)
    k, v = (x[None].expand(2, *x.shape).contiguous() for x in (s["k"], s["v"]))
    with pytest.raises(RuntimeError):
        s["tree"].evict(k, v, table, n, torch.zeros(1, 3, 2, places, device="cuda").expand(2, 3, 2, places), 4)
    assert s["tree"].status() == 0
