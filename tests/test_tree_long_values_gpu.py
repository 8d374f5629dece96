"""Values that are not finite in the token tree's operators for long and shared texts."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests import long_model as L                                                       # noqa: E402
from tests.test_tree_gpu import DT, dba                                                 # noqa: E402,F401
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
