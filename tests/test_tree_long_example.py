"""The example with a prefix that all sentences share, with norms of queries and keys, and with contexts that are thinned."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("dtype,kw", [("f32", dict(shared=20)), ("f32", dict(norm=True)), ("f32", dict(shared=33, norm=True, heads=4, kv_heads=4)),
                                      ("bf16", dict(shared=20, norm=True)), ("bf16", dict(shared=50, B=5, k=5, heads=16, kv_heads=2, dim=128, page_size=8)),
                                      ("bf16", dict(shared=7, norm=True, B=2, k=20, heads=8, kv_heads=4, dim=64, page_size=5))])
def test_constrained_decoding_after_a_shared_prefix(dtype, kw):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from constrained_decode import decode
    _, worst, info = decode(dtype=dtype, check=True, steps=10, **kw)
    # the bounds of the example's other test: logits of the size of 3; fp32 products over a few hundred terms, bf16 some ten roundings a layer; the
    # own part's one more rounding is within them
    assert worst < (2e-4 if dtype == "f32" else 0.25), worst
    assert info["settled"] > 0


@pytest.mark.parametrize("dtype,kw", [("f32", {}), ("bf16", dict(shared=20, norm=True))])
def test_constrained_decoding_with_contexts_that_are_thinned(dtype, kw):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from constrained_decode import decode
    (tokens, length, score, flags), _, info = decode(dtype=dtype, steps=16, prompt=24, keep=12, check=True, **kw)
    assert info["evicted"] > 0 and max(info["context"]) <= 12 and info["settled"] > 0


def test_keeping_everything_changes_nothing():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from constrained_decode import decode
    one, two = (decode(dtype="f32", steps=10, keep=keep)[0] for keep in (0, 1000))
    assert all((a == b).all() for a, b in zip(one, two))
