"""The example that runs the step and the token tree together: every hypothesis' logits against its whole text without a cache."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("dtype,kw", [("f32", {}), ("bf16", {}), ("f32", dict(B=3, k=20, heads=4, kv_heads=4, dim=64, prompt=5)),
                                      ("bf16", dict(B=5, k=5, heads=16, kv_heads=2, dim=128, prompt=30, page_size=5)),
                                      ("bf16", dict(B=2, k=8, heads=8, kv_heads=4, dim=64, layers=3))])
def test_constrained_decoding_with_the_tree_as_its_cache(dtype, kw):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from constrained_decode import EOS, decode
    (tokens, length, score, flags), worst, info = decode(dtype=dtype, check=True, steps=16, **kw)
    # Logits are of the size of 3 (unembedding 3 / sqrt(d) on unit rows).  fp32: products over a few hundred terms and two to
    # three layers, some 1e-5; bf16: every layer's products and sums are rounded to 2^-9, in another order on either side,
    # some ten roundings of values up to 4 standard deviations: 10 * 2^-9 * 12 < 0.25.
    assert worst < (2e-4 if dtype == "f32" else 0.25), worst
    assert info["settled"] > 0
    for b, phrases in enumerate(info["constraints"]):
        if flags[b] & 1:                                     # a completed hypothesis has every constraint
            text = tokens[b, :length[b]].tolist()
            assert text[-1] == EOS
            for p in phrases:
                assert any(text[i:i + len(p)] == p for i in range(len(text)))
