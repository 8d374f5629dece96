"""The example with contexts that are thinned: every open hypothesis' logits against its whole text, in which each token sees what was left for it when it
came, and the weights that tokens have received against those texts' attention."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import constrained_decode
    return constrained_decode


@pytest.mark.parametrize("dtype,kw", [("f32", dict()), ("f32", dict(shared=20)), ("f32", dict(norm=True, B=3, k=20, heads=4, kv_heads=4, keep=7)), ("f32", dict(shared=33, norm=True, page_size=5)),
                                      ("bf16", dict()), ("bf16", dict(shared=20, norm=True)), ("bf16", dict(shared=7, B=2, heads=16, kv_heads=2, dim=128, keep=9, page_size=8)),
                                      ("bf16", dict(norm=True, B=2, k=20, heads=8, kv_heads=4, layers=3))])
def test_logits_and_weights_of_thinned_contexts(example, dtype, kw):
    _, worst, info = example.decode(dtype=dtype, check=True, **{**dict(steps=16, prompt=24, keep=12), **kw})
    assert info["evicted"] > 0 and info["settled"] > 0
    # logits: as where nothing is thinned, whose sums have as many terms or more
    assert worst < (2e-4 if dtype == "f32" else 0.25), worst
    # fp32: a score's 64 products of values up to 4 standard deviations, (64 + 4) 2^-24 of some 30, and as much from hidden states that differ in the last
    # bits: 2.4e-4 of a probability; a weight is a sum of them
    if dtype == "f32":
        assert info["worst_weight"] < 1e-3, info["worst_weight"]


@pytest.mark.parametrize("mistake", ["places", "weights", "positions"])
def test_the_check_sees_what_is_wrong(example, monkeypatch, mistake):
    """A mistake in the plain texts' own books: others stay, a row's attention is left out, a token too few has gone."""
    real = example.Check
    if mistake == "places":
        monkeypatch.setattr(real, "evicted", lambda self, kept, plain=real.evicted: plain(self, torch.where(kept >= 0, torch.arange(kept.shape[-1], device=kept.device), -1)))
    elif mistake == "weights":
        def logits(self, *args, plain=real.logits):
            plain(self, *args)
            self.received = [[[[0.9 * x for x in row] for row in by_head] for by_head in by_sequence] for by_sequence in self.received]
        monkeypatch.setattr(real, "logits", logits)
    else:
        monkeypatch.setattr(real, "step", lambda self, nx, backptr, tokens, offset, plain=real.step: plain(self, nx, backptr, tokens, [max(0, x - 1) for x in offset]))
    call = lambda: example.decode(dtype="f32", check=True, steps=8, prompt=24, keep=12)  # noqa: E731
    if mistake == "positions":
        with pytest.raises(AssertionError):
            call()
        return
    _, worst, info = call()
    assert worst > 2e-3 if mistake == "places" else info["worst_weight"] > 1e-2


def test_the_command_checks_thinned_contexts(example, monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["constrained_decode.py", "--B", "2", "--k", "4", "--steps", "8", "--prompt", "20", "--keep", "10", "--check", "--dtype", "f32"])
    example.main()
    out = capsys.readouterr().out
    assert "tokens evicted" in out and "largest difference of a logit" in out and "of a token's weight" in out
