"""The oracle of log-probabilities from hidden states against sums written out and against differences."""
import numpy as np
import pytest

from oracle import scoring


def _inputs(rng, R=5, d=7, V=11):
    tok = rng.integers(0, V, R)
    tok[2] = -1
    return rng.standard_normal((R, d)), rng.standard_normal((V, d)), tok, rng.standard_normal(R), rng.standard_normal(R)


def test_scores_are_those_of_the_logits():
    h, w, tok, _, _ = _inputs(np.random.default_rng(1))
    s, z = scoring.linear(h, w, tok, 1.3)
    for r in range(len(h)):
        assert np.allclose(z[r], [1.3 * sum(a * b for a, b in zip(h[r], x)) for x in w], rtol=1e-13, atol=1e-13)
        p = np.exp(z[r]) / np.exp(z[r]).sum()
        if tok[r] < 0:
            assert s[r]["logprob"] == 0 and s[r]["entropy"] == 0
        else:
            assert abs(s[r]["logprob"] - np.log(p[tok[r]])) < 1e-12 and abs(s[r]["entropy"] + (p * np.log(p)).sum()) < 1e-12
    alone, _ = scoring.linear(h, w, None, 1.3)
    assert all(abs(alone[r]["entropy"] - s[r]["entropy"]) == 0 for r in range(len(h)) if tok[r] >= 0)


@pytest.mark.parametrize("scale", [0.5, 1.0, 2.0])
def test_gradients_against_differences(scale):
    h, w, tok, g, gh = _inputs(np.random.default_rng(2))

    def f(h, w):
        s, _ = scoring.linear(h, w, tok, scale)
        return sum(g[r] * x["logprob"] + gh[r] * x["entropy"] for r, x in enumerate(s))

    dh, dw, _ = scoring.linear_grad(h, w, tok, g, gh, scale)
    assert (dh[2] == 0).all()
    # central differences of step 1e-5: third derivatives of some 10 leave 1e-9, rounding of sums of some 10 leaves 1e-15 / 1e-5
    for x, dx in ((h, dh), (w, dw)):
        for i in np.ndindex(*x.shape):
            was = x[i]
            x[i] = was + 1e-5
            up = f(h, w)
            x[i] = was - 1e-5
            down = f(h, w)
            x[i] = was
            assert abs((up - down) / 2e-5 - dx[i]) < 1e-7, i


def test_padding_adds_nothing_whatever_it_holds():
    h, w, tok, g, gh = _inputs(np.random.default_rng(3))
    want = scoring.linear_grad(h, w, tok, g, gh)
    h[2] = np.nan
    got = scoring.linear_grad(h, w, tok, g, gh)
    assert all(np.array_equal(a, b) for a, b in zip(want, got))
