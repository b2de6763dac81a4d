"""The 64-bit oracles of the cache and scoring operators, against the definitions by other means."""
import numpy as np
import pytest

from oracle import kv8, scoring


def _e4m3_values():
    v = [m * 2.0 ** -9 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)]
    return np.array([x for x in v if x <= 448.0])


def test_grid_of_e4m3_is_the_nearest_value():
    vals = _e4m3_values()
    rng = np.random.default_rng(0)
    x = np.concatenate([vals, (vals[1:] + vals[:-1]) / 2, rng.uniform(0, 448, 2000), 2.0 ** rng.uniform(-14, 8.8, 2000)])
    got = kv8.to_grid(x, "e4m3")
    assert np.isin(got, vals).all()
    best = np.abs(x[:, None] - vals[None]).min(1)
    assert (np.abs(got - x) == best).all()
    for a in (vals[1:] + vals[:-1]) / 2:  # halfway: the even one of the two (its place in the list is even)
        i = int(np.flatnonzero(vals == kv8.to_grid(np.array([a]), "e4m3")[0])[0])
        assert i % 2 == 0
    assert (kv8.to_grid(-x, "e4m3") == -got).all()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_exponent_is_the_smallest_that_holds(fmt):
    rng = np.random.default_rng(1)
    for a in np.concatenate([2.0 ** rng.uniform(-60, 60, 300), [448.0, 127.0, 448.0 * 2 ** 7, 127.0 / 64, 448.0000001, 1e-45, 0.0]]):
        e = kv8.exponent(a, fmt)
        assert e >= -100 and a <= kv8.TOP[fmt] * 2.0 ** e
        assert e == -100 or a > kv8.TOP[fmt] * 2.0 ** (e - 1)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_many_raises_of_a_scale_cost_at_most_one_smallest_step(fmt):
    rng = np.random.default_rng(2)
    codes, scales = np.zeros((1, 2, 1, 128, 8)), np.ones((1, 2, 1, 4))
    x = rng.standard_normal((32, 1, 8)) * 2.0 ** np.linspace(-6, 14, 32)[:, None, None]  # each token larger than the one before
    for t in range(32):
        kv8.write(codes, scales, fmt, [0], t, x[t:t + 1], -x[t:t + 1])
    k, v = kv8.read(codes, scales, [0], 0, 32)
    s = scales[0, 0, 0, 0]
    bound = np.abs(x) * 2.0 ** -4 + s * 2.0 ** -9 if fmt == "e4m3" else s
    assert (np.abs(k - x) <= bound).all() and (v == -k).all()


def test_gradient_against_differences():
    rng = np.random.default_rng(3)
    z = rng.standard_normal(23) * 2
    z[5] = -np.inf
    tok, g, gh, h = 7, 0.7, -1.3, 1e-5
    f = lambda y: (lambda s: g * s["logprob"] + gh * s["entropy"])(scoring.score(y, tok))  # noqa: E731
    want = scoring.grad(z, tok, g, gh)
    for v in range(23):
        if v == 5:
            assert want[v] == 0
            continue
        a, b = z.copy(), z.copy()
        a[v] -= h
        b[v] += h
        assert abs((f(b) - f(a)) / (2 * h) - want[v]) < 1e-8


def test_scores_of_a_uniform_row_and_order_of_ties():
    s = scoring.score(np.full(8, -3.0e38), 3, top=10)
    assert abs(s["logprob"] + np.log(8)) < 1e-12 and abs(s["entropy"] - np.log(8)) < 1e-12
    assert s["top_token"] == [0, 1, 2, 3, 4, 5, 6, 7, -1, -1]
