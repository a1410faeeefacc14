"""The oracle of the operators on class scores against closed forms, brute
force and finite differences."""
import itertools

import numpy as np
import pytest

from oracle import scores_oracle as S


def test_order_ties_and_absent():
    z = np.array([1.0, 3.0, 1.0, -np.inf, 3.0, -0.0, 0.0, np.nan])
    assert S.order(z).tolist() == [1, 4, 0, 2, 5, 6]
    v, c = S.top_logits(z[None], 9)
    assert c[0].tolist() == [1, 4, 0, 2, 5, 6, -1, -1, -1]
    assert np.isneginf(v[0, 6:]).all()


def test_distill_closed_forms():
    # a teacher that knows every class and equals the student: no loss, no gradient
    rng = np.random.default_rng(0)
    z = rng.standard_normal((5, 6))
    v, c = S.top_logits(z, 6)
    loss, g, cs = S.distill(z, v, c, 1.7, 0.3)
    assert abs(loss) < 1e-15 and np.abs(g).max() < 1e-15 and np.abs(cs).max() < 1e-15
    # one entry: the cross-entropy against that class
    loss, g, _ = S.distill(z, v[:, 1:2], c[:, 1:2], 1.0)
    p = np.exp(z) / np.exp(z).sum(1, keepdims=True)
    r = np.arange(5)
    assert np.isclose(loss, -np.log(p[r, c[:, 1]]).mean(), rtol=1e-14)
    p[r, c[:, 1]] -= 1
    assert np.allclose(g, p / 5, rtol=0, atol=1e-15)


def test_distill_gradient_against_differences():
    rng = np.random.default_rng(1)
    z = rng.standard_normal((4, 9))
    v = rng.standard_normal((4, 5))
    c = rng.integers(-1, 9, (4, 5))
    c[1] = -1                                   # nothing to learn from
    c[2] = [3, 3, 3, 8, -1]                     # one class three times
    mask = np.array([1, 1, 1, 0], np.uint8)
    f = lambda y: S.distill(y, v, c, 2.5, 0.7, mask=mask)[0]  # noqa: E731
    _, g, _ = S.distill(z, v, c, 2.5, 0.7, mask=mask)
    h = 1e-5
    for i, j in itertools.product(range(4), range(9)):
        d = np.zeros_like(z)
        d[i, j] = h
        # central differences: error h^2 / 6 times a third derivative below 1
        assert abs((f(z + d) - f(z - d)) / (2 * h) - g[i, j]) < 1e-9
    assert not g[1].any() and not g[3].any()


@pytest.mark.parametrize("top_k,top_p,min_p", [(0, 1.0, 0.0), (3, 1.0, 0.0), (0, 0.6, 0.0), (0, 1.0, 0.3),
                                               (5, 0.8, 0.05), (1, 0.01, 1.0)])
def test_sample_keeps_and_draws(top_k, top_p, min_p):
    rng = np.random.default_rng(2)
    z = np.round(rng.standard_normal(8), 1)     # with ties now and then
    T = 0.9
    # brute force: the shortest beginning of the order that each filter allows
    o = sorted(range(8), key=lambda c: (-z[c], c))
    w = {c: np.exp((z[c] - z[o[0]]) / T) for c in o}
    m = top_k or 8
    part = o[:m]
    total = sum(w[c] for c in part)
    kp = next(k for k in range(1, m + 1) if sum(w[c] for c in part[:k]) >= top_p * total * (1 - 1e-15))
    kept = [c for c in part[:kp] if w[c] >= min_p]
    assert S.sample_row(z, 0.0, T, top_k, top_p, min_p)[2].tolist() == sorted(kept)
    # u on a fine grid gives every kept class its share
    us = (np.arange(20000) + 0.5) / 20000
    got = [S.sample_row(z, u, T, top_k, top_p, min_p)[0] for u in us]
    s = sum(w[c] for c in kept)
    for c in range(8):
        share = w[c] / s if c in kept else 0.0
        assert abs(np.mean(np.array(got) == c) - share) <= 1.01 / 20000   # one grid point at each end


def test_sample_without_an_answer():
    assert S.sample_row([-np.inf, -np.inf], 0.5, 1.0)[:2] == (-1, 0.0)
    assert S.sample_row([0.0, np.nan], 0.5, 1.0)[:2] == (-1, 0.0)
    assert S.sample_row([0.0, 1.0], 1.0, 1.0)[:2] == (-1, 0.0)
    assert S.sample_row([0.0, 1.0], 1.0, 0.0)[:2] == (1, 1.0)
    assert S.sample_row([-np.inf, 2.0, -np.inf], 0.999, 0.1)[:2] == (1, 1.0)
