"""Pins of the oracle for gathered weights and eviction: against other ways to write the same, and by hand."""
import numpy as np

from oracle import serving_oracle as so


def test_gathered_weights_are_the_columns_of_the_softmax():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((7, 3, 16)), rng.standard_normal((40, 16))
    sees = so.visible(33, 7)
    lse = np.stack([so.attention(q[:, g], k, k, sees)[1] for g in range(3)], 1)
    got, size = so.attention_mass(q, lse, k, sees)
    z = np.where(sees[:, None], np.einsum("tgd,nd->tgn", q, k) / 4, -np.inf)
    w = np.exp(z - z.max(2, keepdims=True))
    assert np.allclose(got, (w / w.sum(2, keepdims=True)).sum((0, 1)), rtol=1e-12)
    assert np.isclose(got.sum(), 21) and (size >= got * np.abs(lse).min()).all()
    lse[2, 1] = np.inf
    assert np.isclose(so.attention_mass(q, lse, k, sees)[0].sum(), 20)


def test_eviction_by_hand():
    #                     f           m     recent
    mass = np.array([0, 5, 1, 7, 5, 5, 2, 9, 0, 0.])
    # ten positions, six remain: one at the front, two at the end, of 1 .. 7 the three heaviest: 7 (9), 3 (7), and of 1, 4, 5 with equal weights the first
    assert so.evict_places(mass, 10, 6, first=1, recent=2) == [0, 1, 7, 3, 8, 9]
    assert so.evict_places(mass, 10, 10, 1, 2) == list(range(10)) == so.evict_places(mass, 10, 99)
    assert so.evict_places(mass, 10, 0) == [] and so.evict_places(mass, 10, 2, first=3, recent=4) == [0, 1, 2, 6, 7, 8, 9]
    assert so.evict_places(np.full(6, np.nan), 6, 2) == [0, 1]
    assert so.evict_places(np.array([np.nan, -np.inf, -1.0]), 3, 2) == [2, 1]


def test_eviction_keeps_the_heaviest():
    rng = np.random.default_rng(1)
    for _ in range(200):
        n = int(rng.integers(0, 60))
        budget, first, recent = (int(rng.integers(0, 70)) for _ in range(3))
        mass = rng.integers(0, 9, n).astype(float)
        place = so.evict_places(mass, n, budget, first, recent)
        f, r = min(first, n), min(recent, n - min(first, n))
        assert len(place) == max(min(budget, n), f + r) and len(set(place)) == len(place)
        m = len(place) - r
        assert place[:f] == list(range(f)) and place[m:] == list(range(n - r, n))
        gone = set(range(n)) - set(place)
        if gone and m > f:
            order = lambda y: (-mass[y], y)  # noqa: E731
            assert max(map(order, place[f:m])) < min(map(order, gone))
        assert all(y == i or y >= m for i, y in enumerate(place[:m]))          # what stays, and what comes from behind
