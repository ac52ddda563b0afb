"""Pins of the oracle for pages and draws (oracle/serving_oracle.py)."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from oracle import verify_oracle as vo


def test_attention_of_a_chain_equals_a_librarys_causal_attention():
    rng = np.random.default_rng(0)
    q, k, v = (rng.standard_normal((9, 8)) for _ in range(3))
    out, lse, mag, _ = so.attention(q[4:], k, v, so.visible(4, 5))
    ref = torch.nn.functional.scaled_dot_product_attention(*(torch.from_numpy(x)[None] for x in (q, k, v)), is_causal=True)[0].numpy()
    assert np.allclose(out, ref[4:], atol=1e-12)
    assert np.all(mag >= np.abs(out) - 1e-12)


def test_attention_of_a_tree_equals_the_tree_oracle():
    rng = np.random.default_rng(1)
    parent, P = np.array([-1, 0, 0, 1, 3, 2]), 7
    q, kt, vt = (rng.standard_normal((6, 1, 8)) for _ in range(3))
    kc, vc = (rng.standard_normal((1, 1, P, 8)) for _ in range(2))
    ref, ref_lse = vo.tree_attention(q, kt, vt, kc, vc, parent, np.array([0, 6]), np.array([P]))
    out, lse, _, _ = so.attention(q[:, 0], np.concatenate([kc[0, 0], kt[:, 0]]), np.concatenate([vc[0, 0], vt[:, 0]]), so.visible(P, 6, parent))
    assert np.allclose(out, ref[:, 0]) and np.allclose(lse, ref_lse[:, 0])


def test_windows():
    chain = np.arange(-1, 9)
    assert np.array_equal(so.visible(5, 10), so.visible(5, 10, chain))
    assert np.array_equal(so.visible(5, 10), so.visible(5, 10, None, 15))
    w = so.visible(5, 10, None, 3, 2)
    assert np.array_equal(w, so.visible(5, 10, chain, 3, 2))
    assert w[0].tolist() == [True, True, False, True, True, True] + [False] * 9      # two sinks, positions 3 to 5
    assert all(w[i].sum() == 5 for i in range(10))


def test_slots_against_a_dictionary():
    rng = np.random.default_rng(2)
    page, rows = 16, 6
    seq, new = rng.integers(0, 50, rows), rng.integers(0, 40, rows)
    table, free = np.full((rows, 8), -7), rng.permutation(100)
    place, at = {}, 0
    for s in range(rows):
        for e in range(-(-int(seq[s]) // page)):
            table[s, e] = free[at]
            at += 1
    free = free[at:]
    got = so.paged_slots(seq, new, table, free, len(free), page, int(new.sum()) + 5)
    for s in range(rows):
        for e in range(-(-int(seq[s] + new[s]) // page)):
            place[s, e] = int(got["table"][s, e])
    assert len(set(place.values())) == len(place)                                     # no page twice
    assert not got["refused"].any() and got["free_count"] == len(free) - (len(place) - at)
    for s in range(rows):
        for j in range(new[s]):
            t, x = got["q_off"][s] + j, int(seq[s]) + j
            assert got["slot_map"][t] == place[s, x // page] * page + x % page and got["position"][t] == x
    assert (got["slot_map"][-5:] == -1).all()


def test_slots_run_out_in_order():
    got = so.paged_slots([16, 16, 5, 16], [1, 20, 3, 1], np.arange(16).reshape(4, 4), [90, 91], 2, 16, 100)
    assert got["refused"].tolist() == [False, True, False, True]                      # the second asks for two of one left; the third for none
    assert got["seq_len"].tolist() == [17, 16, 8, 16] and got["free_count"] == 1 and got["table"][0, 1] == 91


@pytest.mark.parametrize("top_k,top_p,min_p", [(0, 1, 0), (5, 1, 0), (0, 0.7, 0), (0, 1, 0.1), (7, 0.8, 0.02)])
def test_draws_follow_the_filtered_distribution(top_k, top_p, min_p):
    rng = np.random.default_rng(3)
    x = rng.standard_normal(20) * 2
    order = np.argsort(-x)
    p = np.exp(x / 0.9)
    p /= p.sum()
    keep = np.zeros(20, bool)
    chosen = order[:top_k or 20]
    mass = np.cumsum(p[chosen]) / p[chosen].sum()
    chosen = chosen[:int((mass < top_p).sum()) + 1] if top_p < 1 else chosen
    keep[chosen] = True
    keep &= p >= min_p * p.max()
    p = np.where(keep, p, 0) / p[keep].sum()
    us = (np.arange(4000) + 0.5) / 4000
    tokens = np.array([so.sample(x, u, 0.9, top_k, top_p, min_p)[0] for u in us])
    assert np.abs(np.bincount(tokens, minlength=20) / 4000 - p).max() < 1 / 2000      # an interval of 4000 steps is counted to one step at either end
    assert so.sample(x, 0.3, 0.9, top_k, top_p, min_p)[1] == pytest.approx(p[so.sample(x, 0.3, 0.9, top_k, top_p, min_p)[0]])


def test_edges_of_draws():
    inf, nan = np.inf, np.nan
    assert so.sample([1, 3, 3, 2], 0.9, 0.0)[:2] == (1, 1.0)                           # greedy: the first of the largest
    assert so.sample([-inf, nan], 0.5)[:2] == (-1, 0.0)
    assert so.sample([0, inf, 1, inf], 0.6)[:2] == (3, 0.5)
    assert so.sample([nan, 0, -inf, 0], 0.5)[:2] == (3, 0.5)
    assert so.sample([1, 1, 1, 0], 0.99, 1.0, 1)[2] == 3 and so.sample([1, 1, 1, 0], 0.99, 1.0, 0, 0.1)[2] == 3      # ties stay
    low = np.finfo(np.float32).min
    assert so.sample([low, low], 0.7)[:2] == (1, 0.5) and so.sample([low, 0], 0.0)[0] == 1
