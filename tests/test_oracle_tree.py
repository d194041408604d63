"""Pins of the oracle for trees, sampling and acceptance: brute force, the one-token oracle, frequencies."""
import itertools
import math

import numpy as np
import pytest

from oracle import sp_oracle as orc
from oracle import sp_oracle_tree as ort


def test_a_chain_is_token_by_token_decode():
    rng = np.random.default_rng(1)
    S, n, H, Hkv, d = 9, 5, 4, 2, 8
    k, v = rng.standard_normal((2, S, Hkv, d))
    q, kn, vn = rng.standard_normal((n, H, d)), rng.standard_normal((n, Hkv, d)), rng.standard_normal((n, Hkv, d))
    o, absum, _ = ort.tree_attention(q, kn, vn, k, v, [i - 1 for i in range(n)], 0.3)
    for i in range(n):
        one = orc.pruned_decode_step(q[i], kn[i], vn[i], k, v, np.arange(S), kn[:i], vn[:i], 0.3)
        np.testing.assert_allclose(o[i], one, rtol=1e-12)
    assert (absum >= np.abs(o) - 1e-15).all()


def test_brothers_do_not_see_each_other_and_bias_is_a_penalty():
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((2, 3, 1, 4))
    q, kn, vn = rng.standard_normal((3, 1, 4)), rng.standard_normal((3, 1, 4)), rng.standard_normal((3, 1, 4))
    parent = [-1, 0, 0]
    o, _, _ = ort.tree_attention(q, kn, vn, k, v, parent, 1.0)
    kn2, vn2 = kn.copy(), vn.copy()
    kn2[1] += 5
    vn2[1] -= 7
    o2, _, _ = ort.tree_attention(q, kn2, vn2, k, v, parent, 1.0)
    assert np.array_equal(o[[0, 2]], o2[[0, 2]]) and not np.allclose(o[1], o2[1])
    # a steep slope leaves the nearest key alone: each node itself
    pos_old, pos = np.array([0.0, 1.0, 2.0]), np.array([3.0, 4.0, 4.0])
    far, _, _ = ort.tree_attention(q, kn, vn, k, v, parent, 1.0, slopes=np.array([200.0]), pos_q=pos, pos_old=pos_old)
    np.testing.assert_allclose(far[:, 0], vn[:, 0], rtol=1e-9)
    assert ort.lineage([-1, 0, 5, 1], 3) == [0, 1, 3] and ort.lineage([-1, 0, 5, 1], 2) == [2]


def _brute_row(x, u, T, k, p, m):
    """The definition, token by token over a sorted list of (weight, index)."""
    order = sorted((i for i in range(len(x)) if x[i] == x[i] and x[i] != -math.inf), key=lambda i: (-x[i], i))
    if not order:
        return -1
    if T <= 0:
        return order[0]
    w = [math.exp((x[i] - x[order[0]]) / T) for i in order]
    left = [j for j in range(len(w)) if m <= 0 or w[j] >= min(m, 1)]
    left = left[:k] if k > 0 else left
    if p < 1:
        total, some, run = sum(w[j] for j in left), [], 0.0
        for j in left:
            if some and run >= p * total:
                break
            some.append(j)
            run += w[j]
        left = some
    total, run = sum(w[j] for j in left), 0.0
    for j in left:
        run += w[j]
        if run > u * total:
            return order[j]
    return order[left[-1]]


def test_rows_against_the_definition():
    rng = np.random.default_rng(3)
    for T, k, p, m in itertools.product((0.0, 0.5, 2.0), (0, 1, 3), (1.0, 0.6, 0.0), (0.0, 0.3, 1.0)):
        for _ in range(6):
            x = np.round(rng.standard_normal(9) * 2) / 2                       # ties
            x[rng.integers(0, 9)] = rng.choice([-np.inf, np.nan, 0.5])
            u = float(rng.random())
            token, logprob, margin = ort.sample_row(x, u, T, k, p, m)
            if margin > 1e-9:
                assert token == _brute_row(list(x), u, T, k, p, m), (x, u, T, k, p, m)
            assert logprob <= 1e-12
    assert ort.sample_row([-np.inf, np.nan], 0.5)[:2] == (-1, -np.inf)
    assert ort.sample_row([1.0, np.inf, 3.0, np.inf], 0.6)[:2] == (3, -math.log(2))
    assert ort.sample_row([0.0, 0.0, 0.0, 0.0], 0.5, top_p=0.5)[0] == 1        # two of four weigh half
    assert ort.sample_row([2.0, 2.0, 1.0], 7.0)[0] == 2 and ort.sample_row([2.0, 2.0, 1.0], float("nan"))[0] == 0


def test_draws_have_the_distribution():
    x = np.array([1.0, -0.5, 2.0, 0.3])
    n = 20000
    got = np.bincount([ort.sample_row(x, (i + 0.5) / n, 0.7)[0] for i in range(n)], minlength=4) / n
    want = np.exp(x / 0.7)
    np.testing.assert_allclose(got, want / want.sum(), atol=1.01 / n)


def test_walks():
    parent, draft = [-1, 0, 0, 1, 2, 2], [9, 5, 6, 7, 8, 8]
    assert ort.accept_walk(parent, 6, draft, [6, 0, 8, 0, 3, 4], 99) == ([0, 2, 4], 3)
    assert ort.accept_walk(parent, 6, draft, [4, 0, 8, 0, 3, 4], 99) == ([0], 4)
    assert ort.accept_walk(parent, 4, draft, [6, 0, 8, 0, 3, 4], 99) == ([0, 2], 8)
    assert ort.accept_walk(parent, 6, draft, [6, 0, 8, 0, 3, 4], 2) == ([0], 6)
    assert ort.accept_walk(parent, 0, draft, [6, 0, 8, 0, 3, 4], 99) == ([], -1)
    assert ort.accept_walk(parent, 6, [9, -1, 6, 7, 8, 8], [-1] * 6, 99) == ([0], -1)
