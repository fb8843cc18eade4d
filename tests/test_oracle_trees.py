"""Pins of the oracle of drafts that branch (``oracle/trees.py``) against things other than itself (no GPU)."""
import numpy as np
import pytest

from oracle import sampling as osamp
from oracle import trees as ot


def _distribution(rng, V, zeros=0):
    p = rng.random(V) ** 2
    p[rng.permutation(V)[:zeros]] = 0.0
    return p / p.sum()


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("parent", [[-1, 0], [-1, 0, 0], [-1, 0, 0, 0], [-1, 0, 0, 1, 1, 2]])
def test_the_first_token_emitted_has_the_full_models_distribution(drawn, parent):
    """Whatever was drafted: the token behind row 0 - a draft that was kept, or the drawn one - is distributed as p[0].  Over 30 000 rounds a share is off by more than
    5 sqrt(p (1 - p) / N) hardly ever (6e-7 each)."""
    rng = np.random.default_rng(len(parent) + 10 * drawn)
    V, N, n = 5, 30000, len(parent)
    p = np.stack([_distribution(rng, V, 1) for _ in range(n)])
    q = np.stack([_distribution(rng, V) for _ in range(n)])
    counts = np.zeros(V)
    for _ in range(N):
        if drawn:
            token = [0] + [int(rng.choice(V, p=q[parent[i]])) for i in range(1, n)]
        else:                                                        # the most probable ones of q, by rank among the siblings
            token = [0] + [int(np.argsort(-q[parent[i]])[parent[:i].count(parent[i])]) for i in range(1, n)]
        kept, nxt = ot.accept(p, q if drawn else None, token, parent, rng.random(n), rng.random())
        counts[token[kept[1]] if len(kept) > 1 else nxt] += 1
    assert (np.abs(counts / N - p[0]) <= 5 * np.sqrt(p[0] * (1 - p[0]) / N) + 1e-12).all()


def test_chains_are_the_rounds_of_speculative_sampling():
    rng = np.random.default_rng(4)
    for _ in range(300):
        V, k = int(rng.integers(2, 40)), int(rng.integers(0, 6))
        p = np.stack([_distribution(rng, V, V // 3) for _ in range(k + 1)])
        q = np.stack([_distribution(rng, V, V // 3) for _ in range(k + 1)])
        drafts = [int(rng.choice(V, p=q[j])) for j in range(k)]
        u, last = rng.random(k), float(rng.random())
        want = osamp.accept_or_resample(p, q[:k], drafts, u, last)
        kept, nxt = ot.accept(p, q, [0] + drafts, list(range(-1, k)), np.concatenate([[0.5], u]), last)
        assert (len(kept) - 1, nxt) == tuple(want)


def test_words_count_back_from_the_row():
    rng = np.random.default_rng(7)
    for n, back in [(1, 1), (5, 1), (64, 9), (64, 63), (200, 1)]:
        parent = [max(-1, i - int(rng.integers(1, back + 1))) for i in range(n)]
        depth, words = ot.words(parent)
        sees = ot.ancestors(parent)
        for i in range(n):
            full = ot.seen(10 + n, 10 + i, words[i])                 # ten positions were held before
            assert full[:10].all() and (full[10:10 + n] == sees[i]).all()
            assert depth[i] == (depth[parent[i]] + 1 if parent[i] >= 0 else 0)
    assert ot.words(list(range(-1, 99)) + [99] * 60) is not None     # a chain, then a tree
    assert ot.words([-1] + [0] * 64) is not None and ot.words([-1] + [0] * 65) is None
    assert ot.words([-1, 1]) is None and ot.words([-2]) is None


def test_greedy_paths():
    assert ot.agree([7, 8, 9], [5, 7, 7], [-1, 0, 0]) == ([0, 1], 8)     # the first of two that agree
    assert ot.agree([7, 8, 9], [5, 6, 7], [-1, 0, 0]) == ([0, 2], 9)
    assert ot.agree([7, 8, 9, 3], [5, 7, 1, 8], [-1, 0, 0, 1]) == ([0, 1, 3], 3)
    assert ot.agree([7], [5], [-1]) == ([0], 7)
