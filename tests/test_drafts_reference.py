"""The oracle of decoding by drafts against closed forms, its own definitions in other words, and the distribution that it has to give (CPU only)."""
import itertools

import numpy as np
import pytest

from oracle import decoder as OD
from oracle import drafts as DR


def test_who_follows_whom_by_hand():
    assert DR.follows([-1, 0, 0, 1, -1, 4, 7, 6, -2, 8]) == [[0], [0, 1], [0, 2], [0, 1, 3], [4], [4, 5], [], [], [], []]
    assert DR.words([[0, 63], [64, 255], []]).tolist() == [[1 + (1 << 63), 0, 0, 0], [0, 1, 0, 1 << 63], [0, 0, 0, 0]]


@pytest.mark.parametrize("window,softcap", [(0, 0.0), (9, 0.0), (0, 3.0)])
def test_attention_of_a_chain_is_causal_and_of_a_branch_that_of_its_chain(window, softcap):
    rng = np.random.default_rng([1, window])
    Q, K, V = rng.standard_normal((5, 4, 16)), rng.standard_normal((12, 2, 16)), rng.standard_normal((12, 2, 16))
    o, a = DR.attention(Q, K, V, 7, [-1, 0, 1, 2, 3], 0.25, window, softcap)
    want, mass = OD.attention(Q, K, V, 7, 0.25, window, softcap)
    assert np.allclose(o, want) and np.allclose(a, mass)
    o, _ = DR.attention(Q, K, V, 7, [-1, 0, 0, 2, -5], 0.25, window, softcap)
    keep = [0, 1, 2, 3, 4, 5, 6, 7, 9, 10]                       # the branch 0, 2, 3
    want, _ = OD.attention(Q[[0, 2, 3]], K[keep], V[keep], 7, 0.25, window, softcap)
    assert np.allclose(o[[0, 2, 3]], want) and not o[4].any()


def outcome(logits, draft, parents, t, tokens, u):
    """All tokens that a step gives: of the rows that stay, and the one behind them."""
    path, v, _, _ = DR.verify(logits, draft, tokens, parents, u, t)
    return [tokens[r] for r in path[1:]] + [v]


@pytest.mark.parametrize("parents,tokens", [([-1, 0], [9, 2]), ([-1, 0, 0, 0], [9, 2, 2, 1]), ([-1, 0, 0, 1, 1], [9, 0, 3, 1, 2])])
def test_given_drafts_leave_the_targets_distribution(parents, tokens):
    """The first token of a step has the target's probabilities whatever was drafted: over a fine grid of the uniforms that decide about it."""
    rng = np.random.default_rng(2)
    logits, t = rng.standard_normal((len(parents), 4)) * 1.5, 0.8
    p = DR.distribution(logits[0], t)
    tried = [c for c in range(1, len(parents)) if parents[c] == 0]
    n = 24 if len(tried) < 2 else 10
    grid, count, total = (np.arange(n) + 0.5) / n, np.zeros(4), 0
    for us in itertools.product(grid, repeat=len(tried) + 1):
        u = np.full(len(parents), 0.5)
        u[0] = us[0]
        u[tried] = us[1:]
        count[outcome(logits, None, parents, t, tokens, u)[0]] += 1
        total += 1
    assert np.abs(count / total - p).max() < (len(tried) + 1) / n + 1e-9      # each uniform's grid is at most half a cell off at either border


def test_drawn_drafts_leave_the_targets_distribution():
    rng = np.random.default_rng(3)
    logits, draft, t = rng.standard_normal((2, 5)), rng.standard_normal((2, 5)), 1.1
    p, q = DR.distribution(logits[0], t), DR.distribution(draft[0], t)
    grid, got = (np.arange(200) + 0.5) / 200, np.zeros(5)
    for x in range(5):
        for a in grid:
            path, _, _, _ = DR.verify(logits, draft, [0, x], [-1, 0], [0.5, a], t)
            if len(path) == 2:
                got[x] += q[x] / len(grid)
                continue
            for b in grid:
                got[DR.verify(logits, draft, [0, x], [-1, 0], [b, a], t)[1]] += q[x] / len(grid) ** 2
    assert np.abs(got - p).max() < 2 / 200


def test_greedy_drafts_stay_while_they_are_the_largest():
    logits = np.array([[0., 3, 3, 1], [5, 0, 0, 0], [0, 0, 0, 2], [1, 2, 3, 4.]])
    assert DR.verify(logits, None, [7, 1, 0, 3], [-1, 0, 1, 2], [0.9] * 4, 0.0)[:2] == ([0, 1, 2, 3], 3)
    assert DR.verify(logits, None, [7, 2, 1, 0], [-1, 0, 0, 2], [0.0] * 4, -1.0)[:2] == ([0, 2], 3)      # the first of equal ones is token 1
    assert DR.verify(logits, logits, [7, 2, 1, 0], [-1, 0, 0, 2], [0.0] * 4, 0.0)[:2] == ([0], 1)        # drawn: the first child alone


def test_rows_without_a_distribution_and_odd_uniforms():
    x = np.array([[0., 1, 2], [1, 1, 1]])
    for broken in (np.nan, np.inf):
        y = x.copy()
        y[0, 1] = broken
        assert DR.verify(y, None, [0, 2], [-1, 0], [0.5, 0.0], 1.0)[:2] == ([0], -1)
    assert DR.verify(np.full((1, 3), -np.inf), None, [0], [-1], [0.5], 0.0)[1] == -1
    assert DR.verify(x, None, [0, 5], [-1, 0], [1.5, 0.0], 1.0)[:2] == ([0], 2)
    assert DR.verify(x, None, [0, 0], [-1, 0], [np.nan, -3.0], 1.0)[:2] == ([0, 1], 0)
    assert DR.verify(np.array([[0., 0.]]), None, [0], [-1], [0.5], 1.0)[1] == 1      # the border belongs to what follows
    # q = p: nothing is left when a draft is turned away, which no uniform below 1 does
    assert DR.verify(x, x, [0, 1], [-1, 0], [0.5, 1.0], 1.0)[0] == [0, 1]


def test_keeping_moves_tokens_and_rescales_what_grows():
    rng = np.random.default_rng(5)
    c, pages, D = OD.Cache(5, 2, 64, rng), [4, 1, 3], 64
    K, V = (rng.standard_normal((150, 2, D)) * np.exp2(rng.integers(-3, 4, (150, 1, 1))) for _ in range(2))
    c.append(pages, 0, K[:50], V[:50])
    c.append(pages, 50, K[50:], V[50:])
    before = c.values(pages, 150)
    path = [0, 3, 4, 30, 31, 60, 99]
    codes = c.codes.copy()
    assert DR.keep(c, pages, 50, 100, path + [98, 99]) == 7
    after = c.values(pages, 57)
    for was, now in zip(before, after):
        src = list(range(50)) + [50 + r for r in path]
        step = np.maximum(np.abs(was[src]) * 2.0 ** -4, 2.0 ** (4 - 9 - 1))      # rounded again where the block grew: half a step of its scale (at most 2^4 here)
        assert (np.abs(now - was[src]) <= step).all() and (now[:32] == was[:32]).all()
    assert (c.codes[1] == codes[1]).all() and (c.codes[4, :, :, 57:] == codes[4, :, :, 57:]).all()       # what does not stay is left as it is
    again = c.codes.copy()
    assert DR.keep(c, pages, 50, 100, [0, 1, 2, -1, 7]) == 3 and (c.codes == again).all()                # nothing moves
