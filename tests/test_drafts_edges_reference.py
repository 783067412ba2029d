"""The oracle of decoding by drafts where next to nothing is left to draw from (CPU only)."""
import numpy as np

from oracle import drafts as DR


def test_tokens_at_which_both_agree_are_never_drawn_from_what_is_left():
    """p and q are normalised by sums whose roundings differ: what that leaves of equal weights counts as nothing."""
    rng = np.random.default_rng(7)
    x = rng.standard_normal((2, 4000)) * 2.5
    for left in (0.1, 1e-5):
        x[0, 3000] = np.log(np.exp(x[0]).sum()) + np.log(left)
        x[0, 3500] = x[0, 3000] - 4.0
        d = x.copy()
        d[0, [3000, 3500]] = x[0, [3500, 3000]]
        for u in (0.0, np.nan, 2.0 ** -28, 0.5, 1.0):
            path, v, _, margin = DR.verify(x, d, [0, 3500], [-1, 0], [u, 1.0], 1.0)
            assert (path, v) == ([0], 3000) and margin > 2.0 ** -10
    assert DR.verify(x, x, [0, 3], [-1, 0], [0.0, 1.0], 1.0)[0] == [0, 1]


def test_nothing_stays_of_a_tree_whose_first_row_is_not_there():
    """What follows it is not there either, so nothing is kept and nothing drawn; as for a sequence without rows."""
    rng = np.random.default_rng(8)
    x = rng.standard_normal((4, 6)) * 3
    tokens = [0, int(x[0].argmax()), int(x[1].argmax()), int(x[2].argmax())]
    for parents in ([-2, 0, 1, 2], [0, 0, 1, 2], [3, -1, 1, 2], [100000, 0, 0, 0], [-2] * 4):
        assert not DR.follows(parents)[0]
        for t in (0.0, 0.9):
            for draft in (None, x):
                assert DR.verify(x, draft, tokens, parents, [0.0] * 4, t)[:2] == ([], -1)
    assert DR.verify(x, None, tokens, [-1, 0, 1, 2], [0.0] * 4, 0.0)[0] == [0, 1, 2, 3]
