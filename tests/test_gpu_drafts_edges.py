"""GPU parity of verification where next to nothing is left to draw from: drafts that agree with the target but for a few tokens, over several chunks of a row, with the
uniforms at the ends of their range.

The sums and borders are compared as in test_gpu_drafts.py; here the oracle's weights are exactly those of the tokens that differ, since the draft's
probabilities count 2^-44 more in both.  And trees whose first row is not there, of which nothing may stay, through every call of a step."""
import numpy as np
import pytest
import torch

from oracle import drafts as DR
from test_gpu_decoder import dev
from test_gpu_draft_steps import Drafted, judge
from test_gpu_drafts import Verify, check_verify, run_verify

pytestmark = pytest.mark.gpu
ENDS = [0.0, -1.0, float("nan"), 2.0 ** -28, 2.0 ** -24, 0.3, 0.999, 1 - 2.0 ** -24, 1.0]


def nearly_equal(rng, n, vocab, pairs, left, dtype="bf16", pad=0, shift=0):
    """n sequences of a row and a draft behind it that is turned away.  The draft's logits are the target's, but for each of `pairs` (i, j), whose two logits are exchanged: the target has
    about `left` of its probability at i, the draft at j.  The drafted token is the first pair's j."""
    s = Verify(rng, [[-1, 0]] * n, vocab, dtype, True, ts=[0.8] * n)
    t = float(s.ts[0])
    for row in range(0, 2 * n, 2):
        x = s.x[row]
        for k, (i, j) in enumerate(pairs):
            x[i] = t * (np.log(np.exp(x / t).sum()) + np.log(left * 2.0 ** -k))
            x[j] = x[i] - 4.0
        x[:] = dev(x.astype(np.float32)).to(s.logits.dtype).float().cpu().numpy()
        s.d[row] = x
        for i, j in pairs:
            s.d[row, [i, j]] = x[[j, i]]
        s.tokens[row: row + 2] = [0, pairs[0][1]]
    s.u[1::2] = 1 - 2.0 ** -24
    s.logits.copy_(dev(s.x.astype(np.float32)))
    if pad or shift:                                             # the draft's rows begin at other places of a piece of 16 bytes than the target's
        s.draft = torch.zeros(2 * n * (vocab + pad) + shift, dtype=s.logits.dtype, device=s.logits.device)[shift:].reshape(2 * n, vocab + pad)[:, :vocab]
    s.draft.copy_(dev(s.d.astype(np.float32)))
    return s


@pytest.mark.parametrize("left", [0.2, 1e-2, 1e-4, 1e-6])
@pytest.mark.parametrize("dtype,vocab,pad,shift", [("bf16", 8192, 0, 0), ("bf16", 20011, 1, 3), ("f32", 4099, 0, 0), ("f32", 12000, 2, 1), ("bf16", 700, 0, 0)])
def test_what_is_left_lies_in_the_last_chunk_alone(left, dtype, vocab, pad, shift):
    """One token has all that is left: it comes, whatever the uniform is, and not one at which both agree."""
    rng = np.random.default_rng([101, vocab])
    n = 4 * len(ENDS)
    s = nearly_equal(rng, n, vocab, [(vocab - 3, vocab - 40)], left, dtype, pad, shift)
    s.u[::2] = ENDS * 4
    plan = run_verify([s])
    assert plan.kept.tolist() == [1] * n and plan.next.tolist() == [vocab - 3] * n
    check_verify([s], plan, most_near=0.0)


@pytest.mark.parametrize("left", [0.1, 1e-4, 1e-6])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_left_lies_in_several_chunks(left, dtype):
    rng = np.random.default_rng([102, dtype == "f32"])
    n, vocab = 40, 10007
    pairs = [(9990, 9800), (31, 500), (5000, 5001), (2100, 2600)]
    s = nearly_equal(rng, n, vocab, pairs, left, dtype)
    s.u[::2] = rng.random(n)
    s.u[: 2 * len(ENDS): 2] = ENDS
    plan = run_verify([s])
    assert set(plan.next.tolist()) <= {i for i, _ in pairs} and plan.next.tolist()[0] == 31
    check_verify([s], plan)


@pytest.mark.parametrize("vocab", [300, 9001])
def test_nothing_left_by_a_draft_that_cannot_have_been_drawn(vocab):
    """The draft is the target, its token has no probability in either: nothing is left, and the largest logit comes, whatever the uniform is."""
    rng = np.random.default_rng([103, vocab])
    n = len(ENDS)
    s = Verify(rng, [[-1, 0]] * n, vocab, "bf16", True)
    for a, b in ((s.logits, s.x), (s.draft, s.d)):
        b[:] = s.x
        b[:, 7] = -np.inf
        a.copy_(dev(b.astype(np.float32)))
    s.tokens[1::2] = [7] * n
    s.u[::2] = ENDS
    plan = run_verify([s])
    assert plan.kept.tolist() == [1] * n and plan.next.tolist() == s.x[::2].argmax(axis=1).tolist()
    check_verify([s], plan, most_near=0.0)


# ---- first rows that are not there -------------------------------------------------------------------------------

@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("t", [0.0, 0.8])
def test_nothing_stays_of_a_tree_whose_first_row_is_not_there(drawn, t):
    """Next to trees that are there: kept 0, a path of -1, -1 for the next token, whatever the rows behind the first say."""
    rng = np.random.default_rng([104, drawn])
    gone = [[-2, 0, 1, 0], [0, 0, 1, 2], [3, -1, 1, 2], [-2 ** 31, 0], [5], [-2] * 256, [1] + list(range(255))]
    trees = [tree for g in gone for tree in (g, [-1, 0, 0, 1])]
    s = Verify(rng, trees, 5003, drawn=drawn, sharp=6.0, ts=[t] * len(trees))
    s.u[:] *= 0.01                                               # what is tried stays
    row = 0
    for p in trees:
        for i, a in enumerate(p):
            if 0 <= a < i:
                s.tokens[row + i] = int(s.x[row + a].argmax())
        row += len(p)
    plan = run_verify([s])
    assert plan.kept.tolist()[::2] == [0] * len(gone) and plan.next.tolist()[::2] == [-1] * len(gone) and min(plan.kept.tolist()[1::2]) >= 1
    check_verify([s], plan, most_near=0.0)
    path, row = plan.groups[0]["path"].tolist(), 0
    for i, p in enumerate(trees):
        assert i % 2 or path[row: row + len(p)] == [-1] * len(p)
        row += len(p)


def test_a_step_whose_trees_are_not_there_changes_no_sequence():
    """Trees, append, attention, verification and keeping: sequences keep their length, their pages and what lies in them, and go on."""
    c, rng = Drafted(), np.random.default_rng(105)
    blk = c.block
    X = lambda n: torch.from_numpy(rng.standard_normal((n, 256)).astype(np.float32)).to(blk.device).bfloat16()
    c.step([[("a", X(62))], [("b", X(5)), ("c", X(64))], [("d", X(7))]])
    before = [{n: (list(p), k) for n, (p, k) in seqs.items()} for seqs in blk.sequences]
    gone, tree = [-2, 0, 1, 2, 0], [-1, 0, 0, 1]
    out = c.step([[("a", X(5))], [("b", X(4)), ("c", X(5))], [("d", X(1))]], [{"a": gone}, {"b": tree, "c": gone}, None])
    assert not out[0]["o"].any() and not out[1]["o"][4:].any()
    held = [(cache.codes.clone(), cache.scales.clone()) for cache in blk.caches]
    got = c.accept([judge(rng, [gone], 99), judge(rng, [tree, gone], 300), None], [[0.8], [1.0, 0.0], []])
    assert got[0]["a"] == ([], -1) and got[1]["c"] == ([], -1) and got[1]["b"][0][0] == 0
    assert blk.sequences[0]["a"] == list(before[0]["a"]) and blk.sequences[1]["c"] == list(before[1]["c"])
    assert torch.equal(held[0][0], blk.caches[0].codes) and torch.equal(held[0][1], blk.caches[0].scales)
    # a sequence that begins with such a tree has no tokens afterwards
    free = blk.pools[1].n_free
    blk.step([[], [("new", X(5))], []], [None, {"new": gone}, None])
    assert blk.accept([None, judge(rng, [gone], 300), None], [[], [0.7], []])[1] == {"new": ([], -1)}
    assert blk.sequences[1]["new"] == [[], 0] and blk.pools[1].n_free == free
    c.step([[("a", X(3))], [("b", X(1)), ("c", X(1)), ("new", X(2))], [("d", X(1))]])
