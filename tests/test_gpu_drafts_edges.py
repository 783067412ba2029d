"""GPU parity of verification where next to nothing is left to draw from: drafts that agree with the target but for a few tokens, over several chunks of a row, with the
uniforms at the ends of their range.

The sums and borders are compared as in test_gpu_drafts.py; here the oracle's weights are exactly those of the tokens that differ, since a difference under 2^-44 of a weight
counts as none in both."""
import numpy as np
import pytest
import torch

from oracle import drafts as DR
from test_gpu_decoder import dev
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
