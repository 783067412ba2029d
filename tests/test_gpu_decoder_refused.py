"""A decoder block goes on correctly after steps that were refused: the pool runs out at a later sequence or service, a sequence grows past the table of
angles, a name comes twice.  Every stage of the steps that follow is compared with the oracle."""
import numpy as np
import pytest
import torch

from paper_2511_00603_amd import binding as B
from test_gpu_decoder_block import DEV, Checked
from workloads import make_mix

pytestmark = pytest.mark.gpu


def test_decoder_block_after_refused_steps():
    mix = make_mix(4, d=256, ffn=704, rows=[1, 8, 20])
    c = Checked(mix, "bf16")                                     # 24 pages for each service, 512 positions
    blk, rng = c.block, np.random.default_rng(92)
    X = lambda n: torch.from_numpy(rng.standard_normal((n, 256)).astype(np.float32)).to(DEV).bfloat16()
    c.step([[("a", X(60))], [("b%d" % i, X(200)) for i in range(5)], [("d", X(64))]])             # 20 of service 1's 24 pages
    for new, error in (([[("a", X(7))], [("b0", X(3)), ("e", X(300))], []], B.EparaError),        # the pool runs out at a name that is not known yet
                       ([[("a", X(7))], [("b1", X(250)), ("b2", X(60))], [("f", X(2))]], B.EparaError),
                       ([[("a", X(7))], [("b3", X(313))], []], ValueError),                       # more positions than angles
                       ([[("a", X(1)), ("a", X(1))], [], []], ValueError)):
        with pytest.raises(error):
            blk.step(new)
        assert [blk.sequences[0]["a"][1], blk.sequences[1]["b0"][1], sorted(blk.sequences[1])] == [60, 200, ["b%d" % i for i in range(5)]]
        assert [p.n_free for p in blk.pools] == [23, 4, 23]
    blk.release(1, "b4")
    c.step([[("a", X(7))], [("b0", X(3)), ("e", X(300))], [("d", X(1))]])                         # the first of them again
    c.step([[("a", X(1))], [("e", X(1)), ("b0", X(1)), ("b3", X(1))], []])
