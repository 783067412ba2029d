"""A decoder block goes on correctly after steps that were refused: the pool runs out at a later sequence or service, a sequence grows past the table of
angles, a name comes twice.  Every stage of the steps that follow is compared with the oracle."""
import numpy as np
import pytest
import torch

from paper_2511_00603_amd import binding as B
from paper_2511_00603_amd import runtime as R
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


def test_plans_do_not_take_an_empty_table_or_a_scale_of_nothing_for_one_left_out():
    cache = R.PagedCache.empty(2, 1, 64, DEV)
    QKV, Q, O = (torch.zeros(3, n * 64, dtype=torch.bfloat16, device=DEV) for n in (4, 2, 2))
    table = R.SequenceTable([[{"first_row": 0, "rows": 3, "start": 0, "pages": [0]}]], DEV)
    append = {"QKV": QKV, "Q": Q, "cache": cache, "heads": 2}
    for rows in (0, 2):                                          # fewer angles than positions
        with pytest.raises((ValueError, B.EparaError)):
            R.CacheAppendPlan(table, [dict(append, rotary=torch.zeros(rows, 32, 2, device=DEV))], DEV)
    R.CacheAppendPlan(table, [dict(append, rotary=torch.zeros(3, 32, 2, device=DEV))], DEV)
    attn = {"Q": Q, "O": O, "cache": cache, "heads": 2}
    for scale in (0, 0.0, -1.0):
        with pytest.raises(B.EparaError):
            R.CacheAttnPlan(table, [dict(attn, scale=scale)], DEV)
    for scale in (None, 0.25):
        plan = R.CacheAttnPlan(table, [dict(attn, scale=scale)], DEV)
        assert plan.args[0]["scale"] == np.float32(scale or 0.125)
