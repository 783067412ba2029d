"""Layer normalisation at the largest number of rows that a call takes."""
import numpy as np
import pytest
import torch

from oracle import block as OB
from paper_2511_00603_amd import runtime as R
from parity_util import assert_close
from test_gpu_block import DEV, TOL_NORM, dev_bf16, dev_f32, fetch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [8, 4096])
def test_add_layernorm_of_as_many_rows_as_a_call_takes(d):
    """2^31 - 1 rows, the last of them wide or not: the last workgroups' next rows would pass 31 bits."""
    rng, groups, want = np.random.default_rng([112, d]), [], []
    for M, width in ((2**31 - 3, 8), (2, d)):
        gamma, beta = (1 + 0.2 * rng.standard_normal(width)).astype(np.float32), (0.3 * rng.standard_normal(width)).astype(np.float32)
        X, Y = torch.zeros(M, width, dtype=torch.bfloat16, device=DEV), torch.full((M, width), 7.0, dtype=torch.bfloat16, device=DEV)
        groups.append({"X": X, "gamma": dev_f32(gamma), "beta": dev_f32(beta), "Y": Y, "eps": 1e-6})
        for rows in ((slice(0, 9000), slice(M // 2, M // 2 + 9000), slice(M - 9000, M)) if M > 9000 else (slice(0, M),)):
            x, part = dev_bf16(rng.standard_normal((rows.stop - rows.start, width)))
            X[rows] = part
            want.append((Y, rows, OB.add_layer_norm(x, None, gamma.astype(np.float64), beta.astype(np.float64), float(np.float32(1e-6)))[1]))
    R.add_layernorm(R.NormPlan(groups, DEV))
    torch.cuda.synchronize()
    for Y, rows, y in want:
        assert_close(fetch(Y[rows]), y, TOL_NORM, "rows %d to %d" % (rows.start, rows.stop))
    Y = groups[0]["Y"]                                           # all other rows were written
    assert not any((Y[i: i + (1 << 28)] == 7.0).any() for i in range(0, len(Y), 1 << 28))
