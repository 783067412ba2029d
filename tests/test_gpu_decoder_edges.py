"""GPU parity of a decoder block's pieces where their inputs are far from ordinary, against oracle/decoder.py in 64 bits on the same bits.  Tolerances are those of
test_gpu_decoder.py, which derives them."""
import numpy as np
import pytest
import torch

from oracle import decoder as OD
from paper_2511_00603_amd import binding as B
from paper_2511_00603_amd import runtime as R
from test_gpu_decoder import BF, DEV, SLACK, Case, attn_case, check_attn, dev_bf16, fetch, run_attn, sync

pytestmark = pytest.mark.gpu


# ---- attention ---------------------------------------------------------------------------------------------------

def one_sequence(rng, n, rows, D, K, V, q, window=0, softcap=0.0, group=2):
    """The last `rows` of n tokens K, V [n, 1, D] with the queries q [rows, group * D], ready for run_attn and check_attn."""
    case = Case(rng, [n], group, 1, D)
    case.oracle.append(case.pages[0], 0, K, V)
    case.upload()
    q, Q = dev_bf16(q)
    O = torch.zeros(rows, group * D, dtype=torch.bfloat16, device=DEV)
    return (case, [{"first_row": 0, "rows": rows, "start": n - rows, "pages": case.pages[0]}],
            {"Q": Q, "O": O, "cache": case.cache, "heads": group, "window": window, "softcap": softcap}, q.reshape(rows, group, D))


@pytest.mark.parametrize("rows", [1, 3, 16, 90, 200])
@pytest.mark.parametrize("huge", [1e6, 1e10, 1e30])
def test_attention_of_rows_that_do_not_see_a_block_of_huge_values(rows, huge):
    """Blocks of huge values behind a row, or left by its window, take nothing from it: few and many rows, rows on both sides in one tile."""
    for D in (64, 128):
        for lo, hi, window in ((224, 256, 0), (288, 300, 0), (32, 64, 0), (0, 32, 37), (96, 128, 70), (224, 256, 20)):
            n, rng = 300, np.random.default_rng([101, rows, D, lo])
            K, V = rng.standard_normal((n, 1, D)), rng.standard_normal((n, 1, D))
            V[lo:hi] *= huge
            c = one_sequence(rng, n, rows, D, K, V, rng.standard_normal((rows, 2 * D)), window)
            run_attn([c])
            check_attn([c])


@pytest.mark.parametrize("rows", [1, 3, 90])
@pytest.mark.parametrize("huge", [1e-20, 1e-6, 1e6, 1e10, 1e30])
def test_attention_of_blocks_of_huge_values_with_next_to_no_weight(rows, huge):
    """What a block gives is its weight times its values: huge values whose weights are e^-60 and less of the others' take no bits from small ones that have all the weight, and
    tiny values of strong keys leave the others theirs; one order and the other."""
    for D in (64, 128):
        for lo, hi in ((0, 32), (128, 192), (256, 288)):
            n, rng = 330, np.random.default_rng([102, rows, D, lo])
            K, V = rng.standard_normal((n, 1, D)) * 0.3, rng.standard_normal((n, 1, D))
            V[lo:hi] *= huge
            K[:, 0, 0] = 2.0
            K[lo:hi, 0, 0] = 2.0 - (np.log(huge) + 60.0) / 4.0 if huge > 1 else 6.0
            q = rng.standard_normal((rows, 2 * D))
            q[:, 0] = q[:, D] = 4.0 * D ** 0.5
            c = one_sequence(rng, n, rows, D, K, V, q)
            run_attn([c])
            check_attn([c])


@pytest.mark.parametrize("rows", [1, 40, 100])
def test_attention_joins_parts_of_very_different_values(rows):
    """Parts of a long context, each of one magnitude of values (of whole blocks), from 2^-60 to 2^99 in any order, the largest with the least weight: all of them give alike."""
    n, D = 6 * 1024, 64
    rng = np.random.default_rng([105, rows])
    K, V = rng.standard_normal((n, 1, D)) * 0.2, rng.standard_normal((n, 1, D))
    level = np.repeat(rng.integers(-60, 100, 6), 1024)
    V *= np.exp2(level)[:, None, None]
    K[:, 0, 0] = -level * np.log(2.0) / 4.0 + rng.standard_normal(n) * 0.1
    q = rng.standard_normal((rows, D))
    q[:, 0] = 4.0 * D ** 0.5
    c = one_sequence(rng, n, rows, D, K, V, q, group=1)
    plan = run_attn([c])
    assert plan.plan.workspace_bytes > 0
    check_attn([c])


@pytest.mark.parametrize("rows", [1, 90])
def test_attention_of_values_at_the_end_of_the_range(rows):
    """Means of values near bf16's largest are finite as those values are."""
    for D in (64, 128):
        n, rng = 200, np.random.default_rng([104, rows, D])
        K, V = rng.standard_normal((n, 1, D)) * 0.1, np.full((n, 1, D), 3.2e38) * np.sign(rng.standard_normal(D))
        V[40:80] *= 0.25
        c = one_sequence(rng, n, rows, D, K, V, rng.standard_normal((rows, 2 * D)))
        run_attn([c])
        check_attn([c])


@pytest.mark.parametrize("rows", [1, 90])
@pytest.mark.parametrize("softcap", [1e-38, 1e-6, 500.0, 600.0, 1e3, 1e4, 1e5, 1e6, 1e8, 1e15, 1e25, 3e38])
def test_attention_with_caps_far_from_the_scores(rows, softcap):
    """A cap far above the scores leaves them what they are; under one far below them all keys weigh alike (but for their signs); scores of some hundreds about a cap of that size."""
    for D in (64, 128):
        n, rng = 200, np.random.default_rng([106, rows, D])
        K, V = rng.standard_normal((n, 1, D)), rng.standard_normal((n, 1, D))
        q = rng.standard_normal((rows, 2 * D))
        q[0, :D] = 0.0
        q[:, D:] *= 100.0 if softcap < 1e3 else 3.0
        c = one_sequence(rng, n, rows, D, K, V, q, softcap=softcap)
        run_attn([c])
        check_attn([c])


# ---- normalisation -----------------------------------------------------------------------------------------------

def test_rmsnorm_of_as_many_rows_as_a_call_takes():
    """2^31 - 1 rows in two groups: the last workgroups' next rows would pass 31 bits."""
    counts, d, rng = [2**31 - 40001, 40000], 8, np.random.default_rng(111)
    gamma = (1 + 0.2 * rng.standard_normal(d)).astype(np.float32)
    groups, kept = [], []
    for M in counts:
        g = {"X": torch.zeros(M, d, dtype=torch.bfloat16, device=DEV), "gamma": torch.from_numpy(gamma).to(DEV), "eps": 1e-5, "out_scale": 0.01,
             "Y": torch.full((M, d), 0x7F, dtype=torch.uint8, device=DEV)}
        x, X = dev_bf16(rng.standard_normal((30000, d)))
        for rows in (slice(0, 10000), slice(M // 2, M // 2 + 10000), slice(M - 10000, M)):
            part = slice(10000 * (len(kept) % 3), 10000 * (len(kept) % 3) + 10000)
            g["X"][rows] = X[part]
            kept.append((g, rows, x[part]))
        groups.append(g)
    R.add_rmsnorm(R.RmsNormPlan(groups, DEV))
    sync()
    scale = float(np.float32(0.01))
    for g, rows, x in kept:
        _, y = OD.add_rms_norm(x, None, gamma.astype(np.float64), float(np.float32(1e-5)))
        got, limit = OD.e4m3_decode(g["Y"][rows].cpu().numpy()) * scale, np.clip(y, -448 * scale, 448 * scale)
        assert (np.abs(got - limit) <= np.maximum(np.abs(limit) * 2.0 ** -4, scale * 2.0 ** -10) * SLACK).all()
    for g in groups:                                             # all other rows are zeros, and were written
        assert not any((g["Y"][i: i + (1 << 28)] == 0x7F).any() for i in range(0, len(g["Y"]), 1 << 28))


@pytest.mark.parametrize("kind", ["bf16", "row", "service"])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-5])
@pytest.mark.parametrize("with_r", [True, False])
def test_rmsnorm_of_rows_of_any_size(kind, eps, with_r):
    """Rows of zeros, rows whose squares pass fp32's range at either end, and ordinary ones side by side; a row of one large value."""
    rng, groups, want = np.random.default_rng([113, with_r]), [], []
    sizes = np.array([0.0, 1e-38, 1e-30, 1e-25, 1e-19, 1.0, 1e18, 3e19, 1e30, 5e37, 0.0, 1.0])
    for d in (8, 520, 1032, 8192):
        x, X = dev_bf16(rng.standard_normal((len(sizes), d)) * sizes[:, None])
        r, Rt = dev_bf16(rng.standard_normal((len(sizes), d)) * 0.5 * sizes[:, None]) if with_r else (None, None)
        X[-1, 5] = 2.0 ** 100
        x[-1, 5] = 2.0 ** 100
        gamma = (1 + 0.2 * rng.standard_normal(d)).astype(np.float32)
        g = {"X": X, "R": Rt, "gamma": torch.from_numpy(gamma).to(DEV), "S": torch.full_like(X, 7.0), "eps": eps,
             "Y": torch.full((len(sizes), d), 7.0, dtype=torch.bfloat16, device=DEV) if kind == "bf16" else torch.full((len(sizes), d), 0x7F, dtype=torch.uint8, device=DEV)}
        if kind == "row":
            g["row_scales"] = torch.full((len(sizes),), -1.0, device=DEV)
        if kind == "service":
            g["out_scale"] = 0.011
        s = x if r is None else x + r
        e = float(np.float32(eps))
        root = np.sqrt((s * s).mean(axis=1, keepdims=True) + e)
        groups.append(g)
        want.append((s, np.divide(s, root, out=np.zeros_like(s), where=root > 0) * gamma))
    R.add_rmsnorm(R.RmsNormPlan(groups, DEV))
    sync()
    for g, (s, y) in zip(groups, want):
        assert (np.abs(fetch(g["S"]) - s) <= BF * np.abs(s) + 1e-40).all()
        if kind == "bf16":
            assert (np.abs(fetch(g["Y"]) - y) <= BF * np.abs(y) + 1e-40).all()
            continue
        scale = np.full((len(y), 1), float(np.float32(0.011)))
        if kind == "row":
            scale, top = fetch(g["row_scales"])[:, None], np.abs(y).max(axis=1, keepdims=True)
            least = np.where(top > 0, np.maximum(top / 448.0, 2.0 ** -126), 1.0)
            assert (np.abs(scale - least) <= 1e-6 * least).all()
        got, limit = OD.e4m3_decode(g["Y"].cpu().numpy()) * scale, np.clip(y, -448 * scale, 448 * scale)
        assert (np.abs(got - limit) <= np.maximum(np.abs(limit) * 2.0 ** -4, scale * 2.0 ** -10) * SLACK).all()


@pytest.mark.parametrize("window", [2**24, 2**31 - 1])
def test_attention_with_windows_wider_than_any_sequence(window):
    """Positions less such a window would pass 32 bits; rows of padding next to rows that see keys, few and many."""
    rng = np.random.default_rng([107])
    cases = [attn_case(rng, [-5, -300, 0, 100, -2000], [7, 310, 40, 1, 2003], 4, 2, D, window, softcap) for D, softcap in ((64, 0.0), (128, 30.0))]
    run_attn(cases)
    check_attn(cases)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,softcap", [(2501, 0.0), (3030, 20.0), (0, 20.0)])
def test_attention_over_cut_contexts_with_windows_and_capped_scores(D, window, softcap):
    """Contexts in parts that begin where a window does, of few and of many rows; tiles of a sequence with different numbers of parts; the same bits every time."""
    rng = np.random.default_rng([108, D, window])
    c = attn_case(rng, [9000, 4097, 3000, 6000], [1, 5, 64, 200], 4, 1, D, window, softcap)
    plan = run_attn([c])
    check_attn([c])
    assert plan.plan.workspace_bytes > 0
    for few, (start, rows) in ((True, (9000, 1)), (True, (4097, 5)), (False, (3000, 64)), (False, (6000, 200))):
        tile, part = (16, plan.plan.part_pages[0]) if few else (128, plan.plan.part_pages[1])
        counts = set()
        for first in range(0, 4 * rows, tile):
            lo, hi = start + first // 4, start + (min(first + tile, 4 * rows) - 1) // 4
            pages = hi // 64 + 1 - (max(0, lo - window + 1) // 64 if window else 0)
            counts.add(-(-pages // part))
        assert min(counts) > 1                                   # every sequence is cut
        assert len(counts) > 1 or window != 3030 or rows != 200  # and tiles have different numbers of parts here
    got = c[2]["O"].clone()
    for _ in range(3):
        c[2]["O"].fill_(float("nan"))
        R.cache_attention(plan)
        sync()
        assert torch.equal(c[2]["O"].view(torch.int16), got.view(torch.int16))


@pytest.mark.parametrize("rows", [1, 90])
@pytest.mark.parametrize("power", [10, 20, 24, 28, 34, 60, 100])
def test_attention_with_scores_that_leave_fp32_no_fractions(rows, power):
    """Scores of up to 2^power whose differences are as large (each one exact up to the factor log2 e, alike for equal keys): all the weight lies on the largest, shared alike by the keys
    that have it, in blocks of different scales."""
    for D in (64, 128):
        n, rng = 330, np.random.default_rng([109, rows, D])
        K, V = np.zeros((n, 1, D)), rng.standard_normal((n, 1, D)) * np.exp2(np.repeat(rng.integers(-12, 12, 11), 32))[:n, None, None]
        K[:, 0, 0] = -rng.integers(1, 8, n)
        K[rng.choice(n - rows, 6 if rows < 90 else 40, replace=False), 0, 0] = rng.choice([7.0, 6.0])
        q = np.zeros((rows, 2 * D))
        q[:, 0], q[:, D] = 1.0, -1.0
        c = one_sequence(rng, n, rows, D, K, V, q)
        c[2]["scale"] = 2.0 ** (power - 3)
        run_attn([c])
        got = fetch(c[2]["O"]).reshape(rows, 2, D)
        keys, values = c[0].oracle.values(c[1][0]["pages"], n)
        want, mass = OD.attention(c[3], keys, values, n - rows, 2.0 ** (power - 3))
        assert (np.abs(got - want) <= (2.0 ** -8 + 2.0 ** -10) * mass + BF * np.abs(want)).all()


def test_attention_plans_that_share_a_workspace():
    """Two plans with different numbers of workgroups take turns on one workspace, zeroed whenever the plan changes; a plan's own calls need nothing in between."""
    rng = np.random.default_rng(110)
    cases = [attn_case(rng, starts, news, 4, 2, 128) for starts, news in (([9000], [1]), ([3000] * 9, [2, 60, 1, 1, 90, 1, 1, 1, 1]))]
    plans = [R.CacheAttnPlan(R.SequenceTable([c[1]], DEV), [c[2]], DEV) for c in cases]
    size = max(p.plan.workspace_bytes for p in plans)
    shared = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV)
    for p in plans:
        assert p.plan.workspace_bytes > 0
        p.c.d_workspace, p.c.workspace_bytes = shared.data_ptr(), size
    for _ in range(2):
        for c, p in zip(cases, plans):
            B.epara_workspace_init(shared.data_ptr(), -(-4 * sum(p.plan.n_items) // 256) * 256, R.current_stream_handle())
            for _ in range(2):
                c[2]["O"].fill_(float("nan"))
                R.cache_attention(p)
                sync()
                check_attn([c])
