"""GPU parity of decoding by drafts (trees, attention over the cache for them, verification, keeping what stays), through the C ABI, against oracle/drafts.py in 64 bits on the
same bits.

Tolerances.  Trees, paths, tokens and kept codes are whole: equal.  Attention is held to what the causal one is: a weight to 2^-8 of its value (f16 keeps 2^-11), scores' fp32
error 2^-10, and bf16 rounds the output by 2^-8 of itself.  Probabilities: an fp32 exponential's argument is off by up to 2^-24 of its size, which is under 128 where a weight counts (2^-17 of
the weight), the exponential by 2^-22, and the sums of up to 64 in fp32 by 2^-18, in all under 2^-16; the result rounds to fp32 by 2^-24.  Decisions
that lie nearer to their border than that are left out of the comparison (the oracle says how near the nearest is); how many may be is bounded."""
import numpy as np
import pytest
import torch

from oracle import decoder as OD
from oracle import drafts as DR
from oracle import reference as ref
from paper_2511_00603_amd import binding as B
from paper_2511_00603_amd import runtime as R
from test_gpu_decoder import BF, DEV, Case, dev, dev_bf16, fetch, sequences, sync
from workloads import casts

pytestmark = pytest.mark.gpu
NEAR = 2.0 ** -16


def random_tree(rng, n, roots=1, gone=0.0):
    """Parents anywhere before the row; some rows follow the context, some are not there."""
    p = [-1] + [int(rng.integers(max(0, i - 9), i)) for i in range(1, n)]
    for _ in range(roots - 1):
        p[int(rng.integers(0, n))] = -1
    for i in range(n):
        if rng.random() < gone:
            p[i] = int(rng.choice([-2, i, i + 1, 100000, -2 ** 31]))
    return p


def shapes(rng, n):
    return [list(range(-1, n - 1)), [-1] + [0] * (n - 1), [-1] * n, [-2] * n, random_tree(rng, n), random_tree(rng, n, 3, 0.1)]


# ---- trees -------------------------------------------------------------------------------------------------------

def run_trees(services, starts):
    """services: per service a list of parents (lists) -> what the library writes, with rows that belong to no sequence around each."""
    groups, table = [], []
    for trees, start in zip(services, starts):
        row, seqs, parents = 2, [], [-1, -1]
        for p, at in zip(trees, start):
            seqs.append({"first_row": row, "rows": len(p), "start": at, "pages": [0] * max(0, -(-(at + len(p)) // 64))})
            parents += p + [-1]
            row += len(p) + 1
        groups.append({"parents": dev(parents, np.int32), "visible": torch.full((len(parents), 4), -7, dtype=torch.int64, device=DEV),
                       "positions": torch.full((len(parents), 3), -9, dtype=torch.int32, device=DEV)})
        table.append(seqs)
    plan = R.DraftTreePlan(R.SequenceTable(table, DEV), groups, DEV)
    R.draft_trees(plan)
    sync()
    return table, groups


@pytest.mark.parametrize("n", [1, 2, 3, 31, 63, 64, 65, 127, 128, 129, 255, 256])
def test_trees_of_every_shape(n):
    rng = np.random.default_rng([1, n])
    services = [shapes(rng, n), [], shapes(rng, max(1, n // 2)) + [[]]]
    table, groups = run_trees(services, [rng.integers(0, 300, len(s)).tolist() for s in services])
    for trees, seqs, g in zip(services, table, groups):
        visible, positions = g["visible"].cpu().numpy().view(np.uint64), g["positions"].cpu().numpy()
        inside = np.zeros(len(visible), dtype=bool)
        for p, s in zip(trees, seqs):
            rows = slice(s["first_row"], s["first_row"] + s["rows"])
            f = DR.follows(p)
            assert np.array_equal(visible[rows], DR.words(f))
            assert np.array_equal(positions[rows], np.repeat(np.array([s["start"] + max(len(x) - 1, 0) for x in f], dtype=np.int32).reshape(-1, 1), 3, 1))
            inside[rows] = True
        assert (visible[~inside].view(np.int64) == -7).all() and (positions[~inside] == -9).all()


def test_long_sequences_are_no_trees_and_positions_may_be_left_out():
    chain, long = list(range(-1, 39)), [5] * 257
    table, groups = run_trees([[chain, long, [-1] * 1000]], [[3, 70, -40]])
    g, (a, b, c) = groups[0], table[0]
    assert np.array_equal(g["visible"][2:42].cpu().numpy().view(np.uint64), DR.words(DR.follows(chain)))
    assert (g["visible"][b["first_row"]:] == -7).all()
    for s in (a, b, c):
        assert g["positions"][s["first_row"]: s["first_row"] + s["rows"], 1].tolist() == list(range(s["start"], s["start"] + s["rows"]))
    plan = R.DraftTreePlan(R.SequenceTable([[a]], DEV), [{"parents": g["parents"]}], DEV)
    plan.args["positions"] = 0
    B.epara_draft_trees(plan.args, R._upload(plan.args, DEV).data_ptr(), plan.table.c, R.current_stream_handle())
    sync()
    assert np.array_equal(plan.groups[0]["visible"][2:42].cpu().numpy().view(np.uint64), DR.words(DR.follows(chain))) and not plan.groups[0]["positions"].any()


# ---- attention ---------------------------------------------------------------------------------------------------

def tree_case(rng, starts, trees, heads, kv_heads, D, window=0, softcap=0.0, sharp=1.0, strided=False, broken=()):
    """broken: (sequence, row) whose keys and values are NaN."""
    news = [len(p) for p in trees]
    case = Case(rng, [s + n for s, n in zip(starts, news)], heads, kv_heads, D)
    for i, (pages, s, n) in enumerate(zip(case.pages, starts, news)):
        K = rng.standard_normal((s + n, kv_heads, D)) * np.exp(0.5 * rng.standard_normal((s + n, 1, 1)))
        V = rng.standard_normal((s + n, kv_heads, D)) + 0.2
        for seq, row in broken:
            if seq == i:
                K[s + row, :, 3] = V[s + row, :, 5] = np.nan
        if s + n:
            case.oracle.append(pages, 0, K, V)
    case.upload()
    seqs, rows = sequences(case, starts, news)
    q, Q = dev_bf16(rng.standard_normal((rows, heads * D)) * sharp)
    O = torch.full((rows, heads * D + (8 if strided else 0)), float("nan"), dtype=torch.bfloat16, device=DEV)[:, : heads * D]
    if strided:
        wide = torch.full((rows, heads * D + 2 * kv_heads * D), float("nan"), dtype=torch.bfloat16, device=DEV)
        wide[:, : heads * D] = Q
        Q = wide[:, : heads * D]
    visible = np.concatenate([np.zeros((0, 4), dtype=np.uint64)] + [DR.words(DR.follows(p)) if len(p) <= 256 else np.full((len(p), 4), 2 ** 64 - 1, dtype=np.uint64) for p in trees])
    g = {"Q": Q, "O": O, "cache": case.cache, "heads": heads, "window": window, "softcap": softcap, "visible": dev(visible.view(np.int64))}
    return case, seqs, g, q.reshape(rows, heads, D), trees


def run_tree_attn(cases):
    plan = R.TreeAttnPlan(R.SequenceTable([c[1] for c in cases], DEV), [c[2] for c in cases], DEV)
    R.tree_attention(plan)
    sync()
    return plan


def check_tree_attn(cases):
    for case, seqs, g, q, trees in cases:
        got, scale = fetch(g["O"]).reshape(q.shape), float(np.float32(case.D ** -0.5))
        for s, p in zip(seqs, trees):
            rows = slice(s["first_row"], s["first_row"] + s["rows"])
            K, V = case.oracle.values(s["pages"], s["start"] + s["rows"])
            if len(p) > 256 or g["visible"] is None:
                want, mass = OD.attention(q[rows], K, V, s["start"], scale, g["window"], g["softcap"])
            else:
                want, mass = DR.attention(q[rows], K, V, s["start"], p, scale, g["window"], g["softcap"])
            assert np.array_equal(np.isnan(got[rows]), np.isnan(want)), (s["start"], s["rows"])
            off, bound = np.abs(got[rows] - want), (2.0 ** -8 + 2.0 ** -10) * mass + BF * np.abs(want)
            assert (np.nan_to_num(off) <= np.nan_to_num(bound)).all(), (s["start"], s["rows"], np.nanmax(off / np.maximum(bound, 1e-30)))


HEADS = [(8, 2, 128), (3, 3, 64), (16, 1, 128), (12, 4, 64), (32, 2, 64), (2, 2, 128), (5, 1, 64)]


@pytest.mark.parametrize("heads,kv_heads,D", HEADS)
def test_attention_of_trees_that_begin_anywhere_in_a_page(heads, kv_heads, D):
    rng = np.random.default_rng([61, heads, D])
    starts = [0, 1, 15, 16, 31, 32, 33, 62, 63, 64, 65, 127, 128, 191, 300, 1000]
    c = tree_case(rng, starts, [random_tree(rng, n) for n in (8, 1, 2, 16, 7, 3, 8, 1, 13, 5, 8, 20, 4, 9, 8, 30)], heads, kv_heads, D)
    run_tree_attn([c])
    check_tree_attn([c])


@pytest.mark.parametrize("n", [1, 17, 64, 65, 130, 200, 256])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_of_large_trees_over_several_pages(n, D):
    rng = np.random.default_rng([62, n, D])
    c = tree_case(rng, [40, 0, 63, 130], [random_tree(rng, n), random_tree(rng, n, 4), list(range(-1, n - 1)), random_tree(rng, n, 2, 0.2)], 4, 2, D, strided=True)
    run_tree_attn([c])
    check_tree_attn([c])


@pytest.mark.parametrize("n", [5, 40, 100])
def test_rows_that_are_not_there_are_zeros_and_their_keys_unseen(n):
    """Rows that are gone hold NaNs in the cache; a tree without any row; rows next to them are as they were."""
    for D in (64, 128):
        rng = np.random.default_rng([63, n, D])
        p = random_tree(rng, n, 2, 0.25)
        gone = [i for i, f in enumerate(DR.follows(p)) if not f]
        c = tree_case(rng, [70, 5, 0], [p, [-2] * n, p], 4, 2, D, broken=[(0, i) for i in gone] + [(1, i) for i in range(n)] + [(2, i) for i in gone])
        run_tree_attn([c])
        check_tree_attn([c])
        assert (c[2]["O"][n: 2 * n] == 0).all() and torch.isfinite(c[2]["O"]).all()


def test_a_broken_token_is_seen_by_those_that_follow_it_alone():
    rng = np.random.default_rng(64)
    p = [-1, 0, 0, 1, 2, 3, 4, 4]
    c = tree_case(rng, [33], [p], 2, 1, 128, broken=[(0, 2)])
    run_tree_attn([c])
    check_tree_attn([c])
    assert torch.isnan(c[2]["O"]).any(dim=1).tolist() == [2 in f for f in DR.follows(p)]


@pytest.mark.parametrize("window,softcap", [(40, 0.0), (64, 0.0), (65, 5.0), (200, 0.0), (5000, 30.0), (0, 30.0), (0, 0.5), (0, 4000.0)])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_of_trees_with_windows_and_capped_scores(window, softcap, D):
    """A row's window reaches back from its own position, which is before the slot that it lies in."""
    rng = np.random.default_rng([65, window, D])
    c = tree_case(rng, [0, 500, 64, 127, 300], [random_tree(rng, n, 1, 0.03) for n in (40, 1, 7, 33, 40)], 4, 2, D, window, softcap, sharp=2.0)
    run_tree_attn([c])
    check_tree_attn([c])


def test_trees_next_to_prompts_and_services_without_trees():
    """Long sequences are causal (their bits say otherwise and are not read), and so is a service without bits, left padding and all."""
    rng = np.random.default_rng(66)
    cases = [tree_case(rng, [40, 100, 3], [random_tree(rng, 9), [0] * 300, random_tree(rng, 90)], 8, 2, 128), tree_case(rng, [], [], 2, 2, 64),
             tree_case(rng, [10, 200], [[0] * 12, [0] * 80], 6, 6, 64), tree_case(rng, [700], [random_tree(rng, 5)], 24, 2, 128)]
    cases[2][2]["visible"] = None
    run_tree_attn(cases)
    check_tree_attn(cases)


def test_padded_sequences_of_a_service_without_trees():
    """In front of position 0 rows see nothing and get zeros, in each kind of tile, next to a service of trees."""
    rng = np.random.default_rng(69)
    trees = tree_case(rng, [40, 3], [random_tree(rng, 9), random_tree(rng, 70)], 4, 2, 64)
    case = Case(rng, [0, 9, 3, 30, 120], 4, 2, 64)
    starts, news = [-5, -1, -30, -3, -180], [5, 10, 33, 33, 300]
    case.fill([0, 9, 3, 30, 120])
    seqs, rows = sequences(case, starts, news)
    q, Q = dev_bf16(rng.standard_normal((rows, 4 * 64)))
    O = torch.full((rows, 4 * 64), float("nan"), dtype=torch.bfloat16, device=DEV)
    g = {"Q": Q, "O": O, "cache": case.cache, "heads": 4, "window": 0, "softcap": 0.0, "visible": None}
    R.tree_attention(R.TreeAttnPlan(R.SequenceTable([trees[1], seqs], DEV), [trees[2], g], DEV))
    sync()
    check_tree_attn([trees])
    got = fetch(O).reshape(rows, 4, 64)
    for s, n in zip(seqs, news):
        part = slice(s["first_row"], s["first_row"] + n)
        K, V = case.oracle.values(s["pages"], max(s["start"] + n, 0))
        want, mass = OD.attention(q.reshape(rows, 4, 64)[part], K, V, s["start"], 64 ** -0.5)
        assert (np.abs(got[part] - want) <= (2.0 ** -8 + 2.0 ** -10) * mass + BF * np.abs(want)).all(), s["start"]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [4, 16, 40, 100])
def test_trees_behind_long_contexts_are_cut_and_joined(n, D):
    rng = np.random.default_rng([67, n, D])
    c = tree_case(rng, [5000, 2111], [random_tree(rng, n, 1, 0.05), random_tree(rng, n)], 4, 2, D)
    plan = run_tree_attn([c])
    assert plan.plan.workspace_bytes > 0
    check_tree_attn([c])
    first = c[2]["O"].clone()
    for _ in range(3):
        c[2]["O"].fill_(float("nan"))
        R.tree_attention(plan)
        sync()
        assert torch.equal(c[2]["O"].view(torch.int16), first.view(torch.int16))


def test_a_chain_is_causal_attention_in_every_kernel():
    """Both calls against the causal oracle: 12 to 400 rows to a key head, next to enough others that each of the kernels runs."""
    rng = np.random.default_rng(68)
    for news in ((3, 8, 5), (20, 33, 70), (70, 90, 100), (3, 16, 100, 200)):
        c = tree_case(rng, [40, 0, 1000, 77][: len(news)], [list(range(-1, n - 1)) for n in news], 8, 2, 128)
        for call, plan in ((R.tree_attention, R.TreeAttnPlan), (R.cache_attention, R.CacheAttnPlan)):
            c[2]["O"].fill_(float("nan"))
            call(plan(R.SequenceTable([c[1]], DEV), [c[2]], DEV))
            sync()
            check_tree_attn([(c[0], c[1], dict(c[2], visible=None), c[3], c[4])])


# ---- verification ------------------------------------------------------------------------------------------------

class Verify:
    """One service's sequences: logits as rows of a wider buffer that may begin anywhere, and the oracle's view of them."""

    def __init__(self, rng, trees, vocab, dtype="bf16", drawn=False, shift=0, pad=0, sharp=2.5, ts=None):
        self.trees, self.V, n = trees, vocab, sum(len(p) for p in trees)
        size = n * (vocab + pad) + shift
        x = rng.standard_normal(size) * sharp
        d = x + 0.7 * rng.standard_normal(size)

        def laid(a):
            flat = dev(a.astype(np.float32))
            flat = flat.bfloat16() if dtype == "bf16" else flat
            rows = flat[shift:].reshape(n, vocab + pad)[:, :vocab]
            return rows.float().cpu().numpy().astype(np.float64), rows

        (self.x, self.logits), (self.d, self.draft) = laid(x), laid(d)
        self.ts = rng.choice([0.3, 0.7, 1.0, 1.4], len(trees)).astype(np.float32) if ts is None else np.array(ts, dtype=np.float32)
        self.u = rng.random(n).astype(np.float32)
        self.tokens, self.parents, row = [], [], 0
        for p, t in zip(trees, self.ts):
            rank = {}
            for i, a in enumerate(p):
                at = row + (a if 0 <= a < i else 0)
                if drawn:
                    q = DR.distribution(self.d[at], max(float(t), 0.05))
                    self.tokens.append(int(rng.choice(vocab, p=q)))
                else:
                    rank[a] = rank.get(a, -1) + 1
                    self.tokens.append(int(np.argsort(-self.d[at])[min(rank[a], vocab - 1)]))
            self.parents += p
            row += len(p)
        self.drawn = drawn

    def group(self, **kw):
        n = len(self.parents)
        g = {"logits": self.logits, "tokens": dev(self.tokens, np.int32), "parents": dev(self.parents, np.int32), "uniforms": dev(self.u),
             "path": torch.full((n,), -5, dtype=torch.int32, device=DEV), "probs": torch.full((n,), -5.0, device=DEV)}
        if self.drawn:
            g["draft_logits"] = self.draft
        return dict(g, **kw)

    def sequences(self):
        out, row = [], 0
        for p in self.trees:
            out.append({"first_row": row, "rows": len(p), "start": 0, "pages": [0] * -(-len(p) // 64)})
            row += len(p)
        return out


def run_verify(services, groups=None, **kw):
    groups = [s.group() for s in services] if groups is None else groups
    ts = dev(np.concatenate([s.ts for s in services] + [np.zeros(0, np.float32)]).astype(np.float32))
    plan = R.VerifyPlan(R.SequenceTable([s.sequences() for s in services], DEV), groups, DEV, temperatures=ts, **kw)
    plan.kept.fill_(-5)
    plan.next.fill_(-5)
    R.verify_drafts(plan)
    sync()
    return plan


def check_verify(services, plan, most_near=0.02):
    kept, nxt, at, near = plan.kept.tolist(), plan.next.tolist(), 0, 0
    for s, g in zip(services, plan.groups):
        path, probs = g["path"].tolist(), g["probs"].cpu().numpy().astype(np.float64)
        row = 0
        for p, t in zip(s.trees, s.ts):
            rows = slice(row, row + len(p))
            want, v, w, margin = DR.verify(s.x[rows], s.d[rows] if s.drawn else None, s.tokens[rows], p, s.u[rows], float(t))
            assert (np.abs(probs[rows] - w) <= NEAR * w + 1e-37).all(), (at, np.abs(probs[rows] - w).max())
            if margin < NEAR:
                near += 1
            else:
                assert path[rows] == want + [-1] * (len(p) - len(want)), (at, t, margin)
                assert (kept[at], nxt[at]) == (len(want), v), (at, t, margin)
            row, at = row + len(p), at + 1
    assert near <= max(1, most_near * at)


VOCABS = [1, 2, 7, 8, 9, 255, 2047, 2048, 2049, 2055, 5003, 33333]


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("dtype,drawn", [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)])
def test_verification_over_vocabularies_of_every_size(vocab, dtype, drawn):
    """Rows that begin anywhere in a piece of 16 bytes; trees and chains, greedy and not."""
    rng = np.random.default_rng([71, vocab, dtype == "f32", drawn])
    few = vocab > 4000
    trees = [random_tree(rng, int(n)) for n in ([1, 6, 9] if few else [1, 2, 5, 9, 17, 40])] + [list(range(-1, 5))]
    for shift, pad in ((0, 0), (1, 3)) if few else ((0, 0), (1, 0), (3, 5), (7, 8)):
        s = [Verify(rng, trees, vocab, dtype, drawn, shift, pad), Verify(rng, [], vocab, dtype, drawn), Verify(rng, trees[:3], max(1, vocab - 1), dtype, False, ts=[0.0, 0.8, -1.0])]
        check_verify(s, run_verify(s))


@pytest.mark.parametrize("n", [1, 2, 64, 65, 255, 256])
def test_verification_of_trees_of_every_shape(n):
    """Chains, stars (equal tokens among siblings), rows that are not there: their tokens do not count."""
    rng = np.random.default_rng([72, n])
    for drawn in (False, True):
        s = Verify(rng, shapes(rng, n), 300, drawn=drawn, sharp=1.0)
        for i in range(0, len(s.tokens), 3):
            s.tokens[i] = s.tokens[max(0, i - 1)]
        check_verify([s], run_verify([s]))


def test_verification_keeps_long_chains_that_agree():
    """Drafts that are nearly certain: whole chains stay, and the token comes from the last row's own distribution."""
    rng = np.random.default_rng(73)
    for drawn in (False, True):
        s = Verify(rng, [list(range(-1, n - 1)) for n in (2, 5, 33, 256, 1)], 500, drawn=drawn, sharp=12.0)
        s.d[:] = s.x
        s.draft.copy_(s.logits)
        row = 0
        for p in s.trees:
            for i in range(1, len(p)):
                s.tokens[row + i] = int(s.x[row + i - 1].argmax())
            row += len(p)
        plan = run_verify([s])
        check_verify([s], plan)
        assert max(plan.kept.tolist()) > 4


def test_chains_without_parents_and_outputs_that_are_left_out():
    rng = np.random.default_rng(74)
    s = Verify(rng, [list(range(-1, n - 1)) for n in (4, 1, 7)], 1000)
    plan = run_verify([s], [s.group(parents=None)])
    check_verify([s], plan)
    plan.args["probs"] = 0
    d = R._upload(plan.args, DEV)
    plan.c.d_args = d.data_ptr()
    before = plan.kept.tolist(), plan.next.tolist(), plan.groups[0]["path"].tolist()
    plan.groups[0]["probs"].fill_(3.0)
    plan.kept.zero_()
    R.verify_drafts(plan)
    sync()
    assert (plan.kept.tolist(), plan.next.tolist(), plan.groups[0]["path"].tolist()) == before and (plan.groups[0]["probs"] == 3).all()


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_rows_without_a_distribution(drawn, value):
    """One such logit in the root, or further down, or nothing but them; and of masked tokens, which are no reason."""
    rng = np.random.default_rng([75, drawn])
    trees = [list(range(-1, 4))] * 6
    for t in (0.8, 0.0):
        s = Verify(rng, trees, 700, drawn=drawn, ts=[t] * 6)
        for a, b in ((s.logits, s.x), (s.draft, s.d)):
            for row, cols in ((0, slice(5, 6)), (6, slice(699, 700)), (10, slice(None)), (17, slice(0, 1)), (25, slice(0, 650))):
                a[row, cols] = value
                b[row, cols] = value
        check_verify([s], run_verify([s]))


def test_odd_uniforms_temperatures_and_tokens():
    rng = np.random.default_rng(76)
    odd_t = [float("nan"), -3.0, 0.0, 1e-38, 1e-30, 1e-3, 1e30, float("inf"), 50.0, 2.0 ** -100]
    trees = [list(range(-1, 3))] * len(odd_t)
    for drawn in (False, True):
        s = Verify(rng, trees, 333, drawn=drawn, ts=odd_t)
        s.u[::4] = rng.choice([0.0, -1.0, 1.0, 7.0, np.nan, 1 - 2.0 ** -24, np.inf, -np.inf], len(odd_t))
        s.u[1::4] = rng.choice([0.0, -1.0, 1.0, np.nan, 0.5], len(odd_t))
        for i, v in ((1, -1), (6, 333), (11, 2 ** 31 - 1), (13, -2 ** 31)):
            s.tokens[i] = v
        check_verify([s], run_verify([s]), most_near=0.2)


def test_a_draft_equal_to_the_target_is_never_turned_away_and_nothing_left_gives_the_largest():
    rng = np.random.default_rng(77)
    s = Verify(rng, [[-1, 0, 1, 2]] * 40, 97, drawn=True)
    s.draft.copy_(s.logits)
    s.d[:] = s.x
    s.u[:] = 1 - 2.0 ** -24
    row = 0
    for t in s.ts:                                               # tokens that the draft may have drawn, however unlikely
        for i in range(1, 4):
            s.tokens[row + i] = int(rng.choice(np.flatnonzero(DR.distribution(s.x[row + i - 1], float(t)) > 1e-9)))
        row += 4
    plan = run_verify([s])
    assert plan.kept.tolist() == [4] * 40
    # all of the probability lies on tokens that were turned away: none is left by any rounding
    s = Verify(rng, [[-1, 0, 0]], 4, "f32", ts=[1.0])
    s.x[0] = [-np.inf, 2.0, 2.0, -np.inf]
    s.logits[0] = dev(s.x[0].astype(np.float32))
    s.tokens, s.u[:] = [0, 3, 0], 0.0
    plan = run_verify([s])
    assert (plan.kept.tolist(), plan.next.tolist()) == ([1], [1])


def test_tokens_are_drawn_with_the_targets_probabilities():
    """4000 sequences of one row and different uniforms, spread evenly: as many tokens of each kind as its probability says, to one or two at its borders."""
    n, V = 4000, 50
    x = np.random.default_rng(78).standard_normal(V).astype(np.float32)
    s = Verify(np.random.default_rng(79), [[-1]] * n, V, "f32", ts=[0.9] * n)
    s.logits.copy_(dev(x)[None].expand(n, V))
    s.x[:] = x
    s.u[:] = (np.arange(n) + 0.5) / n
    plan = run_verify([s])
    got = np.bincount(plan.next.cpu().numpy(), minlength=V)
    assert np.abs(got - DR.distribution(x, float(np.float32(0.9))) * n).max() <= 1.0 + 1e-6


def test_every_cut_of_the_rows_gives_the_same():
    """1, 2, 4 and 8 pieces to a thread, chunks from one to dozens."""
    rng = np.random.default_rng(80)
    s = [Verify(rng, [random_tree(rng, 9), list(range(-1, 4))], 20011, drawn=d, shift=d) for d in (False, True)]
    plan = run_verify(s)
    table, ts = plan.table, plan.temperatures
    for pieces, draw in ((1, 1), (2, 4), (4, 2), (8, 1), (1, 4)):
        first, at, chunks = np.zeros_like(plan.first), 0, lambda a, n: -(-((int(a["vocab"]) - 1 + 7) // 8 + 1) // (256 * n))
        for i, q in enumerate(table.seqs):
            a = plan.args[q["service"]]
            first[i] = at
            at += int(q["rows"]) * chunks(a, pieces) * (2 if a["draft_logits"] else 1)
        first[-1] = at
        own = B.VerifyPlan(at, pieces, max(chunks(a, draw) for a in plan.args), draw, 1 << 20)
        ws = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)
        d_first = R._upload(first, DEV)
        launch = B.VerifyLaunch(plan.args.ctypes.data, plan.d_args.data_ptr(), first.ctypes.data, d_first.data_ptr(), ts.data_ptr(), plan.kept.data_ptr(), plan.next.data_ptr(),
                                ws.data_ptr(), ws.numel(), table.c, own, len(plan.args), plan.dtype)
        for _ in range(2):
            plan.kept.fill_(-1)
            plan.next.fill_(-1)
            B.epara_verify_drafts(launch, R.current_stream_handle())
            sync()
            check_verify(s, plan)


# ---- keeping -----------------------------------------------------------------------------------------------------

def keep_case(rng, starts, trees, kv_heads, D, wild=False):
    """A cache in whose blocks the exponents differ, with rubbish behind; wild: any bytes, NaN codes and the lowest and highest scales."""
    case = Case(rng, [s + n for s, n in zip(starts, trees)], kv_heads, kv_heads, D)
    for pages, s, n in zip(case.pages, starts, trees):
        if s + n and not wild:
            size = np.exp2(rng.integers(-12, 13, (s + n + 31) // 32)).repeat(32)[: s + n, None, None]
            case.oracle.append(pages, 0, rng.standard_normal((s + n, kv_heads, D)) * size, rng.standard_normal((s + n, kv_heads, D)) * size[::-1])
    case.upload()
    return case


def run_keep(services):
    """services: per service (cases of its layers, starts, rows, paths, kept) -> runs the library and the oracle."""
    table, groups, kept_all = [], [], []
    for g, (layers, starts, rows, paths, kept) in enumerate(services):
        seqs, row, flat = [], 0, []
        for pages, s, n, p in zip(layers[0].pages, starts, rows, paths):
            seqs.append({"first_row": row, "rows": n, "start": s, "pages": pages})
            flat += list(p) + [-1] * (n - len(p))
            row += n
        table.append(seqs)
        path = dev(flat, np.int32) if flat else torch.zeros(0, dtype=torch.int32, device=DEV)
        for c in layers:
            c.pages = layers[0].pages
            groups.append({"service": g, "cache": c.cache, "path": path})
        kept_all += kept
    plan = R.CacheKeepPlan(R.SequenceTable(table, DEV), groups, DEV, kept=dev(kept_all, np.int32))
    R.cache_keep(plan)
    for layers, starts, rows, paths, kept in services:
        for c in layers:
            for pages, s, n, p, k in zip(c.pages, starts, rows, paths, kept):
                if n <= 256:
                    DR.keep(c.oracle, pages, s, n, list(p)[: max(0, min(k, n))])
    sync()
    for layers, *_ in services:
        for c in layers:
            assert np.array_equal(c.cache.scales.cpu().numpy(), c.oracle.scales)
            assert np.array_equal(c.cache.codes.cpu().numpy(), c.oracle.packed())
    return plan


def some_path(rng, n):
    k = int(rng.integers(1, n + 1)) if rng.random() < 0.5 else int(rng.integers(1, min(n, 6) + 1))
    return sorted(rng.choice(n, k, replace=False).tolist())


@pytest.mark.parametrize("kv_heads,D", [(2, 128), (3, 64), (1, 128), (8, 64)])
def test_keeping_paths_of_every_kind(kv_heads, D):
    """Trees that begin and end anywhere in a block, on pages in any order; bit for bit, what is behind included."""
    rng = np.random.default_rng([91, kv_heads, D])
    starts = [0, 1, 31, 32, 33, 63, 64, 100, 5, 127, 500, 90]
    rows = [8, 40, 1, 64, 33, 2, 130, 256, 16, 65, 9, 200]
    paths = [some_path(rng, n) for n in rows]
    layers = [keep_case(rng, starts, rows, kv_heads, D) for _ in range(3)]
    second = [keep_case(rng, starts[:3], rows[:3], 5, 192 - D)]
    run_keep([(layers, starts, rows, paths, [len(p) for p in paths]), ([keep_case(rng, [], [], 1, D)], [], [], [], []),
              (second, starts[:3], rows[:3], paths[:3], [len(p) for p in paths[:3]])])


@pytest.mark.parametrize("D", [64, 128])
def test_keeping_what_need_not_move_and_odd_paths(D):
    """Whole chains, nothing, more than there is; paths that fall, repeat or leave the rows; a sequence that is no tree."""
    rng = np.random.default_rng([92, D])
    rows = [20, 20, 20, 20, 20, 20, 20, 70, 300, 0]
    starts = [10, 50, 30, 20, 0, 40, 60, 31, 5, 64]
    paths = [list(range(20)), [3, 4], [0, 5, 9], [0, 4, 4, 7], [0, 2, 1], [1, 19, 20, 21], [-1, 3], [0, 1, 2, 69], [0, 299], []]
    kept = [20, 0, -4, 4, 3, 4, 2, 100, 2, 5]
    layers = [keep_case(rng, starts, rows, 2, D) for _ in range(2)]
    run_keep([(layers, starts, rows, paths, kept)])


@pytest.mark.parametrize("D", [64, 128])
def test_keeping_copies_any_codes(D):
    """NaN codes stay NaN (a broken token keeps to itself), -0 stays; scale bytes at both ends; earlier tokens of a block that grows are rounded again."""
    rng = np.random.default_rng([93, D])
    starts, rows = [40, 7, 64], [50, 25, 100]
    case = keep_case(rng, starts, rows, 2, D, wild=True)
    case.oracle.scales[:] = rng.choice([0, 31, 100, 127, 130, 180, 247, 255], case.oracle.scales.shape)
    case.upload()
    paths = [[0, 7, 8, 30, 49], [24], [0, 1, 2, 3, 40, 41, 77, 99]]
    codes, scales = case.oracle.codes.copy(), case.oracle.scales.copy()
    run_keep([([case], starts, rows, paths, [len(p) for p in paths])])
    assert not np.array_equal(codes, case.oracle.codes) and not np.array_equal(scales, case.oracle.scales)
