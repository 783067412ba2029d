"""GPU parity of the pieces between a decoder block's dense layers (norm, append, attention over the 8-bit cache, page copies), through the
C ABI, against oracle/decoder.py in 64 bits on the same bits.

Tolerances, from the formats.  bf16 outputs: half a unit in the last place is 2^-9 of the value's power of two, so 2^-8 of the value holds it with
fp32's own errors (~1e-6).  E4M3 outputs: half a step is 2^-4 of a value, or 2^-10 of the scale for subnormal codes; fp32 in front of it may move a
value over a rounding boundary, which the same bound holds with a factor of 1 + 1e-4.  Attention: a weight is held to 2^-8 of its value at least (f16
keeps it to 2^-11), so an output moves by at most 2^-8 of the weighted mean of |v|, and bf16 rounds it by 2^-8 of itself; scores are fp32 sums of
exact products, some 1e-5 in the exponent (2^-10 is allowed for them and the rest)."""
import numpy as np
import pytest
import torch

from oracle import decoder as OD
from oracle import reference as ref
from paper_2511_00603_amd import binding as B
from paper_2511_00603_amd import runtime as R
from workloads import casts

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, SLACK = 2.0 ** -8, 1.0 + 1e-4


def dev_bf16(a):
    """-> (exact values of the bf16 rounding in 64 bits, device tensor)."""
    bits = casts.bf16_bits(np.ascontiguousarray(a, dtype=np.float32))
    return ref.bf16_decode(bits), R.device_tensor_from_bits(bits, B.EPARA_BF16, DEV)


def dev(a, dtype=None):
    return torch.from_numpy(np.array(a, dtype=dtype)).to(DEV)


def fetch(t):
    return t.float().cpu().numpy().astype(np.float64)


def sync():
    torch.cuda.synchronize()


# ---- normalisation -----------------------------------------------------------------------------------------------

def norm_groups(rng, shapes, kind, with_r, with_s, eps=1e-5):
    groups, want = [], []
    for M, d in shapes:
        x, X = dev_bf16(rng.standard_normal((M, d)) * 2 + 0.3)
        r, Rt = dev_bf16(rng.standard_normal((M, d))) if with_r else (None, None)
        gamma = (1 + 0.2 * rng.standard_normal(d)).astype(np.float32)
        g = {"X": X, "R": Rt, "gamma": dev(gamma), "S": torch.full((M, d), 7.0, dtype=torch.bfloat16, device=DEV) if with_s else None, "eps": eps,
             "Y": torch.full((M, d), 7.0, dtype=torch.bfloat16, device=DEV) if kind == "bf16" else torch.full((M, d), 0x7F, dtype=torch.uint8, device=DEV)}
        if kind == "row":
            g["row_scales"] = torch.full((M,), -1.0, device=DEV)
        if kind == "service":
            g["out_scale"] = 0.011
        groups.append(g)
        want.append(OD.add_rms_norm(x, r, gamma.astype(np.float64), float(np.float32(eps))))
    return groups, want


def check_norm(groups, want, kind):
    for i, (g, (s, y)) in enumerate(zip(groups, want)):
        if not y.size:
            continue
        if g["S"] is not None:
            assert (np.abs(fetch(g["S"]) - s) <= BF * np.abs(s) + 1e-30).all(), i
        if kind == "bf16":
            assert (np.abs(fetch(g["Y"]) - y) <= BF * np.abs(y) + 1e-30).all(), i
            continue
        scale = np.full(len(y), float(np.float32(0.011)))
        if kind == "row":
            scale = fetch(g["row_scales"])
            top = np.abs(y).max(axis=1)
            assert (np.abs(scale - np.where(top > 0, top / 448.0, 1.0)) <= 1e-6 * scale).all(), i
        scale = scale[:, None]
        got = OD.e4m3_decode(g["Y"].cpu().numpy()) * scale
        limit = np.clip(y, -448 * scale, 448 * scale)
        assert (np.abs(got - limit) <= np.maximum(np.abs(limit) * 2.0 ** -4, scale * 2.0 ** -10) * SLACK).all(), i


@pytest.mark.parametrize("kind", ["bf16", "row", "service"])
@pytest.mark.parametrize("with_r,with_s", [(True, True), (False, False), (True, False), (False, True)])
def test_rmsnorm_mixed_services(kind, with_r, with_s):
    """Widths that take one to sixteen chunks a lane and leave lanes idle, row counts from none on, in one launch."""
    rng = np.random.default_rng([41, with_r, with_s])
    groups, want = norm_groups(rng, [(105, 4096), (0, 64), (1, 8), (5, 520), (33, 1032), (3, 8192), (0, 768), (67, 64), (2, 5120)], kind, with_r, with_s)
    R.add_rmsnorm(R.RmsNormPlan(groups, DEV))
    sync()
    check_norm(groups, want, kind)


@pytest.mark.parametrize("d", [8, 504, 512, 520, 1016, 1024, 2040, 2048, 2056, 4088, 4096, 4104, 8184, 8192])
def test_rmsnorm_widths(d):
    for kind in ("bf16", "row"):
        groups, want = norm_groups(np.random.default_rng([42, d]), [(9, d)], kind, True, True)
        R.add_rmsnorm(R.RmsNormPlan(groups, DEV))
        sync()
        check_norm(groups, want, kind)


@pytest.mark.parametrize("n", [63, 64, 65, 130])
def test_rmsnorm_many_services(n):
    groups, want = norm_groups(np.random.default_rng(43), [((0, 1, 3, 0, 2)[(i + n) % 5] if i < n - 1 else 0, 64 + 8 * (i % 3)) for i in range(n)], "row", True, True)
    R.add_rmsnorm(R.RmsNormPlan(groups, DEV))
    sync()
    check_norm(groups, want, "row")


def test_rmsnorm_more_rows_than_waves():
    groups, want = norm_groups(np.random.default_rng(44), [(9000, 64), (4500, 256)], "bf16", True, True)
    R.add_rmsnorm(R.RmsNormPlan(groups, DEV))
    sync()
    check_norm(groups, want, "bf16")


def test_rmsnorm_in_place_zero_rows_and_rows_that_are_not_finite():
    rng = np.random.default_rng(45)
    x, X = dev_bf16(rng.standard_normal((20, 768)))
    r, Rt = dev_bf16(rng.standard_normal((20, 768)))
    s, y = OD.add_rms_norm(x, r, np.ones(768), float(np.float32(1e-5)))
    R.add_rmsnorm(R.RmsNormPlan([{"X": X, "R": Rt, "gamma": torch.ones(768, device=DEV), "S": X, "Y": Rt, "eps": 1e-5}], DEV))
    sync()
    assert (np.abs(fetch(X) - s) <= BF * np.abs(s)).all() and (np.abs(fetch(Rt) - y) <= BF * np.abs(y)).all()
    X = torch.randn(4, 256, device=DEV).bfloat16()
    X[0] = 0
    X[2, 5] = float("nan")
    X[3, 7] = float("inf")
    g = {"X": X, "gamma": torch.ones(256, device=DEV), "Y": torch.zeros(4, 256, dtype=torch.uint8, device=DEV), "row_scales": torch.zeros(4, device=DEV)}
    R.add_rmsnorm(R.RmsNormPlan([g], DEV))
    sync()
    scale = g["row_scales"].cpu()
    assert scale[0] == 1.0 and (g["Y"][0] == 0).all() and 0 < scale[1] < 1 and not torch.isfinite(scale[2:]).any()


# ---- the cache ---------------------------------------------------------------------------------------------------

class Case:
    """One service: a cache with rubbish in it (NaN codes and scales too), sequences with pages anywhere in it, and the oracle's copy."""

    def __init__(self, rng, lengths, heads, kv_heads, D, spare=3):
        self.rng, self.H, self.KV, self.D = rng, heads, kv_heads, D
        counts = [-(-n // 64) for n in lengths]
        self.n_pages = sum(counts) + spare
        ids = rng.permutation(self.n_pages)
        self.pages, at = [], 0
        for c in counts:
            self.pages.append([int(p) for p in ids[at: at + c]])
            at += c
        self.oracle = OD.Cache(self.n_pages, kv_heads, D, rng)
        self.cache = R.PagedCache(dev(self.oracle.packed()), dev(self.oracle.scales))

    def fill(self, lengths):
        """Tokens that earlier calls have appended."""
        for pages, n in zip(self.pages, lengths):
            if n:
                K = self.rng.standard_normal((n, self.KV, self.D)) * np.exp(0.5 * self.rng.standard_normal((n, 1, 1)))
                self.oracle.append(pages, 0, K, self.rng.standard_normal((n, self.KV, self.D)) + 0.2)
        self.upload()

    def upload(self):
        self.cache.codes.copy_(dev(self.oracle.packed()))
        self.cache.scales.copy_(dev(self.oracle.scales))


def sequences(case, starts, news):
    out, row = [], 0
    for pages, start, new in zip(case.pages, starts, news):
        out.append({"first_row": row, "rows": new, "start": start, "pages": pages})
        row += new
    return out, row


def append_case(rng, starts, news, heads, kv_heads, D, axes=1, rotary=True, strided=False):
    case = Case(rng, [max(s + n, 0) for s, n in zip(starts, news)], heads, kv_heads, D)
    case.fill([max(s, 0) for s in starts])
    seqs, rows = sequences(case, starts, news)
    qkv, QKV = dev_bf16(rng.standard_normal((rows, (heads + 2 * kv_heads) * D)) * np.exp(rng.standard_normal((rows, 1))))
    if strided:                                                  # a row of a wider buffer
        wide = torch.full((rows, QKV.shape[1] + 24), float("nan"), dtype=torch.bfloat16, device=DEV)
        wide[:, 8: 8 + QKV.shape[1]] = QKV
        QKV = wide[:, 8: 8 + QKV.shape[1]]
    Q = torch.full((rows, heads * D + (16 if strided else 0)), 3.0, dtype=torch.bfloat16, device=DEV)[:, : heads * D]
    longest = max([s + n for s, n in zip(starts, news)] + [1])
    table = OD.rotary_table(longest, D).astype(np.float32)
    pos = np.concatenate([np.zeros((0, 3))] + [np.repeat(np.arange(s, s + n)[:, None], 3, 1) for s, n in zip(starts, news)]).astype(np.int32)
    pairs = [D // 2, 0, 0]
    if axes > 1:
        pairs = [D // 2 - 13 * (axes - 1)] + [13] * (axes - 1) + [0] * (3 - axes)         # odd counts: an axis may begin inside a lane's pairs
        pos = rng.integers(-2, longest + 3, pos.shape).astype(np.int32)                   # positions outside the table take its nearest row
    g = {"QKV": QKV, "Q": Q, "cache": case.cache, "heads": heads, "rotary": dev(table) if rotary else None, "axis_pairs": pairs,
         "positions": dev(pos) if axes > 1 else None}
    x = qkv.reshape(rows, heads + 2 * kv_heads, D)
    if rotary:
        turned = OD.rotate(x[:, : heads + kv_heads], table.astype(np.float64), pos, pairs)
        x = np.concatenate([turned, x[:, heads + kv_heads:]], axis=1)
    return case, seqs, g, x


def run_append(cases):
    """cases: what append_case gives, of several services -> runs them in one call and the oracle's after it."""
    table = R.SequenceTable([c[1] for c in cases], DEV)
    plan = R.CacheAppendPlan(table, [c[2] for c in cases], DEV)
    R.cache_append(plan)
    for case, seqs, g, x in cases:
        for s in seqs:
            rows = slice(s["first_row"], s["first_row"] + s["rows"])
            if s["rows"]:
                case.oracle.append(s["pages"], s["start"], x[rows, case.H: case.H + case.KV], x[rows, case.H + case.KV:])
    sync()
    return plan


def check_append(cases, exact):
    for case, seqs, g, x in cases:
        want = x[:, : case.H].reshape(len(x), case.H * case.D)
        if g["Q"] is not None and len(x):
            assert (np.abs(fetch(g["Q"]) - want) <= BF * np.abs(want) + 1e-6 * np.abs(x).max()).all()
        assert np.array_equal(case.cache.scales.cpu().numpy(), case.oracle.scales)
        got, codes = case.cache.codes.cpu().numpy(), case.oracle.packed()
        if exact:
            assert np.array_equal(got, codes)
            continue
        # a rotated key in fp32 may fall on the other side of a rounding boundary: one step, and rarely
        other = got != codes
        assert other.mean() < 2e-3
        a, b = got[other].astype(int), codes[other].astype(int)
        near = (np.abs((a & 0x7F) - (b & 0x7F)) <= 1) & (((a ^ b) & 0x80 == 0) | (((a | b) & 0x7F) <= 1))
        assert near.all()


@pytest.mark.parametrize("heads,kv_heads,D", [(8, 2, 128), (3, 3, 64), (5, 1, 128), (12, 4, 64), (1, 1, 64), (40, 40, 128)])
def test_append_single_tokens_and_prompts(heads, kv_heads, D):
    """One to hundreds of new tokens behind contexts that end anywhere in a block, without rotation: bit for bit."""
    rng = np.random.default_rng([51, heads, D])
    starts, news = [0, 0, 31, 32, 63, 64, 100, 5, 17, 0, 90], [1, 70, 1, 1, 1, 1, 1, 27, 0, 32, 200 if heads < 20 else 40]
    c = append_case(rng, starts, news, heads, kv_heads, D, rotary=False)
    run_append([c])
    check_append([c], exact=True)


@pytest.mark.parametrize("axes", [1, 2, 3])
@pytest.mark.parametrize("D", [64, 128])
def test_append_rotates_by_one_to_three_axes_over_several_services(axes, D):
    rng = np.random.default_rng([52, axes, D])
    cases = [append_case(rng, [0, 45], [77, 3], 6, 2, D, axes, strided=True), append_case(rng, [200], [1], 4, 4, 192 - D, axes),
             append_case(rng, [], [], 2, 1, D), append_case(rng, [10, 0, 3], [0, 0, 40], 7, 1, D, 1)]
    run_append(cases)
    check_append(cases, exact=False)


def test_append_of_queries_left_where_they_are():
    c = append_case(np.random.default_rng(53), [3, 9], [40, 1], 4, 2, 128, rotary=False)
    c[2]["Q"] = None
    run_append([c])
    check_append([c], exact=True)


def test_append_token_by_token_and_again():
    """The same tokens one by one over three blocks, where scales grow; and a call repeated leaves everything as it is."""
    rng = np.random.default_rng(54)
    case = Case(rng, [90], 2, 2, 128)
    qkv, QKV = dev_bf16(rng.standard_normal((90, 6 * 128)) * np.exp2(rng.integers(-6, 7, (90, 1))))
    x = qkv.reshape(90, 6, 128)
    for t in range(90):
        for again in range(2 if t % 7 == 0 else 1):
            seqs = [{"first_row": t, "rows": 1, "start": t, "pages": case.pages[0]}]
            R.cache_append(R.CacheAppendPlan(R.SequenceTable([seqs], DEV), [{"QKV": QKV, "Q": None, "cache": case.cache, "heads": 2}], DEV))
        case.oracle.append(case.pages[0], t, x[t: t + 1, 2:4], x[t: t + 1, 4:])
    sync()
    assert np.array_equal(case.cache.scales.cpu().numpy(), case.oracle.scales) and np.array_equal(case.cache.codes.cpu().numpy(), case.oracle.packed())


def test_append_padding_zeros_infinities_and_nans():
    """Rows in front of a sequence join nothing; a block of zeros, the largest and the smallest values; broken tokens keep to themselves."""
    for D in (64, 128):
        rng = np.random.default_rng([55, D])
        c = append_case(rng, [-3, -40, 20, 0], [10, 40, 30, 64], 2, 2, D, rotary=False)
        case, seqs, g, x = c
        rows = len(x)
        bad = x.reshape(rows, -1).astype(np.float32)
        bad[50 + 5, 3 * D: 5 * D] = 0.0                          # zeros
        bad[50 + 30: 50 + 62] = 0.0                              # and a block of them
        bad[52, 2 * D + 3] = np.nan                              # key of head 0
        bad[53, 5 * D + D - 1] = np.nan                          # value of head 1
        bad[54, 4 * D: 4 * D + 9] = np.inf                       # values of head 0
        bad[56, 2 * D] = -np.inf
        bad[85] = np.float32(3.3e38)
        bad[140] = 1e-38
        g["QKV"].copy_(dev(bad).bfloat16())
        x = ref.bf16_decode(casts.bf16_bits(bad)).reshape(x.shape)
        c = (case, seqs, g, x)
        run_append([c])
        assert np.array_equal(case.cache.scales.cpu().numpy(), case.oracle.scales)
        assert np.array_equal(case.cache.codes.cpu().numpy(), case.oracle.packed())


def test_append_refuses_before_it_enqueues():
    case = Case(np.random.default_rng(56), [100, 100], 2, 1, 64)
    QKV = torch.zeros(8, 4 * 64, dtype=torch.bfloat16, device=DEV)
    seqs = [{"first_row": 0, "rows": 2, "start": 0, "pages": case.pages[0]}, {"first_row": 2, "rows": 1, "start": 3, "pages": case.pages[0]}]
    with pytest.raises(B.EparaError) as e:                       # the same page for two sequences
        R.cache_append(R.CacheAppendPlan(R.SequenceTable([seqs], DEV), [{"QKV": QKV, "cache": case.cache, "heads": 2}], DEV))
    assert e.value.status == B.EPARA_ERR_SHAPE
    for bad in ({"QKV": QKV.float()}, {"QKV": QKV[:, :128]}, {"QKV": QKV.cpu()}, {"Q": torch.zeros(8, 64, dtype=torch.bfloat16, device=DEV)}, {"rotary": torch.zeros(9, 16, 2, device=DEV)},
                {"axis_pairs": (30, 1, 0)}, {"positions": torch.zeros(8, 3, device=DEV)}):
        with pytest.raises(ValueError):
            R.CacheAppendPlan(R.SequenceTable([seqs[:1]], DEV), [dict({"QKV": QKV, "cache": case.cache, "heads": 2}, **bad)], DEV)
    with pytest.raises(ValueError):
        R.PagedCache(case.cache.codes, case.cache.scales[:, :, :, :1])


# ---- attention ---------------------------------------------------------------------------------------------------

def attn_case(rng, starts, news, heads, kv_heads, D, window=0, softcap=0.0, sharp=1.0, strided=False):
    case = Case(rng, [max(s + n, 0) for s, n in zip(starts, news)], heads, kv_heads, D)
    case.fill([max(s + n, 0) for s, n in zip(starts, news)])
    seqs, rows = sequences(case, starts, news)
    q, Q = dev_bf16(rng.standard_normal((rows, heads * D)) * sharp)
    O = torch.full((rows, heads * D + (8 if strided else 0)), float("nan"), dtype=torch.bfloat16, device=DEV)[:, : heads * D]
    if strided:                                                  # the queries as the first columns of a projection's output
        wide = torch.full((rows, heads * D + 2 * kv_heads * D), float("nan"), dtype=torch.bfloat16, device=DEV)
        wide[:, : heads * D] = Q
        Q = wide[:, : heads * D]
    return case, seqs, {"Q": Q, "O": O, "cache": case.cache, "heads": heads, "window": window, "softcap": softcap}, q.reshape(rows, heads, D)


def run_attn(cases):
    plan = R.CacheAttnPlan(R.SequenceTable([c[1] for c in cases], DEV), [c[2] for c in cases], DEV)
    R.cache_attention(plan)
    sync()
    return plan


def check_attn(cases):
    for case, seqs, g, q in cases:
        got = fetch(g["O"]).reshape(q.shape)
        for s in seqs:
            if not s["rows"]:
                continue
            rows = slice(s["first_row"], s["first_row"] + s["rows"])
            K, V = case.oracle.values(s["pages"], max(s["start"] + s["rows"], 0))
            want, mass = OD.attention(q[rows], K, V, s["start"], float(np.float32(case.D ** -0.5)), g["window"], g["softcap"])
            assert np.array_equal(np.isnan(got[rows]), np.isnan(want)), (s["start"], s["rows"])
            off, bound = np.abs(got[rows] - want), (2.0 ** -8 + 2.0 ** -10) * mass + BF * np.abs(want)
            assert (np.nan_to_num(off) <= np.nan_to_num(bound)).all(), (s["start"], s["rows"], np.nanmax(off / np.maximum(bound, 1e-30)))


HEADS = [(8, 2, 128), (3, 3, 64), (16, 1, 128), (12, 4, 64), (32, 2, 64), (2, 2, 128)]


@pytest.mark.parametrize("heads,kv_heads,D", HEADS)
def test_attention_of_single_tokens(heads, kv_heads, D):
    """One token behind contexts that end at every place of a page that matters, one to many pages."""
    rng = np.random.default_rng([61, heads, D])
    starts = [0, 1, 15, 16, 31, 32, 33, 62, 63, 64, 65, 127, 128, 191, 300, 1000]
    c = attn_case(rng, starts, [1] * len(starts), heads, kv_heads, D)
    run_attn([c])
    check_attn([c])


@pytest.mark.parametrize("heads,kv_heads,D", HEADS)
def test_attention_of_prompts(heads, kv_heads, D):
    """Prompts of one to hundreds of tokens, alone and behind a context, with tiles of rows that end anywhere."""
    rng = np.random.default_rng([62, heads, D])
    c = attn_case(rng, [0, 0, 0, 70, 3, 130, 0], [1, 5, 130, 40, 17, 8, 0], heads, kv_heads, D, strided=True)
    run_attn([c])
    check_attn([c])


@pytest.mark.parametrize("window,softcap", [(1, 0.0), (2, 0.0), (63, 0.0), (64, 0.0), (65, 5.0), (200, 0.0), (5000, 30.0), (0, 30.0), (0, 0.5)])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_with_windows_and_capped_scores(window, softcap, D):
    rng = np.random.default_rng([63, window, D])
    c = attn_case(rng, [0, 500, 64, 127, 300, 0], [150, 1, 1, 66, 3, 40], 4, 2, D, window, softcap, sharp=2.0)
    run_attn([c])
    check_attn([c])


def test_attention_of_several_services_with_different_heads():
    rng = np.random.default_rng(64)
    cases = [attn_case(rng, [40, 0], [1, 90], 8, 2, 128), attn_case(rng, [], [], 2, 2, 64), attn_case(rng, [33], [200], 6, 6, 64, window=50, softcap=20.0),
             attn_case(rng, [0] * 70, [1] * 35 + [0] * 35, 4, 1, 64), attn_case(rng, [700], [1], 24, 2, 128)]
    run_attn(cases)
    check_attn(cases)


def test_attention_of_padding_and_empty_sequences():
    """Rows in front of a sequence are zeros, in a tile of their own and next to rows that see keys."""
    rng = np.random.default_rng(65)
    cases = [attn_case(rng, [-5, -1, -300, -3, -64], [5, 1, 310, 4, 130], 4, 2, D) for D in (64, 128)]
    run_attn(cases)
    check_attn(cases)
    for case, seqs, g, q in cases:
        assert (g["O"][:6] == 0).all()


@pytest.mark.parametrize("D", [64, 128])
def test_attention_over_long_contexts_is_cut_and_joined(D):
    """Contexts that several workgroups share, of few and of many rows, with and without a window; the same bits every time."""
    rng = np.random.default_rng([66, D])
    c = attn_case(rng, [9000, 4097, 3000, 6000], [1, 5, 64, 200], 4, 1, D)
    plan = run_attn([c])
    assert plan.plan.workspace_bytes > 0 and plan.plan.n_items[0] > 3
    got = c[2]["O"].clone()
    for i, s in enumerate(c[1]):
        r = np.random.default_rng(i).choice(s["rows"], min(s["rows"], 6), replace=False)
        K, V = c[0].oracle.values(s["pages"], s["start"] + s["rows"])
        for t in r:
            want, mass = OD.attention(c[3][s["first_row"] + t: s["first_row"] + t + 1], K, V, s["start"] + int(t), D ** -0.5)
            off = np.abs(fetch(got)[s["first_row"] + t].reshape(4, D) - want[0])
            assert (off <= (2.0 ** -8 + 2.0 ** -10) * mass[0] + BF * np.abs(want[0])).all()
    for _ in range(5):
        c[2]["O"].fill_(float("nan"))
        R.cache_attention(plan)
        sync()
        assert torch.equal(c[2]["O"].view(torch.int16), got.view(torch.int16))


def test_attention_of_one_strong_key_and_thousands_of_weak_ones():
    """What a strong key leaves to thousands of others (weights of some 2^-18 each) is kept to the tolerance."""
    D, n = 128, 6000
    for rows in (1, 100):
        case = Case(np.random.default_rng(67), [n], 1, 1, D)
        K, V = np.zeros((n, 1, D)), np.full((n, 1, D), 1.0)
        K[:, 0, 0], K[7, 0, 0], V[7] = -1.0, 12.0, -1.0
        case.oracle.append(case.pages[0], 0, K, V)
        case.upload()
        q = np.zeros((rows, D))
        q[:, 0] = 10.0
        c = (case, [{"first_row": 0, "rows": rows, "start": n - rows, "pages": case.pages[0]}], {"Q": dev_bf16(q)[1], "O": torch.zeros(rows, D, dtype=torch.bfloat16, device=DEV),
             "cache": case.cache, "heads": 1, "window": 0, "softcap": 0.0}, q.reshape(rows, 1, D))
        run_attn([c])
        check_attn([c])
        assert fetch(c[2]["O"]).min() > -1.0


@pytest.mark.parametrize("rows", [1, 90])
def test_attention_with_scores_that_rise_and_fall_by_hundreds(rows):
    """The reference of a row is raised late and often, or never again; also scores far from zero altogether."""
    for D, slope in ((64, 0.8), (128, -0.8), (64, 40.0), (128, 0.0)):
        n = 400
        rng = np.random.default_rng([68, rows, D])
        case = Case(rng, [n], 2, 1, D)
        K, V = rng.standard_normal((n, 1, D)) * 0.3, rng.standard_normal((n, 1, D))
        K[:, 0, 1] = 60.0 + slope * (np.arange(n) - 200)
        case.oracle.append(case.pages[0], 0, K, V)
        case.upload()
        q = rng.standard_normal((rows, 2 * D))
        q[:, 1], q[:, D + 1] = 8.0, -8.0
        q, Q = dev_bf16(q)
        c = (case, [{"first_row": 0, "rows": rows, "start": n - rows, "pages": case.pages[0]}], {"Q": Q, "O": torch.zeros(rows, 2 * D, dtype=torch.bfloat16, device=DEV), "cache": case.cache,
             "heads": 2, "window": 0, "softcap": 0.0}, q.reshape(rows, 2, D))
        run_attn([c])
        check_attn([c])


@pytest.mark.parametrize("rows", [1, 90])
@pytest.mark.parametrize("tiny", [0.0, 1e-20, 1e-5])
def test_attention_with_blocks_of_zero_and_of_tiny_values(rows, tiny):
    """Tokens whose values are (all but) zeros still take their share of the weights, before and behind blocks of ordinary and of huge values."""
    for D in (64, 128):
        n, rng = 300, np.random.default_rng([72, D])
        case = Case(rng, [n], 2, 1, D)
        K, V = rng.standard_normal((n, 1, D)), rng.standard_normal((n, 1, D))
        for lo, hi in ((0, 32), (64, 128), (160, 192)):
            V[lo:hi] *= tiny
        V[224:256] *= 1e6 if rows == 1 else 1.0
        case.oracle.append(case.pages[0], 0, K, V)
        case.upload()
        q, Q = dev_bf16(rng.standard_normal((rows, 2 * D)))
        c = (case, [{"first_row": 0, "rows": rows, "start": n - rows, "pages": case.pages[0]}], {"Q": Q, "O": torch.zeros(rows, 2 * D, dtype=torch.bfloat16, device=DEV), "cache": case.cache,
             "heads": 2, "window": 0, "softcap": 0.0}, q.reshape(rows, 2, D))
        run_attn([c])
        check_attn([c])


@pytest.mark.parametrize("rows", [3, 80])
def test_attention_keeps_broken_tokens_from_rows_that_do_not_see_them(rows):
    for D in (64, 128):
        n, rng = 130, np.random.default_rng([69, D])
        case = Case(rng, [n], 2, 1, D)
        K, V = rng.standard_normal((n, 1, D)), rng.standard_normal((n, 1, D))
        V[n - 2, 0, 5] = np.nan
        K[n - 60, 0, 5] = np.nan if rows == 80 else 0.0
        case.oracle.append(case.pages[0], 0, K, V)
        case.upload()
        q, Q = dev_bf16(rng.standard_normal((rows, 2 * D)))
        c = (case, [{"first_row": 0, "rows": rows, "start": n - rows, "pages": case.pages[0]}], {"Q": Q, "O": torch.zeros(rows, 2 * D, dtype=torch.bfloat16, device=DEV), "cache": case.cache,
             "heads": 2, "window": 40 if rows == 80 else 0, "softcap": 0.0}, q.reshape(rows, 2, D))
        run_attn([c])
        check_attn([c])
        assert torch.isnan(c[2]["O"][-1]).all() and not torch.isnan(c[2]["O"][0]).any()


def test_attention_of_queries_with_nans_zeros_and_wide_ranges():
    rng = np.random.default_rng(70)
    for new, H in ((1, 4), (40, 4)):
        c = attn_case(rng, [100], [new], H, 1, 128)
        q = fetch(c[2]["Q"]).reshape(new, H, 128).copy()
        q[0, 0], q[0, 1, 3], q[0, 2] = 0.0, np.nan, q[0, 2] * np.exp2(rng.integers(-12, 3, 128))
        q, Q = dev_bf16(q.reshape(new, -1))
        c[2]["Q"].copy_(Q)
        c = (c[0], c[1], c[2], q.reshape(new, H, 128))
        run_attn([c])
        check_attn([c])


def test_a_cache_of_more_than_four_gigabytes():
    """Pages at both ends of a cache whose offsets pass 32 bits: appended to, read and copied."""
    KV, D, n_pages = 8, 128, 33500
    cache = R.PagedCache(torch.empty(n_pages, KV, 2, 64 * D, dtype=torch.uint8, device=DEV), torch.empty(n_pages, KV, 2, 2, dtype=torch.uint8, device=DEV))
    assert cache.codes.numel() > 1 << 32
    rng = np.random.default_rng(71)
    pages = [33499, 3, 32768, 0]
    qkv, QKV = dev_bf16(rng.standard_normal((200, 3 * KV * D)))
    x = qkv.reshape(200, 3 * KV, D)
    seqs = [{"first_row": 0, "rows": 200, "start": 0, "pages": pages}]
    R.cache_append(R.CacheAppendPlan(R.SequenceTable([seqs], DEV), [{"QKV": QKV, "cache": cache, "heads": KV}], DEV))
    R.copy_pages(R.PageCopyPlan([{"cache": cache, "moves": [(33499, 7), (3, 33000)]}], DEV))
    seqs = [{"first_row": 0, "rows": 200, "start": 0, "pages": [7, 33000, 32768, 0]}]
    O = torch.zeros(200, KV * D, dtype=torch.bfloat16, device=DEV)
    R.cache_attention(R.CacheAttnPlan(R.SequenceTable([seqs], DEV), [{"Q": QKV[:, : KV * D], "O": O, "cache": cache, "heads": KV}], DEV))
    sync()
    small = OD.Cache(4, KV, D)
    small.append([0, 1, 2, 3], 0, x[:, KV: 2 * KV], x[:, 2 * KV:])
    got = cache.codes[pages].cpu().numpy()
    assert np.array_equal(got[:3], small.packed()[:3]) and np.array_equal(cache.codes[[7, 33000]].cpu().numpy(), got[:2])
    K, V = small.values([0, 1, 2, 3], 200)
    want, mass = OD.attention(x[:, :KV], K, V, 0, D ** -0.5)
    assert (np.abs(fetch(O).reshape(200, KV, D) - want) <= (2.0 ** -8 + 2.0 ** -10) * mass + BF * np.abs(want)).all()


# ---- pages, streams, graphs --------------------------------------------------------------------------------------

def test_copies_of_pages_in_several_caches():
    rng = np.random.default_rng(81)
    groups, want = [], []
    shared = [(1, 5), (1, 0), (7, 2), (8, 9)]
    for i, (KV, D, moves) in enumerate([(3, 128, shared), (3, 128, shared), (1, 64, []), (5, 64, [(0, 11)]), (2, 128, shared), (1, 64, [(4, 3)])]):
        codes, scales = (rng.integers(0, 256, s).astype(np.uint8) for s in ((12, KV, 2, 64 * D), (12, KV, 2, 2)))
        groups.append({"cache": R.PagedCache(dev(codes), dev(scales)), "moves": moves})
        for src, dst in moves:
            codes[dst], scales[dst] = codes[src], scales[src]
        want.append((codes, scales))
    R.copy_pages(R.PageCopyPlan(groups, DEV))
    sync()
    for g, (codes, scales) in zip(groups, want):
        assert np.array_equal(g["cache"].codes.cpu().numpy(), codes) and np.array_equal(g["cache"].scales.cpu().numpy(), scales)


@pytest.mark.parametrize("n", [64, 65, 100])
def test_copies_in_many_layers(n):
    codes, scales = torch.randint(0, 256, (n, 4, 1, 2, 4096), dtype=torch.uint8, device=DEV), torch.randint(0, 256, (n, 4, 1, 2, 2), dtype=torch.uint8, device=DEV)
    want = codes.clone(), scales.clone()
    moves = [(0, 3), (1, 2)]
    R.copy_pages(R.PageCopyPlan([{"cache": R.PagedCache(codes[i], scales[i]), "moves": moves} for i in range(n)], DEV))
    sync()
    for t, w in zip((codes, scales), want):
        assert torch.equal(t[:, :2], w[:, :2]) and torch.equal(t[:, 3], w[:, 0]) and torch.equal(t[:, 2], w[:, 1])


def test_the_calls_on_a_stream_of_their_own_and_in_a_graph():
    """A step (norm, append, attention over a cut context) on a side stream, then captured and replayed: every replay gives the eager bits for inputs that
    change between the replays."""
    rng = np.random.default_rng(82)
    case, seqs, a, q = attn_case(rng, [4000, 64, 700], [1, 1, 90], 8, 2, 128)
    rows = len(q)
    QKV, Q, O = torch.zeros(rows, 12 * 128, dtype=torch.bfloat16, device=DEV), torch.zeros(rows, 1024, dtype=torch.bfloat16, device=DEV), torch.zeros(rows, 1024, dtype=torch.bfloat16, device=DEV)
    X = torch.zeros(rows, 12 * 128, dtype=torch.bfloat16, device=DEV)
    table = R.SequenceTable([seqs], DEV)
    norm = R.RmsNormPlan([{"X": X, "gamma": torch.ones(12 * 128, device=DEV), "Y": QKV}], DEV)
    rotary = dev(OD.rotary_table(4001, 128).astype(np.float32))
    append = R.CacheAppendPlan(table, [{"QKV": QKV, "Q": Q, "cache": case.cache, "heads": 8, "rotary": rotary}], DEV)
    attn = R.CacheAttnPlan(table, [{"Q": Q, "O": O, "cache": case.cache, "heads": 8}], DEV)
    assert attn.plan.workspace_bytes > 0 and attn.plan.n_items[1] > 0

    def step():
        R.add_rmsnorm(norm)
        R.cache_append(append)
        R.cache_attention(attn)

    inputs = [torch.randn(rows, 12 * 128, device=DEV).bfloat16() for _ in range(4)]
    start_codes, start_scales, eager = case.cache.codes.clone(), case.cache.scales.clone(), []
    for x in inputs:
        X.copy_(x)
        case.cache.codes.copy_(start_codes)
        case.cache.scales.copy_(start_scales)
        step()
        sync()
        eager.append((O.clone(), case.cache.codes.clone()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for x, (o, codes) in zip(inputs, eager):
            X.copy_(x)
            case.cache.codes.copy_(start_codes)
            case.cache.scales.copy_(start_scales)
            O.zero_()
            step()
            side.synchronize()
            assert torch.equal(O.view(torch.int16), o.view(torch.int16)) and torch.equal(case.cache.codes, codes)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(2):
        for x, (o, codes) in zip(inputs, eager):
            X.copy_(x)
            case.cache.codes.copy_(start_codes)
            case.cache.scales.copy_(start_scales)
            O.zero_()
            graph.replay()
            sync()
            assert torch.equal(O.view(torch.int16), o.view(torch.int16)) and torch.equal(case.cache.codes, codes)
