"""CPU-side checks of the decoder block's calls: layouts of the structs, refusals (every call looks at the host copies of its
arguments before anything is enqueued, so each case here returns before a launch), plans, and the bookkeeping of pages against the oracle's."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from oracle import decoder as OD
from paper_2511_00603_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
D = 0x7000000                                    # a pretend device address: never dereferenced on these paths
vp = ctypes.c_void_p


def table_of(seqs, pages, **kw):
    """-> (SequenceTable, what keeps it alive)."""
    s, p = np.array(seqs, dtype=B.SEQUENCE), np.array(pages, dtype=np.int32)
    t = B.SequenceTable(s.ctypes.data if len(s) else None, D if len(s) else None, p.ctypes.data if len(p) else None, D if len(p) else None, len(s), len(p))
    for k, v in kw.items():
        setattr(t, k, v)
    return t, (s, p)


def test_struct_sizes_match_the_header():
    assert [t.itemsize for t in (B.RMSNORM_ARGS, B.SEQUENCE, B.APPEND_ARGS, B.CACHE_ATTN_ARGS, B.PAGE_MOVE, B.PAGE_COPY)] == [72, 24, 88, 80, 8, 40]
    assert [ctypes.sizeof(t) for t in (B.SequenceTable, B.CacheAttnPlan, B.CacheAttnLaunch, B.PagePool)] == [40, 24, 120, 24]


def test_rmsnorm_argument_checks():
    L = B.lib()

    def call(dtype=B.EPARA_BF16, G=1, **kw):
        a = np.zeros(1, dtype=B.RMSNORM_ARGS)
        a[0] = (D, D + 0x10000, D + 0x20000, D + 0x30000, D + 0x40000, 0, 0, 4096, 1e-6, 1.0, 0, 0)
        for k, v in kw.items():
            a[0][k] = v
        return L.epara_add_rmsnorm(a.ctypes.data, vp(D + 0x60000), G, dtype, None)

    bits8 = B.EPARA_FP8_E4M3
    assert L.epara_add_rmsnorm(None, None, 0, B.EPARA_BF16, None) == B.EPARA_OK
    assert call() == B.EPARA_OK and call(bits8) == B.EPARA_OK and call(bits8, row_scales=D) == B.EPARA_OK        # no rows: nothing to enqueue
    assert call(B.EPARA_F32) == B.EPARA_ERR_DTYPE and call(7) == B.EPARA_ERR_DTYPE
    assert L.epara_add_rmsnorm(None, vp(D), 1, B.EPARA_BF16, None) == B.EPARA_ERR_NULL
    for bad in (dict(G=-1), dict(M=-1), dict(d=0), dict(d=12), dict(d=B.EPARA_NORM_MAX_D + 8), dict(eps=-1.0), dict(eps=np.inf), dict(eps=np.nan),
                dict(first_row=1), dict(row_scales=D), dict(M=4, Y=D + 0x30000), dict(dtype=bits8, M=4, out_inv_scale=0.0),
                dict(dtype=bits8, M=4, out_inv_scale=np.nan), dict(dtype=bits8, M=4, out_inv_scale=np.inf), dict(dtype=bits8, M=4, Y=D), dict(dtype=bits8, M=4, Y=D + 0x10000)):
        assert call(**bad) == B.EPARA_ERR_SHAPE, bad
    for missing in ("X", "gamma", "Y"):
        assert call(M=4, **{missing: 0}) == B.EPARA_ERR_NULL, missing
    for field in ("X", "R", "gamma", "S", "Y"):
        assert call(M=4, **{field: D + 8}) == B.EPARA_ERR_ALIGN, field
    assert call(bits8, M=4, row_scales=D + 2) == B.EPARA_ERR_ALIGN


SEQ = (0, 0, 3, 60, 0, 1)                        # three tokens at 60 .. 62 of a sequence of one page


def append_args(**kw):
    a = np.zeros(1, dtype=B.APPEND_ARGS)
    a[0] = (D, D + 0x100000, D + 0x200000, D + 0x300000, D + 0x400000, 0, 8, 8, 2, 128, 10, 12 * 128, 8 * 128, 100, (64, 0))
    for k, v in kw.items():
        a[0][k] = v
    return a


BAD_SEQUENCES = [
    (1, 0, 3, 60, 0, 1), (-1, 0, 3, 60, 0, 1),               # no such service
    (0, -1, 3, 60, 0, 1), (0, 6, 3, 60, 0, 1), (0, 0, -1, 60, 0, 1),      # rows outside the service's
    (0, 0, 3, 62, 0, 1), (0, 0, 3, 60, 0, 0), (0, 0, 3, 60, 1, 1), (0, 0, 3, 60, -1, 1), (0, 0, 3, 60, 0, -1),      # tokens outside the pages, pages outside the table
    (0, 0, 3, -B.EPARA_CACHE_MAX_TOKENS - 1, 0, 1),
]


def test_append_argument_checks():
    L = B.lib()

    def plan(args, seqs=(SEQ,), pages=(4,), **kw):
        t, keep = table_of(list(seqs), list(pages), **kw)
        first = np.zeros(len(seqs) + 1, dtype=np.int32)
        return L.epara_plan_cache_append(args.ctypes.data, len(args), ctypes.addressof(t), first.ctypes.data), first

    def call(args, first, seqs=(SEQ,), pages=(4,), d_args=D):
        t, keep = table_of(list(seqs), list(pages))
        first = np.array(first, dtype=np.int32)
        return L.epara_cache_append(args.ctypes.data, d_args, len(args), ctypes.addressof(t), first.ctypes.data, D, None)

    rc, first = plan(append_args())
    assert rc == B.EPARA_OK and first[0] == 0 and first[1] > 2          # two key heads and the queries
    for bad in (dict(rows=-1), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(head_dim=96), dict(n_pages=-1), dict(n_pages=4), dict(qkv_stride=12 * 128 - 8),
                dict(qkv_stride=12 * 128 + 4), dict(q_stride=8 * 128 - 8), dict(q_stride=8 * 128 + 4), dict(axis_pairs=(-1, 0)), dict(axis_pairs=(60, 5)),
                dict(n_positions=0), dict(n_positions=62), dict(Q=D), dict(heads=130, kv_heads=2, qkv_stride=20000, q_stride=20000)):
        assert plan(append_args(**bad))[0] == B.EPARA_ERR_SHAPE, bad
    assert plan(append_args(n_positions=62, positions=D))[0] == B.EPARA_OK      # with positions of their own the table may be shorter
    for missing in ("QKV", "codes", "scales", "Q"):
        assert plan(append_args(**{missing: 0}))[0] == B.EPARA_ERR_NULL, missing
    assert plan(append_args(Q=0, rotary=0))[0] == B.EPARA_OK                    # queries may stay where they are, unrotated
    for field, at in (("QKV", 8), ("Q", 8), ("codes", 8), ("scales", 2), ("rotary", 8), ("positions", 2)):
        assert plan(append_args(**{field: D + at}))[0] == B.EPARA_ERR_ALIGN, field
    for s in BAD_SEQUENCES:
        assert plan(append_args(), [s])[0] == B.EPARA_ERR_SHAPE, s
    for page in (-1, 10):
        assert plan(append_args(), pages=[page])[0] == B.EPARA_ERR_SHAPE
    assert plan(append_args(), n_seqs=-1)[0] == B.EPARA_ERR_SHAPE
    for field in ("h_seqs", "d_seqs", "h_pages", "d_pages"):
        assert plan(append_args(), **{field: None})[0] == B.EPARA_ERR_NULL, field
    assert L.epara_plan_cache_append(None, 1, None, None) == B.EPARA_ERR_NULL
    # pages that a call does not need are not looked at: the first of three, and all of a sequence of padding
    assert plan(append_args(n_positions=300), [(0, 0, 3, 125, 0, 3)], [-1, 5, 6])[0] == B.EPARA_OK
    rc, first = plan(append_args(), [(0, 0, 3, -3, 0, 0)], [])
    assert rc == B.EPARA_OK and first[1] > 0
    assert plan(append_args(), [(0, 0, 0, 0, 0, 0)], [])[1].tolist() == [0, 0]
    # the call: running sums that are not the plan's, a page written twice, no device arguments
    assert call(append_args(), [0, 1]) == B.EPARA_ERR_SHAPE
    two = [(0, 0, 3, 60, 0, 1), (0, 3, 2, 10, 1, 1)]
    _, first = plan(append_args(), two, [4, 4])
    assert call(append_args(), first, two, [4, 4]) == B.EPARA_ERR_SHAPE
    assert call(append_args(), plan(append_args())[1], d_args=None) == B.EPARA_ERR_NULL
    none = [(0, 0, 0, 0, 0, 0)]
    assert call(append_args(), [0, 0], none, []) == B.EPARA_OK


def attn_args(**kw):
    a = np.zeros(1, dtype=B.CACHE_ATTN_ARGS)
    a[0] = (D, D + 0x100000, D + 0x200000, D + 0x300000, 8, 8, 2, 128, 10, 8 * 128, 8 * 128, 0, 0.088, 0.0, (0, 0))
    for k, v in kw.items():
        a[0][k] = v
    return a


def attn_plan(args, seqs=(SEQ,), pages=(4,), units=256, **kw):
    t, keep = table_of(list(seqs), list(pages), **kw)
    first, p = np.zeros(2 * (len(seqs) + 1), dtype=np.int32), B.CacheAttnPlan()
    rc = B.lib().epara_plan_cache_attention(args.ctypes.data, len(args), ctypes.addressof(t), units, first.ctypes.data, ctypes.addressof(p))
    return rc, first, p


def test_attention_argument_checks():
    L = B.lib()
    assert attn_plan(attn_args())[0] == B.EPARA_OK
    for bad in (dict(rows=-1), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(head_dim=32), dict(n_pages=4), dict(q_stride=1016), dict(o_stride=1028), dict(window=-1),
                dict(scale=0.0), dict(scale=-1.0), dict(scale=np.nan), dict(scale=np.inf), dict(softcap=-1.0), dict(softcap=np.nan), dict(softcap=np.inf), dict(O=D)):
        assert attn_plan(attn_args(**bad))[0] == B.EPARA_ERR_SHAPE, bad
    for missing in ("Q", "O", "codes", "scales"):
        assert attn_plan(attn_args(**{missing: 0}))[0] == B.EPARA_ERR_NULL, missing
    for field, at in (("Q", 8), ("O", 8), ("codes", 8), ("scales", 2)):
        assert attn_plan(attn_args(**{field: D + at}))[0] == B.EPARA_ERR_ALIGN, field
    for s in BAD_SEQUENCES:
        assert attn_plan(attn_args(), [s])[0] == B.EPARA_ERR_SHAPE, s
    for units in (0, -1, 1 << 20):
        assert attn_plan(attn_args(), units=units)[0] == B.EPARA_ERR_SHAPE
    assert attn_plan(attn_args(), pages=[-1])[0] == B.EPARA_ERR_SHAPE
    # a window leaves the pages behind it alone
    far = [(0, 0, 3, 200, 0, 4)]
    assert attn_plan(attn_args(), far, [-1, -1, 3, 4])[0] == B.EPARA_ERR_SHAPE
    assert attn_plan(attn_args(window=70), far, [-1, -1, 3, 4])[0] == B.EPARA_OK
    assert attn_plan(attn_args(window=74), far, [-1, -1, 3, 4])[0] == B.EPARA_ERR_SHAPE

    def call(args, seqs, pages, first, plan, workspace=D, nbytes=None, d_args=D):
        t, keep = table_of(list(seqs), list(pages))
        launch = B.CacheAttnLaunch(args.ctypes.data, d_args, first.ctypes.data, D, workspace, plan.workspace_bytes if nbytes is None else nbytes, t, plan, len(args), 0)
        return L.epara_cache_attention(ctypes.addressof(launch), None)

    args, long = attn_args(n_pages=500), [(0, 0, 1, 300 * 64 - 1, 0, 300)]
    rc, first, plan = attn_plan(args, long, range(300))
    assert rc == B.EPARA_OK and plan.workspace_bytes > 0 and first[1] == plan.n_items[0] > 2       # a long context is cut
    assert call(args, long, range(300), first, plan, workspace=None) == B.EPARA_ERR_NULL
    assert call(args, long, range(300), first, plan, workspace=D + 16) == B.EPARA_ERR_ALIGN
    assert call(args, long, range(300), first, plan, nbytes=plan.workspace_bytes - 1) == B.EPARA_ERR_CAPACITY
    assert call(args, long, range(300), first, plan, d_args=None) == B.EPARA_ERR_NULL
    assert call(args, long, range(300), first + 1, plan) == B.EPARA_ERR_SHAPE
    plan.n_items[0] += 1
    assert call(args, long, range(300), first, plan) == B.EPARA_ERR_SHAPE
    plan.part_pages[0] = 0
    assert call(args, long, range(300), first, plan) == B.EPARA_ERR_SHAPE
    assert L.epara_cache_attention(None, None) == B.EPARA_ERR_NULL
    rc, first, plan = attn_plan(attn_args(), [(0, 0, 0, 5, 0, 1)], [1])
    assert plan.n_items[0] == plan.n_items[1] == 0 and call(attn_args(), [(0, 0, 0, 5, 0, 1)], [1], first, plan) == B.EPARA_OK


@pytest.mark.parametrize("seed", range(4))
def test_attention_plans_count_the_work_of_every_sequence(seed):
    """Running sums that never fall, start at nothing and end at the number of workgroups; every sequence with rows has work in one of the two kinds and a
    multiple of its key heads; a workspace exactly where something is cut."""
    rng = np.random.default_rng([9, seed])
    seqs, at = [], 0
    for _ in range(40):
        rows, ctx = int(rng.integers(0, 4) if rng.random() < 0.6 else rng.integers(0, 700)), int(rng.integers(0, 5000))
        n = -(-(ctx + rows) // 64)
        seqs.append((0, 0, rows, ctx, at, n))
        at += n
    args = attn_args(rows=700, n_pages=at + 1, window=int(rng.integers(0, 2) * 900))
    rc, first, plan = attn_plan(args, seqs, range(at))
    assert rc == B.EPARA_OK
    few, many = first[:41], first[41:]
    assert few[0] == many[0] == 0 and few[-1] == plan.n_items[0] and many[-1] == plan.n_items[1]
    a, b = np.diff(few), np.diff(many)
    rows = np.array([s[2] for s in seqs])
    assert ((a > 0) + (b > 0) == (rows > 0)).all() and (a % 2 == 0).all() and (b % 2 == 0).all()
    spans = np.array([(s[3] + s[2] - 1) // 64 + 1 - (max(0, s[3] - 899) // 64 if args[0]["window"] else 0) for s in seqs])
    cut = any(a[i] and spans[i] > plan.part_pages[0] or b[i] and spans[i] > plan.part_pages[1] + 30 for i in range(40))
    assert (plan.workspace_bytes > 0) or not cut


def test_copy_argument_checks():
    L = B.lib()

    def call(moves=((1, 2),), G=1, d=D, **kw):
        c, m = np.zeros(G, dtype=B.PAGE_COPY), np.array(list(moves), dtype=B.PAGE_MOVE)
        for g in range(G):
            c[g] = (D, D, 10, 2, 128, 0, len(m), g * len(m) * 2)
        for k, v in kw.items():
            c[G - 1][k] = v
        return L.epara_copy_pages(c.ctypes.data, d, G, m.ctypes.data, d, len(m), None)

    assert L.epara_copy_pages(None, None, 0, None, None, 0, None) == B.EPARA_OK
    assert call(moves=()) == B.EPARA_OK
    assert L.epara_copy_pages(None, D, 1, None, None, 0, None) == B.EPARA_ERR_NULL
    for bad in ([(1, 1)], [(-1, 2)], [(1, 10)], [(10, 1)], [(1, 2), (3, 2)], [(1, 2), (2, 3)], [(2, 3), (1, 2)]):
        assert call(bad) == B.EPARA_ERR_SHAPE, bad
    for bad in (dict(n_pages=2), dict(kv_heads=0), dict(head_dim=80), dict(first_move=1), dict(n_moves=2), dict(n_moves=-1), dict(first_chunk=1), dict(G=2, first_chunk=0)):
        assert call(**bad) == B.EPARA_ERR_SHAPE, bad
    assert call(codes=0) == B.EPARA_ERR_NULL and call(scales=0) == B.EPARA_ERR_NULL and call(d=None) == B.EPARA_ERR_NULL
    assert call(codes=D + 8) == B.EPARA_ERR_ALIGN and call(scales=D + 2) == B.EPARA_ERR_ALIGN
    assert call(G=3, n_pages=2) == B.EPARA_ERR_SHAPE                     # a layer with fewer pages is looked at by itself


def pool_of(n):
    refs, free = np.zeros(n, dtype=np.int32), np.zeros(n, dtype=np.int32)
    return B.epara_page_pool_init(refs, free), refs, free


@pytest.mark.parametrize("seed", range(6))
def test_pages_follow_the_oracle_through_random_lives(seed):
    rng = np.random.default_rng([10, seed])
    n = int(rng.integers(5, 60))
    pool, refs, free = pool_of(n)
    ref, live = OD.Pages(n), []                                          # live: [pages, tokens]
    for _ in range(200):
        what = rng.random()
        if what < 0.4:
            tokens = int(rng.integers(1, 400))
            k = -(-tokens // 64)
            if k <= pool.n_free:
                got = B.epara_pages_take(pool, k).tolist()
                assert got == ref.take(k)
                live.append([got, tokens])
            else:
                with pytest.raises(B.EparaError):
                    B.epara_pages_take(pool, k)
        elif what < 0.65 and live and pool.n_free:
            pages, tokens = live[int(rng.integers(len(live)))]
            tokens = int(rng.integers(0, tokens + 1))
            child, move = B.epara_pages_fork(pool, pages, tokens)
            want, moves = ref.fork(pages, tokens)
            assert child.tolist() == want and [tuple(m) for m in move.tolist()] == moves
            live.append([want, tokens])
        elif what < 0.9 and live:
            pages, _ = live.pop(int(rng.integers(len(live))))
            B.epara_pages_free(pool, pages)
            ref.free(pages)
        else:
            flat = np.array([p for pages, _ in live for p in pages + [-1]], dtype=np.int32)
            moves = B.epara_pages_compact(pool, flat)
            want, tables = ref.compact([pages + [-1] for pages, _ in live])
            assert [tuple(m) for m in moves.tolist()] == want and flat.tolist() == [p for t in tables for p in t]
            for seq, t in zip(live, tables):
                seq[0] = t[:-1]
        assert refs.tolist() == ref.refs and free[: pool.n_free].tolist() == ref.free_pages


def test_pages_refuse_what_nobody_holds_and_change_nothing():
    pool, refs, free = pool_of(6)
    a = B.epara_pages_take(pool, 4)
    before = (refs.copy(), pool.n_free)

    def refused(f, status):
        with pytest.raises(B.EparaError) as e:
            f()
        assert e.value.status == status and np.array_equal(refs, before[0]) and pool.n_free == before[1]

    refused(lambda: B.epara_pages_take(pool, 3), B.EPARA_ERR_CAPACITY)
    refused(lambda: B.epara_pages_take(pool, -1), B.EPARA_ERR_SHAPE)
    refused(lambda: B.epara_pages_free(pool, [0, 1, 5]), B.EPARA_ERR_SHAPE)
    refused(lambda: B.epara_pages_free(pool, [0, 0]), B.EPARA_ERR_SHAPE)        # held once, named twice
    refused(lambda: B.epara_pages_free(pool, [0, 6]), B.EPARA_ERR_SHAPE)
    refused(lambda: B.epara_pages_fork(pool, [0, 5], 100), B.EPARA_ERR_SHAPE)
    refused(lambda: B.epara_pages_fork(pool, [0, 1], -1), B.EPARA_ERR_SHAPE)
    refused(lambda: B.epara_pages_compact(pool, np.array([0, 5], dtype=np.int32)), B.EPARA_ERR_SHAPE)
    with pytest.raises(ValueError):
        B.epara_pages_fork(pool, [0], 100)
    with pytest.raises(ValueError):
        B.epara_pages_compact(pool, [0, 1])
    B.epara_pages_take(pool, 2)
    before = (refs.copy(), 0)
    refused(lambda: B.epara_pages_fork(pool, a, 100), B.EPARA_ERR_CAPACITY)     # a part-filled last page needs a fresh one
    assert B.epara_pages_fork(pool, a, 128)[1].size == 0                        # whole pages do not
    L = B.lib()
    n = np.zeros(1, dtype=np.int32)
    assert L.epara_page_pool_init(None, None, None, 3) == B.EPARA_ERR_NULL
    assert L.epara_page_pool_init(ctypes.addressof(pool), refs.ctypes.data, free.ctypes.data, -1) == B.EPARA_ERR_SHAPE
    # more moves than the list holds: how many there are is still said
    B.epara_pages_free(pool, a[:2])
    B.epara_pages_free(pool, a[:2])
    t = np.array([4, 5, 2, 3], dtype=np.int32)
    move = np.zeros(1, dtype=B.PAGE_MOVE)
    assert L.epara_pages_compact(ctypes.addressof(pool), t.ctypes.data, 4, move.ctypes.data, 1, n.ctypes.data) == B.EPARA_ERR_CAPACITY
    assert n[0] == 2 and t.tolist() == [4, 5, 2, 3]


def test_cache_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    """The checks, plans and bookkeeping with their own driver under the sanitizers (host code only)."""
    exe = str(tmp_path / "sanitize_cache")
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-static-libasan", "-g", "-O1"]
    subprocess.check_call(["g++", "-std=c++17"] + san + ["-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_2511_00603_amd", "csrc"),
                           os.path.join(ROOT, "tests", "sanitize_cache.cpp"), os.path.join(ROOT, "paper_2511_00603_amd", "csrc", "epara_cache_host.cpp"), "-o", exe])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1")
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0 and "sanitize_cache: ok" in r.stdout and "runtime error" not in r.stdout, r.stdout[-4000:]


def test_rows_that_two_sequences_would_write_are_refused():
    """Two sequences of a service with a row in common would write it in a race: attention's output, and an append's queries.  Rows that are only read may be shared, in any order."""
    L = B.lib()

    def attention(seqs, pages=range(8)):
        args = attn_args(rows=20)
        rc, first, plan = attn_plan(args, seqs, pages)
        assert rc == B.EPARA_OK
        t, keep = table_of(seqs, list(pages))
        # no device arguments: a call that is not refused ends there, before it enqueues anything
        launch = B.CacheAttnLaunch(args.ctypes.data, None, first.ctypes.data, D, None, 0, t, plan, 1, 0)
        return L.epara_cache_attention(ctypes.addressof(launch), None)

    def append(seqs, **kw):
        args = append_args(rows=20, **kw)
        t, keep = table_of(seqs, list(range(8)))
        first = np.zeros(len(seqs) + 1, dtype=np.int32)
        assert L.epara_plan_cache_append(args.ctypes.data, 1, ctypes.addressof(t), first.ctypes.data) == B.EPARA_OK
        return L.epara_cache_append(args.ctypes.data, None, 1, ctypes.addressof(t), first.ctypes.data, D, None)

    seq = lambda row, rows, page: (0, row, rows, 10, page, 1)
    apart = [[seq(0, 3, 0), seq(3, 4, 1), seq(7, 1, 2)], [seq(7, 1, 2), seq(0, 3, 0), seq(3, 4, 1)], [seq(5, 0, 0), seq(3, 4, 1), seq(5, 0, 2), seq(19, 1, 3)]]
    shared = [[seq(0, 3, 0), seq(2, 4, 1)], [seq(2, 4, 0), seq(0, 3, 1)], [seq(5, 2, 0), seq(0, 20, 1)], [seq(8, 1, 0), seq(2, 1, 1), seq(8, 1, 2)]]
    for s in apart:
        assert attention(s) == B.EPARA_ERR_NULL and append(s) == B.EPARA_ERR_NULL, s
    for s in shared:
        assert attention(s) == B.EPARA_ERR_SHAPE and append(s) == B.EPARA_ERR_SHAPE, s
        assert append(s, Q=0, rotary=0) == B.EPARA_ERR_NULL, s
    # rows of two services are rows of two tensors
    args = np.concatenate([attn_args(), attn_args()])
    t, keep = table_of([(0, 0, 3, 10, 0, 1), (1, 0, 3, 10, 1, 1)], [1, 2])
    first, p = np.zeros(6, dtype=np.int32), B.CacheAttnPlan()
    assert L.epara_plan_cache_attention(args.ctypes.data, 2, ctypes.addressof(t), 256, first.ctypes.data, ctypes.addressof(p)) == B.EPARA_OK
    launch = B.CacheAttnLaunch(args.ctypes.data, None, first.ctypes.data, D, None, 0, t, p, 2, 0)
    assert L.epara_cache_attention(ctypes.addressof(launch), None) == B.EPARA_ERR_NULL


def test_copies_that_collide_in_a_cache_named_twice_are_refused():
    """A cache may come in several entries; their moves are then those of one cache: a destination twice, or a source of another entry, is a race."""
    L = B.lib()

    def call(*entries):
        """entries: (codes, moves); without device arguments a call that is not refused ends there."""
        moves, c, chunks = [m for _, own in entries for m in own], np.zeros(len(entries), dtype=B.PAGE_COPY), 0
        for i, (codes, own) in enumerate(entries):
            c[i] = (codes, codes + 0x10000, 10, 2, 128, sum(len(o) for _, o in entries[:i]), len(own), chunks)
            chunks += 2 * len(own)
        m = np.array(moves, dtype=B.PAGE_MOVE)
        return L.epara_copy_pages(c.ctypes.data, None, len(c), m.ctypes.data, None, len(m), None)

    other = D + 0x100000
    for entries in ([(D, [(1, 2)]), (D, [(3, 4)])], [(D, [(1, 2)]), (other, [(1, 2)]), (D, [(1, 5)])], [(D, []), (D, [(1, 2)]), (D, [])]):
        assert call(*entries) == B.EPARA_ERR_NULL, entries
    for second in ([(3, 2)], [(2, 3)], [(5, 1)], [(1, 2)], [(6, 7), (4, 2)]):
        assert call((D, [(1, 2)]), (D, second)) == B.EPARA_ERR_SHAPE, second
        assert call((D, second), (other, [(0, 9)]), (D, [(1, 2)])) == B.EPARA_ERR_SHAPE, second
    # the same list for a cache that is named twice, and entries that see the cache's pages differently
    c, m = np.zeros(2, dtype=B.PAGE_COPY), np.array([(1, 2)], dtype=B.PAGE_MOVE)
    for second in ((D, D, 10, 2, 128, 0, 1, 2), (D, D, 10, 4, 64, 0, 1, 2)):
        c[0], c[1] = (D, D, 10, 2, 128, 0, 1, 0), second
        assert L.epara_copy_pages(c.ctypes.data, None, 2, m.ctypes.data, None, 1, None) == B.EPARA_ERR_SHAPE


def test_sequences_whose_window_has_left_pages_behind_fork_too():
    """Entries of -1 stand for pages that were given back, for fork as for free and compact; a part-filled last page has to be there."""
    pool, refs, free = pool_of(8)
    ref = OD.Pages(8)
    pages = B.epara_pages_take(pool, 4).tolist()
    assert pages == ref.take(4)
    B.epara_pages_free(pool, pages[:2])
    ref.free(pages[:2])
    left = [-1, -1] + pages[2:]
    for tokens in (256, 250, 192, 128, 100):
        if tokens == 100:                                        # its last page, of which 36 tokens are the child's, is gone
            before = refs.copy(), pool.n_free
            with pytest.raises(B.EparaError) as e:
                B.epara_pages_fork(pool, left, tokens)
            assert e.value.status == B.EPARA_ERR_SHAPE and np.array_equal(refs, before[0]) and pool.n_free == before[1]
            continue
        child, move = B.epara_pages_fork(pool, left, tokens)
        want, moves = ref.fork(left, tokens)
        assert child.tolist() == want and [tuple(m) for m in move.tolist()] == moves and child[:2].tolist() == [-1, -1]
        assert refs.tolist() == ref.refs and free[: pool.n_free].tolist() == ref.free_pages
        B.epara_pages_free(pool, child)
        ref.free(want)
    for bad in (-2, 8, int(free[0])):
        with pytest.raises(B.EparaError):
            B.epara_pages_fork(pool, [bad] + left[1:], 256)
