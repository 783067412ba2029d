"""CPU-side checks of decoding by drafts: layouts of the structs, refusals (every call looks at the host copies of its arguments before anything is enqueued, so each case here
returns before a launch), and plans."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2511_00603_amd import binding as B
from test_cache_abi import BAD_SEQUENCES, D, attn_args, table_of

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SEQ = (0, 0, 3, 60, 0, 1)


def test_struct_sizes_match_the_header():
    assert [t.itemsize for t in (B.TREE_ARGS, B.VERIFY_ARGS, B.KEEP_ARGS)] == [32, 72, 56]
    assert [ctypes.sizeof(t) for t in (B.TreeAttnPlan, B.TreeAttnLaunch, B.VerifyPlan, B.VerifyLaunch)] == [40, 152, 24, 144]


def tree_args(**kw):
    a = np.zeros(1, dtype=B.TREE_ARGS)
    a[0] = (D, D + 0x1000, D + 0x2000, 8, 0)
    for k, v in kw.items():
        a[0][k] = v
    return a


def test_tree_argument_checks():
    L = B.lib()

    def call(args, seqs=(SEQ,), pages=(4,), d_args=None, **kw):
        t, keep = table_of(list(seqs), list(pages), **kw)
        return L.epara_draft_trees(args.ctypes.data, d_args, len(args), ctypes.addressof(t), None)

    assert call(tree_args()) == B.EPARA_ERR_NULL                # all is well but for the device's copy
    assert call(tree_args(), [], []) == B.EPARA_OK              # no sequences: nothing to enqueue
    assert call(tree_args(rows=-1)) == B.EPARA_ERR_SHAPE
    for s in BAD_SEQUENCES:
        assert call(tree_args(), [s]) == B.EPARA_ERR_SHAPE, s
    assert call(tree_args(), [(0, 0, 3, -1, 0, 1)]) == B.EPARA_ERR_SHAPE                 # a tree in front of position 0
    assert call(tree_args(rows=400), [(0, 0, 300, -10, 0, 5)], range(5)) == B.EPARA_ERR_NULL      # what is no tree may be padded
    assert call(tree_args(), [SEQ, (0, 2, 3, 0, 0, 1)]) == B.EPARA_ERR_SHAPE             # a row of two sequences
    for missing in ("parents", "visible"):
        assert call(tree_args(**{missing: 0})) == B.EPARA_ERR_NULL
    assert call(tree_args(positions=0)) == B.EPARA_ERR_NULL     # (positions may be left out: the device's copy is what is missing)
    for field, at in (("parents", 2), ("visible", 8), ("positions", 2)):
        assert call(tree_args(**{field: D + at})) == B.EPARA_ERR_ALIGN
    assert L.epara_draft_trees(None, None, 1, None, None) == B.EPARA_ERR_NULL and L.epara_draft_trees(None, None, -1, None, None) == B.EPARA_ERR_SHAPE
    assert call(tree_args(), d_seqs=None) == B.EPARA_ERR_NULL


def tree_plan(args, trees, seqs=(SEQ,), pages=(4,), units=256, **kw):
    t, keep = table_of(list(seqs), list(pages), **kw)
    first, p = np.zeros(3 * (len(seqs) + 1), dtype=np.int32), B.TreeAttnPlan()
    rc = B.lib().epara_plan_tree_attention(args.ctypes.data, trees.ctypes.data, len(args), ctypes.addressof(t), units, first.ctypes.data, ctypes.addressof(p))
    return rc, first, p


def test_tree_attention_argument_checks():
    L = B.lib()
    assert tree_plan(attn_args(), tree_args())[0] == B.EPARA_OK
    for bad in (dict(rows=-1), dict(kv_heads=3), dict(head_dim=32), dict(q_stride=1016), dict(window=-1), dict(scale=0.0), dict(softcap=np.nan), dict(O=D)):
        assert tree_plan(attn_args(**bad), tree_args())[0] == B.EPARA_ERR_SHAPE, bad
    for s in BAD_SEQUENCES:
        assert tree_plan(attn_args(), tree_args(), [s])[0] == B.EPARA_ERR_SHAPE, s
    # of trees alone: before position 0, more rows than a window, bits of another number of rows, bits that are not aligned
    assert tree_plan(attn_args(), tree_args(), [(0, 0, 3, -1, 0, 1)])[0] == B.EPARA_ERR_SHAPE
    assert tree_plan(attn_args(window=2), tree_args())[0] == B.EPARA_ERR_SHAPE and tree_plan(attn_args(window=3), tree_args())[0] == B.EPARA_OK
    assert tree_plan(attn_args(), tree_args(rows=7))[0] == B.EPARA_ERR_SHAPE and tree_plan(attn_args(), tree_args(visible=D + 8))[0] == B.EPARA_ERR_ALIGN
    # a service without bits is causal
    none = tree_args(visible=0, rows=0)
    assert tree_plan(attn_args(window=2), none)[0] == B.EPARA_OK and tree_plan(attn_args(), none, [(0, 0, 3, -1, 0, 1)])[0] == B.EPARA_OK
    assert L.epara_plan_tree_attention(attn_args().ctypes.data, None, 1, None, 256, None, None) == B.EPARA_ERR_NULL
    # a window reaches back from the tree's first row, whose page has to be there
    far = [(0, 0, 8, 200, 0, 4)]
    assert tree_plan(attn_args(window=73), tree_args(), far, [-1, -1, 3, 4])[0] == B.EPARA_OK
    assert tree_plan(attn_args(window=74), tree_args(), far, [-1, -1, 3, 4])[0] == B.EPARA_ERR_SHAPE

    def call(args, trees, seqs, pages, first, plan, workspace=D, nbytes=None, d_args=D, d_trees=None):
        t, keep = table_of(list(seqs), list(pages))
        l = B.TreeAttnLaunch(args.ctypes.data, d_args, trees.ctypes.data, d_trees, first.ctypes.data, D, workspace, plan.workspace_bytes if nbytes is None else nbytes, t, plan, len(args), 0)
        return L.epara_tree_attention(ctypes.addressof(l), None)

    args, trees, long = attn_args(n_pages=500), tree_args(), [(0, 0, 8, 299 * 64, 0, 300)]
    rc, first, plan = tree_plan(args, trees, long, range(300))
    assert rc == B.EPARA_OK and plan.workspace_bytes > 0 and sum(plan.n_items) > 2
    assert call(args, trees, long, range(300), first, plan) == B.EPARA_ERR_NULL
    assert call(args, trees, long, range(300), first, plan, workspace=None) == B.EPARA_ERR_NULL
    assert call(args, trees, long, range(300), first, plan, workspace=D + 16) == B.EPARA_ERR_ALIGN
    assert call(args, trees, long, range(300), first, plan, nbytes=plan.workspace_bytes - 1) == B.EPARA_ERR_CAPACITY
    assert call(args, trees, long, range(300), first + 1, plan) == B.EPARA_ERR_SHAPE
    for field in ("n_items", "part_pages"):
        other = type(plan).from_buffer_copy(plan)
        getattr(other, field)[0] = 0 if field == "part_pages" else plan.n_items[0] + 1
        assert call(args, trees, long, range(300), first, other) == B.EPARA_ERR_SHAPE
    assert L.epara_tree_attention(None, None) == B.EPARA_ERR_NULL
    assert tree_plan(attn_args(), tree_args(), units=0)[0] == B.EPARA_ERR_SHAPE


@pytest.mark.parametrize("seed", range(4))
def test_tree_attention_plans_count_the_work_of_every_sequence(seed):
    rng = np.random.default_rng([9, seed])
    seqs, at = [], 0
    for _ in range(40):
        rows, ctx = int(rng.integers(0, 40) if rng.random() < 0.7 else rng.integers(0, 700)), int(rng.integers(0, 5000))
        n = -(-(ctx + rows) // 64)
        seqs.append((0, 0, rows, ctx, at, n))
        at += n
    args = attn_args(rows=700, n_pages=at + 1, window=int(rng.integers(0, 2) * 900))
    rc, first, plan = tree_plan(args, tree_args(rows=700), seqs, range(at))
    assert rc == B.EPARA_OK
    kinds = np.diff(first.reshape(3, 41), axis=1)
    rows = np.array([s[2] for s in seqs])
    assert (kinds >= 0).all() and (first.reshape(3, 41)[:, 0] == 0).all() and first.reshape(3, 41)[:, -1].tolist() == list(plan.n_items)
    assert ((kinds > 0).sum(axis=0) == (rows > 0)).all() and (kinds % 2 == 0).all()      # one kind each, whole key heads
    assert (plan.workspace_bytes > 0) == any((kinds[k] > 2 * -(-rows * 4 // (32 if k < 2 else 128))).any() for k in range(3))


def verify_args(**kw):
    a = np.zeros(1, dtype=B.VERIFY_ARGS)
    a[0] = (D, 0, D + 0x100, D + 0x200, D + 0x300, D + 0x400, D + 0x500, 8, 1000, 1000, 0)
    for k, v in kw.items():
        a[0][k] = v
    return a


def test_verify_argument_checks():
    L = B.lib()

    def plan(args, seqs=(SEQ,), dtype=B.EPARA_BF16, units=256, **kw):
        t, keep = table_of(list(seqs), [], **kw)
        first, p = np.zeros(len(seqs) + 1, dtype=np.int32), B.VerifyPlan()
        return L.epara_plan_verify_drafts(args.ctypes.data, len(args), ctypes.addressof(t), dtype, units, first.ctypes.data, ctypes.addressof(p)), first, p

    assert plan(verify_args())[0] == B.EPARA_OK and plan(verify_args(), dtype=B.EPARA_F32)[0] == B.EPARA_OK
    assert plan(verify_args(), dtype=B.EPARA_FP8_E4M3)[0] == B.EPARA_ERR_DTYPE
    for bad in (dict(rows=-1), dict(vocab=0), dict(vocab=-3), dict(stride=999), dict(vocab=1 << 29, stride=1 << 29), dict(draft_logits=D, draft_stride=999)):
        assert plan(verify_args(**bad))[0] == B.EPARA_ERR_SHAPE, bad
    for s in ((1, 0, 3, 0, 0, 0), (-1, 0, 3, 0, 0, 0), (0, -1, 3, 0, 0, 0), (0, 6, 3, 0, 0, 0), (0, 0, -1, 0, 0, 0)):
        assert plan(verify_args(), [s])[0] == B.EPARA_ERR_SHAPE, s
    assert plan(verify_args(rows=300), [(0, 0, 257, 0, 0, 0)])[0] == B.EPARA_ERR_SHAPE and plan(verify_args(rows=300), [(0, 0, 256, 0, 0, 0)])[0] == B.EPARA_OK
    assert plan(verify_args(), [(0, 0, 3, -99, 7, -5)])[0] == B.EPARA_OK                 # places and pages are not looked at
    for missing in ("logits", "tokens", "uniforms", "path"):
        assert plan(verify_args(**{missing: 0}))[0] == B.EPARA_ERR_NULL, missing
    assert plan(verify_args(parents=0, probs=0))[0] == B.EPARA_OK
    for field in ("tokens", "parents", "uniforms", "path", "probs"):
        assert plan(verify_args(**{field: D + 2}))[0] == B.EPARA_ERR_ALIGN, field
    assert plan(verify_args(logits=D + 1))[0] == B.EPARA_ERR_ALIGN and plan(verify_args(logits=D + 2))[0] == B.EPARA_OK
    assert plan(verify_args(logits=D + 2), dtype=B.EPARA_F32)[0] == B.EPARA_ERR_ALIGN
    assert plan(verify_args(), units=0)[0] == B.EPARA_ERR_SHAPE and plan(verify_args(), d_seqs=None)[0] == B.EPARA_ERR_NULL

    def call(args, first, p, seqs=(SEQ,), **kw):
        t, keep = table_of(list(seqs), [])
        l = B.VerifyLaunch(args.ctypes.data, None, first.ctypes.data, D, D, D, D, D, p.workspace_bytes, t, p, len(args), B.EPARA_BF16)
        for k, v in kw.items():
            setattr(l, k, v)
        return L.epara_verify_drafts(ctypes.addressof(l), None)

    rc, first, p = plan(verify_args())
    assert call(verify_args(), first, p) == B.EPARA_ERR_NULL                             # no device arguments
    for missing in ("h_first", "d_kept", "d_next", "d_workspace"):
        assert call(verify_args(), first, p, d_args=D, **{missing: None}) == B.EPARA_ERR_NULL, missing
    assert call(verify_args(), first, p, d_workspace=D + 64) == B.EPARA_ERR_ALIGN and call(verify_args(), first, p, d_kept=D + 2) == B.EPARA_ERR_ALIGN
    assert call(verify_args(), first, p, workspace_bytes=p.workspace_bytes - 1) == B.EPARA_ERR_CAPACITY
    assert call(verify_args(), first + 1, p) == B.EPARA_ERR_SHAPE
    for field in ("n_items", "pieces", "draw_chunks", "draw_pieces"):
        other = type(p).from_buffer_copy(p)
        setattr(other, field, 5)
        assert call(verify_args(), first, other) == B.EPARA_ERR_SHAPE, field
    two = [SEQ, (0, 2, 3, 0, 0, 0)]
    rc, first, p = plan(verify_args(), two)
    assert call(verify_args(), first, p, two) == B.EPARA_ERR_SHAPE                       # a row of two sequences
    assert L.epara_verify_drafts(None, None) == B.EPARA_ERR_NULL
    rc, first, p = plan(verify_args(), [])
    assert call(verify_args(), first, p, []) == B.EPARA_OK


def keep_args(**kw):
    a = np.zeros(1, dtype=B.KEEP_ARGS)
    a[0] = (D, D + 0x1000, D + 0x2000, 0, 0, 8, 10, 2, 128, 0, 0)
    for k, v in kw.items():
        a[0][k] = v
    return a


def test_keep_argument_checks():
    L = B.lib()

    def call(args, seqs=(SEQ,), pages=(4,), d_caches=None, kept=D, **kw):
        t, keep = table_of(list(seqs), list(pages), **kw)
        return L.epara_cache_keep(args.ctypes.data, d_caches, len(args), ctypes.addressof(t), kept, None)

    assert call(keep_args()) == B.EPARA_ERR_NULL and call(keep_args(), d_caches=D, kept=None) == B.EPARA_ERR_NULL
    assert call(keep_args(), d_caches=D, kept=D + 2) == B.EPARA_ERR_ALIGN
    assert call(keep_args(), [], []) == B.EPARA_OK
    for bad in (dict(service=-1), dict(first_seq=1), dict(first_item=1), dict(rows=2), dict(rows=-1), dict(n_pages=4), dict(n_pages=-1), dict(kv_heads=0), dict(head_dim=96), dict(service=1)):
        assert call(keep_args(**bad)) == B.EPARA_ERR_SHAPE, bad
    for missing in ("codes", "scales", "path"):
        assert call(keep_args(**{missing: 0})) == B.EPARA_ERR_NULL, missing
    for field, at in (("codes", 8), ("scales", 2), ("path", 2)):
        assert call(keep_args(**{field: D + at})) == B.EPARA_ERR_ALIGN, field
    for s in ((0, -1, 3, 60, 0, 1), (0, 0, -1, 60, 0, 1), (0, 0, 3, 62, 0, 1), (0, 0, 3, 60, 1, 1), (0, 0, 3, -1, 0, 1), (0, 6, 3, 60, 0, 1)):
        assert call(keep_args(), [s]) == B.EPARA_ERR_SHAPE, s
    assert call(keep_args(), pages=[-1]) == B.EPARA_ERR_SHAPE
    two = [SEQ, (0, 3, 3, 0, 1, 1)]
    assert call(keep_args(), two, [4, 4]) == B.EPARA_ERR_SHAPE and call(keep_args(), two, [4, 5]) == B.EPARA_ERR_NULL      # a page of two sequences
    both = np.concatenate([keep_args(), keep_args(first_item=2)])
    assert call(both) == B.EPARA_ERR_SHAPE                                               # a cache twice
    both[1]["codes"] = D + 0x100000
    assert call(both) == B.EPARA_ERR_NULL
    # pages in front of the drafts are not looked at, and a long sequence's are not either
    assert call(keep_args(), [(0, 0, 3, 130, 0, 3)], [-1, -1, 5]) == B.EPARA_ERR_NULL
    assert call(keep_args(rows=300), [(0, 0, 300, 0, 0, 5)], [-1] * 5) == B.EPARA_ERR_NULL
    assert L.epara_cache_keep(None, None, 1, None, None, None) == B.EPARA_ERR_NULL and L.epara_cache_keep(None, None, -1, None, None, None) == B.EPARA_ERR_SHAPE


def test_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    exe, csrc = str(tmp_path / "sanitize_drafts"), os.path.join(ROOT, "paper_2511_00603_amd", "csrc")
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-static-libasan", "-g", "-O1"]
    subprocess.check_call(["g++", "-std=c++17"] + san + ["-I" + os.path.join(ROOT, "include"), "-I" + csrc, os.path.join(ROOT, "tests", "sanitize_drafts.cpp"),
                           os.path.join(csrc, "epara_cache_host.cpp"), os.path.join(csrc, "epara_drafts_host.cpp"), "-o", exe])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1")
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0 and "sanitize_drafts: ok" in r.stdout, r.stdout[-4000:]
