"""Decoding by drafts as a program runs it: whole decoder blocks over several services whose steps mix prompts, chains and trees of drafted tokens; verification, the caches closed up, and the
steps that follow; and a step's calls captured into a graph and replayed.  Attention and caches are checked on the very tensors that the step read."""
import numpy as np
import pytest
import torch

from oracle import decoder as OD
from oracle import drafts as DR
from paper_2511_00603_amd import runtime as R
from paper_2511_00603_amd.decoder import DecoderBlock
from parity_util import TOL, assert_close
from test_gpu_drafts import run_keep, keep_case, random_tree
from workloads import make_decoder_block, make_mix

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def fetch(t):
    return t.float().cpu().numpy().astype(np.float64)


class Drafted:
    def __init__(self):
        mix = make_mix(4, d=256, ffn=704, rows=[1, 8, 20])
        self.params = make_decoder_block(mix, kv_heads=2, head_dim=64)
        self.block = DecoderBlock(mix, self.params, n_pages=24, device=DEV, max_tokens=512)
        self.caches = [OD.Cache(24, p.kv_heads, p.head_dim) for p in self.params]

    def step(self, new, parents=None):
        """The caches and the attention of a step, row by row against the oracle."""
        blk = self.block
        before = [{n: s[1] for n, s in seqs.items()} for seqs in blk.sequences]
        out = blk.step(new, parents)
        torch.cuda.synchronize()
        table = fetch(blk.rotary)
        for g, (p, items, t) in enumerate(zip(self.params, new, out)):
            H, KV, D, row = p.heads, p.kv_heads, p.head_dim, 0
            for name, X in items:
                n, start, pages = int(X.shape[0]), before[g].get(name, 0), blk.sequences[g][name][0]
                tree = list(((parents or [{}] * 9)[g] or {}).get(name, range(-1, n - 1)))
                at = np.array([start + max(len(f) - 1, 0) for f in DR.follows(tree)])
                rows = slice(row, row + n)
                qkv = fetch(t["qkv"])[rows].reshape(n, H + 2 * KV, D)
                turned = OD.rotate(qkv[:, : H + KV], table, np.repeat(at[:, None], 3, 1), (D // 2, 0, 0))
                self.caches[g].append(pages, start, turned[:, H:], qkv[:, H + KV:])
                assert_close(fetch(t["q"])[rows], turned[:, :H].reshape(n, H * D), 2.0 ** -8, "queries")
                K, V = self.caches[g].values(pages, start + n)
                want, _ = DR.attention(fetch(t["q"])[rows].reshape(n, H, D), K, V, start, tree, float(np.float32(D ** -0.5)))
                assert_close(fetch(t["o"])[rows], want.reshape(n, H * D), TOL["bf16"], "attention of %s" % (name,))
                row += n
        return out

    def accept(self, judged, temperatures):
        blk = self.block
        waiting = [dict(w) for w in blk.drafts]
        pages = [{n: list(s[0]) for n, s in seqs.items()} for seqs in blk.sequences]
        got = blk.accept(judged, temperatures)
        assert not any(blk.drafts)
        for g, (w, j) in enumerate(zip(waiting, judged)):
            row = 0
            for i, (name, (start, p)) in enumerate(w.items()):
                rows = slice(row, row + len(p))
                draft = None if j.get("draft_logits") is None else fetch(j["draft_logits"])[rows]
                path, v, _, margin = DR.verify(fetch(j["logits"])[rows], draft, j["tokens"].tolist()[rows], p, fetch(j["uniforms"])[rows], temperatures[g][i])
                assert margin > 2.0 ** -16 and got[g][name] == (path, v)
                DR.keep(self.caches[g], pages[g][name], start, len(p), path)
                now = blk.sequences[g][name]
                assert now[1] == start + len(path) and now[0] == pages[g][name][: -(-now[1] // 64)]
                row += len(p)
        for c, o, seqs in zip(blk.caches, self.caches, blk.sequences):
            for held, n in seqs.values():                        # a rotated key may fall on the other side of a rounding: one step of its code
                K, V = o.values(held, n)
                codes, scales = c.codes.cpu().numpy(), c.scales.cpu().numpy()
                lib = OD.Cache(len(codes), codes.shape[1], K.shape[2])
                t, d = np.arange(64)[:, None], np.arange(K.shape[2])[None]
                D = K.shape[2]
                key = ((((t // 4) % 4) * (D // 16) + d // 16) * 16 + 4 * (t // 16) + t % 4) * 16 + d % 16
                value = ((d // 16 * 4 + t // 16) * 16 + d % 16) * 16 + t % 16
                lib.codes[:, :, 0], lib.codes[:, :, 1] = codes[:, :, 0][:, :, key], codes[:, :, 1][:, :, value]
                lib.scales[:] = scales
                for a, b in zip(lib.values(held, n), (K, V)):
                    assert (np.abs(a - b) <= np.maximum(np.abs(b), np.abs(a)) * 2.0 ** -2.9 + 2.0 ** -9 * np.abs(b).max()).all()
                    assert (a != b).mean() < 0.01
        return got


def judge(rng, trees, vocab, drawn=False, sharp=4.0):
    n = sum(len(p) for p in trees)
    x = rng.standard_normal((n, vocab)) * sharp
    d = x + 0.5 * rng.standard_normal((n, vocab))
    tokens, row = [], 0
    for p in trees:
        rank = {}
        for i, a in enumerate(p):
            rank[a] = rank.get(a, -1) + 1
            tokens.append(int(np.argsort(-d[row + max(a, 0)])[rank[a]]))
        row += len(p)
    j = {"logits": torch.from_numpy(x.astype(np.float32)).to(DEV).bfloat16(), "tokens": torch.tensor(tokens, dtype=torch.int32, device=DEV),
         "uniforms": torch.from_numpy(rng.random(n).astype(np.float32)).to(DEV)}
    if drawn:
        j["draft_logits"] = torch.from_numpy(d.astype(np.float32)).to(DEV).bfloat16()
    return j


def test_decoder_blocks_with_drafts():
    c, rng = Drafted(), np.random.default_rng(93)
    blk = c.block
    X = lambda n: torch.from_numpy(rng.standard_normal((n, 256)).astype(np.float32)).to(DEV).bfloat16()
    tree = [-1, 0, 0, 1, 1, 2, 5, 3]
    c.step([[("a", X(60))], [("b", X(5)), ("c", X(130))], [("d", X(300))]])
    # a tree, a chain next to a prompt, nothing
    c.step([[("a", X(8))], [("b", X(4)), ("e", X(70))], []], [{"a": tree}, {"b": [-1, 0, 1, 2]}, None])
    with pytest.raises(ValueError):
        blk.step([[("a", X(1))], [], []])
    with pytest.raises(ValueError):
        blk.fork(0, "a", "a2")
    assert blk.sequences[0]["a"][1] == 60 and blk.sequences[1]["b"][1] == 5 and blk.sequences[1]["e"][1] == 70
    for bad in ([None, None, None], [judge(rng, [tree], 99), None, None], [judge(rng, [tree[:3]], 99), judge(rng, [[-1, 0, 1, 2]], 99), None]):
        with pytest.raises(ValueError):
            blk.accept(bad, [[1.0], [0.0], []])
    judged = [judge(rng, [tree], 99), judge(rng, [[-1, 0, 1, 2]], 50), None]
    c.accept(judged, [[0.8], [0.0], []])
    # and on: one token, then trees of several sequences and a service at once, drawn ones in another call
    c.step([[("a", X(1))], [("b", X(1))], [("d", X(1))]])
    trees = [random_tree(rng, 40), random_tree(rng, 9)]
    c.step([[("a", X(3))], [("b", X(40)), ("c", X(9))], []], [None, {"b": trees[0], "c": trees[1]}, None])
    c.accept([None, judge(rng, trees, 700), None], [[], [1.1, 0.0], []])
    chains = [[-1, 0, 1, 2, 3]] * 2
    c.step([[], [("c", X(5)), ("b", X(5))], [("d", X(5))]], [None, {"c": chains[0], "b": chains[1]}, {"d": chains[0]}])
    c.accept([None, judge(rng, chains, 321, True), judge(rng, chains[:1], 64, True, 9.0)], [[], [0.7, 1.0], [0.5]])
    c.step([[("a", X(2))], [("b", X(1)), ("c", X(1))], [("d", X(1))]])
    for g, names in enumerate((["a"], ["b", "c", "e"], ["d"])):
        for n in names:
            blk.release(g, n)
        assert blk.pools[g].n_free == 24


def test_a_captured_step_of_drafts_replays_as_it_ran():
    """Trees, append, attention, verification and keeping in one graph, on another stream than the current one; inputs change between the replays, with eager work in between."""
    rng = np.random.default_rng(94)
    n_seqs, rows, H, KV, D, vocab, starts = 3, 12, 4, 2, 64, 5003, [100, 31, 5000]
    pages, at = [], 0
    for s in starts:
        k = -(-(s + rows) // 64)
        pages.append(list(range(at, at + k)))
        at += k
    gen = torch.Generator(device=DEV)
    gen.manual_seed(7)
    randn = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    cache = R.PagedCache(torch.randint(0, 0x60, (at, KV, 2, 64 * D), generator=gen, device=DEV, dtype=torch.uint8), torch.full((at, KV, 2, 2), 120, dtype=torch.uint8, device=DEV))
    start_codes, start_scales = cache.codes.clone(), cache.scales.clone()
    n = n_seqs * rows
    QKV, Q, O = randn(n, (H + 2 * KV) * D).bfloat16(), torch.empty(n, H * D, dtype=torch.bfloat16, device=DEV), torch.empty(n, H * D, dtype=torch.bfloat16, device=DEV)
    parents = torch.tensor(sum((random_tree(rng, rows) for _ in starts), []), dtype=torch.int32, device=DEV)
    logits, tokens, uniforms = randn(n, vocab).bfloat16() * 3, torch.randint(0, vocab, (n,), generator=gen, device=DEV, dtype=torch.int32), torch.rand(n, generator=gen, device=DEV)
    rotary = randn(6000, D // 2, 2)
    table = R.SequenceTable([[{"first_row": i * rows, "rows": rows, "start": s, "pages": p} for i, (s, p) in enumerate(zip(starts, pages))]], DEV)
    trees = R.DraftTreePlan(table, [{"parents": parents}], DEV)
    t = trees.groups[0]
    append = R.CacheAppendPlan(table, [{"QKV": QKV, "Q": Q, "cache": cache, "heads": H, "rotary": rotary, "positions": t["positions"]}], DEV)
    attend = R.TreeAttnPlan(table, [{"Q": Q, "O": O, "cache": cache, "heads": H, "visible": t["visible"]}], DEV)
    verify = R.VerifyPlan(table, [{"logits": logits, "tokens": tokens, "uniforms": uniforms, "parents": parents}], DEV, temperatures=torch.tensor([0.9, 0.0, 0.6], device=DEV))
    keep = R.CacheKeepPlan(table, [{"service": 0, "cache": cache, "path": verify.groups[0]["path"]}], DEV, verify.kept)
    assert attend.plan.workspace_bytes > 0

    def step():
        R.draft_trees(trees)
        R.cache_append(append)
        R.tree_attention(attend)
        R.verify_drafts(verify)
        R.cache_keep(keep)

    def reset():
        cache.codes.copy_(start_codes)
        cache.scales.copy_(start_scales)
        O.fill_(float("nan"))
        for x in (verify.kept, verify.next, verify.groups[0]["path"]):
            x.fill_(-9)
        verify.groups[0]["probs"].fill_(-9)

    def results():
        torch.cuda.synchronize()
        return [x.clone() for x in (cache.codes, cache.scales, O.view(torch.int16), verify.kept, verify.next, verify.groups[0]["path"], verify.groups[0]["probs"], t["visible"], t["positions"])]

    reset()
    step()
    want = results()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    reset()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    for k in range(4):
        reset()
        torch.cuda.synchronize()
        graph.replay()
        for a, b in zip(results(), want):
            assert torch.equal(a, b)
        # other drafts: of the same sizes, some of them not there
        parents.copy_(torch.tensor(sum((random_tree(rng, rows, 1, 0.1 * k) for _ in starts), []), dtype=torch.int32, device=DEV))
        tokens.copy_(logits.float().argmax(dim=1)[torch.arange(n, device=DEV) // rows * rows + parents.clamp(0, rows - 1)].int())
        uniforms.copy_(torch.rand(n, generator=gen, device=DEV))
        QKV.mul_(0.7)
        reset()
        step()
        want = results()
    assert max(want[3].tolist()) > 1


def test_keeping_with_caches_of_many_layers_and_services():
    rng = np.random.default_rng(95)
    services = []
    for g in range(5):
        n = int(rng.integers(0, 4))
        starts, rows = rng.integers(0, 150, n).tolist(), rng.integers(1, 40, n).tolist()
        paths = [sorted(rng.choice(r, int(rng.integers(1, r + 1)), replace=False).tolist()) for r in rows]
        services.append(([keep_case(rng, starts, rows, 1 + g, 64 if g % 2 else 128) for _ in range(15)], starts, rows, paths, [len(p) for p in paths]))
    run_keep(services)
