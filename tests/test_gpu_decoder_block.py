"""A decoder block run as a program would: prompts, single tokens, a fork, a release and a compaction over several services, every stage of every step
against the oracle on the very tensors that the stage read on the GPU."""
import numpy as np
import pytest
import torch

from oracle import decoder as OD
from oracle import reference as ref
from paper_2511_00603_amd import binding as B
from paper_2511_00603_amd.decoder import DecoderBlock
from parity_util import TOL, assert_close
from workloads import make_decoder_block, make_mix

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def fetch(t):
    return t.float().cpu().numpy().astype(np.float64)


class Checked:
    def __init__(self, mix, ffn):
        self.params = make_decoder_block(mix, kv_heads=2, head_dim=64)
        s_h = [0.02] * len(self.params)
        self.block = DecoderBlock(mix, self.params, n_pages=24, device=DEV, ffn=ffn, s_x=0.012, s_h=s_h, max_tokens=512)
        self.ffn, self.s_h = ffn, s_h
        self.caches = [OD.Cache(24, p.kv_heads, p.head_dim) for p in self.params]

    def step(self, new):
        blk = self.block
        before = [{n: s[1] for n, s in seqs.items()} for seqs in blk.sequences]
        out = blk.step(new)
        torch.cuda.synchronize()
        table = fetch(blk.rotary)
        for g, (p, items, t) in enumerate(zip(self.params, new, out)):
            if not items:
                continue
            H, KV, D = p.heads, p.kv_heads, p.head_dim
            bits, scale = blk.bits[g]
            w = {n: ref.bf16_decode(b) if b.dtype == np.uint16 else ref.e4m3_decode(b, scale[n]) for n, b in bits.items()}
            eps, x = float(np.float32(p.eps)), fetch(t["x"])
            g64 = lambda a: a.astype(np.float64)
            got = {n: fetch(v) for n, v in t.items() if v.dtype == torch.bfloat16}
            assert_close(got["y1"], OD.add_rms_norm(x, None, g64(p.gamma1), eps)[1], 2.0 ** -8, "first norm")
            assert_close(got["qkv"], ref.dense_forward(got["y1"], w["qkv"], None, "none"), TOL["bf16"], "QKV")
            row = 0
            for name, X in items:
                n, start, pages = int(X.shape[0]), before[g].get(name, 0), blk.sequences[g][name][0]
                rows = slice(row, row + n)
                qkv = got["qkv"][rows].reshape(n, H + 2 * KV, D)
                turned = OD.rotate(qkv[:, : H + KV], table, np.repeat(np.arange(start, start + n)[:, None], 3, 1), (D // 2, 0, 0))
                self.caches[g].append(pages, start, turned[:, H:], qkv[:, H + KV:])
                assert_close(got["q"][rows], turned[:, :H].reshape(n, H * D), 2.0 ** -8, "queries")
                K, V = self.caches[g].values(pages, start + n)
                want, _ = OD.attention(got["q"][rows].reshape(n, H, D), K, V, start, float(np.float32(D ** -0.5)))
                assert_close(got["o"][rows], want.reshape(n, H * D), TOL["bf16"], "attention of %s" % (name,))
                row += n
            assert_close(got["proj"], ref.dense_forward(got["o"], w["proj"], None, "none"), TOL["bf16"], "projection")
            s2, y2 = OD.add_rms_norm(x, got["proj"], g64(p.gamma2), eps)
            assert_close(got["s2"], s2, 2.0 ** -8, "sum after attention")
            if self.ffn == "fp8":
                codes, s_x = t["y2"].cpu().numpy(), float(np.float32(blk.s_x))
                read = OD.e4m3_decode(codes) * s_x
                limit = np.clip(y2, -448 * s_x, 448 * s_x)
                assert (np.abs(read - limit) <= np.maximum(np.abs(limit) * 2.0 ** -4, s_x * 2.0 ** -10) * 1.0001).all()
            else:
                read = got["y2"]
                assert_close(read, y2, 2.0 ** -8, "second norm")
            a, u = ref.dense_forward(read, w["gate"], None, "none"), ref.dense_forward(read, w["up"], None, "none")
            h = a / (1 + np.exp(-a)) * u
            if self.ffn == "fp8":                            # the codes of H that the GPU wrote are what its second product reads
                h = OD.e4m3_decode(t["h"].cpu().numpy()) * float(np.float32(self.s_h[g]))
            assert_close(got["f"], ref.dense_forward(h, w["down"], None, "none"), TOL[self.ffn], "FFN")
            s3, y3 = OD.add_rms_norm(got["s2"], got["f"], g64(p.gamma1), eps)
            assert_close(got["s3"], s3, 2.0 ** -8, "block output")
            assert_close(got["y3"], y3, 2.0 ** -8, "block output, normalised")
        return out


@pytest.mark.parametrize("ffn", ["bf16", "fp8"])
def test_decoder_block_with_prompts_tokens_forks_and_compaction(ffn):
    mix = make_mix(4, d=256, ffn=704, rows=[1, 8, 20])
    c = Checked(mix, ffn)
    blk, rng = c.block, np.random.default_rng(91)
    X = lambda n: torch.from_numpy(rng.standard_normal((n, 256)).astype(np.float32)).to(DEV).bfloat16()
    c.step([[("a", X(70))], [("b", X(5)), ("c", X(130))], []])                                    # prompts; a service without work
    c.step([[("a", X(1))], [("c", X(1)), ("b", X(1))], [("d", X(64)), ("e", X(3))]])              # tokens next to prompts
    blk.fork(1, "c", "c2")                                                                        # two whole pages shared, the third copied
    pages, own = blk.sequences[1]["c"][0], blk.sequences[1]["c2"][0]
    assert pages[:2] == own[:2] and pages[2] != own[2]
    c.caches[1].codes[own[2]], c.caches[1].scales[own[2]] = c.caches[1].codes[pages[2]], c.caches[1].scales[pages[2]]
    c.step([[("a", X(1))], [("c", X(2)), ("c2", X(1))], [("e", X(62))]])                          # both go their own way
    blk.release(1, "b")
    blk.release(2, "d")
    for g in (1, 2):
        old = {n: list(s[0]) for n, s in blk.sequences[g].items()}
        codes, scales = c.caches[g].codes.copy(), c.caches[g].scales.copy()
        assert blk.compact(g) > 0
        for n, s in blk.sequences[g].items():
            for src, dst in zip(old[n], s[0]):
                c.caches[g].codes[dst], c.caches[g].scales[dst] = codes[src], scales[src]
        assert max(p for s in blk.sequences[g].values() for p in s[0]) < 24 - blk.pools[g].n_free
    c.step([[], [("c2", X(1)), ("c", X(1))], [("e", X(1))]])
    for g, names in enumerate((["a"], ["c", "c2"], ["e"])):
        for n in names:
            blk.release(g, n)
        assert blk.pools[g].n_free == 24
