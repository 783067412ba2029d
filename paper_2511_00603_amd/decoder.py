"""Runs the SwiGLU services of a decode or prefill mix as whole pre-norm decoder blocks over paged 8-bit caches:

    y1 = RMS(x) -> QKV -> rotary positions, keys and values join the cache -> attention over the cache -> projection
    -> s2 = x + proj, y2 = RMS(s2) -> SwiGLU FFN -> s3 = s2 + ffn, y3 = RMS(s3)      (the sum that enters the next block, normalised for it)

Every service has its own weights, cache and sequences; a step takes new tokens for any of them, prompts and single tokens alike, through
ten launches.  With an fp8 FFN the second normalisation writes E4M3 codes with the service's static scale, which the gated forward reads.
Sequences may be forked (whole pages are shared, a part-filled one is copied), released, and their pages compacted."""
import numpy as np
import torch

from workloads import casts

from . import binding as B
from . import runtime as R


class DecoderBlock:
    def __init__(self, mix, params, n_pages, device="cuda:0", ffn="bf16", s_x=0.02, s_h=None, rotary_base=10000.0, max_tokens=4096):
        self.device, self.params, self.ffn = torch.device(device), params, B.DTYPE_BY_NAME[ffn]
        self.s_x, self.s_h = (s_x, s_h or [1.0] * len(params)) if ffn == "fp8" else (1.0, [1.0] * len(params))
        dev, bf, fp8 = self.device, B.EPARA_BF16, ffn == "fp8"
        f32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(dev)
        self.bits, self.weights, self.caches, self.pools, self.sequences = [], [], [], [], []
        for svc, p in zip(mix.services, params):
            bits = {"qkv": casts.bf16_bits(p.Wqkv), "proj": casts.bf16_bits(p.Wproj)}
            scale = {"qkv": 1.0, "proj": 1.0}
            for name, W in (("gate", svc.Wgate), ("up", svc.Wup), ("down", svc.Wdown)):
                scale[name] = casts.e4m3_scale(W) if fp8 else 1.0
                bits[name] = casts.e4m3_codes(W, scale[name]) if fp8 else casts.bf16_bits(W)
            kind = lambda n: self.ffn if n in ("gate", "up", "down") else bf
            self.bits.append((bits, scale))
            self.weights.append({n: (R.pack_weights(R.device_tensor_from_bits(w, kind(n), dev), kind(n)), w.shape) for n, w in bits.items()})
            self.caches.append(R.PagedCache.empty(n_pages, p.kv_heads, p.head_dim, dev))
            self.pools.append(R.PagePool(n_pages))
            self.sequences.append({})                            # name -> [pages, tokens]
        self.gammas = [(f32(p.gamma1), f32(p.gamma2)) for p in params]
        D = max(p.head_dim for p in params)
        if any(p.head_dim != D for p in params):
            raise ValueError("one rotary table: the services' heads have to be of one size")
        angle = np.arange(max_tokens)[:, None] * rotary_base ** (-np.arange(D // 2) * 2.0 / D)[None]
        self.rotary = f32(np.stack([np.cos(angle), np.sin(angle)], axis=-1))

    # ---- sequences
    def fork(self, service, name, child):
        pages, tokens = self.sequences[service][name]
        if child in self.sequences[service]:
            raise ValueError("sequence %r exists" % (child,))
        own, moves = self.pools[service].fork(pages, tokens)
        try:
            self._copy(service, moves)
        except BaseException:
            self.pools[service].free(own)
            raise
        self.sequences[service][child] = [own.tolist(), tokens]

    def release(self, service, name):
        self.pools[service].free(self.sequences[service].pop(name)[0])

    def compact(self, service):
        """-> how many pages moved."""
        seqs, pool, at = self.sequences[service], self.pools[service], 0
        table = np.array([p for pages, _ in seqs.values() for p in pages], dtype=np.int32)
        before = pool.state()
        moves = pool.compact(table)
        try:
            self._copy(service, moves)
        except BaseException:
            pool.restore(before)
            raise
        for s in seqs.values():
            s[0] = table[at: at + len(s[0])].tolist()
            at += len(s[0])
        return len(moves)

    def _copy(self, service, moves):
        if len(moves):
            R.copy_pages(R.PageCopyPlan([{"cache": self.caches[service], "moves": moves}], self.device))

    # ---- one step
    def step(self, new):
        """new: per service a list of (sequence name, X [tokens, d] bf16 on the GPU) -> per service a dict of the step's tensors, rows in the order of the list.  A name that
        is not known yet begins a sequence.  A step that raises leaves all sequences and pages as they were: EparaError (ERR_CAPACITY) where a service has too few
        free pages, ValueError for a name twice, tokens of another shape, or more positions than the table of angles has."""
        work = self._admit(new)
        try:
            tensors = self._launch(new, work)
        except BaseException:
            self._give_back(work)
            raise
        self._commit(work)
        return tensors

    def _admit(self, new):
        """-> per service a list of (name, position of the first new token, tokens, pages with the new ones, the new ones): checked, and the pages taken; no sequence is
        changed yet."""
        if len(new) != len(self.params):
            raise ValueError("%d services, tokens for %d" % (len(self.params), len(new)))
        work, limit = [], int(self.rotary.shape[0])
        for g, (items, p) in enumerate(zip(new, self.params)):
            if len({name for name, _ in items}) != len(items):
                raise ValueError("a sequence is named twice in one step")
            for name, X in items:
                if X.dim() != 2 or X.shape[1] != p.Wqkv.shape[0] or X.dtype != torch.bfloat16:
                    raise ValueError("sequence %r: tokens are bfloat16 [n, %d]" % (name, p.Wqkv.shape[0]))
                if self.sequences[g].get(name, [[], 0])[1] + int(X.shape[0]) > limit:
                    raise ValueError("sequence %r: more than %d positions" % (name, limit))
        try:
            for g, items in enumerate(new):
                work.append([])
                for name, X in items:
                    pages, start = self.sequences[g].get(name, [[], 0])
                    n = int(X.shape[0])
                    fresh = self.pools[g].take(max(0, -(-(start + n) // B.EPARA_CACHE_PAGE) - len(pages))).tolist()
                    work[g].append((name, start, n, pages + fresh, fresh))
        except BaseException:
            self._give_back(work)
            raise
        return work

    def _give_back(self, work):
        for g, items in enumerate(work):
            for _, _, _, _, fresh in reversed(items):
                self.pools[g].free(fresh[::-1])

    def _commit(self, work):
        for g, items in enumerate(work):
            for name, start, n, pages, _ in items:
                self.sequences[g][name] = [pages, start + n]

    def _launch(self, new, work):
        dev, bf = self.device, B.EPARA_BF16
        table, tensors = [], []
        for g, (items, p) in enumerate(zip(new, self.params)):
            seqs, row = [], 0
            for _, start, n, pages, _ in work[g]:
                seqs.append({"first_row": row, "rows": n, "start": start, "pages": pages})
                row += n
            table.append(seqs)
            d, width = p.Wqkv.shape
            f = self.weights[g]["gate"][1][1]
            buf = lambda N, t=torch.bfloat16: torch.empty((row, N), dtype=t, device=dev)
            t = {"x": torch.cat([X for _, X in items]) if items else buf(d), "y1": buf(d), "qkv": buf(width), "q": buf(p.heads * p.head_dim), "o": buf(p.heads * p.head_dim),
                 "proj": buf(d), "s2": buf(d), "y2": buf(d, torch.uint8 if self.ffn == B.EPARA_FP8_E4M3 else torch.bfloat16), "h": buf(f, torch.uint8 if self.ffn == B.EPARA_FP8_E4M3 else torch.bfloat16),
                 "f": buf(d), "s3": buf(d), "y3": buf(d)}
            tensors.append(t)
        R.add_rmsnorm(self._norm(tensors, "x", None, 0, None, "y1"))
        R.grouped_forward(self._forward(tensors, "qkv", "y1", "qkv"), bf)
        seqs = R.SequenceTable(table, dev)
        R.cache_append(R.CacheAppendPlan(seqs, [{"QKV": t["qkv"], "Q": t["q"], "cache": c, "heads": p.heads, "rotary": self.rotary}
                                                for t, c, p in zip(tensors, self.caches, self.params)], dev))
        R.cache_attention(R.CacheAttnPlan(seqs, [{"Q": t["q"], "O": t["o"], "cache": c, "heads": p.heads} for t, c, p in zip(tensors, self.caches, self.params)], dev))
        R.grouped_forward(self._forward(tensors, "proj", "o", "proj"), bf)
        R.add_rmsnorm(self._norm(tensors, "x", "proj", 1, "s2", "y2"))
        up, down = self._ffn(tensors)
        R.grouped_ffn_swiglu(up, down, self.ffn, bf)
        R.add_rmsnorm(self._norm(tensors, "s2", "f", 0, "s3", "y3"))
        return tensors

    def _norm(self, tensors, x, r, which, s, y):
        return R.RmsNormPlan([{"X": t[x], "R": None if r is None else t[r], "gamma": gamma[which], "S": None if s is None else t[s], "Y": t[y], "eps": p.eps, "out_scale": self.s_x}
                              for t, gamma, p in zip(tensors, self.gammas, self.params)], self.device)

    def _forward(self, tensors, name, src, dst):
        args = [R.group_args(t[src], w[name][0], t[dst], t[src].shape[0], w[name][1][0], w[name][1][1], "none") for t, w in zip(tensors, self.weights)]
        return R.LaunchPlan(np.array(args, dtype=B.GROUP_ARGS), B.EPARA_BF16, self.device)

    def _ffn(self, tensors):
        ffn = np.zeros(len(tensors), dtype=B.FFN_DESC)
        for g, (t, w, (_, s)) in enumerate(zip(tensors, self.weights, self.bits)):
            d, f = w["gate"][1]
            ffn[g] = (t["y2"].data_ptr(), w["gate"][0].data_ptr(), w["up"][0].data_ptr(), w["down"][0].data_ptr(), t["h"].data_ptr(), t["f"].data_ptr(),
                      t["x"].shape[0], d, f, self.s_x, s["gate"], s["up"], self.s_h[g], s["down"])
        up, down = B.epara_ffn_swiglu_args(ffn, self.ffn)
        return R.LaunchPlan(up, self.ffn, self.device), R.LaunchPlan(down, self.ffn, self.device)
