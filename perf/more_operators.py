"""Measured cases of decoding by drafts over an 8-bit paged cache: several tokens of a request are proposed at once, as a chain or a tree, one pass
over the model looks at all of them, and those that the target agrees to stay in the cache.

  tree     from the rows' parents: which rows each of them follows (256 bits) and its rotary position
  attend   attention of the drafted rows over the cache: a row sees the tokens before the drafts, itself and the rows that it follows
  verify   which drafts stay, given the target's logits (and the draft's) and a random number for each row, and the token drawn behind them
  keep     the keys and values of the rows that stay close up in the caches of all layers

`own` chooses between the plain form, elementary torch operations, and the framework's kernels.
"""
import math
import random

import torch

own = False

DEV = "cuda"
PAGE, BLOCK = 64, 32                  # tokens of a page; tokens that share a scale
BIAS, LOWEST = 127, -96               # a scale's byte is its exponent + 127; the smallest exponent that is used
MOST = 256                            # rows of a tree
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
NONE = -2                             # parent of a row that is not there


# ---- cases -----------------------------------------------------------------------------------------------------

def listed():
    return [
        # the drafts of one request: bound by latency
        {"name": "tree_one", "op": "tree", "seqs": "1", "rows": "8..8", "start": "777..777", "layout": 11},
        # the trees of 105 requests of four services, and some requests of two further ones with longer chains
        {"name": "tree_requests", "op": "tree", "seqs": "1,8,32,64,40,60", "rows": "33..256", "start": "0..8191", "layout": 12},
        # eight drafts of one request
        {"name": "attend_one", "op": "attend", "seqs": "1", "rows": "8..8", "start": "4000..4000", "heads": 32, "kv_heads": 8, "head_dim": 128, "window": 0, "softcap": 0.0, "layout": 21},
        # small trees of 105 requests with contexts of all lengths
        {"name": "attend_requests", "op": "attend", "seqs": "1,8,32,64", "rows": "9..16", "start": "0..4095", "heads": 32, "kv_heads": 8, "head_dim": 128, "window": 0, "softcap": 0.0, "layout": 22},
        # trees of 64 of a few requests, every head with its own keys
        {"name": "attend_wide", "op": "attend", "seqs": "4,4", "rows": "64..64", "start": "2000..8000", "heads": 40, "kv_heads": 40, "head_dim": 128, "window": 0, "softcap": 0.0, "layout": 23},
        # one request with a long context and a wide tree, heads of 64
        {"name": "attend_long", "op": "attend", "seqs": "1", "rows": "61..61", "start": "32767..32767", "heads": 12, "kv_heads": 4, "head_dim": 64, "window": 0, "softcap": 30.0, "layout": 24},
        # a chain of five drafts of one request: bound by latency
        {"name": "verify_one", "op": "verify", "seqs": "1", "rows": "6..6", "vocab": 32000, "dtype": "bf16", "draft": False, "chain": True, "greedy": 0.0, "layout": 31},
        # chains of four drafts of 64 requests, drawn from the draft's own probabilities
        {"name": "verify_chains", "op": "verify", "seqs": "64", "rows": "5..5", "vocab": 131072, "dtype": "bf16", "draft": True, "chain": True, "greedy": 0.0, "layout": 32},
        # trees of given tokens of two services, a vocabulary of odd size (rows of logits begin anywhere)
        {"name": "verify_trees", "op": "verify", "seqs": "3,5", "rows": "40..64", "vocab": 50021, "dtype": "bf16", "draft": False, "chain": False, "greedy": 0.2, "layout": 33},
        # logits in 32 bits, many requests, half of them greedy
        {"name": "verify_wide", "op": "verify", "seqs": "8,24", "rows": "3..16", "vocab": 100003, "dtype": "f32", "draft": False, "chain": False, "greedy": 0.5, "layout": 34},
        # one request, the caches of 32 layers
        {"name": "keep_one", "op": "keep", "seqs": "1", "rows": "8..8", "start": "0..4000", "kv_heads": 8, "head_dim": 128, "layers": 32, "layout": 41},
        # the requests of two services, the caches of 16 layers each
        {"name": "keep_requests", "op": "keep", "seqs": "8,32", "rows": "9..64", "start": "0..300", "kv_heads": 8, "head_dim": 128, "layers": 16, "layout": 42},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tree", "attend", "attend", "attend", "verify", "verify", "keep"])
    services, layout = rng.choice([1, 2, 3]), rng.randrange(1 << 20)
    hi = _log(rng, 1, 64)
    rows = "%d..%d" % (max(1, hi // rng.choice([1, 2, 3])), hi)
    n = _log(rng, 1, 48)
    seqs = ",".join([str(max(1, n // services))] * services)
    case = {"op": op, "seqs": seqs, "rows": rows, "start": "0..%d" % _log(rng, 30, 8000), "layout": layout}
    if op == "tree":
        top = _log(rng, 1, 256)
        case["rows"] = "%d..%d" % (max(1, top // 2), top)
        return case
    if op == "verify":
        vocab = _log(rng, 100, 131072)
        most = max(1, int(40e6 / vocab / hi))                     # at most 40 million logits
        del case["start"]
        case.update({"seqs": ",".join([str(max(1, min(n, most) // services))] * services), "vocab": vocab, "dtype": rng.choice(["bf16", "bf16", "f32"]), "draft": rng.random() < 0.4,
                     "greedy": rng.choice([0.0, 0.0, 0.3, 1.0])})
        case["chain"] = case["draft"] or rng.random() < 0.4
        return case
    kv, group, dim = rng.choice([1, 2, 4, 5, 8]), rng.choice([1, 2, 3, 4, 8]), rng.choice([64, 128, 128])
    if op == "keep":
        case.update({"start": "0..%d" % _log(rng, 30, 1000), "kv_heads": kv, "head_dim": dim, "layers": rng.choice([1, 2, 4, 8])})
        return case
    if rng.random() < 0.25:                                       # one request with a long context
        case.update({"seqs": "1", "start": "%d..32000" % _log(rng, 100, 32000)})
    if rng.random() < 0.15:                                       # the largest trees
        case.update({"seqs": "2", "rows": "100..256"})
    cost = kv * group * _span(case["rows"])[1] * _span(case["start"])[1] * services
    case["seqs"] = ",".join([str(max(1, min(int(case["seqs"].split(",")[0]), int(120e6 / cost))))] * len(case["seqs"].split(",")))      # as many as the largest listed case does
    case.update({"heads": kv * group, "kv_heads": kv, "head_dim": dim, "window": rng.choice([0, 0, 0, _log(rng, 256, 4000)]), "softcap": rng.choice([0.0, 0.0, 30.0])})
    return case


def _span(text):
    lo, hi = text.split("..")
    return int(lo), int(hi)


def _parents(rng, n, kind):
    """A chain, or a tree whose rows come level by level as a rule; now and then several rows that follow the context, and rows at the end that are not there."""
    if kind == "chain":
        return list(range(-1, n - 1))
    out = [-1] + [rng.randint((i - 1) // 4, (i - 1) // 2) for i in range(1, n)]
    if kind == "any":
        if n > 4 and rng.random() < 0.3:
            out[rng.randrange(1, n)] = -1
        if n > 8 and rng.random() < 0.5:
            gone = rng.randint(1, n // 4)
            out[n - gone:] = [NONE] * gone
    return out


def _sequences(case):
    """Per service a list of sequences (first row, rows, start, pages, parents): from the case alone."""
    rng = random.Random(case["layout"])
    kind = "any" if case["op"] != "verify" else "chain" if case["chain"] else "tree"
    out = []
    for n in map(int, case["seqs"].split(",")):
        row, seqs, taken = 0, [], 0
        for _ in range(n):
            rows, start = rng.randint(*_span(case["rows"])), rng.randint(*_span(case.get("start", "0..0")))
            count = -(-(start + rows) // PAGE)
            seqs.append([row, rows, start, count, _parents(rng, rows, kind)])
            row, taken = row + rows, taken + count
        ids = list(range(taken))
        rng.shuffle(ids)                                          # the pages of a sequence lie anywhere
        for s in seqs:
            s[3], ids = ids[:s[3]], ids[s[3]:]
        out.append((row, taken, seqs))
    return out


def _follows(parents):
    """Per row the rows that it follows, itself among them; none where it is not there."""
    out = []
    for i, p in enumerate(parents):
        out.append([i] if p == -1 else out[p] + [i] if 0 <= p < i and out[p] else [])
    return out


def _kept(case):
    """Per sequence of a service the rows that stay: what a row follows, for a row drawn from the case."""
    rng = random.Random(case["layout"] + 1)
    return [[rng.choice([f for f in _follows(q[4]) if f and f[0] == 0]) for q in seqs] for _, _, seqs in _sequences(case)]


def work(case):
    n_bytes = flops = 0
    for rows, _, seqs in _sequences(case):
        if case["op"] == "tree":
            n_bytes += rows * (4 + 32 + 12)
        elif case["op"] == "verify":
            size = 4 if case["dtype"] == "f32" else 2
            drafts = sum(len({p for p in q[4] if p >= 0}) for q in seqs) if case["draft"] else 0       # rows that another one follows
            n_bytes += (rows + drafts) * case["vocab"] * size + rows * 20
            flops += 4 * (rows + drafts) * case["vocab"]
        elif case["op"] == "attend":
            H, KV, D = case["heads"], case["kv_heads"], case["head_dim"]
            n_bytes += rows * (H * D * 4 + 32)
            for _, new, start, _, parents in seqs:
                context = min(start, case["window"]) if case["window"] else start
                n_bytes += (context + new) * KV * 2 * D
                flops += 4 * H * D * sum(context + len(f) for f in _follows(parents) if f)
    if case["op"] == "keep":
        n_bytes = sum(len(k) for service in _kept(case) for k in service) * case["layers"] * case["kv_heads"] * 4 * case["head_dim"]
    return {"bytes": n_bytes, "flops": flops}


# ---- inputs ----------------------------------------------------------------------------------------------------

def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def _pack(K, V):
    """Codes of keys and values [.., 64, D] in a page's order: keys in pieces of 16 dims x 16 tokens (4 from each quarter of the page), values
    transposed in pieces of 16 tokens x 16 dims."""
    lead, D = K.shape[:-2], K.shape[-1]
    k = K.reshape(-1, 4, 4, 4, D // 16, 16).permute(0, 2, 4, 1, 3, 5).reshape(*lead, PAGE * D)
    v = V.reshape(-1, 4, 16, D // 16, 16).permute(0, 3, 1, 4, 2).reshape(*lead, PAGE * D)
    return torch.stack([k, v], dim=-2)


def _unpack(codes, D):
    """The inverse of _pack: codes [.., 2, 64 * D] -> keys, values [.., 64, D]."""
    lead = codes.shape[:-2]
    K = codes[..., 0, :].reshape(-1, 4, D // 16, 4, 4, 16).permute(0, 3, 1, 4, 2, 5).reshape(*lead, PAGE, D)
    V = codes[..., 1, :].reshape(-1, D // 16, 4, 16, 16).permute(0, 2, 4, 1, 3).reshape(*lead, PAGE, D)
    return K, V


def _exponent(amax):
    """The smallest e >= LOWEST with amax <= 448 * 2^e: 448 = 0.875 * 2^9."""
    f, x = torch.frexp(amax)
    return torch.where(amax > 0, x - 9 + (f > 0.875), LOWEST).clamp(min=LOWEST)


def _filled(gen, L, P, H, D):
    """Caches as earlier tokens left them: (codes [L, P, H, 2, 64 D], scales).  A few channels of the keys are several times wider than the others, and blocks are of different size."""
    wide = 1 + 3 * (torch.rand(H, 1, D, generator=gen, device=DEV) < 0.04).float()
    size = torch.exp2(torch.randint(-1, 2, (L, P, H, 2, 1, 1), generator=gen, device=DEV).float()).expand(L, P, H, 2, BLOCK, 1).reshape(L, P, H, PAGE, 1)
    packed, exps = [], []
    for x in (_normal(gen, L, P, H, PAGE, D) * wide * size, (_normal(gen, L, P, H, PAGE, D) * 0.5 + 0.1) * size):
        x = x.reshape(L, P, H, 2, BLOCK, D)
        e = _exponent(x.abs().amax(dim=(4, 5)))
        packed.append((x * torch.exp2(-e.float())[..., None, None]).to(E4M3).view(torch.uint8).reshape(L, P, H, PAGE, D))
        exps.append((e + BIAS).to(torch.uint8))
    return _pack(*packed).contiguous(), torch.stack(exps, dim=3).contiguous()


def _indices(seqs):
    """What the plain form looks rows up with: at [n, R], the row of the service that row r of sequence i is (its last one behind the end); live; per row its sequence and place."""
    new = torch.tensor([q[1] for q in seqs], device=DEV)
    first = torch.tensor([q[0] for q in seqs], device=DEV)
    R = max(q[1] for q in seqs)
    r = torch.arange(R, device=DEV)
    return {"at": first[:, None] + torch.minimum(r, new[:, None] - 1), "live": r < new[:, None], "seq": torch.repeat_interleave(torch.arange(len(seqs), device=DEV), new),
            "place": torch.cat([torch.arange(q[1], device=DEV) for q in seqs]), "first": first, "start": torch.tensor([q[2] for q in seqs], device=DEV)}


def _words(rows):
    """Sets of rows as four words of 64 bits each."""
    words = [[sum(1 << (j - 64 * w) for j in f if j // 64 == w) for w in range(4)] for f in rows]
    return torch.tensor([[w - (1 << 64) if w >> 63 else w for w in ws] for ws in words], dtype=torch.int64, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op = case["op"]
    st = {"case": case, "services": []}
    for (rows, pages, seqs), kept in zip(_sequences(case), _kept(case) if op == "keep" else [None] * 99):
        s = {"seqs": seqs, "rows": rows, **_indices(seqs)}
        s["parents"] = torch.tensor([p for q in seqs for p in q[4]], device=DEV, dtype=torch.int32)
        if op == "tree":                                          # the order of the nodes is what the seed changes: a permutation of each row's siblings
            some = torch.rand(rows, generator=gen, device=DEV) < 0.2
            s["parents"] = torch.where(some & (s["parents"] > 0), s["parents"] - 1, s["parents"])
            s["visible"], s["positions"] = torch.zeros(rows, 4, device=DEV, dtype=torch.int64), torch.zeros(rows, 3, device=DEV, dtype=torch.int32)
        elif op == "attend":
            H, KV, D = case["heads"], case["kv_heads"], case["head_dim"]
            longest = max(len(q[3]) for q in seqs)
            s["pages"] = torch.tensor([q[3] + [0] * (longest - len(q[3])) for q in seqs], device=DEV)
            codes, scales = _filled(gen, 1, pages, KV, D)
            s["codes"], s["scales"], s["heads"] = codes[0], scales[0], H
            s["visible"] = _words([f for q in seqs for f in _follows(q[4])])
            s["Q"] = _normal(gen, rows, H * D).bfloat16()
            s["O"] = torch.empty_like(s["Q"])
            s["window"], s["softcap"], s["scale"] = case["window"], case["softcap"], D ** -0.5
        elif op == "verify":
            _logits(gen, case, s)
        else:
            s["layers"] = _filled(gen, case["layers"], pages, case["kv_heads"], case["head_dim"])
            s["path"] = torch.tensor([v for q, k in zip(seqs, kept) for v in k + [-1] * (q[1] - len(k))], device=DEV, dtype=torch.int32)
            s["kept"] = torch.tensor([len(k) for k in kept], device=DEV, dtype=torch.int32)
            touched = [(i, k) for i, q in enumerate(seqs) for k in range(q[2] // PAGE, len(q[3]))]      # the pages that drafts lie in
            index = {ik: j for j, ik in enumerate(touched)}
            s["page"] = torch.tensor([seqs[i][3][k] for i, k in touched], device=DEV)
            s["earlier"] = (torch.tensor([seqs[i][2] - k * PAGE for i, k in touched], device=DEV)[:, None] > torch.arange(PAGE, device=DEV)).reshape(-1)      # tokens before the drafts
            s["slot"] = torch.tensor([index[i, (q[2] + r) // PAGE] * PAGE + (q[2] + r) % PAGE for i, q in enumerate(seqs) for r in range(q[1])], device=DEV)
        st["services"].append(s)
    if own:
        _plan(st)
    return st


def _logits(gen, case, s):
    """Logits as a model has them: a few tokens take most of the probability.  Drafts are drawn from the draft's probabilities, or are its likeliest tokens, one rank a sibling."""
    rows, V, n = s["rows"], case["vocab"], len(s["seqs"])
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    x = _normal(gen, rows, V) * 2.5
    d = x + 0.8 * _normal(gen, rows, V)
    s["logits"], d = x.to(dtype), d.to(dtype)
    s["temperatures"] = torch.where(torch.rand(n, generator=gen, device=DEV) < case["greedy"], 0.0, 0.4 + 0.8 * torch.rand(n, generator=gen, device=DEV))
    parent = s["at"][s["seq"], 0] + s["parents"].clamp(min=0)
    if case["draft"]:
        t = s["temperatures"][s["seq"]].clamp(min=1e-3)[:, None]
        s["draft_logits"] = d
        token = (d.float() / t - torch.log(-torch.log(torch.rand(rows, V, generator=gen, device=DEV).clamp(1e-20, 1 - 1e-7)))).argmax(dim=1)
        s["tokens"] = token[parent].int()
    else:
        rank = torch.zeros(rows, dtype=torch.int64)
        seen = {}
        for i, p in enumerate(parent.tolist()):
            rank[i] = seen[p] = seen.get(p, -1) + 1
        s["draft_logits"], top = None, d.float().topk(min(V, int(rank.max()) + 1), dim=1).indices
        s["tokens"] = top[parent, rank.to(DEV).clamp(max=top.shape[1] - 1)].int()
    s["uniforms"] = torch.rand(rows, generator=gen, device=DEV)


def _plan(st):
    """What a program of the framework keeps for these calls: the plan, and the buffers that it writes."""
    from paper_2511_00603_amd import runtime as R
    op, services = st["case"]["op"], st["services"]
    has_pages = op in ("attend", "keep")
    table = R.SequenceTable([[{"first_row": q[0], "rows": q[1], "start": q[2] if op != "verify" else 0, "pages": q[3] if has_pages else [0] * len(q[3])} for q in s["seqs"]] for s in services], DEV)
    if op == "tree":
        st["call"], st["plan"] = R.draft_trees, R.DraftTreePlan(table, services, DEV)
        st["out"] = [{"visible": s["visible"], "positions": s["positions"]} for s in services]
    elif op == "attend":
        st["call"], st["plan"] = R.tree_attention, R.TreeAttnPlan(table, [dict(s, cache=R.PagedCache(s["codes"], s["scales"])) for s in services], DEV)
        st["out"] = [s["O"] for s in services]
    elif op == "verify":
        plan = R.VerifyPlan(table, services, DEV, temperatures=torch.cat([s["temperatures"] for s in services]))
        st["call"], st["plan"], st["out"] = R.verify_drafts, plan, []
        ends = 0
        for s, g in zip(services, plan.groups):
            begin, ends = ends, ends + len(s["seqs"])
            st["out"].append({"path": g["path"], "probs": g["probs"], "kept": plan.kept[begin:ends], "next": plan.next[begin:ends]})
    else:
        groups = [{"service": g, "cache": R.PagedCache(codes, scales), "path": s["path"]} for g, s in enumerate(services) for codes, scales in zip(*s["layers"])]
        st["call"], st["plan"] = R.cache_keep, R.CacheKeepPlan(table, groups, DEV, kept=torch.cat([s["kept"] for s in services]))
        st["out"] = [{"codes": s["layers"][0].view(E4M3), "scales": s["layers"][1].view(E8M0)} for s in services]


# ---- one pass --------------------------------------------------------------------------------------------------

def run(st):
    if own:
        st["call"](st["plan"])
        return st["out"]
    return [{"tree": _tree, "attend": _attend, "verify": _verify, "keep": _keep}[st["case"]["op"]](st["case"], s) for s in st["services"]]


def _ancestors(s):
    """[n, R, R]: row j is row i or one that it follows; none where row i is not there.  Paths double: after k steps they are 2^k long."""
    R = s["at"].shape[1]
    r = torch.arange(R, device=DEV)
    p = s["parents"].long()[s["at"]]
    good = s["live"] & ((p == -1) | ((p >= 0) & (p < r)))
    up = torch.where(good & (p >= 0), p, torch.where(good, R, R + 1))             # R: the context; R + 1: nowhere
    seen = torch.zeros(*up.shape, R + 2, device=DEV, dtype=torch.bool)
    seen.scatter_(2, up[..., None], True)
    seen[:, r, r] = True
    ends = torch.tensor([[R, R + 1]], device=DEV).expand(len(up), 2)
    none = torch.zeros(len(up), 2, R + 2, device=DEV, dtype=torch.bool)
    for _ in range(R.bit_length()):
        seen = seen | torch.cat([seen, none], dim=1).gather(1, up[..., None].expand(-1, -1, R + 2))
        up = torch.cat([up, ends], dim=1).gather(1, up)
    return seen[..., :R] & ~seen[..., R + 1:]


def _tree(case, s):
    a = _ancestors(s)
    n, R = a.shape[:2]
    bits = torch.nn.functional.pad(a, (0, MOST - R)).reshape(n, R, 4, 64).long()
    words = (bits << torch.arange(64, device=DEV)).sum(dim=3)
    depth = (a.sum(dim=2) - 1).clamp(min=0)
    position = (s["start"][:, None] + depth)[s["seq"], s["place"]]
    return {"visible": words[s["seq"], s["place"]], "positions": position[:, None].expand(-1, 3).int()}


def _attend(case, s):
    H, KV, D, G = case["heads"], case["kv_heads"], case["head_dim"], case["heads"] // case["kv_heads"]
    n, R = s["at"].shape
    L = s["pages"].shape[1] * PAGE
    K, V = _unpack(s["codes"][s["pages"].reshape(-1)], D)
    scale = torch.exp2(s["scales"][s["pages"].reshape(-1)].float() - BIAS).repeat_interleave(BLOCK, dim=3)   # [n * pages, KV, 2, 64]
    lay = lambda x, e: (x.view(E4M3).float() * e[..., None]).reshape(n, -1, KV, PAGE, D).transpose(1, 2).reshape(n * KV, L, D)
    K, V = lay(K, scale[:, :, 0]), lay(V, scale[:, :, 1])
    q = s["Q"].float().reshape(-1, H, D)[s["at"]].reshape(n, R, KV, G, D).transpose(1, 2).reshape(n * KV, R * G, D)
    score = torch.bmm(q, K.transpose(1, 2).contiguous()) * s["scale"]
    if s["softcap"]:
        score = s["softcap"] * torch.tanh(score / s["softcap"])
    bits = (s["visible"][s["at"]][..., None] >> torch.arange(64, device=DEV) & 1).bool().reshape(n, R, MOST)
    there = bits.any(dim=2)
    key = torch.arange(L, device=DEV)
    begin = s["start"][:, None] + bits.sum(dim=2) - s["window"] if s["window"] else torch.zeros_like(s["at"])      # the first key that the window leaves
    behind = (key - s["start"][:, None])[:, None].expand(n, R, L)
    seen = torch.where(behind < 0, there[..., None] & (key >= begin[..., None]), bits.gather(2, behind.clamp(0, MOST - 1)) & (behind < MOST))
    score = score.reshape(n, KV, R, G, L).masked_fill_(~seen[:, None, :, None, :], -math.inf).reshape(n * KV, R * G, L)
    score = torch.exp(score - score.amax(dim=2, keepdim=True))
    o = torch.bmm(score, V) / score.sum(dim=2, keepdim=True)
    o = o.reshape(n, KV, R, G, D).transpose(1, 2).reshape(n, R, H * D)
    return torch.where(there[..., None], o, 0.0)[s["seq"], s["place"]].bfloat16()


def _softmax_at(x, t, row, token):
    """softmax(x / t)[row, token], the largest of each row of x and where it is."""
    top, where = x.max(dim=1)
    e = torch.exp((x - top[:, None]) / t[:, None])
    return torch.exp((x[row, token] - top[row]) / t[row]) / e.sum(dim=1)[row], where


def _verify(case, s):
    n, R = s["at"].shape
    rows, r = s["rows"], torch.arange(R, device=DEV)
    t = s["temperatures"][s["seq"]]
    greedy, t1 = t <= 0, torch.where(t > 0, t, 1.0)
    p, token = s["parents"].long(), s["tokens"].long()
    drafted = (p >= 0) & (p < s["place"])
    parent = s["at"][s["seq"], 0] + torch.where(drafted, p, 0)
    x = s["logits"].float()
    prob, top = _softmax_at(x, t1, parent, token)
    prob = torch.where(drafted, torch.where(greedy, (top[parent] == token).float(), prob), 0.0)
    # ---- rows against rows of the same sequence: which are siblings, which came before
    pick = lambda v: v[s["at"]]
    live, par, tok, u, w = s["live"] & pick(drafted), pick(p), pick(token), pick(s["uniforms"]), pick(prob)
    earlier = (par[:, :, None] == par[:, None, :]) & live[:, :, None] & live[:, None, :] & (r[:, None] > r[None, :])      # [n, i, j]: j is an elder sibling of i
    again = (earlier & (tok[:, :, None] == tok[:, None, :])).any(dim=2)
    mass = 1 - (earlier & ~again[:, None, :]).float().mul(w[:, None, :]).sum(dim=2)
    yes = live & ~again & (u * mass < w)
    if case["draft"]:
        q, _ = _softmax_at(s["draft_logits"].float(), t1, parent, token)
        yes = live & ~earlier.any(dim=2) & torch.where(pick(greedy), w > 0, u * pick(q) < w)
    chosen = yes & ~(earlier & yes[:, None, :]).any(dim=2)
    chosen[:, 0] = True
    a = _ancestors(s)
    on_path = a[:, :, 0] & ~(a & ~chosen[:, None, :]).any(dim=2)
    kept, last = on_path.sum(dim=1), torch.where(on_path, r, 0).amax(dim=1)
    path = torch.where(r < kept[:, None], torch.where(on_path, r, R).sort(dim=1).values, -1)
    # ---- the token behind the last row that stays: in 64 bits, for borders of the running sum lie close
    at = s["at"].gather(1, last[:, None])[:, 0]
    t64 = t1[at].double()[:, None]
    l = s["logits"][at].double()
    weight = torch.exp((l - l.amax(dim=1, keepdim=True)) / t64)
    child = live & (par == last[:, None])
    if case["draft"]:
        d = s["draft_logits"][at].double()
        q = torch.exp((d - d.amax(dim=1, keepdim=True)) / t64)
        rest = (weight / weight.sum(dim=1, keepdim=True) - q / q.sum(dim=1, keepdim=True)).clamp(min=0)
        weight = torch.where(child.any(dim=1, keepdim=True), rest, weight)
    else:
        weight = weight.scatter_add(1, torch.where(child, tok, tok[:, :1]), torch.where(child, -math.inf, 0.0).double()).clamp(min=0)
    cum = weight.cumsum(dim=1)
    goal = u[:, :1].double() * cum[:, -1:]
    token = torch.searchsorted(cum, goal, right=True)[:, 0].clamp(max=case["vocab"] - 1)
    token = torch.where(greedy[at], top[at], token)
    return {"path": path[s["seq"], s["place"]].int(), "probs": prob, "kept": kept.int(), "next": token.int()}


def _keep(case, s):
    D, KV, (codes, scales) = case["head_dim"], case["kv_heads"], s["layers"]
    Ls, J = codes.shape[0], len(s["page"])
    stays = s["place"] < s["kept"][s["seq"]]
    dst = s["slot"][stays]
    src = s["slot"][s["at"][s["seq"], 0] + s["path"].clamp(min=0)][stays]
    old = torch.stack(_unpack(codes[:, s["page"]], D), dim=3).permute(1, 4, 0, 2, 3, 5).reshape(J * PAGE, Ls, KV, 2, D)       # a token's codes, by slot
    before = scales[:, s["page"]].int().permute(1, 4, 0, 2, 3).reshape(J * 2, Ls, KV, 2) - BIAS                              # a block's exponents
    wanted = torch.full_like(before, -999).scatter_reduce(0, (dst // BLOCK)[:, None, None, None].expand(-1, Ls, KV, 2), before[src // BLOCK], "amax")
    joined = wanted > -999
    e = torch.where(joined, torch.where(s["earlier"][::BLOCK, None, None, None], torch.maximum(before, wanted), wanted), before)
    value = old.view(E4M3).float() * torch.exp2((before - e).float()).repeat_interleave(BLOCK, dim=0)[..., None]            # earlier tokens of a block that grows
    moved = old[src].view(E4M3).float() * torch.exp2((before[src // BLOCK] - e[dst // BLOCK]).float())[..., None]
    new = torch.where(s["earlier"][:, None, None, None, None], value.to(E4M3).view(torch.uint8), old)                        # what does not stay, and what lies behind, is left as it is
    new = new.index_put((dst,), moved.to(E4M3).view(torch.uint8))
    new = new.reshape(J, PAGE, Ls, KV, 2, D).permute(2, 0, 3, 4, 1, 5)
    codes[:, s["page"]] = _pack(new[:, :, :, 0], new[:, :, :, 1])
    scales[:, s["page"]] = (e + BIAS).to(torch.uint8).reshape(J, 2, Ls, KV, 2).permute(2, 0, 3, 4, 1)
    return {"codes": codes.view(E4M3), "scales": scales.view(E8M0)}


# ---- in 64 bits, from the definitions -----------------------------------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "tree":
        return None                                               # whole numbers
    return [{"attend": _attend64, "verify": _verify64, "keep": _keep64}[case["op"]](case, s) for s in st["services"]]


def _attend64(case, s):
    H, KV, D, G = case["heads"], case["kv_heads"], case["head_dim"], case["heads"] // case["kv_heads"]
    out = torch.zeros(s["rows"], H, D, device=DEV, dtype=torch.float64)
    for row, new, start, pages, parents in s["seqs"]:
        ids = torch.tensor(pages, device=DEV)
        K, V = _unpack(s["codes"][ids], D)
        e = torch.exp2(s["scales"][ids].double() - BIAS)          # [pages, KV, 2, 2]
        hidden = torch.ones(new, start + new, device=DEV, dtype=torch.bool)
        for i, f in enumerate(_follows(parents)):
            if f:
                hidden[i, max(0, start + len(f) - s["window"]) if s["window"] else 0: start] = False
                hidden[i, [start + j for j in f]] = False
        there = ~hidden.all(dim=1)
        for h in range(KV):
            k = (K[:, h].view(E4M3).double().reshape(-1, 2, BLOCK, D) * e[:, h, 0, :, None, None]).reshape(-1, D)[: start + new]
            v = (V[:, h].view(E4M3).double().reshape(-1, 2, BLOCK, D) * e[:, h, 1, :, None, None]).reshape(-1, D)[: start + new]
            for g in range(G):
                q = s["Q"][row: row + new, (h * G + g) * D: (h * G + g + 1) * D].double()
                z = q @ k.T * s["scale"]
                if s["softcap"]:
                    z = s["softcap"] * torch.tanh(z / s["softcap"])
                o = torch.softmax(z.masked_fill(hidden, -math.inf), dim=1) @ v
                out[row: row + new, h * G + g] = torch.where(there[:, None], o, 0.0)
    return out.reshape(-1, H * D)


def _verify64(case, s):
    """The probabilities; what is whole has no value in 64 bits."""
    out = torch.zeros(s["rows"], device=DEV, dtype=torch.float64)
    tokens = s["tokens"].tolist()
    for i, (row, new, _, _, parents) in enumerate(s["seqs"]):
        t, x = float(s["temperatures"][i]), s["logits"][row: row + new].double()
        p = torch.softmax(x / t, dim=1) if t > 0 else torch.nn.functional.one_hot(x.argmax(dim=1), case["vocab"]).double()
        for r in range(1, new):
            if 0 <= parents[r] < r:
                out[row + r] = p[parents[r], tokens[row + r]]
    return {"path": None, "probs": out, "kept": None, "next": None}


def _keep64(case, s):
    """The codes' values before they are rounded, sequence by sequence and block by block."""
    D, (codes, scales) = case["head_dim"], s["layers"]
    K, V = (c.view(E4M3).double() for c in _unpack(codes, D))
    e = scales.double() - BIAS                                    # [L, P, KV, 2, 2]
    path, kept = s["path"].tolist(), s["kept"].tolist()
    for (row, _, start, pages, _), n in zip(s["seqs"], kept):
        src = [start + j for j in path[row: row + n]]
        was = e.clone()
        for b in range(start // BLOCK, (start + n - 1) // BLOCK + 1):
            lo, hi = max(start, b * BLOCK), min(start + n, (b + 1) * BLOCK)
            page, half = pages[b // 2], b % 2
            from_ = src[lo - start: hi - start]
            for which, cache in ((0, K), (1, V)):
                exps = [was[:, pages[j // PAGE], :, which, j % PAGE // BLOCK] for j in from_]
                top = torch.stack(exps + ([was[:, page, :, which, half]] if lo > b * BLOCK else [])).amax(dim=0)
                fresh = [cache[:, pages[j // PAGE], :, j % PAGE] * torch.exp2(x - top)[..., None] for j, x in zip(from_, exps)]
                base = half * BLOCK
                cache[:, page, :, base: base + lo - b * BLOCK] *= torch.exp2(was[:, page, :, which, half] - top)[..., None, None]
                cache[:, page, :, base + lo - b * BLOCK: base + hi - b * BLOCK] = torch.stack(fresh, dim=2)
                e[:, page, :, which, half] = top
    return {"codes": _pack(K, V), "scales": torch.exp2(e)}
