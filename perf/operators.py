"""Measured cases of the operators of a decoder block that works on an 8-bit paged cache.

  norm     s = x + r, y = s / rms(s) * gamma, y in bf16 or in E4M3 codes with a scale per row or per service
  append   rotary positions (one to three axes) for new queries and keys; keys and values join the cache in E4M3
           with a power-of-two scale for each block of 32 tokens and head
  attend   causal attention of new rows over the cache (shared key heads, window, capped scores)
  copy     pages of the cache copied to other pages (forks, compaction)

`own` chooses between the plain form, elementary torch operations in 32 bits, and the framework's kernels.
"""
import math
import random

import torch

own = False

DEV = "cuda"
PAGE, BLOCK = 64, 32                  # tokens of a page; tokens that share a scale
BIAS, LOWEST = 127, -96               # a scale's byte is its exponent + 127; the smallest exponent that is used
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
TOP = 448.0
EPS = 1e-5


# ---- cases -----------------------------------------------------------------------------------------------------

def listed():
    return [
        # one token of every request of four co-located services (1, 8, 32 and 64 requests), width 4096: the smallest calls, bound by latency
        {"name": "norm_tokens", "op": "norm", "rows": "1,8,32,64", "d": 4096, "out": "bf16", "residual": True},
        # the prompts of two services, 8192 rows of width 5120, in bf16 for a bf16 projection
        {"name": "norm_prompts", "op": "norm", "rows": "4301,3891", "d": 5120, "out": "bf16", "residual": True},
        # the same rows in 8 bits with a scale per row
        {"name": "norm_prompts_rows8", "op": "norm", "rows": "4301,3891", "d": 5120, "out": "row", "residual": True},
        # one token of 105 requests joins the caches of four services; most blocks are partly filled
        {"name": "append_tokens", "op": "append", "seqs": "1,8,32,64", "new": "1..1", "start": "0..4095", "heads": 32, "kv_heads": 8, "head_dim": 128, "axes": 1, "layout": 11},
        # prompts of 512 to 2048 tokens of two services, every head with its own keys
        {"name": "append_prompts", "op": "append", "seqs": "3,3", "new": "512..2048", "start": "0..0", "heads": 40, "kv_heads": 40, "head_dim": 128, "axes": 1, "layout": 12},
        # frames of a video (time, height, width) behind a text of odd length, heads of 64
        {"name": "append_frames", "op": "append", "seqs": "5", "new": "197..1024", "start": "1..77", "heads": 12, "kv_heads": 4, "head_dim": 64, "axes": 3, "layout": 13},
        # one token of one request with a long context: few rows, the long axis has to be split
        {"name": "attend_token_long", "op": "attend", "seqs": "1", "new": "1..1", "start": "32767..32767", "heads": 32, "kv_heads": 8, "head_dim": 128, "window": 0, "softcap": 0.0, "layout": 21},
        # one token of 105 requests with contexts of all lengths
        {"name": "attend_tokens", "op": "attend", "seqs": "1,8,32,64", "new": "1..1", "start": "0..4095", "heads": 32, "kv_heads": 8, "head_dim": 128, "window": 0, "softcap": 0.0, "layout": 22},
        # prompts of 512 to 2048 tokens of two services, every head with its own keys: the largest products
        {"name": "attend_prompts", "op": "attend", "seqs": "3,3", "new": "512..2048", "start": "0..0", "heads": 40, "kv_heads": 40, "head_dim": 128, "window": 0, "softcap": 0.0, "layout": 23},
        # pieces of long prompts next to contexts in the cache, with a window and capped scores
        {"name": "attend_pieces", "op": "attend", "seqs": "3", "new": "257..512", "start": "3000..7000", "heads": 32, "kv_heads": 8, "head_dim": 128, "window": 4096, "softcap": 50.0, "layout": 24},
        # the part-filled last pages of forked requests
        {"name": "copy_forks", "op": "copy", "pages": 256, "moves": 9, "kv_heads": 8, "head_dim": 128, "layout": 31},
        # a compaction that moves a large part of a cache
        {"name": "copy_compaction", "op": "copy", "pages": 8192, "moves": 3001, "kv_heads": 8, "head_dim": 128, "layout": 32},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "append", "attend", "attend", "copy"])
    if op == "norm":
        total, n = _log(rng, 1, 8192), rng.choice([1, 2, 3, 5])
        rows = [max(1, int(total * rng.uniform(0.5, 1.0) / n)) for _ in range(n)]
        return {"op": op, "rows": ",".join(map(str, rows)), "d": 8 * _log(rng, 8, 1024), "out": rng.choice(["bf16", "row", "service"]), "residual": rng.random() < 0.8}
    if op == "copy":
        pages = _log(rng, 16, 8192)
        return {"op": op, "pages": pages, "moves": max(1, int(pages * rng.uniform(0.02, 0.4))), "kv_heads": rng.choice([1, 2, 5, 8]), "head_dim": rng.choice([64, 128]), "layout": rng.randrange(1 << 20)}
    kv, group, dim = rng.choice([1, 2, 4, 5, 8]), rng.choice([1, 2, 3, 4, 8]), rng.choice([64, 128, 128])
    services = rng.choice([1, 2, 3])
    shape = {"heads": kv * group, "kv_heads": kv, "head_dim": dim, "layout": rng.randrange(1 << 20)}
    if rng.random() < 0.5:                                        # one token of many requests, or a few
        n = _log(rng, 1, 48)
        seqs, hi = [max(1, n // services)] * services, _log(rng, 100, 8192)
        new, start = "1..%d" % rng.choice([1, 1, 1, 5]), "0..%d" % hi
    else:                                                         # prompts, or pieces of them
        hi = _log(rng, 16, 2048)
        seqs = [rng.choice([1, 2, 3])] * services
        new, start = "%d..%d" % (max(1, hi // 4), hi), rng.choice(["0..0", "0..%d" % _log(rng, 2, 3000)])
    shape.update({"op": op, "seqs": ",".join(map(str, seqs)), "new": new, "start": start})
    if op == "append":
        shape["axes"] = rng.choice([1, 1, 2, 3])
    else:
        shape.update({"window": rng.choice([0, 0, _log(rng, 20, 4000)]), "softcap": rng.choice([0.0, 0.0, 30.0])})
    return shape


def _span(text):
    lo, hi = text.split("..")
    return int(lo), int(hi)


def _sequences(case):
    """Per service a list of sequences (first row, new rows, start, pages): from the case alone."""
    rng = random.Random(case["layout"])
    out = []
    for n in map(int, case["seqs"].split(",")):
        row, seqs, taken = 0, [], 0
        for _ in range(n):
            new, start = rng.randint(*_span(case["new"])), rng.randint(*_span(case["start"]))
            count = -(-(start + new) // PAGE)
            seqs.append([row, new, start, count])
            row, taken = row + new, taken + count
        ids = list(range(taken))
        rng.shuffle(ids)                                          # the pages of a sequence lie anywhere
        for s in seqs:
            s[3], ids = ids[:s[3]], ids[s[3]:]
        out.append((row, taken, seqs))
    return out


def work(case):
    if case["op"] == "norm":
        total, out = sum(map(int, case["rows"].split(","))), 2 if case["out"] == "bf16" else 1
        per = 2 * (2 if case["residual"] else 1) + 2 + out
        return {"bytes": total * case["d"] * per + 4 * case["d"] * len(case["rows"].split(",")), "flops": 6 * total * case["d"]}
    if case["op"] == "copy":
        page = case["kv_heads"] * 2 * (PAGE * case["head_dim"] + 2)
        return {"bytes": 2 * case["moves"] * page, "flops": 0}
    H, KV, D, n_bytes, flops = case["heads"], case["kv_heads"], case["head_dim"], 0, 0
    for rows, _, seqs in _sequences(case):
        if case["op"] == "append":
            n_bytes += rows * D * (4 * H + 6 * KV)                # bf16 in; queries out in bf16, keys and values in 8 bits
            flops += rows * D * 3 * (H + KV)
            continue
        n_bytes += rows * H * D * 4
        for _, new, start, _ in seqs:
            lo = max(0, start - case["window"] + 1) if case["window"] else 0
            n_bytes += (start + new - lo) * KV * 2 * D
            seen = sum(min(start + i + 1, case["window"] or start + i + 1) for i in range(new))
            flops += 4 * seen * H * D
    return {"bytes": n_bytes, "flops": flops}


# ---- inputs ----------------------------------------------------------------------------------------------------

def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def _pack(K, V):
    """Codes of keys and values [pages, kv_heads, 64, D] in a page's order: keys in pieces of 16 dims x 16 tokens (4 from each quarter of
    the page), values transposed in pieces of 16 tokens x 16 dims."""
    P, H, _, D = K.shape
    k = K.reshape(P, H, 4, 4, 4, D // 16, 16).permute(0, 1, 3, 5, 2, 4, 6).reshape(P, H, PAGE * D)
    v = V.reshape(P, H, 4, 16, D // 16, 16).permute(0, 1, 4, 2, 5, 3).reshape(P, H, PAGE * D)
    return torch.stack([k, v], dim=2).contiguous()


def _unpack(codes, D):
    """The inverse of _pack: codes [pages, kv_heads, 2, 64 * D] -> keys, values [pages, kv_heads, 64, D]."""
    P, H = codes.shape[:2]
    K = codes[:, :, 0].reshape(P, H, 4, D // 16, 4, 4, 16).permute(0, 1, 4, 2, 5, 3, 6).reshape(P, H, PAGE, D)
    V = codes[:, :, 1].reshape(P, H, D // 16, 4, 16, 16).permute(0, 1, 3, 5, 2, 4).reshape(P, H, PAGE, D)
    return K, V


def _filled(gen, P, H, D):
    """A cache as earlier tokens left it: (codes, scales).  A few channels of the keys are several times wider than the others."""
    wide = 1 + 3 * (torch.rand(H, 1, D, generator=gen, device=DEV) < 0.04).float()
    k, v = _normal(gen, P, H, PAGE, D) * wide, _normal(gen, P, H, PAGE, D) * 0.5 + 0.1
    packed, exps = [], []
    for x in (k, v):
        x = x.reshape(P, H, 2, BLOCK, D)
        e = _exponent(x.abs().amax(dim=(3, 4)))
        packed.append((x * torch.exp2(-e.float())[..., None, None]).to(E4M3).view(torch.uint8).reshape(P, H, PAGE, D))
        exps.append((e + BIAS).to(torch.uint8))
    return _pack(*packed), torch.stack(exps, dim=2).contiguous()


def _table(case, service):
    """(page, slot) of every position of every sequence, padded: [n, longest] page ids."""
    longest = max(len(s[3]) for s in service)
    return torch.tensor([s[3] + [0] * (longest - len(s[3])) for s in service], device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    st = {"case": case}
    op = case["op"]
    if op == "norm":
        d, st["services"] = case["d"], []
        for M in map(int, case["rows"].split(",")):
            s = {"X": _normal(gen, M, d) * 2, "R": _normal(gen, M, d) if case["residual"] else None, "gamma": 1 + 0.2 * _normal(gen, d), "eps": EPS}
            s["X"] = s["X"].bfloat16()
            s["R"] = None if s["R"] is None else s["R"].bfloat16()
            s["S"] = torch.empty_like(s["X"])
            s["Y"] = torch.empty(M, d, device=DEV, dtype=torch.bfloat16 if case["out"] == "bf16" else torch.uint8)
            s["row_scales"] = torch.empty(M, device=DEV) if case["out"] == "row" else None
            s["out_scale"] = 0.0125 if case["out"] == "service" else None
            st["services"].append(s)
    elif op == "copy":
        st["codes"], st["scales"] = _filled(gen, case["pages"], case["kv_heads"], case["head_dim"])
        ids = list(range(case["pages"]))
        random.Random(case["layout"]).shuffle(ids)
        n = min(case["moves"], case["pages"] // 2)
        st["moves"] = list(zip(ids[:n], ids[n:2 * n]))
        st["src"], st["dst"] = (torch.tensor([m[i] for m in st["moves"]], device=DEV) for i in (0, 1))
    else:
        H, KV, D, st["services"] = case["heads"], case["kv_heads"], case["head_dim"], []
        for rows, pages, seqs in _sequences(case):
            s = {"seqs": seqs, "pages": _table(case, seqs), "heads": H}
            s["codes"], s["scales"] = _filled(gen, pages, KV, D)
            s["start"], s["new"] = (torch.tensor([q[i] for q in seqs], device=DEV) for i in (2, 1))
            s["row_seq"] = torch.repeat_interleave(torch.arange(len(seqs), device=DEV), s["new"])
            s["row_pos"] = torch.cat([torch.arange(q[2], q[2] + q[1], device=DEV) for q in seqs])
            s["row_in"] = torch.cat([torch.arange(q[1], device=DEV) for q in seqs])
            if op == "append":
                joined = [(i, k) for i, q in enumerate(seqs) for k in range(q[2] // PAGE, len(q[3]))]      # the pages that new tokens join
                index = {ik: j for j, ik in enumerate(joined)}
                s["row_page"] = torch.tensor([index[i, (q[2] + r) // PAGE] for i, q in enumerate(seqs) for r in range(q[1])], device=DEV)
                s["page"], s["page_base"], s["page_start"], s["page_end"] = torch.tensor(
                    [(seqs[i][3][k], k * PAGE, seqs[i][2], seqs[i][2] + seqs[i][1]) for i, k in joined], device=DEV).unbind(1)
                last = max(q[1] + q[2] for q in seqs)
                s["QKV"] = torch.cat([_normal(gen, rows, (H + KV) * D), _normal(gen, rows, KV * D) * 0.5], dim=1).bfloat16()
                s["Q"] = torch.empty(rows, H * D, device=DEV, dtype=torch.bfloat16)
                angle = torch.arange(last, device=DEV).double()[:, None] * 10000.0 ** (-torch.arange(D // 2, device=DEV).double() * 2 / D)
                s["rotary"] = torch.stack([angle.cos(), angle.sin()], dim=-1).float()
                axes = case["axes"]
                s["axis_pairs"] = [D // 2 - (axes - 1) * (D // 8)] + [D // 8] * (axes - 1) + [0] * (3 - axes)
                s["positions"] = None
                if axes > 1:                                      # frames of 14 x 14 behind the text
                    at = s["row_pos"]
                    s["positions"] = torch.stack([at // 196, at // 14 % 14, at % 14], dim=1).clamp(max=last - 1).int()
            else:
                s["Q"] = _normal(gen, rows, H * D).bfloat16()
                s["O"] = torch.empty_like(s["Q"])
                s["window"], s["softcap"], s["scale"] = case["window"], case["softcap"], D ** -0.5
            st["services"].append(s)
    if own:
        _plan(st)
    return st


def _plan(st):
    """What a program of the framework keeps for these calls: the plan, and the buffers that it writes."""
    from paper_2511_00603_amd import runtime as R
    op, services = st["case"]["op"], st.get("services")
    if op == "norm":
        st["call"], st["plan"] = R.add_rmsnorm, R.RmsNormPlan(services, DEV)
        st["out"] = [{"S": s["S"], "Y": s["Y"].view(E4M3) if s["Y"].dtype == torch.uint8 else s["Y"], "row_scales": s["row_scales"]} for s in services]
        return
    if op == "copy":
        st["call"], st["plan"] = R.copy_pages, R.PageCopyPlan([{"cache": R.PagedCache(st["codes"], st["scales"]), "moves": st["moves"]}], DEV)
        st["out"] = {"codes": st["codes"].view(E4M3), "scales": st["scales"].view(E8M0)}
        return
    table = R.SequenceTable([[{"first_row": q[0], "rows": q[1], "start": q[2], "pages": q[3]} for q in s["seqs"]] for s in services], DEV)
    groups = [dict(s, cache=R.PagedCache(s["codes"], s["scales"])) for s in services]
    if op == "append":
        st["call"], st["plan"] = R.cache_append, R.CacheAppendPlan(table, groups, DEV)
        st["out"] = [{"Q": s["Q"], "codes": s["codes"].view(E4M3), "scales": s["scales"].view(E8M0)} for s in services]
    else:
        st["call"], st["plan"] = R.cache_attention, R.CacheAttnPlan(table, groups, DEV)
        st["out"] = [s["O"] for s in services]


# ---- one pass --------------------------------------------------------------------------------------------------

def run(st):
    if own:
        st["call"](st["plan"])
        return st["out"]
    op = st["case"]["op"]
    if op != "copy":
        return [{"norm": _norm, "append": _append, "attend": _attend}[op](st["case"], s) for s in st["services"]]
    st["codes"][st["dst"]] = st["codes"][st["src"]]
    st["scales"][st["dst"]] = st["scales"][st["src"]]
    return {"codes": st["codes"].view(E4M3), "scales": st["scales"].view(E8M0)}


def _exponent(amax):
    """The smallest e >= LOWEST with amax <= 448 * 2^e: 448 = 0.875 * 2^9."""
    f, x = torch.frexp(amax)
    return torch.where(amax > 0, x - 9 + (f > 0.875), LOWEST).clamp(min=LOWEST)


def _norm(case, s):
    x = s["X"].float()
    if s["R"] is not None:
        x = x + s["R"].float()
    y = x * torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS) * s["gamma"]
    if case["out"] == "bf16":
        return {"S": x.bfloat16(), "Y": y.bfloat16(), "row_scales": None}
    scales = None
    if case["out"] == "row":
        amax = y.abs().amax(dim=1)
        scales = torch.where(amax > 0, amax / TOP, 1.0)
        y = y * (1 / scales)[:, None]
    else:
        y = y * (1 / s["out_scale"])
    return {"S": x.bfloat16(), "Y": y.clamp(-TOP, TOP).to(E4M3), "row_scales": scales}


def _rotated(x, s):
    """x [rows, heads, D] in float: pair (i, i + D / 2) turned by the angle of the row's position on the pair's axis."""
    half = x.shape[-1] // 2
    if s["positions"] is None:
        cs = s["rotary"][s["row_pos"]]                            # [rows, D / 2, 2]
    else:
        axis = torch.repeat_interleave(torch.arange(3, device=DEV), torch.tensor(s["axis_pairs"], device=DEV))
        cs = s["rotary"][s["positions"][:, axis].long(), torch.arange(half, device=DEV)]
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _append(case, s):
    H, KV, D = case["heads"], case["kv_heads"], case["head_dim"]
    rows = s["QKV"].shape[0]
    q, k, v = s["QKV"].float().split([H * D, KV * D, KV * D], dim=1)
    Q = _rotated(q.reshape(rows, H, D), s).reshape(rows, H * D).bfloat16()
    kv = torch.stack([_rotated(k.reshape(rows, KV, D), s), v.reshape(rows, KV, D)], dim=2)       # [rows, KV, 2, D]
    P = len(s["page"])                                            # the pages that new tokens join
    staged = torch.zeros(P, PAGE, KV, 2, D, device=DEV)
    staged[s["row_page"], s["row_pos"] % PAGE] = kv
    at = s["page_base"][:, None] + torch.arange(PAGE, device=DEV)
    is_old = at < s["page_start"][:, None]                        # tokens that were there before
    is_new = ~is_old & (at < s["page_end"][:, None])
    staged = staged.permute(0, 2, 3, 1, 4).reshape(P, KV, 2, 2, BLOCK, D)
    is_new, is_old = is_new.reshape(P, 1, 1, 2, BLOCK), is_old.reshape(P, 1, 1, 2, BLOCK)
    wanted = _exponent(staged.abs().amax(dim=(4, 5)))
    before = s["scales"][s["page"]].int() - BIAS                  # [P, KV, 2, 2]
    e = torch.where(is_new.any(dim=4), torch.where(is_old.any(dim=4), torch.maximum(wanted, before), wanted), before)
    old = torch.stack(_unpack(s["codes"][s["page"]], D), dim=2).reshape(P, KV, 2, 2, BLOCK, D).view(E4M3).float()
    value = torch.where(is_new[..., None], staged * torch.exp2(-e.float())[..., None, None],
                        torch.where(is_old[..., None], old * torch.exp2((before - e).float())[..., None, None], old))
    new = value.to(E4M3).view(torch.uint8).reshape(P, KV, 2, PAGE, D)
    s["codes"][s["page"]] = _pack(new[:, :, 0], new[:, :, 1])
    s["scales"][s["page"]] = (e + BIAS).to(torch.uint8)
    return {"Q": Q, "codes": s["codes"].view(E4M3), "scales": s["scales"].view(E8M0)}


def _attend(case, s):
    H, KV, D, G = case["heads"], case["kv_heads"], case["head_dim"], case["heads"] // case["kv_heads"]
    n, longest = s["pages"].shape[0], int(max(q[1] for q in s["seqs"]))
    L = s["pages"].shape[1] * PAGE
    K, V = _unpack(s["codes"][s["pages"].reshape(-1)], D)
    scale = torch.exp2(s["scales"][s["pages"].reshape(-1)].float() - BIAS).repeat_interleave(BLOCK, dim=3)   # [n * pages, KV, 2, 64]
    lay = lambda x, e: (x.view(E4M3).float() * e[..., None]).reshape(n, -1, KV, PAGE, D).transpose(1, 2).reshape(n * KV, L, D)
    K, V = lay(K, scale[:, :, 0]), lay(V, scale[:, :, 1])
    q = torch.zeros(n, longest, H, D, device=DEV)
    q[s["row_seq"], s["row_in"]] = s["Q"].float().reshape(-1, H, D)
    q = q.reshape(n, longest, KV, G, D).transpose(1, 2).reshape(n * KV, longest * G, D)
    score = torch.bmm(q, K.transpose(1, 2).contiguous()) * s["scale"]
    if s["softcap"]:
        score = s["softcap"] * torch.tanh(score / s["softcap"])
    pos, key = s["start"][:, None] + torch.arange(longest, device=DEV), torch.arange(L, device=DEV)
    seen = key <= pos[..., None]
    if s["window"]:
        seen &= key > pos[..., None] - s["window"]
    score = score.reshape(n, KV, longest, G, L).masked_fill_(~seen[:, None, :, None, :], -math.inf).reshape(n * KV, longest * G, L)
    score = torch.exp(score - score.amax(dim=2, keepdim=True))
    o = torch.bmm(score, V) / score.sum(dim=2, keepdim=True)
    o = o.reshape(n, KV, longest, G, D).transpose(1, 2).reshape(n, longest, H * D)
    return o[s["row_seq"], s["row_in"]].bfloat16()


# ---- in 64 bits, from the definitions -----------------------------------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "copy":
        codes, scales = st["codes"].view(E4M3).double(), torch.exp2(st["scales"].double() - BIAS)
        a, b = codes.clone(), scales.clone()
        for src, dst in st["moves"]:
            a[dst], b[dst] = codes[src], scales[src]
        return {"codes": a, "scales": b}
    return [{"norm": _norm64, "append": _append64, "attend": _attend64}[case["op"]](case, s) for s in st["services"]]


def _norm64(case, s):
    x = s["X"].double() + (0 if s["R"] is None else s["R"].double())
    y = x / ((x ** 2).mean(dim=1, keepdim=True) + EPS).sqrt() * s["gamma"].double()
    if case["out"] == "bf16":
        return {"S": x, "Y": y, "row_scales": None}
    if case["out"] == "service":
        return {"S": x, "Y": (y / s["out_scale"]).clamp(-TOP, TOP), "row_scales": None}
    scales = y.abs().amax(dim=1) / TOP
    return {"S": x, "Y": y / scales[:, None], "row_scales": scales}


def _append64(case, s):
    """The codes' values before they are rounded, sequence by sequence and block by block."""
    H, KV, D = case["heads"], case["kv_heads"], case["head_dim"]
    M, half = s["QKV"].shape[0], D // 2
    x = s["QKV"].double().reshape(M, H + 2 * KV, D)
    at = s["row_pos"][:, None].expand(M, 3) if s["positions"] is None else s["positions"].long()
    turned = x.clone()
    first = 0
    for axis, pairs in enumerate(s["axis_pairs"]):
        i = slice(first, first + pairs)
        j = slice(half + first, half + first + pairs)
        w = s["rotary"].double()[at[:, axis], i]                  # [M, pairs, 2]
        c, t = w[:, None, :, 0], w[:, None, :, 1]
        turned[:, : H + KV, i] = x[:, : H + KV, i] * c - x[:, : H + KV, j] * t
        turned[:, : H + KV, j] = x[:, : H + KV, j] * c + x[:, : H + KV, i] * t
        first += pairs
    K, V = (c.view(E4M3).double() for c in _unpack(s["codes"], D))
    scales = s["scales"].clone()
    for row, new, start, pages in s["seqs"]:
        for b in range(start // BLOCK, (start + new - 1) // BLOCK + 1):
            lo, hi = max(start, b * BLOCK), min(start + new, (b + 1) * BLOCK)
            page, half_page = pages[b // 2], b % 2
            base = half_page * BLOCK
            for which, cache, first in ((0, K, H), (1, V, H + KV)):
                fresh = turned[row + lo - start: row + hi - start, first: first + KV]          # [n, KV, D]
                amax = fresh.abs().amax(dim=(0, 2)) / TOP
                e = torch.ceil(torch.log2(amax.clamp(min=2.0 ** LOWEST)))
                had = lo - b * BLOCK
                if had:
                    before = scales[page, :, which, half_page].double() - BIAS
                    e = torch.maximum(e, before)
                    cache[page, :, base: base + had] *= torch.exp2(before - e)[:, None, None]
                cache[page, :, base + had: base + had + hi - lo] = (fresh * torch.exp2(-e)[None, :, None]).transpose(0, 1)
                scales[page, :, which, half_page] = (e + BIAS).to(torch.uint8)
    return {"Q": turned[:, :H].reshape(M, H * D), "codes": _pack(K, V), "scales": torch.exp2(scales.double() - BIAS)}


def _attend64(case, s):
    H, KV, D, G = case["heads"], case["kv_heads"], case["head_dim"], case["heads"] // case["kv_heads"]
    out = torch.zeros(s["Q"].shape[0], H, D, device=DEV, dtype=torch.float64)
    for row, new, start, pages in s["seqs"]:
        ids = torch.tensor(pages, device=DEV)
        K, V = _unpack(s["codes"][ids], D)
        e = torch.exp2(s["scales"][ids].double() - BIAS)          # [pages, KV, 2, 2]
        for h in range(KV):
            k = (K[:, h].view(E4M3).double().reshape(-1, 2, BLOCK, D) * e[:, h, 0, :, None, None]).reshape(-1, D)[: start + new]
            v = (V[:, h].view(E4M3).double().reshape(-1, 2, BLOCK, D) * e[:, h, 1, :, None, None]).reshape(-1, D)[: start + new]
            pos, key = torch.arange(start, start + new, device=DEV)[:, None], torch.arange(start + new, device=DEV)[None]
            hidden = (key > pos) | ((key <= pos - s["window"]) if s["window"] else torch.zeros_like(key > pos))
            for g in range(G):
                q = s["Q"][row: row + new, (h * G + g) * D: (h * G + g + 1) * D].double()
                z = q @ k.T * s["scale"]
                if s["softcap"]:
                    z = s["softcap"] * torch.tanh(z / s["softcap"])
                out[row: row + new, h * G + g] = torch.softmax(z.masked_fill(hidden, -math.inf), dim=1) @ v
    return out.reshape(-1, H * D)
