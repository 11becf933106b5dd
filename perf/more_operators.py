"""Operators on a cache of 16 or 8 bits and on drafted tokens, as cases to measure.

  append   aflex_cache_append    rotary embedding and K/V append, quantised as it is written; drafted trees' rows at their own positions
  convert  aflex_cache_convert   a bf16 cache quantised to 8 bits, an 8-bit cache read back to bf16
  attend   aflex_attn_draft      attention of single tokens, drafted chains and drafted trees over a cache of either kind
  accept   aflex_cache_accept    the accepted path of a drafted tree moved together in the caches of all layers

`run` computes an operator in plain torch operations (own = False) or calls the framework (own = True).
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
DEV = "cuda"
TOP = {"int8": 127.0, "e4m3": 448.0}                       # the largest code
STORE = {"bf16": torch.bfloat16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
LEAST = 2.0 ** -64                                         # the smallest scale


# ------------------------------------------------------------------------------------------ the cases
def listed():
    def c(name, op, **kw):
        base = dict(name=name, op=op, fmt="int8", back=False, batch=1, rows=1, tree=False, hq=64, hkv=8, d=128, lo=16, hi=128, norm=False,
                    theta=1.0e6, layers=1)
        base.update(kw)
        return base
    return [
        # one decode step of the tiny layer: four sequences, what counts is the launch
        c("append-tiny", "append", batch=4, hq=8, hkv=2, d=64, norm=True, theta=1.0e4),
        # drafted trees of a decode batch, Qwen3-32B-shaped layer with q / k norms
        c("append-trees", "append", fmt="e4m3", batch=32, rows=13, tree=True, lo=512, hi=4096, norm=True),
        # ragged prompt chunks behind cached prefixes
        c("append-chunks", "append", batch=7, rows=1171, lo=1171, hi=5400, norm=True),
        # the caches of a decode batch handed over from the prefill pool
        c("quantise-32", "convert", batch=32, lo=512, hi=4096),
        # one prompt's cache given back to an operator that reads bf16
        c("readback-1", "convert", fmt="e4m3", back=True, lo=5003, hi=5003),
        # one user with a long context
        c("attend-long", "attend", lo=131072, hi=131072),
        # a decode batch of conversations
        c("attend-32", "attend", fmt="e4m3", batch=32, lo=512, hi=4096),
        # a loaded Mixtral-shaped layer with long prompts
        c("attend-256", "attend", batch=256, hq=32, lo=512, hi=8192),
        # five drafted tokens in a row per sequence to verify over the bf16 cache, small heads
        c("attend-chain", "attend", fmt="bf16", batch=13, rows=5, hq=16, hkv=4, d=64, lo=700, hi=6000),
        # large drafted trees of a few users, to verify over the 8-bit cache
        c("attend-trees", "attend", batch=8, rows=61, tree=True, lo=2048, hi=16384),
        # one small tree was verified, the tiny model's layers
        c("accept-tiny", "accept", fmt="bf16", batch=3, rows=9, hq=8, hkv=2, d=64, layers=2),
        # a decode batch's trees were verified, all layers of a large model
        c("accept-64", "accept", batch=32, rows=29, lo=256, hi=512, layers=64),
    ]


def draw(rng):
    logint = lambda a, b: int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))  # noqa: E731
    op = rng.choice(("append", "convert", "attend", "attend", "accept"))
    hkv = rng.choice((1, 2, 4, 8))
    g = rng.choice((1, 2, 4, 8))
    c = dict(op=op, fmt=rng.choice(("bf16", "int8", "e4m3")), back=rng.random() < 0.5, batch=logint(1, 160), rows=1, tree=False, hq=hkv * g,
             hkv=hkv, d=rng.choice((64, 128)), norm=rng.random() < 0.5, theta=rng.choice((1.0e4, 5.0e5, 1.0e6)), layers=1)
    if op == "convert" and c["fmt"] == "bf16":
        c["fmt"] = "int8"
    if op == "accept":
        c["rows"], c["layers"] = rng.randint(2, 60), logint(1, 64)
        c["batch"] = min(c["batch"], 40)
        c["hi"] = logint(64, max(65, min(2000, 1000000 // (c["batch"] * c["layers"]))))
        c["lo"] = max(c["rows"], c["hi"] // 2)
        c["hi"] = max(c["hi"], c["lo"])
        return c
    # tokens of all caches together: at most about 400 K, so that a state stays small
    most = max(80, min(100000, 400000 // c["batch"]))
    c["hi"] = logint(33, most)
    c["lo"] = max(1, int(c["hi"] * rng.uniform(0.05, 1.0)))
    kind = rng.random()
    if op == "append" and kind < 0.4:
        c["batch"] = min(c["batch"], 24)
        c["rows"] = min(c["lo"], logint(2, max(2, 8000 // c["batch"])))
    elif op in ("append", "attend") and kind < 0.8:
        c["batch"] = min(c["batch"], 40)
        c["rows"] = min(c["lo"], logint(2, 64))
        c["tree"] = rng.random() < 0.6
    return c


def _lens(case):
    """Cached tokens of every sequence, the new ones included: spread over [lo, hi], the same for every seed."""
    gold = 0.6180339887498949
    return [case["lo"] + int((case["hi"] - case["lo"] + 1) * ((0.37 + b * gold) % 1.0)) for b in range(case["batch"])]


def _new(case):
    """Rows of every sequence; ragged where there are several."""
    if case["rows"] > 1 and case["op"] != "accept":
        return [max(1, case["rows"] - (b * 37) % (case["rows"] // 2 + 1)) for b in range(case["batch"])]
    return [case["rows"]] * case["batch"]


def _path_len(case, b):
    """Accepted tokens of a sequence's tree; none for some."""
    return (3 + 5 * b) % min(9, case["rows"] + 1)


def work(case):
    lens, new, hq, hkv, d = _lens(case), _new(case), case["hq"], case["hkv"], case["d"]
    rows = sum(new)
    token = hkv * d * 4 if case["fmt"] == "bf16" else hkv * (2 * d + 8)          # K and V of a token, its scales among them
    if case["op"] == "append":
        return {"bytes": rows * ((2 * hq + 2 * hkv) * d * 2 + token), "flops": rows * (hq + hkv) * d * 6}
    if case["op"] == "convert":
        return {"bytes": sum(lens) * (token + hkv * d * 4), "flops": sum(lens) * hkv * d * 4}
    if case["op"] == "accept":
        moved = sum(_path_len(case, b) for b in range(case["batch"]))
        return {"bytes": 2 * moved * token * case["layers"], "flops": 0}
    return {"bytes": sum(lens) * token + rows * hq * (4 * d + 4), "flops": 4 * d * hq * sum(n * m for n, m in zip(lens, new))}


# ------------------------------------------------------------------------------------------ inputs
def _quantise(x, fmt):
    """Codes and scales of the last axis: scale = max |x| / TOP in 32 bits, code = x * (1 / scale) rounded to nearest, halves to even."""
    x = x.float()
    scale = (x.abs().amax(-1) * float(np.float32(1.0 / TOP[fmt]))).clamp(min=LEAST)
    y = (x * torch.reciprocal(scale)[..., None]).clamp(-TOP[fmt], TOP[fmt])
    return (torch.round(y) if fmt == "int8" else y).to(STORE[fmt]), scale


def _trees(case, new, rng):
    """Ancestors (each row's own token among them) of every drafted token, as bits, and depths, sequence after sequence."""
    words = (max(new) + 31) // 32
    mask, depth = np.zeros((sum(new), words), dtype=np.uint32), np.zeros(sum(new), dtype=np.int64)
    r = 0
    for m in new:
        for j in range(m):
            # a few children of the root, then mostly chains with side branches
            parent = -1 if j == 0 or rng.random() < 0.08 else int(rng.integers(max(0, j - 6), j))
            if parent >= 0:
                mask[r + j] = mask[r + parent]
                depth[r + j] = depth[r + parent] + 1
            mask[r + j, j // 32] |= np.uint32(1 << (j % 32))
        r += m
    return mask, depth


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    lens, new, hkv, d, fmt = _lens(case), _new(case), case["hkv"], case["d"], case["fmt"]
    B, T = case["batch"], sum(new)
    npg = [(n + PAGE - 1) // PAGE for n in lens]
    total = sum(npg) + 8
    perm = rng.permutation(total)
    table = np.zeros((B, max(npg)), dtype=np.int32)
    at = 0
    for b, n in enumerate(npg):
        table[b, :n] = perm[at:at + n]
        at += n
    s = {"case": case, "table": torch.from_numpy(table).to(DEV), "lens": torch.tensor(lens, dtype=torch.int32, device=DEV)}
    gain = torch.exp(0.7 * torch.randn(hkv, 1, d, generator=g, device=DEV)).to(torch.bfloat16)     # some key channels are much larger
    draw16 = lambda *shape: torch.randn(*shape, generator=g, device=DEV, dtype=torch.bfloat16)  # noqa: E731

    def pool(kind):
        """k, v and their scales (None for bf16) of one layer."""
        k, v = draw16(total, hkv, PAGE, d).mul_(gain), draw16(total, hkv, PAGE, d)
        if kind == "bf16":
            return k, v, None, None
        (k, ks), (v, vs) = _quantise(k, kind), _quantise(v, kind)
        return k, v, ks, vs

    if case["op"] == "convert":
        s["src"] = pool(fmt if case["back"] else "bf16")
        to = "bf16" if case["back"] else fmt
        empty = lambda t, *shape: torch.zeros(*shape, device=DEV).to(t)  # noqa: E731
        shape = (total, hkv, PAGE, d)
        s["dst"] = (empty(STORE[to], *shape), empty(STORE[to], *shape), *((None, None) if to == "bf16" else (empty(torch.float32, *shape[:3]) for _ in range(2))))
        # every cached token's page and slot, the same in both caches
        seq = np.repeat(np.arange(B), lens)
        tok = np.concatenate([np.arange(n) for n in lens])
        s["page"], s["slot"] = torch.from_numpy(table[seq, tok // PAGE].astype(np.int64)).to(DEV), torch.from_numpy(tok % PAGE).to(DEV)
        return s
    layers = [pool(fmt) for _ in range(case["layers"])]
    s["stacks"] = [None if t[0] is None else torch.stack(t) for t in zip(*layers)]               # of all layers, one after another
    s["caches"] = [tuple(None if t is None else t[l] for t in s["stacks"]) for l in range(case["layers"])]
    del layers
    if case["op"] == "accept":
        base = np.array([n - case["rows"] for n in lens], dtype=np.int32)
        path, count = np.zeros((B, case["rows"]), dtype=np.int32), np.zeros(B, dtype=np.int32)
        for b in range(B):
            n = _path_len(case, b)
            # levels of a tree: an accepted token either stays where it is or comes from behind the accepted ones
            stay = int(rng.integers(0, n + 1)) if n < case["rows"] else n
            rest = np.arange(n, case["rows"])
            stay = max(stay, n - len(rest))
            path[b, :stay] = np.arange(stay)
            path[b, stay:n] = np.sort(rng.choice(rest, n - stay, replace=False))
            count[b] = n
        s["base"], s["path"], s["count"] = (torch.from_numpy(x).to(DEV) for x in (base, path, count))
        seq = np.repeat(np.arange(B), count)
        k = np.concatenate([np.arange(n) for n in count])
        frm, to = base[seq] + path[seq, k], base[seq] + k
        for name, t in (("from", frm), ("to", to)):
            s[name] = (torch.from_numpy(table[seq, t // PAGE].astype(np.int64)).to(DEV), torch.from_numpy(t.astype(np.int64) % PAGE).to(DEV))
        return s
    offs = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    s["offsets"] = torch.from_numpy(offs).to(DEV) if case["rows"] > 1 else None
    seq = np.repeat(np.arange(B), new)
    idx = np.concatenate([np.arange(m) for m in new])
    ctx = np.array(lens)[seq] - np.array(new)[seq]
    mask, depth = _trees(case, new, rng) if case["tree"] else (None, idx)
    s["mask"] = torch.from_numpy(mask.view(np.int32)).to(DEV) if case["tree"] else None
    s["positions"] = torch.from_numpy((ctx + depth).astype(np.int32)).to(DEV) if case["tree"] else None
    s["seq"], s["idx"], s["pos"] = (torch.from_numpy(x).to(DEV) for x in (seq, idx, ctx + depth))
    s["slot"] = torch.from_numpy(ctx + idx).to(DEV)                          # where each row's token lies in its sequence
    if case["op"] == "append":
        s["qkv"] = draw16(T, (case["hq"] + 2 * hkv) * d)
        norm = lambda: (1 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16) if case["norm"] else None  # noqa: E731
        s["wq"], s["wk"] = norm(), norm()
        s["q"] = torch.empty(T, case["hq"], d, dtype=torch.bfloat16, device=DEV)
    else:
        s["q"] = draw16(T, case["hq"], d)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(T, case["hq"], dtype=torch.float32, device=DEV)
    return s


_handle = []                      # the library context that a serving process keeps


def _framework(s):
    """The context for the framework's calls, made once a process; the descriptors are made once a state."""
    from paper_2608_01891_b200 import aflex as AF
    if not _handle:
        _handle.append(AF.Context(0, 128 << 20))
    if "desc" not in s:
        c = s["case"]
        s["desc"] = AF.attn_desc(c["hq"], c["hkv"], c["d"])
        make = lambda p: AF.make_cache(p[0], p[1], s["table"], s["lens"], p[2], p[3])  # noqa: E731
        if c["op"] == "convert":
            s["from_cache"], s["to_cache"] = make(s["src"]), make(s["dst"])
        else:
            s["made"] = [make(p) for p in s["caches"]]
        s["draft"] = AF.draft_rows(s["offsets"], s["positions"], s["mask"]) if s.get("offsets") is not None else None
    return _handle[0]


# ------------------------------------------------------------------------------------------ plain forms
def _append_plain(s):
    c = s["case"]
    hq, hkv, d, fmt = c["hq"], c["hkv"], c["d"], c["fmt"]
    x = s["qkv"].view(-1, hq + 2 * hkv, d)
    i = torch.arange(d // 2, device=DEV, dtype=torch.float64)
    ang = s["pos"].double()[:, None] * c["theta"] ** (-2.0 * i / d)
    cos, sin = torch.cos(ang)[:, None, :], torch.sin(ang)[:, None, :]
    eps = float(np.float32(1e-6))

    def turn(v, w, cos, sin):
        if w is not None:
            v = v * (1.0 / torch.sqrt((v * v).mean(2, keepdim=True) + eps)) * w.to(v.dtype)
        a, b = v[..., : d // 2], v[..., d // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], 2)

    s["q"].copy_(turn(x[:, :hq].float(), s["wq"], cos.float(), sin.float()))
    # keys in 64 bits: their codes are whole numbers, which have to come out the same
    k, v = turn(x[:, hq:hq + hkv].double(), s["wk"], cos, sin).to(torch.bfloat16), x[:, hq + hkv:]
    kc, vc, ks, vs = s["caches"][0]
    page, slot = s["table"][s["seq"], s["slot"] // PAGE].long(), s["slot"] % PAGE
    if fmt == "bf16":
        kc[page, :, slot], vc[page, :, slot] = k, v
        return {"q": s["q"], "k": kc, "v": vc}
    (k, k_scale), (v, v_scale) = _quantise(k, fmt), _quantise(v, fmt)
    raw = lambda t: t.view(torch.int8)  # noqa: E731
    raw(kc)[page, :, slot], raw(vc)[page, :, slot] = raw(k), raw(v)
    ks[page, :, slot], vs[page, :, slot] = k_scale, v_scale
    return {"q": s["q"], "k": kc, "v": vc, "k_scales": ks, "v_scales": vs}


def _convert_plain(s):
    c, page, slot = s["case"], s["page"], s["slot"]
    raw = lambda t: t.view(torch.int8) if t.dtype == torch.float8_e4m3fn else t  # noqa: E731
    values = lambda t, at: raw(t)[at].view(t.dtype).float()  # noqa: E731
    (k, v, ks, vs), (k2, v2, ks2, vs2) = s["src"], s["dst"]
    at = (page, slice(None), slot)
    if c["back"]:
        k2[at] = (values(k, at) * ks[at][..., None]).to(torch.bfloat16)
        v2[at] = (values(v, at) * vs[at][..., None]).to(torch.bfloat16)
        return {"k": k2, "v": v2}
    code, ks2[at] = _quantise(k[at], c["fmt"])
    raw(k2)[at] = raw(code)
    code, vs2[at] = _quantise(v[at], c["fmt"])
    raw(v2)[at] = raw(code)
    return {"k": k2, "v": v2, "k_scales": ks2, "v_scales": vs2}


def _visible(s, m, N):
    """[batch, m, N]: which cached tokens each row sees, rows past a sequence's last see none."""
    c = s["case"]
    B = c["batch"]
    new = torch.bincount(s["seq"], minlength=B)
    ctx = (s["lens"] - new)[:, None, None]
    t, i = torch.arange(N, device=DEV), torch.arange(m, device=DEV)[:, None]
    if s["mask"] is None:
        return (t <= ctx + i) & (i < new[:, None, None])
    bits = torch.zeros(B, m, s["mask"].shape[1], dtype=torch.int64, device=DEV)
    bits[s["seq"], s["idx"]] = s["mask"].long()
    j = (t - ctx).expand(B, 1, N)
    word = torch.gather(bits, 2, (j // 32).clamp(0, bits.shape[2] - 1).expand(B, m, N))
    seen = (word >> (j % 32)) & 1
    return ((j < 0) | ((j < new[:, None, None]) & (seen == 1))) & (i < new[:, None, None])


def _attend_plain(s):
    c = s["case"]
    B, hq, hkv, d, m = c["batch"], c["hq"], c["hkv"], c["d"], max(_new(c))
    G = hq // hkv
    k, v, ks, vs = s["caches"][0]
    table = s["table"].long()
    N = table.shape[1] * PAGE

    def gather(x, scale):
        """[batch, hkv, N, d] in 32 bits."""
        y = (x.view(torch.int8)[table].view(x.dtype) if x.dtype == torch.float8_e4m3fn else x[table]).float()
        if scale is not None:
            y = y * scale[table][..., None]
        return y.permute(0, 2, 1, 3, 4).reshape(B, hkv, N, d)

    q = torch.zeros(B, m, hq, d, device=DEV)
    q[s["seq"], s["idx"]] = s["q"].float()
    q = q.view(B, m, hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, m * G, d)
    x = torch.matmul(q, gather(k, ks).transpose(2, 3)) * (1.0 / math.sqrt(d))
    see = _visible(s, m, N)[:, None, :, None, :]
    x = x.view(B, hkv, m, G, N)
    x = torch.where(see, x, torch.full_like(x, -math.inf))
    top = x.amax(4, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = torch.exp(x - top)
    del x
    total = p.sum(4, keepdim=True)
    out = torch.matmul(p.view(B, hkv, m * G, N), gather(v, vs)).view(B, hkv, m, G, d) / torch.where(total > 0, total, torch.ones_like(total))
    rows = lambda y: y.permute(0, 2, 1, 3, 4).reshape(B, m, hq, -1)[s["seq"], s["idx"]]  # noqa: E731
    return {"out": rows(out).to(torch.bfloat16), "lse": rows(top + torch.log(total))[..., 0]}


def _accept_plain(s):
    (page0, slot0), (page1, slot1) = s["from"], s["to"]
    raw = lambda t: t.view(torch.int8) if t.dtype == torch.float8_e4m3fn else t  # noqa: E731
    for t in s["stacks"]:
        if t is not None:
            raw(t)[:, page1, :, slot1] = raw(t)[:, page0, :, slot0]
    return {"caches": [t for t in s["stacks"] if t is not None]}


def run(s):
    c = s["case"]
    op = c["op"]
    if not own:
        return {"append": _append_plain, "convert": _convert_plain, "attend": _attend_plain, "accept": _accept_plain}[op](s)
    ctx = _framework(s)
    desc = s["desc"]
    if op == "attend":
        ctx.attn_draft(desc, s["q"], s["made"][0], s["out"], s["lse"], draft=s["draft"])
        return {"out": s["out"], "lse": s["lse"]}
    if op == "append":
        ctx.cache_append(desc, s["qkv"], s["made"][0], s["q"], s["wq"], s["wk"], 1e-6, c["theta"], draft=s["draft"])
        k, v, ks, vs = s["caches"][0]
        return {"q": s["q"], "k": k, "v": v} if ks is None else {"q": s["q"], "k": k, "v": v, "k_scales": ks, "v_scales": vs}
    if op == "convert":
        ctx.cache_convert(desc, s["from_cache"], s["to_cache"], c["batch"])
        k, v, ks, vs = s["dst"]
        return {"k": k, "v": v} if ks is None else {"k": k, "v": v, "k_scales": ks, "v_scales": vs}
    ctx.cache_accept(desc, s["made"], c["batch"], s["base"], s["path"], s["count"])
    return {"caches": [t for t in s["stacks"] if t is not None]}


# ------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    if case["op"] == "accept":
        return None                                                  # nothing is computed
    s = prepare(case, seed)
    hq, hkv, d, G, fmt = case["hq"], case["hkv"], case["d"], case["hq"] // case["hkv"], case["fmt"]
    lens, new = _lens(case), _new(case)
    table = s["table"].long()

    def codes_of(x):
        """Scale, and the quotient that the code is the rounding of."""
        scale = torch.clamp(x.abs().max(-1)[0] / TOP[fmt], min=LEAST)
        return x / scale[..., None], scale

    if case["op"] == "convert":
        (k, v, ks, vs), (k2, v2, ks2, vs2) = s["src"], s["dst"]
        page, slot = s["page"], s["slot"]
        if case["back"]:
            for x, sc, y in ((k, ks, "k"), (v, vs, "v")):
                full = torch.zeros(x.shape, dtype=torch.float64, device=DEV)
                full[page, :, slot] = (x.double() * sc.double()[..., None])[page, :, slot]
                s[y] = full
            return {"k": s["k"], "v": s["v"]}
        res = {}
        for name, x in (("k", k), ("v", v)):
            y, sc = codes_of(x.double()[page, :, slot])
            codes = torch.zeros(x.shape, dtype=torch.float64, device=DEV)
            scales = torch.zeros(x.shape[:3], dtype=torch.float64, device=DEV)
            codes[page, :, slot], scales[page, :, slot] = y, sc
            res[name], res[name + "_scales"] = (codes if fmt == "e4m3" else None), scales
        return {"k": res["k"], "v": res["v"], "k_scales": res["k_scales"], "v_scales": res["v_scales"]}
    if case["op"] == "append":
        k, v, ks, vs = s["caches"][0]
        x = s["qkv"].double().view(-1, hq + 2 * hkv, d)
        inv = torch.tensor([case["theta"] ** (-2.0 * i / d) for i in range(d // 2)], dtype=torch.float64, device=DEV)
        z = torch.polar(torch.ones(x.shape[0], d // 2, dtype=torch.float64, device=DEV), s["pos"].double()[:, None] * inv)[:, None]

        def turned(heads, w):
            if w is not None:
                heads = heads / (heads.square().sum(2, keepdim=True) / d + float(np.float32(1e-6))).sqrt() * w.double()
            y = torch.complex(heads[..., : d // 2].contiguous(), heads[..., d // 2:].contiguous()) * z
            return torch.cat([y.real, y.imag], 2)

        q64, key, value = turned(x[:, :hq], s["wq"]), turned(x[:, hq:hq + hkv], s["wk"]), x[:, hq + hkv:]
        page, slot = table[s["seq"], s["slot"] // PAGE], s["slot"] % PAGE
        k64, v64 = k.double(), v.double()
        if fmt == "bf16":
            k64[page, :, slot], v64[page, :, slot] = key, value
            return {"q": q64, "k": k64, "v": v64}
        ks64, vs64 = ks.double(), vs.double()
        # (the cache holds bf16 keys' codes: the rounding before is part of the definition)
        k64[page, :, slot], ks64[page, :, slot] = codes_of(key.to(torch.bfloat16).double())
        v64[page, :, slot], vs64[page, :, slot] = codes_of(value)
        return {"q": q64, "k": k64 if fmt == "e4m3" else None, "v": v64 if fmt == "e4m3" else None, "k_scales": ks64, "v_scales": vs64}
    if sum(n * m for n, m in zip(lens, new)) * hq * d > 4.0e12:
        return None
    k, v, ks, vs = s["caches"][0]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(out.shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    mask = None if s["mask"] is None else s["mask"].cpu().numpy().view(np.uint32)
    r = 0
    for b, (n, m) in enumerate(zip(lens, new)):
        ids = table[b, : (n + PAGE - 1) // PAGE]
        see = np.ones((m, n), dtype=bool)
        for i in range(m):
            for j in range(m):
                see[i, n - m + j] = j <= i if mask is None else bool((int(mask[r + i, j // 32]) >> (j % 32)) & 1)
        see = torch.from_numpy(see).to(DEV).repeat_interleave(G, 0)
        for g in range(hkv):
            flat = lambda x, sc: (x[ids, g].double() if sc is None else x.view(torch.int8)[ids, g].view(x.dtype).double() * sc[ids, g].double()[..., None]).reshape(-1, d)[:n]  # noqa: E731
            x = s["q"][r:r + m, g * G:g * G + G].double().reshape(m * G, d) @ flat(k, ks).T / math.sqrt(d)
            x = x.masked_fill(~see, -math.inf)
            lse[r:r + m, g * G:g * G + G] = torch.logsumexp(x, 1).view(m, G)
            out[r:r + m, g * G:g * G + G] = (torch.softmax(x, 1) @ flat(v, vs)).view(m, G, d)
        r += m
    return {"out": out, "lse": lse}
