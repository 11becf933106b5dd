"""The page-sparse decode attention operators, as cases to measure.

  append   aflex_rope_append_bounds   rotary embedding, K/V append and the touched pages' key bounds
  bounds   aflex_page_bounds          the key bounds of pages that something else filled
  select   aflex_page_select          the pages of the cache that each row's queries should read
  attend   aflex_attn_decode_pages    attention of each row over its listed pages

`run` computes an operator in plain torch operations (own = False) or calls the framework (own = True).
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
DEV = "cuda"
E_MIN, E_MAX = -60, 50            # shared exponents of the bounds and of the quantised queries


# ------------------------------------------------------------------------------------------ the cases
def listed():
    def c(name, op, **kw):
        base = dict(name=name, op=op, batch=1, rows=1, hq=64, hkv=8, d=128, lo=16, hi=128, top=0, sink=1, window=2, norm=False, theta=1.0e6)
        base.update(kw)
        return base
    return [
        # one decode step of the tiny layer: four sequences, what counts is the launch
        c("append-tiny", "append", batch=4, hq=8, hkv=2, d=64, lo=16, hi=128, norm=True, theta=1.0e4),
        # one decode step of a loaded Mixtral-shaped layer
        c("append-256", "append", batch=256, hq=32, lo=512, hi=2048),
        # ragged prompt chunks behind cached prefixes, Qwen3-32B-shaped layer with q / k norms
        c("append-chunks", "append", batch=7, rows=1171, lo=1171, hi=5400, norm=True),
        # a chunk of one prompt's cache that another engine filled
        c("bounds-short", "bounds", batch=3, hq=8, hkv=2, d=64, lo=17, hi=700),
        # the caches of a decode batch handed over from the prefill pool
        c("bounds-32", "bounds", batch=32, lo=512, hi=4096),
        # one user with a long context
        c("select-long", "select", batch=1, lo=131072, hi=131072, top=128),
        # a decode batch of conversations
        c("select-32", "select", batch=32, lo=512, hi=4096, top=64),
        # five drafted tokens per sequence to verify
        c("select-verify", "select", batch=16, rows=5, hq=32, lo=1024, hi=8192, top=96, window=4),
        # one user with a long context
        c("attend-long", "attend", batch=1, lo=131072, hi=131072, top=128),
        # a decode batch of conversations
        c("attend-32", "attend", batch=32, lo=512, hi=4096, top=64),
        # a loaded Mixtral-shaped layer with long prompts
        c("attend-256", "attend", batch=256, hq=32, lo=512, hi=8192, top=128),
        # four drafted tokens per sequence to verify, small heads
        c("attend-verify", "attend", batch=13, rows=4, hq=16, hkv=4, d=64, lo=700, hi=6000, top=50),
    ]


def draw(rng):
    logint = lambda a, b: int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))  # noqa: E731
    op = rng.choice(("append", "bounds", "select", "attend"))
    hkv = rng.choice((1, 2, 4, 8))
    g = rng.choice((1, 2, 4, 8))
    c = dict(op=op, batch=logint(1, 160), rows=1, hq=hkv * g, hkv=hkv, d=rng.choice((64, 128)), top=0,
             sink=rng.choice((0, 1, 2)), window=rng.choice((1, 2, 5)), norm=rng.random() < 0.5, theta=rng.choice((1.0e4, 5.0e5, 1.0e6)))
    # tokens of all caches together: at most about 400 K, so that a state stays small
    most = max(40, min(100000, 400000 // c["batch"]))
    c["hi"] = logint(33, most)
    c["lo"] = max(1, int(c["hi"] * rng.uniform(0.05, 1.0)))
    if op == "append" and rng.random() < 0.5:
        c["batch"] = min(c["batch"], 24)
        c["rows"] = min(c["lo"], logint(2, max(2, 8000 // c["batch"])))
    if op in ("select", "attend"):
        c["top"] = max(c["sink"] + c["window"], logint(4, 160))
        if rng.random() < 0.4:
            c["batch"] = min(c["batch"], 40)
            c["rows"] = min(c["lo"], rng.randint(2, 6))
    return c


def _lens(case):
    """Cached tokens of every sequence, the new ones included: spread over [lo, hi], the same for every seed."""
    gold = 0.6180339887498949
    return [case["lo"] + int((case["hi"] - case["lo"] + 1) * ((0.37 + b * gold) % 1.0)) for b in range(case["batch"])]


def _new(case):
    """Rows of every sequence; ragged for prompt chunks."""
    if case["op"] == "append" and case["rows"] > 1:
        return [max(1, case["rows"] - (b * 37) % (case["rows"] // 2 + 1)) for b in range(case["batch"])]
    return [case["rows"]] * case["batch"]


def work(case):
    lens, new, hq, hkv, d = _lens(case), _new(case), case["hq"], case["hkv"], case["d"]
    rows = sum(new)
    bound = 2 * d + d // 32
    pages = lambda n: (n + PAGE - 1) // PAGE  # noqa: E731
    if case["op"] == "append":
        touched = [(n - m) // PAGE for n, m in zip(lens, new)]
        old = sum(((n - m) % PAGE) for n, m in zip(lens, new))
        npg = sum(pages(n) - t for n, t in zip(lens, touched))
        byt = 2 * rows * (hq + 2 * hkv) * d * 2 + old * hkv * d * 2 + npg * hkv * bound
        return {"bytes": byt, "flops": rows * (hq + hkv) * d * 6}
    if case["op"] == "bounds":
        return {"bytes": sum(lens) * hkv * d * 2 + sum(pages(n) for n in lens) * hkv * bound, "flops": sum(lens) * hkv * d * 2}
    byt, flops = 0, 0
    for n, m in zip(lens, new):
        if case["op"] == "select":
            most = pages(n)
            cand = max(0, most - case["sink"] - case["window"]) if most > case["top"] else 0
            byt += cand * hkv * bound + m * hkv * (case["top"] + 1) * 4 + m * hq * d * 2
            flops += m * cand * hq * d * 2
        else:
            tok = [min(p + 1, case["top"] * PAGE - (PAGE - 1 - p % PAGE) if p // PAGE + 1 > case["top"] else p + 1) for p in range(n - m, n)]
            # rows of one sequence may list the same pages: at least the longest list has to be read
            byt += max(tok) * hkv * d * 4 + m * hq * d * 4 + m * hkv * (case["top"] + 1) * 4 + m * hq * 4
            flops += sum(tok) * hq * d * 4
    return {"bytes": byt, "flops": flops}


# ------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    lens, new, hkv, d = _lens(case), _new(case), case["hkv"], case["d"]
    B, T = case["batch"], sum(new)
    npg = [(n + PAGE - 1) // PAGE for n in lens]
    total = sum(npg) + 8
    perm = rng.permutation(total)
    table = np.zeros((B, max(npg)), dtype=np.int32)
    at = 0
    for b, n in enumerate(npg):
        table[b, :n] = perm[at:at + n]
        at += n
    s = {"case": case}
    # keys: some channels are much larger than others, and the tokens of a page resemble one another
    gain = torch.exp(0.7 * torch.randn(hkv, 1, d, generator=g, device=DEV))
    drift = torch.randn(total, hkv, 1, d, generator=g, device=DEV, dtype=torch.bfloat16)
    s["k"] = torch.randn(total, hkv, PAGE, d, generator=g, device=DEV, dtype=torch.bfloat16)
    s["k"].add_(drift).mul_(gain.to(torch.bfloat16))
    s["v"] = torch.randn(total, hkv, PAGE, d, generator=g, device=DEV, dtype=torch.bfloat16) if case["op"] in ("append", "attend") else s["k"]
    s["table"] = torch.from_numpy(table).to(DEV)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    offs = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    s["offsets"] = torch.from_numpy(offs).to(DEV) if case["rows"] > 1 else None
    s["codes"] = torch.zeros(total, hkv, d // 8, 2, 8, dtype=torch.int8, device=DEV)
    s["scales"] = torch.zeros(total, hkv, d // 32, dtype=torch.uint8, device=DEV)
    # where each row sits: its sequence and its position
    seq = np.repeat(np.arange(B), new)
    pos = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, new)])
    s["seq"], s["pos"] = torch.from_numpy(seq).to(DEV), torch.from_numpy(pos).to(DEV)
    if case["op"] == "append":
        s["qkv"] = torch.randn(T, (case["hq"] + 2 * hkv) * d, generator=g, device=DEV, dtype=torch.bfloat16)
        norm = lambda: (1 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16) if case["norm"] else None  # noqa: E731
        s["wq"], s["wk"] = norm(), norm()
        s["q"] = torch.empty(T, case["hq"], d, dtype=torch.bfloat16, device=DEV)
        # rows that end a page or a chunk: after them the page's keys are all there
        ends = (pos % PAGE == PAGE - 1) | (np.arange(T) == offs[1:][seq] - 1)
        s["ends"] = torch.from_numpy(np.nonzero(ends)[0]).to(DEV)
    else:
        s["q"] = torch.randn(T, case["hq"], d, generator=g, device=DEV, dtype=torch.bfloat16)
    if case["op"] in ("select", "bounds"):
        s["full_pages"] = torch.from_numpy(np.concatenate([table[b, :n] for b, n in enumerate(npg)]).astype(np.int64)).to(DEV)
        s["full_valid"] = torch.from_numpy(np.concatenate([np.minimum(PAGE, lens[b] - PAGE * np.arange(n)) for b, n in enumerate(npg)])).to(DEV)
    if case["op"] == "select":
        _bounds_plain(s, s["full_pages"], s["full_valid"])
        s["list"] = torch.empty(T, hkv, case["top"], dtype=torch.int32, device=DEV)
        s["count"] = torch.empty(T, hkv, dtype=torch.int32, device=DEV)
    if case["op"] == "attend":
        n = s["pos"] // PAGE + 1                                     # pages that a row can see
        width = int(n.max())
        key = torch.rand(T, hkv, width, generator=g, device=DEV)
        j = torch.arange(width, device=DEV)
        key = torch.where(j < n[:, None, None], key, torch.full_like(key, 2.0))
        key = torch.where(j == n[:, None, None] - 1, torch.full_like(key, -1.0), key)
        top = min(case["top"], width)
        chosen, order = torch.sort(key, dim=2, stable=True)
        lst = torch.where(chosen[:, :, :top] < 1.5, order[:, :, :top], torch.full_like(order[:, :, :top], width))
        lst = torch.sort(lst, dim=2)[0]
        lst = torch.where(lst < width, lst, torch.full_like(lst, -1))
        s["list"] = torch.full((T, hkv, case["top"]), -1, dtype=torch.int32, device=DEV)
        s["list"][:, :, :top] = lst.to(torch.int32)
        s["count"] = (s["list"] >= 0).sum(2).to(torch.int32)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(T, case["hq"], dtype=torch.float32, device=DEV)
    return s


_handle = []                      # the library context that a serving process keeps


def _framework(s):
    """The context for the framework's calls, made once a process; the descriptors are made once a state."""
    from paper_2608_01891_b200 import aflex as AF
    if not _handle:
        _handle.append(AF.Context(0, 64 << 20))
    if "desc" not in s:
        s["desc"] = AF.attn_desc(s["case"]["hq"], s["case"]["hkv"], s["case"]["d"])
        s["kv"] = AF.make_kv(s["k"], s["v"], s["table"], s["lens"])
        s["bounds"] = AF.make_page_bounds(s["codes"], s["scales"])
    return _handle[0]


# ------------------------------------------------------------------------------------------ plain forms
def _exponent(a):
    """Smallest e with a <= 127 * 2^e, in [E_MIN, E_MAX]; E_MIN where a is 0."""
    m, x = torch.frexp(a)
    e = torch.where(m * 128 > 127, x - 6, x - 7)
    e = torch.where(a == 0, torch.full_like(e, E_MIN), e)
    return torch.where(torch.isinf(a), torch.full_like(e, E_MAX), e).clamp(E_MIN, E_MAX)


def _pow2(e, like):
    return torch.ldexp(torch.ones_like(e, dtype=like), e)


def _bounds_plain(s, pages, valid):
    """Writes the bounds of the given physical pages, the first `valid` slots of each."""
    hkv, d = s["k"].shape[1], s["k"].shape[3]
    k = s["k"][pages].float()
    there = (torch.arange(PAGE, device=DEV) < valid[:, None])[:, None, :, None] & ~torch.isnan(k)
    hi = torch.where(there, k, torch.full_like(k, -math.inf)).amax(2)
    lo = torch.where(there, k, torch.full_like(k, math.inf)).amin(2)
    none = hi < lo
    hi = torch.where(none, torch.zeros_like(hi), hi).view(-1, hkv, d // 32, 32)
    lo = torch.where(none, torch.zeros_like(lo), lo).view(-1, hkv, d // 32, 32)
    e = _exponent(torch.maximum(hi.abs(), lo.abs()).amax(3))
    inv = _pow2(-e, torch.float32)[..., None]
    hi = torch.ceil(hi * inv).clamp(-127, 127).to(torch.int8).view(-1, hkv, d // 8, 1, 8)
    lo = torch.floor(lo * inv).clamp(-127, 127).to(torch.int8).view(-1, hkv, d // 8, 1, 8)
    s["codes"][pages] = torch.cat([hi, lo], 3)
    s["scales"][pages] = (e + 127).to(torch.uint8)


def _append_plain(s):
    c = s["case"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
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
    # keys in 64 bits: their bounds are whole numbers, which have to come out the same
    k = turn(x[:, hq:hq + hkv].double(), s["wk"], cos, sin).to(torch.bfloat16)
    page = s["table"][s["seq"], s["pos"] // PAGE].long()
    slot = s["pos"] % PAGE
    s["k"][page, :, slot] = k
    s["v"][page, :, slot] = x[:, hq + hkv:]
    _bounds_plain(s, page[s["ends"]], slot[s["ends"]] + 1)
    return {"q": s["q"], "k": s["k"], "v": s["v"], "codes": s["codes"], "scales": s["scales"]}


def _select_plain(s):
    c = s["case"]
    hkv, d, top = c["hkv"], c["d"], c["top"]
    G, C, B, R = c["hq"] // hkv, d // 32, c["batch"], c["rows"]
    q = s["q"].float().view(B, R, hkv, G, C, 32)
    q = torch.where(torch.isnan(q), torch.zeros_like(q), q)
    f = _exponent(q.abs().amax(5))
    qi = torch.round(q * _pow2(-f, torch.float32)[..., None]).clamp(-127, 127)
    table = s["table"].long()
    N = table.shape[1]
    b = s["codes"][table].float().view(B, N, hkv, C, 4, 2, 8)
    hi, lo = b[..., 0, :].reshape(B, N, hkv, C, 32), b[..., 1, :].reshape(B, N, hkv, C, 32)
    # sums of at most 32 products of at most 127 * 127: exact in 32 bits, in any order
    dot = torch.einsum("brhgcx,bnhcx->brhgcn", qi.clamp(min=0), hi) + torch.einsum("brhgcx,bnhcx->brhgcn", qi.clamp(max=0), lo)
    e = s["scales"][table].to(torch.int32).permute(0, 2, 3, 1) - 127                      # [B, hkv, C, N]
    v = dot * _pow2(e, torch.float32)[:, None, :, None] * _pow2(f, torch.float32)[..., None]
    score = v[..., 0, :]
    for k in range(1, C):
        score = score + v[..., k, :]
    score = score.amax(3).view(B * R, hkv, N)
    n = (s["pos"] // PAGE + 1)[:, None, None]
    j = torch.arange(N, device=DEV)
    forced = (j < n) & ((j < c["sink"]) | (j >= n - c["window"]) | (n <= top))
    rest = (j < n) & ~forced
    order = torch.sort(torch.where(rest, score, torch.full_like(score, -math.inf)), dim=2, descending=True, stable=True)[1]
    rank = torch.empty_like(order).scatter_(2, order, j.expand_as(order).contiguous())
    taken = forced | (rest & (rank < top - c["sink"] - c["window"]))
    at = torch.where(taken, torch.cumsum(taken, 2) - 1, torch.full_like(rank, top))
    lst = torch.full((B * R, hkv, top + 1), -1, dtype=torch.int32, device=DEV)
    lst.scatter_(2, at, j.to(torch.int32).expand_as(at).contiguous())
    return {"list": lst[:, :, :top], "count": taken.sum(2).to(torch.int32)}


def _attend_plain(s):
    c = s["case"]
    hkv, d, G = c["hkv"], c["d"], c["hq"] // c["hkv"]
    T = s["q"].shape[0]
    lst = s["list"].long()
    page = s["table"].long()[s["seq"][:, None, None], lst.clamp(min=0)]
    head = torch.arange(hkv, device=DEV)[None, :, None]
    tok = lst[..., None] * PAGE + torch.arange(PAGE, device=DEV)
    there = ((lst >= 0)[..., None] & (tok <= s["pos"][:, None, None, None])).view(T, hkv, 1, -1)
    k = s["k"][page, head].float().view(T, hkv, -1, d)
    x = torch.matmul(s["q"].float().view(T, hkv, G, d), k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    del k
    x = torch.where(there, x, torch.full_like(x, -math.inf))
    m = x.amax(3, keepdim=True)
    m0 = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    p = torch.exp(x - m0)
    l = p.sum(3, keepdim=True)
    v = s["v"][page, head].float().view(T, hkv, -1, d)
    v = torch.where(there.view(T, hkv, -1, 1), v, torch.zeros_like(v))
    out = torch.matmul(p, v) / torch.where(l > 0, l, torch.ones_like(l))
    return {"out": out.to(torch.bfloat16).view(T, c["hq"], d), "lse": (m0 + torch.log(l)).view(T, c["hq"])}


def run(s):
    c = s["case"]
    op = c["op"]
    if not own:
        if op == "append":
            return _append_plain(s)
        if op == "bounds":
            _bounds_plain(s, s["full_pages"], s["full_valid"])
            return {"codes": s["codes"], "scales": s["scales"]}
        return _select_plain(s) if op == "select" else _attend_plain(s)
    ctx = _framework(s)
    desc, kv, bounds = s["desc"], s["kv"], s["bounds"]
    if op == "attend":
        ctx.attn_decode_pages(desc, s["q"], kv, s["list"], s["count"], s["out"], s["lse"], q_offsets=s["offsets"])
        return {"out": s["out"], "lse": s["lse"]}
    if op == "append":
        ctx.rope_append_bounds(desc, s["qkv"], kv, bounds, s["q"], s["wq"], s["wk"], 1e-6, c["theta"], q_offsets=s["offsets"])
        return {"q": s["q"], "k": s["k"], "v": s["v"], "codes": s["codes"], "scales": s["scales"]}
    if op == "bounds":
        ctx.page_bounds(desc, kv, bounds, c["batch"])
        return {"codes": s["codes"], "scales": s["scales"]}
    ctx.page_select(desc, s["q"], kv, bounds, c["top"], s["list"], s["count"], sink_pages=c["sink"], window_pages=c["window"], q_offsets=s["offsets"])
    return {"list": s["list"], "count": s["count"]}


# ------------------------------------------------------------------------------------------ 64 bits
def _exact_bounds(k, codes, scales, page, valid):
    """Definition of one page's bounds, head by head and block by block, in 64 bits."""
    x = k[page, :, :valid].double()                                  # [hkv, valid, d]
    hi, lo = x.max(1)[0], x.min(1)[0]
    d = hi.shape[1]
    for c in range(d // 32):
        h, l = hi[:, 32 * c:32 * c + 32], lo[:, 32 * c:32 * c + 32]
        a = torch.maximum(h.abs(), l.abs()).max(1, keepdim=True)[0]
        e = torch.ceil(torch.log2(a / 127))
        e = torch.where(a / 127 <= 2.0 ** (e - 1), e - 1, torch.where(a / 127 > 2.0 ** e, e + 1, e)).clamp(E_MIN, E_MAX)
        e = torch.where(a > 0, e, torch.full_like(e, E_MIN))
        codes[page, :, 4 * c:4 * c + 4, 0] = torch.ceil(h / 2.0 ** e).clamp(-127, 127).to(torch.int8).view(-1, 4, 8)
        codes[page, :, 4 * c:4 * c + 4, 1] = torch.floor(l / 2.0 ** e).clamp(-127, 127).to(torch.int8).view(-1, 4, 8)
        scales[page, :, c] = (e[:, 0] + 127).to(torch.uint8)


def exact(case, seed):
    s = prepare(case, seed)
    hq, hkv, d, G = case["hq"], case["hkv"], case["d"], case["hq"] // case["hkv"]
    lens, new = _lens(case), _new(case)
    table = s["table"].cpu().numpy()
    if case["op"] in ("bounds", "select") and sum(lens) > 30 * PAGE * 100:
        return None                                                  # page by page it would take too long
    if case["op"] == "bounds":
        for b, n in enumerate(lens):
            for t in range(0, n, PAGE):
                _exact_bounds(s["k"], s["codes"], s["scales"], int(table[b, t // PAGE]), min(PAGE, n - t))
        return {"codes": s["codes"], "scales": s["scales"]}
    if case["op"] == "append":
        k64, v64 = s["k"].double(), s["v"].double()
        q64 = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
        inv = torch.tensor([case["theta"] ** (-2.0 * i / d) for i in range(d // 2)], dtype=torch.float64, device=DEV)
        r = 0
        for b, (n, m) in enumerate(zip(lens, new)):
            p = torch.arange(n - m, n, device=DEV)
            x = s["qkv"][r:r + m].double().view(m, hq + 2 * hkv, d)
            z = torch.polar(torch.ones(m, d // 2, dtype=torch.float64, device=DEV), p.double()[:, None] * inv)[:, None]
            for heads, w, is_q in ((x[:, :hq], s["wq"], True), (x[:, hq:hq + hkv], s["wk"], False)):
                if w is not None:
                    rms = (heads.square().sum(2, keepdim=True) / d + float(np.float32(1e-6))).sqrt()
                    heads = heads / rms * w.double()
                y = torch.complex(heads[..., : d // 2].contiguous(), heads[..., d // 2:].contiguous()) * z
                y = torch.cat([y.real, y.imag], 2)
                if is_q:
                    q64[r:r + m] = y
                else:
                    k64[torch.from_numpy(table[b]).to(DEV).long()[p // PAGE], :, p % PAGE] = y
            v64[torch.from_numpy(table[b]).to(DEV).long()[p // PAGE], :, p % PAGE] = x[:, hq + hkv:]
            r += m
        return {"q": q64, "k": k64, "v": v64, "codes": None, "scales": None}
    if case["op"] == "select":
        lists = np.full((s["q"].shape[0], hkv, case["top"]), -1, dtype=np.int32)
        counts = np.zeros((s["q"].shape[0], hkv), dtype=np.int32)
        codes, scales = s["codes"].cpu().numpy().astype(np.int64), s["scales"].cpu().numpy().astype(np.int64) - 127
        q = s["q"].double().cpu().numpy()
        seq, pos = s["seq"].cpu().numpy(), s["pos"].cpu().numpy()
        for r in range(q.shape[0]):
            n = int(pos[r]) // PAGE + 1
            pg = table[seq[r], :n]
            for g in range(hkv):
                if n <= case["top"]:
                    take = list(range(n))
                else:
                    best = np.full(n, -np.inf, dtype=np.float32)
                    for h in range(g * G, g * G + G):
                        total = None
                        for c in range(d // 32):
                            x = q[r, h, 32 * c:32 * c + 32]
                            a, f = np.abs(x).max(), E_MIN
                            while a > 127 * 2.0 ** f and f < E_MAX:
                                f += 1
                            xi = np.clip(np.rint(x / 2.0 ** f), -127, 127).astype(np.int64)
                            blk = codes[pg, g, 4 * c:4 * c + 4]
                            i = np.maximum(xi * blk[:, :, 0].reshape(n, 32), xi * blk[:, :, 1].reshape(n, 32)).sum(1)
                            v = (i * 2.0 ** (scales[pg, g, c] + f)).astype(np.float32)
                            total = v if total is None else (total + v).astype(np.float32)
                        best = np.maximum(best, total)
                    mid = range(case["sink"], n - case["window"])
                    mid = sorted(mid, key=lambda j: (-best[j], j))[: case["top"] - case["sink"] - case["window"]]
                    take = sorted(list(range(case["sink"])) + list(mid) + list(range(n - case["window"], n)))
                lists[r, g, : len(take)], counts[r, g] = take, len(take)
        return {"list": torch.from_numpy(lists), "count": torch.from_numpy(counts)}
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(out.shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    seq, pos, lists = s["seq"].cpu().numpy(), s["pos"].cpu().numpy(), s["list"].cpu().numpy()
    if out.shape[0] * hkv > 4000:
        return None
    for r in range(out.shape[0]):
        for g in range(hkv):
            js = lists[r, g][lists[r, g] >= 0]
            idx = torch.from_numpy(table[seq[r], js].astype(np.int64)).to(DEV)
            keep = torch.from_numpy((js[:, None] * PAGE + np.arange(PAGE) <= pos[r]).reshape(-1)).to(DEV)
            k, v = s["k"][idx, g].double().view(-1, d)[keep], s["v"][idx, g].double().view(-1, d)[keep]
            x = s["q"][r, g * G:g * G + G].double() @ k.T / math.sqrt(d)
            lse[r, g * G:g * G + G] = torch.logsumexp(x, 1)
            out[r, g * G:g * G + G] = torch.softmax(x, 1) @ v
    return {"out": out, "lse": lse}
