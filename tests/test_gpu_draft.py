"""Caches of 16 or 8 bits and drafted tokens (aflex_cache_append, aflex_cache_convert, aflex_attn_draft, aflex_cache_accept,
aflex_draft_layers) on the GPU against the plain definitions in 64 bits, at the sizes where such operators go wrong, and run together."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as DO
from paper_2608_01891_b200 import aflex as AF
from tests.helpers import f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF_STEP = 2.0 ** -8                     # bf16: a rounding is off by at most eps / 2, relative to the value
TYPES = {"bf16": torch.bfloat16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
FORMATS = list(TYPES)
EPS = float(np.float32(1e-6))


@pytest.fixture
def ctx():
    c = AF.Context(0, 1 << 27)
    yield c
    c.close()


def raw(t):
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


def values(t):
    """A cache tensor's codes or values in 64 bits on the host."""
    return t.detach().to(torch.float32).cpu().to(torch.float64).numpy()


class Cache:
    """A paged cache with shuffled pages.  Slots and pages of no sequence hold NaN (or the codes and scales of garbage) unless asked otherwise."""

    def __init__(self, lens, Hkv, D, fmt, seed=0, poison=True, max_pages=None):
        g = torch.Generator().manual_seed(seed)
        self.lens = np.asarray(lens, dtype=np.int32)
        npg = (np.maximum(self.lens, 0) + 15) // 16
        self.total = int(npg.sum()) + 3
        width = max_pages or max(1, int(npg.max()))
        perm = np.random.default_rng(seed).permutation(self.total)
        self.table = np.full((len(lens), width), -7, dtype=np.int32)      # entries past a sequence's pages are never looked at
        at = 0
        for b, n in enumerate(npg):
            self.table[b, :n] = perm[at:at + n]
            at += n
        shape = (self.total, Hkv, 16, D)
        k = (torch.randn(shape, generator=g) * torch.exp(0.7 * torch.randn(Hkv, 1, D, generator=g))).to(torch.bfloat16)
        v = torch.randn(shape, generator=g).to(torch.bfloat16)
        used = torch.zeros(self.total, 16, dtype=torch.bool)
        for b, n in enumerate(self.lens):
            for j in range(int(n)):
                used[int(self.table[b, j // 16]), j % 16] = True
        self.used, self.fmt, self.Hkv, self.D = used, fmt, Hkv, D
        if fmt == "bf16":
            self.tensors = [k, v, None, None]
        else:
            (kc, ks), (vc, vs) = DO.quantise(f64(k), fmt), DO.quantise(f64(v), fmt)
            cast = lambda x: torch.from_numpy(x).float().to(TYPES[fmt])  # noqa: E731
            self.tensors = [cast(kc), cast(vc), torch.from_numpy(ks).float(), torch.from_numpy(vs).float()]
        if poison:
            for t in self.tensors:
                if t is None:
                    continue
                free = ~used[:, None, :].expand(self.total, Hkv, 16)
                if t.dtype == torch.int8:
                    t[free] = -128
                elif t.dtype == torch.float8_e4m3fn:
                    t.view(torch.uint8)[free] = 0x7f                       # NaN
                else:
                    t[free] = float("nan")
        self.put()

    def put(self):
        self.dev = [None if t is None else raw(t).to(DEV).view(t.dtype) for t in self.tensors]
        self.td, self.ld = torch.from_numpy(self.table).to(DEV), torch.from_numpy(self.lens).to(DEV)
        self.cache = AF.make_cache(self.dev[0], self.dev[1], self.td, self.ld, self.dev[2], self.dev[3])

    def stands_for(self):
        """k, v in 64 bits."""
        k, v, ks, vs = self.tensors
        if self.fmt == "bf16":
            return f64(k), f64(v)
        return values(k) * f64(ks)[..., None], values(v) * f64(vs)[..., None]


def offsets_of(new):
    return None if new is None else np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


def random_masks(rng, new, kind):
    """Masks as whole numbers and as device words; kind: "tree", "any" (a row may see none of the drafted tokens), "none"."""
    if kind == "chain" or new is None:
        return None, None
    words, ints = max(1, (max(new) + 31) // 32), []
    for m in new:
        seen = []
        for i in range(m):
            if kind == "tree":
                parent = int(rng.integers(-1, i)) if i else -1
                seen.append((seen[parent] if parent >= 0 else 0) | 1 << i)
            elif kind == "none":
                seen.append(0)
            else:
                seen.append(int.from_bytes(rng.bytes(64), "little") & ((1 << m) - 1) if rng.random() < 0.8 else 0)
        ints += seen
    a = np.array([[(s >> 32 * w) & 0xffffffff for w in range(words)] for s in ints], dtype=np.uint32).reshape(len(ints), words)
    return ints, torch.from_numpy(a.view(np.int32)).to(DEV)


# --------------------------------------------------------------------------- append
APPEND = [  # Hq, Hkv, D, norm, theta, lens, new tokens (None: one row per sequence), positions of a tree
    (8, 2, 64, True, 1e4, [1, 16, 17, 15, 32, 33], None, False),
    (8, 8, 128, False, 1e6, [1, 2, 160, 31], None, False),
    (64, 8, 128, True, 1e6, [5, 48, 49], None, False),
    (8, 1, 128, True, 5e5, [4000], None, False),
    (5, 5, 64, False, 1e4, list(range(1, 40)), None, False),
    (1, 1, 64, True, 1e4, [16], [16], False),
    (16, 4, 128, True, 1e6, [37, 16, 100, 33, 5, 64], [37, 0, 1, 17, 5, 33], True),
    (8, 2, 64, False, 1e4, [70, 300, 18], [3, 259, 2], True),
    (4, 1, 64, True, 1e4, [20 + i % 9 for i in range(300)], [1 + i % 4 for i in range(300)], False),
    (32, 8, 128, True, 1e6, [500], [490], False),
]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("Hq,Hkv,D,norm,theta,lens,new,tree", APPEND)
def test_append_matches_the_definition(ctx, fmt, Hq, Hkv, D, norm, theta, lens, new, tree):
    c = Cache(lens, Hkv, D, fmt, seed=len(lens) + D)
    offs = offsets_of(new)
    T = len(lens) if new is None else int(offs[-1])
    pad = 0 if new is None else 5
    g = torch.Generator().manual_seed(7)
    qkv = torch.randn(T + pad, (Hq + 2 * Hkv) * D, generator=g).to(torch.bfloat16)
    qkv[0, Hq * D:(Hq + 1) * D] = 0                                       # a head of zeros: the least scale
    gain = lambda: (1 + 0.1 * torch.randn(D, generator=g)).to(torch.bfloat16) if norm else None  # noqa: E731
    wq, wk = gain(), gain()
    pos = None
    if tree:
        pos = np.random.default_rng(3).integers(0, 200000, T + pad).astype(np.int32)
        pos[1:T // 2] = pos[0] + np.arange(1, T // 2) // 2                # some equal, some one on
    q = torch.full((T + pad, Hq, D), 3.25, dtype=torch.bfloat16, device=DEV)
    dev = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    dr = None if new is None else AF.draft_rows(torch.from_numpy(offs).to(DEV), None if pos is None else torch.from_numpy(pos).to(DEV))
    ctx.cache_append(AF.attn_desc(Hq, Hkv, D), qkv.to(DEV), c.cache, q, dev(wq), dev(wk), 1e-6, theta, draft=dr)
    assert ctx.device_status() == AF.OK
    want_q, size, put = DO.append(f64(qkv), c.table, lens, offs, pos, Hq, Hkv, None if wq is None else f64(wq), None if wk is None else f64(wk), EPS, theta)
    # q: one rounding to bf16, and in 32 bits: norm (D products and adds, a reciprocal root), sine, cosine (2 steps each),
    # two products and a sum, each within 2^-23 of |a| + |b|
    err = np.abs(f64(q)[:T] - want_q[:T])
    assert (err <= HALF_STEP * np.abs(want_q[:T]) + (D + 16) * 2.0 ** -23 * size[:T]).all()
    assert (q[T:] == 3.25).all()                                          # padding rows stay
    # keys are formed in 64 bits, so codes and scales are the same, bit for bit; everything else in the cache is as it was
    want = [None if t is None else values(t).copy() for t in c.tensors]
    for page, slot, key, value in put:
        for at, x in ((0, key), (1, value)):
            if fmt == "bf16":
                want[at][page, :, slot] = x
            else:
                want[at][page, :, slot], want[at + 2][page, :, slot] = DO.quantise(x, fmt)
    for got, w in zip(c.dev, want):
        if w is not None:
            np.testing.assert_array_equal(values(got), w)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_of_infinities_and_extreme_sizes(ctx, fmt):
    Hq, Hkv, D = 2, 2, 64
    c = Cache([7] * 6, Hkv, D, fmt)
    qkv = torch.randn(6, (Hq + 2 * Hkv) * D).to(torch.bfloat16)
    v0 = (Hq + Hkv) * D
    qkv[0, v0 + 3], qkv[1, v0 + 5], qkv[2, v0 + 9] = float("inf"), float("nan"), -float("inf")
    qkv[3, v0:] *= 1e38 / qkv[3, v0:].abs().max()
    qkv[4, v0:] *= 1e-30
    qkv[5, v0:] = torch.tensor([2.0 ** -133, -(2.0 ** -130)] * D).to(torch.bfloat16)
    q = torch.zeros(6, Hq, D, dtype=torch.bfloat16, device=DEV)
    ctx.cache_append(AF.attn_desc(Hq, Hkv, D), qkv.to(DEV), c.cache, q, None, None, 1e-6, 1e4)
    assert ctx.device_status() == AF.OK
    for b in range(6):
        x = f64(qkv[b, v0:].view(Hkv, D))
        got = values(c.dev[1])[c.table[b, 0], :, 6]
        if fmt == "bf16":
            np.testing.assert_array_equal(got, x)
        else:
            code, scale = DO.quantise(x, fmt)
            np.testing.assert_array_equal(got, code)
            np.testing.assert_array_equal(f64(c.dev[3])[c.table[b, 0], :, 6], scale)


def test_append_does_not_depend_on_chunking_and_agrees_with_the_bf16_operator(ctx):
    Hq, Hkv, D, n, m = 16, 2, 128, 61, 45
    g = torch.Generator().manual_seed(1)
    qkv = torch.randn(m, (Hq + 2 * Hkv) * D, generator=g).to(torch.bfloat16).to(DEV)
    w = (1 + 0.1 * torch.randn(D, generator=g)).to(torch.bfloat16).to(DEV)
    desc = AF.attn_desc(Hq, Hkv, D)
    got = []
    for fmt in ("int8", "bf16"):
        for cuts in ([0, 45], [0, 1, 2, 19, 20, 45], list(range(46))):
            c = Cache([n], Hkv, D, fmt, seed=5, poison=False)
            q = torch.zeros(m, Hq, D, dtype=torch.bfloat16, device=DEV)
            for a, b in zip(cuts[:-1], cuts[1:]):
                c.ld.fill_(n - m + b)
                ctx.cache_append(desc, qkv[a:b], c.cache, q[a:b], w, w, 1e-6, 1e6, draft=AF.draft_rows(torch.tensor([0, b - a], dtype=torch.int32, device=DEV)))
            torch.cuda.synchronize()
            got.append([q] + [t for t in c.dev if t is not None])
    for x in (got[1], got[2]):
        assert all(torch.equal(a, b) for a, b in zip(got[0], x))
    for x in (got[4], got[5]):
        assert all(torch.equal(a, b) for a, b in zip(got[3], x))
    # one token at a time through the operator that was there (its rotary embedding of keys is in fp32)
    c = Cache([n], Hkv, D, "bf16", seed=5, poison=False)
    q = torch.zeros(m, Hq, D, dtype=torch.bfloat16, device=DEV)
    kv = AF.make_kv(c.dev[0], c.dev[1], c.td, c.ld)
    for i in range(m):
        c.ld.fill_(n - m + i + 1)
        ctx.rope_append(desc, qkv[i:i + 1], kv, q[i:i + 1], w, w, 1e-6, 1e6)
    torch.cuda.synchronize()
    # both round to bf16 once, after fp32 arithmetic on terms of |a| + |b| <= 8 or so: at most one bf16 step apart
    assert (np.abs(f64(q) - f64(got[3][0])) <= 2 * HALF_STEP * np.abs(f64(q)) + (D + 16) * 2.0 ** -20).all()
    assert torch.equal(c.dev[1], got[3][2])


# --------------------------------------------------------------------------- conversion
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("Hkv,D,lens,first", [
    (2, 64, [0, 1, 15, 16, 17, 700], None),
    (8, 128, [33, 128, 1], None),
    (1, 128, [100, 64, 31, 5], [17, 64, 30, 0]),
    (4, 64, [5000], [2501]),
])
def test_convert_there_and_back(ctx, fmt, Hkv, D, lens, first):
    src = Cache(lens, Hkv, D, "bf16", seed=3)
    dst = Cache(lens, Hkv, D, fmt, seed=4)                                # other pages
    back = Cache(lens, Hkv, D, "bf16", seed=9)
    desc = AF.attn_desc(Hkv, Hkv, D)
    f = None if first is None else torch.tensor(first, dtype=torch.int32, device=DEV)
    ctx.cache_convert(desc, src.cache, dst.cache, len(lens), first_token=f)
    ctx.cache_convert(desc, dst.cache, back.cache, len(lens), first_token=f)
    assert ctx.device_status() == AF.OK
    want = [values(t).copy() for t in dst.tensors]
    want_back = [f64(t).copy() for t in back.tensors[:2]]
    for b, n in enumerate(lens):
        for t in range(0 if first is None else first[b], n):
            s, d, e = (int(c.table[b, t // 16]) for c in (src, dst, back))
            for at in (0, 1):
                code, scale = DO.quantise(f64(src.tensors[at])[s, :, t % 16], fmt)
                want[at][d, :, t % 16], want[at + 2][d, :, t % 16] = code, scale
                want_back[at][e, :, t % 16] = DO.to_bf16((code.astype(np.float32) * scale.astype(np.float32)[:, None]).astype(np.float64))
    for got, w in zip(dst.dev, want):
        np.testing.assert_array_equal(values(got), w)
    for got, w in zip(back.dev, want_back):
        np.testing.assert_array_equal(values(got), w)


# --------------------------------------------------------------------------- attention
ATTEND = [  # Hq, Hkv, D, lens, rows per sequence (None: one), kind of mask
    (8, 2, 64, [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129], None, "chain"),
    (64, 8, 128, [1, 300, 1000, 16], None, "chain"),
    (8, 8, 128, [40, 5, 257], None, "chain"),
    (4, 2, 64, [3000], None, "chain"),
    (16, 4, 64, [37, 16, 100, 33, 5, 64], [37, 0, 1, 17, 5, 33], "chain"),
    (16, 4, 128, [37, 16, 100, 33, 5, 64], [37, 0, 1, 17, 5, 33], "any"),
    (64, 8, 128, [70, 300, 61], [61, 64, 33], "tree"),
    (8, 8, 64, [70, 129, 20], [61, 65, 20], "any"),
    (4, 1, 64, [20 + i % 9 for i in range(300)], [1 + i % 4 for i in range(300)], "tree"),
    (8, 1, 128, [20000, 17], [5, 17], "tree"),
    (32, 8, 128, [500], [490], "chain"),
    (8, 1, 128, [130, 70], [130, 70], "none"),                            # nothing to attend to
    (8, 4, 128, [1500, 1100], [700, 300], "chain"),
    (8, 1, 64, [400, 1000], [300, 150], "any"),
    (4, 4, 64, [900, 33, 700], [600, 20, 257], "chain"),                  # more rows per tile than tokens per unit
    (8, 1, 128, [9000, 5000, 129], [24, 3, 129], "tree"),                 # tiles in one place and in two, shared by several CTAs
    (16, 2, 128, [130, 1], [16, 1], "chain"),
]


def within(got, want, bound):
    with np.errstate(invalid="ignore"):
        over = ~(np.abs(got - want) <= bound)
    if over.any():
        at = tuple(np.argwhere(over)[0])
        pytest.fail(f"{over.sum()} of {over.size} off, the first at {at}: {got[at]} for {want[at]}, bound {bound[at]}")


def check_attention(out, lse, q, c, offs, ints, T, weight):
    """Against the definition.  weight: what one weight of V is off by, relative to itself."""
    k, v = c.stands_for()
    k, v = np.nan_to_num(k), np.nan_to_num(v)
    vs = None if c.fmt == "bf16" else np.nan_to_num(f64(c.tensors[3]))
    want, want_lse, size, spread, codes = DO.attend(f64(q)[:T], k, v, c.table, c.lens, offs, ints, v_scales=vs)
    n, D = int(max(c.lens)), c.D
    # a score in 32 bits: D products and adds of at most `size` together, the scales, the logarithm of V's scale (below 64, 2^-21), the exponential
    off = (D + 16) * 2.0 ** -23 * size + 2.0 ** -19
    # numerator and denominator are each off by their weights' part of spread (or of the sum), and by the additions of n terms in 32 bits
    rel = weight + off + n * 2.0 ** -24
    # a code's weight p_j scale_j in fp16, the largest of them at 2^8 or more: subnormal steps are 2^-24, so it is off by up to 2^-25 however small
    # it is, which is 2^-33 of the largest
    within(f64(out)[:T], want, HALF_STEP * np.abs(want) + 2 * (1 + HALF_STEP) * rel[..., None] * spread + (1 + HALF_STEP) * 2.0 ** -33 * codes + 1e-30)
    some = np.isfinite(want_lse)
    got = f64(lse)[:T]
    assert (np.isneginf(got) == ~some).all()
    within(got[some], want_lse[some], (off + n * 2.0 ** -24)[some] + 2.0 ** -22 * (1 + np.abs(want_lse[some])))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("Hq,Hkv,D,lens,new,kind", ATTEND)
def test_attention_matches_the_definition(ctx, fmt, Hq, Hkv, D, lens, new, kind):
    c = Cache(lens, Hkv, D, fmt, seed=len(lens) + D + Hq)
    offs = offsets_of(new)
    T, pad = (len(lens), 0) if new is None else (int(offs[-1]), 3)
    ints, mask = random_masks(np.random.default_rng(Hq + D), new, kind)
    if mask is not None:
        mask = torch.cat([mask, torch.full((pad, mask.shape[1]), -1, dtype=torch.int32, device=DEV)])
    g = torch.Generator().manual_seed(5)
    q = (torch.randn(T + pad, Hq, D, generator=g) * torch.exp(torch.randn(T + pad, Hq, 1, generator=g))).to(torch.bfloat16).to(DEV)
    out, lse = torch.full_like(q, 7.5), torch.full((T + pad, Hq), 7.5, device=DEV)
    dr = None if new is None else AF.draft_rows(torch.from_numpy(offs).to(DEV), None, mask)
    ctx.attn_draft(AF.attn_desc(Hq, Hkv, D), q, c.cache, out, lse, draft=dr)
    assert ctx.device_status() == AF.OK
    assert (out[T:] == 7.5).all() and (lse[T:] == 7.5).all()
    # weights: the sum of two bf16 values (2^-9 of 2^-9), or fp16 (2^-12 of the value; none lost that counts, V's scales being alike)
    check_attention(out, lse, q, c, offs, ints, T, 2.0 ** -17 if fmt == "bf16" else 2.0 ** -12)
    # the same bits from run to run, and without lse
    again = torch.full_like(q, 7.5)
    ctx.attn_draft(AF.attn_desc(Hq, Hkv, D), q, c.cache, again, draft=dr)
    assert ctx.device_status() == AF.OK
    assert torch.equal(out, again)


@pytest.mark.parametrize("fmt", FORMATS)
def test_values_of_very_different_size(ctx, fmt):
    """Tokens whose V is 2^30 times another's: which of them counts is up to the scores, not to the largest scale there is."""
    Hq, Hkv, D, n = 8, 1, 128, 200
    c = Cache([n], Hkv, D, fmt, seed=2)
    g = torch.Generator().manual_seed(3)
    k = torch.randn(n, D, generator=g)
    v = torch.randn(n, D, generator=g) * torch.pow(2.0, torch.randint(-30, 31, (n, 1), generator=g).float())
    v[5] = 0
    q = torch.randn(1, Hq, D, generator=g)
    k[7] = 3 * q[0, 1]                                                     # this one takes nearly everything of head 1 ..
    v[7] *= 2.0 ** -40
    k[5] = 3 * q[0, 2]                                                     # .. and one of zeros nearly everything of head 2
    for t in range(n):
        page, slot = int(c.table[0, t // 16]), t % 16
        for at, x in ((0, k[t]), (1, v[t])):
            x = x.to(torch.bfloat16)
            if fmt == "bf16":
                c.tensors[at][page, 0, slot] = x
            else:
                code, scale = DO.quantise(f64(x), fmt)
                c.tensors[at][page, 0, slot] = torch.from_numpy(code).float().to(TYPES[fmt])
                c.tensors[at + 2][page, 0, slot] = float(scale)
    c.put()
    q = q.to(torch.bfloat16).to(DEV)
    out, lse = torch.zeros_like(q), torch.zeros(1, Hq, device=DEV)
    ctx.attn_draft(AF.attn_desc(Hq, Hkv, D), q, c.cache, out, lse)
    assert ctx.device_status() == AF.OK
    check_attention(out, lse, q, c, None, None, 1, 2.0 ** -17 if fmt == "bf16" else 2.0 ** -12)


@pytest.mark.parametrize("Hq", [8, 32])
@pytest.mark.parametrize("fmt", FORMATS)
def test_masked_infinities_do_not_spread(ctx, fmt, Hq):
    """Drafted tokens with NaN and infinities: rows that do not see them come out the same bit for bit as with numbers in their place."""
    Hkv, D, lens, new = 4, 128, [90, 40, 33], [20, 40, 17]
    offs = offsets_of(new)
    T = int(offs[-1])
    ints, mask = random_masks(np.random.default_rng(1), new, "tree")
    q = torch.randn(T, Hq, D, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    dr = AF.draft_rows(torch.from_numpy(offs).to(DEV), None, mask)
    got = []
    bad = {0: 3, 1: 11, 2: 0}                                              # sequence: drafted token
    for dirty in (False, True):
        c = Cache(lens, Hkv, D, fmt, seed=8)
        if dirty:
            for b, j in bad.items():
                t = lens[b] - new[b] + j
                page, slot = int(c.table[b, t // 16]), t % 16
                if fmt == "bf16":
                    c.tensors[0][page, :, slot, 5] = float("nan")
                    c.tensors[1][page, :, slot, 9] = float("inf") if b else float("nan")
                else:
                    for at in (0, 1):
                        c.tensors[at].view(torch.uint8)[page, :, slot] = 0
                        c.tensors[at + 2][page, :, slot] = float("nan")
            c.put()
        out, lse = torch.zeros_like(q), torch.zeros(T, Hq, device=DEV)
        ctx.attn_draft(AF.attn_desc(Hq, Hkv, D), q, c.cache, out, lse, draft=dr)
        assert ctx.device_status() == AF.OK
        got.append((out, lse))
    for r, (b, i, m) in enumerate(DO.rows_of(lens, offs)):
        if ints[r] >> bad[b] & 1:
            assert torch.isnan(got[1][0][r]).any(1).all()
        else:
            assert torch.equal(got[0][0][r], got[1][0][r]) and torch.equal(got[0][1][r], got[1][1][r]), (b, i)


@pytest.mark.parametrize("Hq", [8, 64])
@pytest.mark.parametrize("fmt", FORMATS)
def test_infinite_queries_and_scores(ctx, fmt, Hq):
    """A query that is not finite makes its own head NaN; equal scores of any size are no trouble."""
    Hkv, D = 8, 64
    c = Cache([50, 20], Hkv, D, fmt, seed=1)
    q = torch.randn(2, Hq, D).to(torch.bfloat16)
    q[0, 3, 7], q[1, 0, 0] = float("inf"), float("nan")
    q[1, 2] = 0
    q = q.to(DEV)
    out, lse = torch.zeros_like(q), torch.zeros(2, Hq, device=DEV)
    ctx.attn_draft(AF.attn_desc(Hq, Hkv, D), q, c.cache, out, lse)
    assert ctx.device_status() == AF.OK
    nan = torch.isnan(out).any(2).cpu()
    want = torch.zeros(2, Hq, dtype=torch.bool)
    want[0, 3] = want[1, 0] = True
    assert torch.equal(nan, want) and torch.equal(torch.isnan(lse).cpu(), want)


@pytest.mark.parametrize("fmt", FORMATS)
def test_bad_lengths_and_pages_are_reported(ctx, fmt):
    Hq, Hkv, D = 8, 2, 128
    q = torch.randn(3, Hq, D).to(torch.bfloat16).to(DEV)
    good = Cache([50, 20, 37], Hkv, D, fmt, seed=1)
    ref = torch.zeros_like(q)
    ctx.attn_draft(AF.attn_desc(Hq, Hkv, D), q, good.cache, ref)
    assert ctx.device_status() == AF.OK
    c = Cache([50, 20, 37], Hkv, D, fmt, seed=1)
    c.ld[1] = 16 * c.table.shape[1] + 1
    out, lse = torch.full_like(q, 9.0), torch.full((3, Hq), 9.0, device=DEV)
    ctx.attn_draft(AF.attn_desc(Hq, Hkv, D), q, c.cache, out, lse)
    assert ctx.device_status() == AF.ERR_BOUNDS
    assert torch.equal(out[0], ref[0]) and torch.equal(out[2], ref[2]) and (out[1] == 0).all() and torch.isneginf(lse[1]).all()
    c = Cache([50, 20, 37], Hkv, D, fmt, seed=1, poison=False)
    c.td[2, 1] = c.total
    ctx.attn_draft(AF.attn_desc(Hq, Hkv, D), q, c.cache, out, lse)
    assert ctx.device_status() == AF.ERR_BOUNDS
    assert torch.equal(out[0], ref[0]) and torch.equal(out[1], ref[1])
    # append: the bad sequence writes nothing, the bad page's row its query only
    c = Cache([50, 20, 37], Hkv, D, fmt, seed=1, poison=False)
    before = [None if t is None else raw(t).clone() for t in c.dev]
    c.ld[1] = 0
    c.td[2, 2] = -1
    qkv = torch.randn(3, (Hq + 2 * Hkv) * D).to(torch.bfloat16).to(DEV)
    out.fill_(9.0)
    ctx.cache_append(AF.attn_desc(Hq, Hkv, D), qkv, c.cache, out, None, None, 1e-6, 1e4)
    assert ctx.device_status() == AF.ERR_BOUNDS
    assert (out[1] == 9).all() and not (out[2] == 9).any() and not (out[0] == 9).any()
    page, slot = int(c.table[0, 3]), 49 % 16
    for a, b in zip(before, c.dev):
        if a is not None:
            a[page, :, slot] = raw(b)[page, :, slot]
            assert torch.equal(a, raw(b))
    # conversion: the bad page is left out
    if fmt != "bf16":
        src, dst = Cache([50, 20, 37], Hkv, D, "bf16", seed=1), Cache([50, 20, 37], Hkv, D, fmt, seed=2, poison=False)
        page = int(dst.table[2, 1])
        was = raw(dst.dev[0])[page].clone()
        dst.td[2, 1] = dst.total
        ctx.cache_convert(AF.attn_desc(Hq, Hkv, D), src.cache, dst.cache, 3)
        assert ctx.device_status() == AF.ERR_BOUNDS
        assert torch.equal(raw(dst.dev[0])[page], was)


# --------------------------------------------------------------------------- acceptance
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("Hkv,D,layers", [(2, 64, 1), (8, 128, 3), (1, 128, 70)])
def test_accept_moves_the_path(ctx, fmt, Hkv, D, layers):
    """Paths whose places are sources of later moves, longer than a step, empty, and of tokens that stay."""
    lens = [80, 61, 40, 33, 100, 200]
    base = np.array([17, 0, 39, 1, 60, 70], dtype=np.int32)
    paths = [[0, 1, 2, 5, 6, 9, 30, 62], list(range(1, 61)), [0], [], [3], sorted(np.random.default_rng(2).choice(130, 77, replace=False).tolist())]
    cs = [Cache(lens, Hkv, D, fmt, seed=4 + l % 3) for l in range(layers)]
    path = np.full((len(lens), 90), -5, dtype=np.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = p
    n = torch.tensor([len(p) for p in paths], dtype=torch.int32, device=DEV)
    ctx.cache_accept(AF.attn_desc(Hkv, Hkv, D), [c.cache for c in cs], len(lens), torch.from_numpy(base).to(DEV), torch.from_numpy(path).to(DEV), n)
    assert ctx.device_status() == AF.OK
    for c in cs:
        for t, got in zip(c.tensors, c.dev):
            if t is None:
                continue
            want = raw(t).clone()
            for b, p in enumerate(paths):
                for k, s in enumerate(p):
                    f, to = int(base[b]) + s, int(base[b]) + k
                    want[int(c.table[b, to // 16]), :, to % 16] = raw(t)[int(c.table[b, f // 16]), :, f % 16]
            assert torch.equal(want.view(torch.uint8), raw(got).cpu().view(torch.uint8))


def test_bad_paths_move_nothing(ctx):
    lens, Hkv, D = [40] * 6, 2, 64
    c = Cache(lens, Hkv, D, "int8", poison=False)
    before = [t.clone() for t in c.dev]
    path = torch.tensor([[1, 3, 2, 0], [1, 1, 0, 0], [-1, 2, 3, 4], [1, 2, 3, 30], [0, 1, 2, 3], [1, 2, 0, 0]], dtype=torch.int32, device=DEV)
    n = torch.tensor([3, 2, 2, 4, 5, 2], dtype=torch.int32, device=DEV)
    base = torch.tensor([10, 10, 10, 10, 10, -1], dtype=torch.int32, device=DEV)
    ctx.cache_accept(AF.attn_desc(Hkv, Hkv, D), [c.cache], 6, base, path, n)
    assert ctx.device_status() == AF.ERR_BOUNDS
    assert all(torch.equal(a, b) for a, b in zip(before, c.dev))


# --------------------------------------------------------------------------- together, streams, graphs
@pytest.mark.parametrize("fmt", FORMATS)
def test_a_step_of_drafting_verifying_and_accepting(ctx, fmt):
    """A tree is appended and attended; its rows are those of the branches decoded one token at a time; after the acceptance of a branch the cache
    is the one that decoding the branch alone leaves."""
    Hq, Hkv, D, ctx_len = 8, 2, 128, 37
    parents = [-1, 0, 0, 1, 2, 2, 4]
    branch = [0, 2, 4, 6]
    m = len(parents)
    mask, depth = AF.tree_rows([parents])
    g = torch.Generator().manual_seed(6)
    qkv = torch.randn(m, (Hq + 2 * Hkv) * D, generator=g).to(torch.bfloat16).to(DEV)
    desc = AF.attn_desc(Hq, Hkv, D)
    c = Cache([ctx_len + m], Hkv, D, fmt, seed=3, poison=False)
    alone = Cache([ctx_len + m], Hkv, D, fmt, seed=3, poison=False)
    q, out = torch.zeros(m, Hq, D, dtype=torch.bfloat16, device=DEV), torch.zeros(m, Hq, D, dtype=torch.bfloat16, device=DEV)
    lse = torch.zeros(m, Hq, device=DEV)
    dr = AF.draft_rows(torch.tensor([0, m], dtype=torch.int32, device=DEV), (ctx_len + depth).to(torch.int32).to(DEV), mask.to(DEV))
    ctx.cache_append(desc, qkv, c.cache, q, None, None, 1e-6, 1e6, draft=dr)
    ctx.attn_draft(desc, q, c.cache, out, lse, draft=dr)
    for k, i in enumerate(branch):
        alone.ld.fill_(ctx_len + k + 1)
        q1, o1, l1 = (torch.zeros(1, *s.shape[1:], dtype=s.dtype, device=DEV) for s in (q, out, lse))
        ctx.cache_append(desc, qkv[i:i + 1], alone.cache, q1, None, None, 1e-6, 1e6)
        ctx.attn_draft(desc, q1, alone.cache, o1, l1)
        torch.cuda.synchronize()
        assert torch.equal(q1[0], q[i])
        # both are within the definition's tolerance; the additions come in another order
        assert (np.abs(f64(o1[0]) - f64(out[i])) <= 2 * HALF_STEP * np.abs(f64(o1[0])) + 2.0 ** -9).all()
        assert (np.abs(f64(l1[0]) - f64(lse[i])) <= 1e-5 * (1 + np.abs(f64(lse[i])))).all()
    ctx.cache_accept(desc, [c.cache], 1, torch.tensor([ctx_len], dtype=torch.int32, device=DEV), torch.tensor([branch], dtype=torch.int32, device=DEV),
                     torch.tensor([len(branch)], dtype=torch.int32, device=DEV))
    assert ctx.device_status() == AF.OK
    for t in range(ctx_len + len(branch)):
        for a, b in zip(c.dev, alone.dev):
            if a is not None:
                assert torch.equal(raw(a)[int(c.table[0, t // 16]), :, t % 16], raw(b)[int(alone.table[0, t // 16]), :, t % 16])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows", [1, 7, 40])
def test_captured_and_replayed(ctx, fmt, rows):
    """A graph of append, attention and acceptance, replayed with other contents; another stream than the default one."""
    Hq, Hkv, D, lens = 16, 4, 128, [300, 150, 90]
    desc = AF.attn_desc(Hq, Hkv, D)
    c = Cache(lens, Hkv, D, fmt, seed=3, poison=False)
    new = [rows] * 3
    T = sum(new)
    dr = None if rows == 1 else AF.draft_rows(torch.from_numpy(offsets_of(new)).to(DEV))
    qkv = torch.randn(T, (Hq + 2 * Hkv) * D).to(torch.bfloat16).to(DEV)
    q, out = (torch.zeros(T, Hq, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    base, path, n = c.ld - rows, torch.tensor([[rows - 1]] * 3, dtype=torch.int32, device=DEV), torch.ones(3, dtype=torch.int32, device=DEV)

    def step(stream=None):
        ctx.cache_append(desc, qkv, c.cache, q, None, None, 1e-6, 1e6, draft=dr, stream=stream)
        ctx.attn_draft(desc, q, c.cache, out, draft=dr, stream=stream)
        ctx.cache_accept(desc, [c.cache], 3, base, path, n, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (1, 2):
        qkv.copy_(torch.randn(qkv.shape, generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        got = [out.clone()] + [raw(t).clone() for t in c.dev if t is not None]
        out.zero_()
        step()
        assert ctx.device_status() == AF.OK
        assert all(torch.equal(a, b) for a, b in zip(got, [out] + [raw(t) for t in c.dev if t is not None]))


def test_one_token_over_bf16_agrees_with_decode_attention(ctx):
    Hq, Hkv, D, lens = 32, 8, 128, [1, 100, 3000, 17, 64]
    c = Cache(lens, Hkv, D, "bf16", seed=1)
    q = torch.randn(5, Hq, D).to(torch.bfloat16).to(DEV)
    a, b, la, lb = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(5, Hq, device=DEV), torch.zeros(5, Hq, device=DEV)
    desc = AF.attn_desc(Hq, Hkv, D)
    ctx.attn_decode(desc, q, AF.make_kv(c.dev[0], c.dev[1], c.td, c.ld), a, la)
    ctx.attn_draft(desc, q, c.cache, b, lb)
    assert ctx.device_status() == AF.OK
    # both round to bf16 once; the older operator's weights are bf16 (2^-9 each)
    assert (np.abs(f64(a) - f64(b)) <= 2 * HALF_STEP * np.abs(f64(b)) + 2.0 ** -8 * np.abs(f64(c.tensors[1]).copy())[np.isfinite(f64(c.tensors[1]))].max()).all()
    assert (np.abs(f64(la) - f64(lb)) <= 1e-5 * (1 + np.abs(f64(lb)))).all()


def test_offsets_beyond_32_bits(ctx):
    """A cache of more than 2^32 bytes, whose last pages are used."""
    Hq, Hkv, D = 8, 8, 128
    pages = (1 << 32) // (Hkv * 16 * D) + 40                               # int8: more than 2^32 bytes of K
    desc = AF.attn_desc(Hq, Hkv, D)
    k, v, ks, vs = AF.empty_cache(pages, Hkv, D, torch.int8, DEV)
    table = torch.arange(pages - 4, pages, dtype=torch.int32, device=DEV).view(1, 4)
    lens = torch.tensor([60], dtype=torch.int32, device=DEV)
    big = AF.make_cache(k, v, table, lens, ks, vs)
    small = AF.empty_cache(4, Hkv, D, torch.int8, DEV)
    little = AF.make_cache(small[0], small[1], torch.arange(4, dtype=torch.int32, device=DEV).view(1, 4), lens, small[2], small[3])
    qkv = torch.randn(60, (Hq + 2 * Hkv) * D).to(torch.bfloat16).to(DEV)
    dr = AF.draft_rows(torch.tensor([0, 60], dtype=torch.int32, device=DEV))
    got = []
    for c in (big, little):
        q, out = (torch.zeros(60, Hq, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        ctx.cache_append(desc, qkv, c, q, None, None, 1e-6, 1e6, draft=dr)
        ctx.attn_draft(desc, q, c, out, draft=dr)
        ctx.cache_accept(desc, [c], 1, torch.tensor([0], dtype=torch.int32, device=DEV), torch.tensor([[5, 50]], dtype=torch.int32, device=DEV),
                         torch.tensor([2], dtype=torch.int32, device=DEV))
        assert ctx.device_status() == AF.OK
        got.append(out)
    assert torch.equal(got[0], got[1])
    for a, b in zip((k, v, ks, vs), small):
        assert torch.equal(a[pages - 4:], b)
    back = AF.empty_cache(4, Hkv, D, torch.bfloat16, DEV)
    for c in (big, little):
        ctx.cache_convert(desc, c, AF.make_cache(back[0], back[1], torch.arange(4, dtype=torch.int32, device=DEV).view(1, 4), lens), 1)
        assert ctx.device_status() == AF.OK
        got.append(back[0].clone())
    assert torch.equal(got[2], got[3])


# --------------------------------------------------------------------------- whole layers
@pytest.mark.parametrize("experts", [0, 4])
@pytest.mark.parametrize("fmt", FORMATS)
def test_layers_agree_with_the_operators_one_by_one(ctx, fmt, experts):
    Hq, Hkv, D, H, I, L = 8, 2, 64, 256, 512, 2
    lens, new = [40, 21, 70], [5, 1, 9]
    offs = offsets_of(new)
    T = int(offs[-1])
    _, mask = random_masks(np.random.default_rng(5), new, "tree")
    pos = torch.from_numpy(np.concatenate([np.arange(n - m, n) for n, m in zip(lens, new)]).astype(np.int32)).to(DEV)
    dr = AF.draft_rows(torch.from_numpy(offs).to(DEV), pos, mask)
    g = torch.Generator().manual_seed(4)
    w = lambda *s: (torch.randn(*s, generator=g) * s[-1] ** -0.5).to(torch.bfloat16).to(DEV)  # noqa: E731
    ones = lambda n: (1 + 0.1 * torch.randn(n, generator=g)).to(torch.bfloat16).to(DEV)  # noqa: E731
    desc = AF.attn_desc(Hq, Hkv, D)
    e = (experts,) if experts else ()
    weights = [dict(o=w(H, Hq * D), gate=w(*e, I, H), up=w(*e, I, H), down=w(*e, H, I), router=w(experts, H) if experts else None, qkv=w((Hq + 2 * Hkv) * D, H),
                    ln1=ones(H), ln2=ones(H), qn=ones(D), kn=ones(D)) for _ in range(L)]
    layers = [AF.decoder_desc(AF.layer_desc(desc, H, I, x["o"], x["gate"], x["up"], x["down"], experts, 2 if experts else 0, x["router"]),
                              x["qkv"], x["ln1"], x["ln2"], x["qn"], x["kn"], 1e-6, 1e4) for x in weights]
    a, b = ([Cache(lens, Hkv, D, fmt, seed=l, poison=False) for l in range(L)] for _ in range(2))
    x = torch.randn(T, H, generator=g).to(torch.bfloat16).to(DEV)
    got = torch.zeros_like(x)
    assert AF.draft_workspace_bytes(layers[0], T) <= 1 << 27
    ctx.draft_layers(layers, [c.cache for c in a], x, got, draft=dr)
    assert ctx.device_status() == AF.OK
    h = x.clone()
    new_ = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    for l, (p, c) in enumerate(zip(weights, b)):
        xn, qkv, q, o, y = new_(T, H), new_(T, (Hq + 2 * Hkv) * D), new_(T, Hq, D), new_(T, Hq, D), new_(T, H)
        ctx.add_rmsnorm(h, None, p["ln1"], 1e-6, y=xn)
        ctx.linear(xn, p["qkv"], qkv)
        ctx.cache_append(desc, qkv, c.cache, q, p["qn"], p["kn"], 1e-6, 1e4, draft=dr)
        ctx.attn_draft(desc, q, c.cache, o, draft=dr)
        ctx.linear(o.view(T, Hq * D), p["o"], y)
        ctx.add_rmsnorm(h, y, p["ln2"], 1e-6, res_out=h, y=xn)
        if experts:
            ctx.ffn_moe(xn, p["gate"], p["up"], p["down"], 2, y, w_router=p["router"])
        else:
            ctx.ffn_dense(xn, p["gate"], p["up"], p["down"], y)
        ctx.add_rmsnorm(h, y, None, 0.0, res_out=h)
    assert ctx.device_status() == AF.OK
    # the chain's steps are the same products, summed in another order and rounded to bf16 in the same places but for the normalisation
    # (each tensor's roundings: 2^-8 of its size; a layer has about six of them in a row): four layers' worth for two
    assert np.abs(f64(got) - f64(h)).max() <= 24 * HALF_STEP * np.abs(f64(h)).max()
    assert torch.equal(raw(a[0].dev[1]), raw(b[0].dev[1]))                 # the first layer's values are rounded the same


def test_layers_of_single_tokens_agree_with_the_dense_chain(ctx):
    Hq, Hkv, D, H, I = 8, 2, 128, 512, 1024
    lens = [40, 21, 70, 1, 16]
    g = torch.Generator().manual_seed(4)
    w = lambda *s: (torch.randn(*s, generator=g) * s[-1] ** -0.5).to(torch.bfloat16).to(DEV)  # noqa: E731
    ones = lambda n: (1 + 0.1 * torch.randn(n, generator=g)).to(torch.bfloat16).to(DEV)  # noqa: E731
    desc = AF.attn_desc(Hq, Hkv, D)
    layers = [AF.decoder_desc(AF.layer_desc(desc, H, I, w(H, Hq * D), w(I, H), w(I, H), w(H, I)), w((Hq + 2 * Hkv) * D, H), ones(H), ones(H), None, None,
                              1e-6, 1e6) for _ in range(2)]
    a, b = ([Cache(lens, Hkv, D, "bf16", seed=l, poison=False) for l in range(2)] for _ in range(2))
    x = torch.randn(5, H, generator=g).to(torch.bfloat16).to(DEV)
    ya, yb = torch.zeros_like(x), torch.zeros_like(x)
    ctx.draft_layers(layers, [c.cache for c in a], x, ya)
    ctx.decoder_layers(layers, [AF.make_kv(c.dev[0], c.dev[1], c.td, c.ld) for c in b], x, yb)
    assert ctx.device_status() == AF.OK
    # keys rotated in 64 or 32 bits, weights of 16 or 8 bits: a bf16 step here and there in each of the two layers
    assert np.abs(f64(ya) - f64(yb)).max() <= 16 * HALF_STEP * np.abs(f64(yb)).max()


def test_a_workspace_that_is_too_small_is_refused():
    desc = AF.attn_desc(8, 2, 128)
    c = Cache([5], 2, 128, "int8")
    q = torch.zeros(1, 8, 128, dtype=torch.bfloat16, device=DEV)
    need = AF.attn_draft_workspace_bytes(desc)
    small, fits = AF.Context(0, need - 256), AF.Context(0, need)
    with pytest.raises(AF.AflexError) as e:
        small.attn_draft(desc, q, c.cache, q.clone())
    assert e.value.status == AF.ERR_WORKSPACE and str(need) in str(e.value)
    fits.attn_draft(desc, q, c.cache, q.clone())
    assert fits.device_status() == AF.OK
    small.close()
    fits.close()
