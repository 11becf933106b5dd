"""Attention of drafted tokens and the operators around it where one value decides: references that move twice in a step of the tensor-core kernel,
codes that are no numbers, values of any size, a channel of large keys, paths with bad pages, scores of any size,
masks of other widths."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as DO
from paper_2608_01891_b200 import aflex as AF
from test_gpu_draft import DEV, FORMATS, TYPES, Cache, check_attention, ctx, f64, offsets_of, random_masks  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu
WEIGHT = {"bf16": 2.0 ** -17, "int8": 2.0 ** -12, "e4m3": 2.0 ** -12}     # what a weight of V is off by (test_gpu_draft.py)


def put_token(c, b, t, g, k=None, v=None):
    """K and V (bf16 values [D] on the host) of token t of sequence b, KV head g, as the cache's format holds them."""
    page, slot = int(c.table[b, t // 16]), t % 16
    for at, x in ((0, k), (1, v)):
        if x is None:
            continue
        if c.fmt == "bf16":
            c.tensors[at][page, g, slot] = x
        else:
            code, scale = DO.quantise(f64(x), c.fmt)
            c.tensors[at][page, g, slot] = torch.from_numpy(code).float().to(TYPES[c.fmt])
            c.tensors[at + 2][page, g, slot] = float(scale)


def attend(ctx, c, q, draft=None, scale=0.0):  # noqa: F811
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV)
    ctx.attn_draft(AF.attn_desc(q.shape[1], c.Hkv, c.D, scale), q, c.cache, out, lse, draft=draft)
    assert ctx.device_status() == AF.OK
    return out, lse


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("Hq,Hkv,D,m", [(32, 4, 128, 40), (32, 4, 128, 6), (16, 4, 64, 20)])
def test_references_move_in_both_halves_of_every_step(ctx, fmt, Hq, Hkv, D, m):  # noqa: F811
    """Scores that grow by 24 (in units of the exponent) in both halves of every 128 tokens: what was summed before has to be scaled by both."""
    n, gen = 640, torch.Generator().manual_seed(21)
    c = Cache([n], Hkv, D, fmt, seed=20)
    level = torch.zeros(n)
    for t in range(0, n, 64):
        level[t + 10:] += 17.0 * D ** 0.5 / 8
    for g in range(Hkv):
        k = 0.5 * torch.randn(n, D, generator=gen)
        k[:, 0] = level
        for t in range(n):
            put_token(c, 0, t, g, k=k[t].to(torch.bfloat16))
    c.put()
    q = torch.randn(m, Hq, D, generator=gen)
    q[:, :, 0] = 8.0
    q = q.to(torch.bfloat16).to(DEV)
    offs = offsets_of([m])
    out, lse = attend(ctx, c, q, AF.draft_rows(torch.from_numpy(offs).to(DEV)))
    check_attention(out, lse, q, c, offs, None, m, WEIGHT[fmt])


MASKED = [  # Hq, Hkv, D, lens, rows per sequence: tiles of 8 lines, of 16, of 256 in two places, of 256
    (8, 4, 128, [90, 40, 33], [3, 4, 5]),
    (8, 4, 64, [90, 40, 33], [3, 4, 5]),
    (16, 4, 128, [90, 40, 33], [3, 4, 5]),
    (16, 4, 64, [90, 140, 33], [3, 4, 12]),
    (8, 4, 128, [90, 40, 33], [20, 40, 17]),
    (16, 2, 128, [390, 40, 33], [40, 33, 17]),
    (32, 4, 64, [290, 40, 133], [20, 40, 17]),
]


@pytest.mark.parametrize("scale", ["number", "nan"])
@pytest.mark.parametrize("Hq,Hkv,D,lens,new", MASKED)
def test_codes_that_are_no_numbers_do_not_spread(ctx, Hq, Hkv, D, lens, new, scale):  # noqa: F811
    """e4m3 has two codes of NaN.  In K or V of a drafted token they reach the rows that see it, and leave the others' bits as they are."""
    offs = offsets_of(new)
    T = int(offs[-1])
    ints, mask = random_masks(np.random.default_rng(1), new, "tree")
    q = torch.randn(T, Hq, D, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    draft = AF.draft_rows(torch.from_numpy(offs).to(DEV), None, mask)
    bad = {0: 1, 1: 3, 2: 0}                                               # sequence: drafted token
    clean = Cache(lens, Hkv, D, "e4m3", seed=8)
    want, want_lse = attend(ctx, clean, q, draft)
    for at in (0, 1):
        c = Cache(lens, Hkv, D, "e4m3", seed=8)
        for b, j in bad.items():
            t = lens[b] - new[b] + j
            page, slot = int(c.table[b, t // 16]), t % 16
            for g in range(Hkv):
                # both codes, in different parts of the head; one head has a single one, in its last channel
                where = [(D - 1, 0x7f)] if g == 1 else [(3, 0x7f), (4, 0xff), (D // 2 + 9, 0xff)]
                for ch, code in where:
                    c.tensors[at].view(torch.uint8)[page, g, slot, ch] = code
                if scale == "nan":
                    c.tensors[at + 2][page, g, slot] = float("nan")
        c.put()
        out, lse = attend(ctx, c, q, draft)
        for r, (b, i, m) in enumerate(DO.rows_of(lens, offs)):
            if ints[r] >> bad[b] & 1:
                assert torch.isnan(out[r]).any(1).all(), (at, b, i)
            else:
                assert torch.equal(want[r], out[r]) and torch.equal(want_lse[r], lse[r]), (at, b, i)


@pytest.mark.parametrize("Hq,Hkv,D,lens,new", MASKED)
def test_a_code_that_is_no_number_in_an_earlier_token(ctx, Hq, Hkv, D, lens, new):  # noqa: F811
    """Every row of its sequence sees it, in the channel at least; other sequences and KV heads do not."""
    offs = offsets_of(new)
    T = int(offs[-1])
    q = torch.randn(T, Hq, D, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    draft = AF.draft_rows(torch.from_numpy(offs).to(DEV))
    got = []
    for t in (None, 2, lens[0] - new[0] - 1):                              # in the first step; beside the drafted tokens
        c = Cache(lens, Hkv, D, "e4m3", seed=8)
        if t is not None:
            c.tensors[1].view(torch.uint8)[int(c.table[0, t // 16]), 1, t % 16, 7] = 0xff
            c.put()
        got.append(attend(ctx, c, q, draft))
    G = Hq // Hkv
    mine = torch.zeros(T, Hq, dtype=torch.bool)
    mine[:new[0], G:2 * G] = True
    for out, lse in got[1:]:
        assert torch.isnan(out[:new[0], G:2 * G, 7]).all()
        assert torch.equal(out[~mine], got[0][0][~mine]) and torch.equal(lse[~mine], got[0][1][~mine])


LINES = [  # Hq, Hkv, D, rows: tiles of 8 lines, of 16, of 256 in two places, of 256
    (8, 1, 128, 1), (8, 2, 64, 2), (8, 1, 128, 2), (8, 1, 64, 2), (8, 1, 128, 8), (8, 1, 64, 8), (8, 1, 128, 40), (8, 1, 64, 40)]


def check_values(ctx, fmt, Hq, Hkv, D, m, large, big):  # noqa: F811
    """Tokens of zeros (every second one), of numbers near 1, and of up to 4 times `big` (those of `large`)."""
    n, gen = 700, torch.Generator().manual_seed(31)
    c = Cache([n], Hkv, D, fmt, seed=30)
    for g in range(Hkv):
        v = torch.randn(n, D, generator=gen)
        v[::2] = 0
        for t in large:
            v[t] = big * torch.randn(D, generator=gen)
        for t in range(n):
            put_token(c, 0, t, g, v=v[t].to(torch.bfloat16))
    c.put()
    q = (2.0 * torch.randn(m, Hq, D, generator=gen)).to(torch.bfloat16).to(DEV)
    offs = offsets_of([m])
    out, lse = attend(ctx, c, q, AF.draft_rows(torch.from_numpy(offs).to(DEV)))
    check_attention(out, lse, q, c, offs, None, m, WEIGHT[fmt])


LARGE = {"one": [333], "early": range(0, 60), "late": range(600, 700), "mixed": range(0, 700, 3)}


@pytest.mark.parametrize("Hq,Hkv,D,m", LINES)
@pytest.mark.parametrize("where", list(LARGE))
def test_very_large_values_of_a_bf16_cache(ctx, Hq, Hkv, D, m, where):  # noqa: F811
    """Sums of weights times values up to 2^122 stay finite."""
    check_values(ctx, "bf16", Hq, Hkv, D, m, LARGE[where], 2.0 ** 120)


@pytest.mark.parametrize("big", [2.0 ** 60, 2.0 ** 120])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,D,m", LINES)
@pytest.mark.parametrize("where", list(LARGE))
def test_values_of_zero_beside_very_large_ones(ctx, fmt, Hq, Hkv, D, m, where, big):  # noqa: F811
    """The sum of the weights counts every token by its score alone, whatever its value's size: in the same pages, before and behind one another, in
    pieces of several CTAs."""
    check_values(ctx, fmt, Hq, Hkv, D, m, LARGE[where], big)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("Hq,Hkv,D,m", LINES)
def test_values_that_are_all_zero(ctx, fmt, Hq, Hkv, D, m):  # noqa: F811
    n = 700
    c = Cache([n], Hkv, D, fmt, seed=30)
    for g in range(Hkv):
        for t in range(n):
            put_token(c, 0, t, g, v=torch.zeros(D, dtype=torch.bfloat16))
    c.put()
    q = (2.0 * torch.randn(m, Hq, D, generator=torch.Generator().manual_seed(3))).to(torch.bfloat16).to(DEV)
    offs = offsets_of([m])
    out, lse = attend(ctx, c, q, AF.draft_rows(torch.from_numpy(offs).to(DEV)))
    assert (out == 0).all()
    check_attention(out, lse, q, c, offs, None, m, WEIGHT[fmt])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("Hq,Hkv,D,m", [(8, 2, 64, 1), (8, 1, 128, 1), (8, 1, 128, 2), (8, 1, 128, 8), (8, 1, 64, 40)])
def test_scores_beside_a_channel_of_large_keys(ctx, fmt, Hq, Hkv, D, m):  # noqa: F811
    """One key channel is 127 times the others, whose codes are then of one bit, and the queries' sum is far from zero.  A score is a sum of products
    that 32 bits hold exactly, so lse is off by roundings of a handful of numbers below 64 (in units of log2) only: 2^-18 each at most."""
    n, gen = 60, torch.Generator().manual_seed(41)
    c = Cache([n], Hkv, D, fmt, seed=40)
    for g in range(Hkv):
        k = torch.randint(0, 2, (n, D), generator=gen).float() * 2 - 1
        k[:, 5] = 127
        for t in range(n):
            put_token(c, 0, t, g, k=k[t].to(torch.bfloat16))
    c.put()
    q = 0.125 + 1.875 * torch.rand(m, Hq, D, generator=gen)                # (8 bits each, steps of 2^-10 and more)
    q[:, :, 5] = 0
    q = q.to(torch.bfloat16).to(DEV)
    offs = offsets_of([m])
    out, lse = attend(ctx, c, q, AF.draft_rows(torch.from_numpy(offs).to(DEV)))
    k, v = (np.nan_to_num(x) for x in c.stands_for())
    _, want, *_ = DO.attend(f64(q), k, v, c.table, c.lens, offs, None)
    assert np.abs(f64(lse) - want).max() <= 4 * 2.0 ** -18


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("Hkv,D", [(2, 64), (8, 128)])
def test_a_path_with_a_bad_page_moves_nothing(ctx, fmt, Hkv, D):  # noqa: F811
    """A path is moved whole or not at all: a page id that is none, of its first tokens or of its last, as source or as destination, leaves the
    sequence as it is in that cache; the other sequences and caches are compacted."""
    lens = [90, 90, 120, 120, 60]
    base = np.array([10, 10, 8, 8, 3], dtype=np.int32)
    paths = [[1, 20, 60], [1, 20, 60], list(range(5, 105)), list(range(5, 105)), [0, 2, 40]]
    spoilt = {0: 1, 1: 4, 2: 6, 3: 0}                                      # sequence: page of its table (of a source, a source, a source, a destination)
    path = np.zeros((len(lens), 100), dtype=np.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = p
    dev = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    n = torch.tensor([len(p) for p in paths], dtype=torch.int32, device=DEV)
    cs = [Cache(lens, Hkv, D, fmt, seed=s, poison=False) for s in (1, 2)]
    for b, page in spoilt.items():
        cs[0].td[b, page] = -1 if b % 2 else cs[0].total
    ctx.cache_accept(AF.attn_desc(Hkv, Hkv, D), [c.cache for c in cs], len(lens), dev(base), dev(path), n)
    assert ctx.device_status() == AF.ERR_BOUNDS
    for c in cs:
        for t, got in zip(c.tensors, c.dev):
            if t is None:
                continue
            raw = lambda x: x.view(torch.int32 if x.dim() == 3 else torch.uint8)  # noqa: E731
            want = t.clone()
            for b, p in enumerate(paths):
                for k, s in enumerate(p):
                    if c is cs[0] and b in spoilt:
                        continue
                    f, to = int(base[b]) + s, int(base[b]) + k
                    raw(want)[int(c.table[b, to // 16]), :, to % 16] = raw(t)[int(c.table[b, f // 16]), :, f % 16]
            assert torch.equal(raw(want), raw(got.cpu()))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("scale", [0.37, 1e-4, -0.2])
@pytest.mark.parametrize("Hq,Hkv,D,m", [(8, 1, 128, 1), (8, 1, 64, 2), (8, 1, 128, 8), (8, 1, 64, 40)])
def test_scores_are_scaled_as_the_descriptor_says(ctx, fmt, Hq, Hkv, D, m, scale):  # noqa: F811
    c = Cache([300], Hkv, D, fmt, seed=50)
    q = torch.randn(m, Hq, D, generator=torch.Generator().manual_seed(51)).to(torch.bfloat16).to(DEV)
    offs = offsets_of([m])
    out, lse = attend(ctx, c, q, AF.draft_rows(torch.from_numpy(offs).to(DEV)), scale)
    # (check_attention knows the usual scale: as if the queries were longer or shorter)
    by = float(np.float32(scale)) * D ** 0.5
    check_attention(out, lse, q.double().cpu() * by, c, offs, None, m, WEIGHT[fmt])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("Hq,Hkv,D,m", [(8, 1, 128, 1), (8, 1, 64, 2), (8, 1, 128, 8), (8, 1, 64, 40)])
def test_infinite_scores_of_finite_queries(ctx, fmt, Hq, Hkv, D, m):  # noqa: F811
    """A score of -infinity weighs nothing, one of +infinity makes its head NaN, and neither touches the other heads."""
    n, far = 300, 7
    c = Cache([n], Hkv, D, fmt, seed=60)
    for t in range(n):
        k = torch.randn(D, generator=torch.Generator().manual_seed(t))
        k[3], k[4] = 0, 0
        put_token(c, 0, t, 0, k=k.to(torch.bfloat16))
    k = torch.zeros(D)
    k[3] = 2.0 ** 100
    put_token(c, 0, far, 0, k=k.to(torch.bfloat16))
    c.put()
    q = torch.randn(m, Hq, D, generator=torch.Generator().manual_seed(61))
    q[:, :, 3], q[:, 1], q[:, 2] = 0, 0, 0
    q[:, 1, 3], q[:, 2, 3] = -2.0 ** 100, 2.0 ** 100
    q[:, 1, 4] = 2.0 ** 100                                                # (where all keys are 0)
    q = q.to(torch.bfloat16).to(DEV)
    offs = offsets_of([m])
    out, lse = attend(ctx, c, q, AF.draft_rows(torch.from_numpy(offs).to(DEV)))
    assert torch.isnan(out[:, 2]).any(1).all() and torch.isnan(lse[:, 2]).all()
    assert torch.isfinite(out[:, [0, 1, 3, 4, 5, 6, 7]]).all()
    # head 1: all other tokens have the score 0, and the far one is not there
    v = np.nan_to_num(c.stands_for()[1])
    flat = v[c.table[0], 0].reshape(-1, D)[:n]
    for i in range(m):
        see = [t for t in range(n - m + i + 1) if t != far]
        want, spread = flat[see].mean(0), np.abs(flat[see]).mean(0)
        err = np.abs(f64(out)[i, 1] - want)
        assert (err <= 2.0 ** -8 * np.abs(want) + 2 * (WEIGHT[fmt] + n * 2.0 ** -24 + 2.0 ** -19) * spread + 2.0 ** -32 * np.abs(flat).max()).all()
        assert abs(float(lse[i, 1]) - np.log(len(see))) <= 2.0 ** -17


@pytest.mark.parametrize("fmt", FORMATS)
def test_masks_of_single_rows(ctx, fmt):  # noqa: F811
    """One row per sequence, with a mask: a row may be told not to see its own token."""
    Hq, Hkv, D, lens = 8, 2, 64, [1, 1, 40, 40, 130, 129]
    c = Cache(lens, Hkv, D, fmt, seed=70)
    q = torch.randn(len(lens), Hq, D, generator=torch.Generator().manual_seed(71)).to(torch.bfloat16).to(DEV)
    ints = [1, 0, 1, 0, 6, 7]                                              # (bits of tokens that there are not change nothing)
    out, lse = attend(ctx, c, q, AF.draft_rows(None, None, torch.tensor(ints, dtype=torch.int32, device=DEV).view(-1, 1)))
    check_attention(out, lse, q, c, None, ints, len(lens), WEIGHT[fmt])
    assert (out[1] == 0).all() and torch.isneginf(lse[1]).all()


@pytest.mark.parametrize("words", [1, 2, 5])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("Hq,Hkv,D,lens,new", [(2, 2, 64, [300, 64, 90, 70], [8, 64, 3, 70]), (8, 1, 128, [300, 64, 90], [80, 64, 3])])
def test_masks_of_more_or_fewer_words_than_rows(ctx, fmt, Hq, Hkv, D, lens, new, words):  # noqa: F811
    """Drafted tokens behind the last word are not seen; words behind the last token are not looked at."""
    offs = offsets_of(new)
    T = int(offs[-1])
    rng = np.random.default_rng(72)
    a = rng.integers(0, 1 << 32, (T, words), dtype=np.uint64).astype(np.uint32)
    ints = [sum(int(x) << 32 * w for w, x in enumerate(row)) for row in a]
    c = Cache(lens, Hkv, D, fmt, seed=73)
    q = torch.randn(T, Hq, D, generator=torch.Generator().manual_seed(74)).to(torch.bfloat16).to(DEV)
    out, lse = attend(ctx, c, q, AF.draft_rows(torch.from_numpy(offs).to(DEV), None, torch.from_numpy(a.view(np.int32)).to(DEV)))
    check_attention(out, lse, q, c, offs, ints, T, WEIGHT[fmt])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("others", [3, 40])
def test_a_chunk_among_single_tokens(ctx, fmt, others):  # noqa: F811
    """The form of the tiles is chosen for all sequences: single tokens on the tensor-core kernel, and a prompt chunk in tiles of 16 lines."""
    Hq, Hkv, D = 8, 2, 64
    new = [1] * others + [150] + [1] * 2
    lens = [1 + 37 * i % 300 for i in range(others)] + [400, 16, 129]
    offs = offsets_of(new)
    T = int(offs[-1])
    c = Cache(lens, Hkv, D, fmt, seed=75)
    q = torch.randn(T, Hq, D, generator=torch.Generator().manual_seed(76)).to(torch.bfloat16).to(DEV)
    out, lse = attend(ctx, c, q, AF.draft_rows(torch.from_numpy(offs).to(DEV)))
    check_attention(out, lse, q, c, offs, None, T, WEIGHT[fmt])


@pytest.mark.parametrize("bad", [[1999], [0], [31, 32, 700, 1500], "all"])
def test_codes_that_are_no_numbers_in_a_long_chunk(ctx, bad):  # noqa: F811
    """A prompt chunk over an e4m3 cache: rows from a bad token on are NaN, rows before it are as they are without it."""
    Hq, Hkv, D, m, before = 8, 1, 128, 2000, 100
    pages = (m + before + 15) // 16
    k, v, ks, vs = AF.empty_cache(pages, Hkv, D, torch.float8_e4m3fn, DEV)
    g = torch.Generator(device=DEV).manual_seed(80)
    for x in (k, v):
        x.view(torch.uint8).copy_(torch.randint(0, 126, x.shape, generator=g, device=DEV, dtype=torch.uint8))
    ks.fill_(1e-3)
    vs.fill_(1e-2)
    cache = AF.make_cache(k, v, torch.randperm(pages, generator=g, device=DEV).to(torch.int32).view(1, -1), torch.tensor([m + before], dtype=torch.int32, device=DEV), ks, vs)
    table = cache._keep[2].cpu()
    q = torch.randn(m, Hq, D, generator=g, device=DEV).to(torch.bfloat16)
    draft = AF.draft_rows(torch.tensor([0, m], dtype=torch.int32, device=DEV))
    outs = []
    for dirty in (False, True):
        for j in (range(m) if bad == "all" else bad) if dirty else ():
            v.view(torch.uint8)[int(table[0, (before + j) // 16]), 0, (before + j) % 16, j % D] = 0xff
        out = torch.zeros_like(q)
        ctx.attn_draft(AF.attn_desc(Hq, Hkv, D), q, cache, out, draft=draft)
        assert ctx.device_status() == AF.OK
        outs.append(out)
    first = 0 if bad == "all" else bad[0]
    assert torch.isnan(outs[1][first:]).any(2).all() and torch.equal(outs[0][:first], outs[1][:first])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,batch", [(3, 2), (200, 2), (200, 1)])
def test_a_call_of_padding_only(ctx, fmt, rows, batch):  # noqa: F811
    """No sequence has a drafted token: nothing is read, written or reported, whatever the lengths are."""
    Hq, Hkv, D = 8, 2, 64
    c = Cache([40, 0][:batch], Hkv, D, fmt, seed=90)
    before = [None if t is None else t.view(torch.uint8).clone() for t in c.dev]
    q, qkv = torch.full((rows, Hq, D), float("nan"), dtype=torch.bfloat16, device=DEV), torch.full((rows, (Hq + 2 * Hkv) * D), float("nan"), dtype=torch.bfloat16, device=DEV)
    out, lse, q_out = torch.full_like(q, 7.5), torch.full((rows, Hq), 7.5, device=DEV), torch.full_like(q, 7.5)
    draft = AF.draft_rows(torch.zeros(batch + 1, dtype=torch.int32, device=DEV))
    desc = AF.attn_desc(Hq, Hkv, D)
    ctx.cache_append(desc, qkv, c.cache, q_out, None, None, 1e-6, 1e4, draft=draft)
    ctx.attn_draft(desc, q, c.cache, out, lse, draft=draft)
    assert ctx.device_status() == AF.OK
    assert (out == 7.5).all() and (lse == 7.5).all() and (q_out == 7.5).all()
    assert all(a is None or torch.equal(a, b.view(torch.uint8)) for a, b in zip(before, c.dev))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("most", [1, 3, 60])
def test_thousands_of_sequences(ctx, fmt, most):  # noqa: F811
    """More sequences than threads plan them, many of them without a row; up to 60 rows put them on the tensor cores."""
    Hq, Hkv, D, batch = 2, 1, 64, 3000
    rng = np.random.default_rng(91)
    new = [1] * batch if most == 1 else (rng.integers(0, most + 1, batch) * (rng.random(batch) < 0.3)).tolist()
    lens = [max(1, m) + int(x) for m, x in zip(new, rng.integers(0, 40, batch))]
    if most == 60:                                                         # (few sequences with many rows: an average above the rule's border)
        new, lens, batch = new[:200], lens[:200], 200
        new = [60 if m else 25 for m in new]
        lens = [max(n, m) for n, m in zip(lens, new)]
    offs = offsets_of(new)
    T = int(offs[-1])
    c = Cache(lens, Hkv, D, fmt, seed=92)
    q = torch.randn(T, Hq, D, generator=torch.Generator().manual_seed(93)).to(torch.bfloat16).to(DEV)
    out, lse = attend(ctx, c, q, None if most == 1 else AF.draft_rows(torch.from_numpy(offs).to(DEV)))
    check_attention(out, lse, q, c, None if most == 1 else offs, None, T, WEIGHT[fmt])
