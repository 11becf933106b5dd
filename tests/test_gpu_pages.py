"""Page-sparse decode attention (aflex_rope_append_bounds, aflex_page_bounds, aflex_page_select, aflex_attn_decode_pages) on the
GPU against the plain definitions in 64 bits, at the sizes where such operators go wrong, and run together as a decode step."""
import numpy as np
import pytest
import torch

from oracle import oracle as O
from oracle import pages_oracle as PO
from paper_2608_01891_b200 import aflex as AF
from paper_2608_01891_b200 import inputs as IN
from tests.helpers import f64, u16

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF_STEP = 2.0 ** -8                     # bf16: a rounding is off by at most eps / 2, relative to the value


@pytest.fixture
def ctx():
    c = AF.Context(0, 1 << 26)
    yield c
    c.close()


class Cache:
    """A paged cache with shuffled pages; slots and pages of no sequence hold NaN unless asked otherwise."""

    def __init__(self, lens, Hkv, D, seed=0, max_pages=None, poison=True, new=None):
        g = torch.Generator().manual_seed(seed)
        lens = np.asarray(lens, dtype=np.int32)
        npg = (lens + 15) // 16
        total = int(npg.sum()) + 3
        width = max_pages or max(1, int(npg.max()))
        perm = np.random.default_rng(seed).permutation(total)
        self.table = np.full((len(lens), width), -7, dtype=np.int32)      # entries past a sequence's pages are never looked at
        self.k = (torch.randn(total, Hkv, 16, D, generator=g) * torch.exp(0.7 * torch.randn(Hkv, 1, D, generator=g))).to(torch.bfloat16)
        self.v = torch.randn(total, Hkv, 16, D, generator=g).to(torch.bfloat16)
        at = 0
        for b, n in enumerate(npg):
            self.table[b, :n] = perm[at:at + n]
            at += n
        if poison:
            used = np.zeros((total, 16), dtype=bool)
            for b, n in enumerate(lens):
                for j in range(int(n)):
                    used[self.table[b, j // 16], j % 16] = True
            free = torch.from_numpy(~used)
            for t in (self.k, self.v):
                t.permute(0, 2, 1, 3)[free] = float("nan")
        self.lens, self.Hkv, self.D, self.total = lens, Hkv, D, total
        self.put()

    def put(self):
        self.kd, self.vd = self.k.to(DEV), self.v.to(DEV)
        self.td, self.ld = torch.from_numpy(self.table).to(DEV), torch.from_numpy(self.lens).to(DEV)
        self.kv = AF.make_kv(self.kd, self.vd, self.td, self.ld)
        self.codes, self.scales = AF.empty_page_bounds(self.total, self.Hkv, self.D, DEV)
        self.codes.fill_(55)
        self.scales.fill_(200)
        self.bounds = AF.make_page_bounds(self.codes, self.scales)

    def want_bounds(self, k, lens=None, first=None):
        """codes and scales of every page the sequences hold (k: stored keys), the others as they were."""
        codes, scales = np.full(tuple(self.codes.shape), 55, np.int8), np.full(tuple(self.scales.shape), 200, np.uint8)
        for b, n in enumerate(self.lens if lens is None else lens):
            for i in range((int(n) + 15) // 16):
                if first is not None and (i + 1) * 16 <= first[b]:
                    continue
                for g in range(self.Hkv):
                    p = self.table[b, i]
                    codes[p, g], scales[p, g] = PO.page_bounds(k[p, g, :min(16, int(n) - 16 * i)])
        return codes, scales


def bits(t):
    return t.detach().cpu().view(torch.int16)


# --------------------------------------------------------------------------- append
APPEND = [  # Hq, Hkv, D, norm, theta, lens, new tokens (None: one row per sequence)
    (8, 2, 64, True, 1e4, [1, 16, 17, 15, 32, 33], None),
    (8, 8, 128, False, 1e6, [1, 2, 160, 31], None),
    (64, 8, 128, True, 1e6, [5, 48, 49], None),
    (8, 1, 128, True, 5e5, [4000], None),
    (5, 5, 64, False, 1e4, list(range(1, 40)), None),
    (1, 1, 64, True, 1e4, [16], [16]),
    (16, 4, 128, True, 1e6, [37, 16, 100, 33, 5, 64], [37, 0, 1, 17, 5, 33]),
    (8, 2, 64, False, 1e4, [70, 300, 18], [3, 259, 2]),
    (4, 1, 64, True, 1e4, [20 + i % 9 for i in range(300)], [1 + i % 4 for i in range(300)]),     # more sequences than threads
    (32, 8, 128, True, 1e6, [500], [490]),
]


@pytest.mark.parametrize("Hq,Hkv,D,norm,theta,lens,new", APPEND)
def test_append_matches_the_definition(ctx, Hq, Hkv, D, norm, theta, lens, new):
    c = Cache(lens, Hkv, D, seed=len(lens) + D)
    offs = None if new is None else np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = len(lens) if new is None else int(offs[-1])
    pad = 0 if new is None else 5
    g = torch.Generator().manual_seed(7)
    qkv = torch.randn(T + pad, (Hq + 2 * Hkv) * D, generator=g).to(torch.bfloat16)
    gain = lambda: (1 + 0.1 * torch.randn(D, generator=g)).to(torch.bfloat16) if norm else None  # noqa: E731
    wq, wk = gain(), gain()
    q = torch.full((T + pad, Hq, D), 3.25, dtype=torch.bfloat16, device=DEV)
    dev = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    od = None if offs is None else torch.from_numpy(offs).to(DEV)
    ctx.rope_append_bounds(AF.attn_desc(Hq, Hkv, D), qkv.to(DEV), c.kv, c.bounds, q, dev(wq), dev(wk), 1e-6, theta, q_offsets=od)
    assert ctx.device_status() == AF.OK
    k, v = f64(c.k).copy(), f64(c.v).copy()
    want_q, size = PO.rope_append(f64(qkv), k, v, c.table, lens, Hq, Hkv, None if wq is None else f64(wq), None if wk is None else f64(wk),
                                  float(np.float32(1e-6)), theta, offs)
    # q: one rounding to bf16, and in 32 bits: norm (D products and adds, a reciprocal root), sine, cosine (2 steps each),
    # two products and a sum, each within 2^-23 of |a| + |b|
    err = np.abs(f64(q)[:T] - want_q[:T])
    assert (err <= HALF_STEP * np.abs(want_q[:T]) + (D + 16) * 2.0 ** -23 * size[:T]).all()
    assert (q[T:] == 3.25).all()                                          # padding rows stay
    # keys are formed in 64 bits: the stored bf16 is the same; everything else in the caches is as it was
    np.testing.assert_array_equal(f64(c.kd), k)
    np.testing.assert_array_equal(f64(c.vd), v)
    # bounds: of the touched pages only, as a function of the stored keys
    m = [1] * len(lens) if new is None else new
    first = [int(n) - mm if mm else 1 << 30 for n, mm in zip(lens, m)]
    codes, scales = c.want_bounds(k, first=[(f // 16) * 16 + 1 for f in first])
    np.testing.assert_array_equal(c.codes.cpu().numpy(), codes)
    np.testing.assert_array_equal(c.scales.cpu().numpy(), scales)


def test_append_agrees_with_the_one_token_operator_and_does_not_depend_on_chunking(ctx):
    Hq, Hkv, D = 16, 2, 128
    g = torch.Generator().manual_seed(1)
    n, m = 61, 45
    qkv = torch.randn(m, (Hq + 2 * Hkv) * D, generator=g).to(torch.bfloat16).to(DEV)
    w = (1 + 0.1 * torch.randn(D, generator=g)).to(torch.bfloat16).to(DEV)
    desc = AF.attn_desc(Hq, Hkv, D)
    got = []
    for cuts in ([0, 45], [0, 1, 2, 19, 20, 45], list(range(46))):
        c = Cache([n], Hkv, D, seed=5)
        q = torch.zeros(m, Hq, D, dtype=torch.bfloat16, device=DEV)
        for a, b in zip(cuts[:-1], cuts[1:]):
            c.ld.fill_(n - m + b)
            off = torch.tensor([0, b - a], dtype=torch.int32, device=DEV)
            ctx.rope_append_bounds(desc, qkv[a:b], c.kv, c.bounds, q[a:b], w, w, 1e-6, 1e6, q_offsets=off)
        got.append([bits(q), bits(c.kd), bits(c.vd), c.codes.cpu(), c.scales.cpu()])
    for other in got[1:]:
        assert all(torch.equal(x, y) for x, y in zip(got[0], other))
    c = Cache([n], Hkv, D, seed=5)
    q1 = torch.zeros(1, Hq, D, dtype=torch.bfloat16, device=DEV)
    ctx.rope_append(desc, qkv[-1:], c.kv, q1, w, w, 1e-6, 1e6)
    page = c.table[0, (n - 1) // 16]
    # two 32-bit computations of one value, each rounded to bf16: a step apart at most
    for a, b in ((f64(q1)[0], f64(q)[-1]), (f64(c.kd)[page, :, (n - 1) % 16], got[0][1].view(torch.bfloat16).double().numpy()[page, :, (n - 1) % 16])):
        assert (np.abs(a - b) <= 2 * HALF_STEP * np.maximum(np.abs(a), np.abs(b)) + 1e-5).all()
    assert ctx.device_status() == AF.OK


def test_append_far_positions(ctx):
    """Position 3,000,000: the angle is far beyond 32-bit accuracy."""
    n, D = 3_000_001, 128
    pages = (n + 15) // 16
    table = np.zeros((1, pages), dtype=np.int32)
    table[0, -1] = 1
    k = torch.zeros(2, 1, 16, D, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    codes, scales = AF.empty_page_bounds(2, 1, D, DEV)
    kv = AF.make_kv(k, v, torch.from_numpy(table).to(DEV), torch.tensor([n], dtype=torch.int32, device=DEV))
    qkv = torch.randn(1, 3 * D, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    q = torch.zeros(1, 1, D, dtype=torch.bfloat16, device=DEV)
    ctx.rope_append_bounds(AF.attn_desc(1, 1, D), qkv.to(DEV), kv, AF.make_page_bounds(codes, scales), q, None, None, 1e-6, 1e4)
    ko, vo = np.zeros((2, 1, 16, D)), np.zeros((2, 1, 16, D))
    want, size = PO.rope_append(f64(qkv), ko, vo, table, [n], 1, 1, None, None, 1e-6, 1e4)
    assert (np.abs(f64(q) - want) <= HALF_STEP * np.abs(want) + 16 * 2.0 ** -23 * size).all()
    np.testing.assert_array_equal(f64(k), ko)


def test_append_bad_inputs_are_reported_and_write_nothing(ctx):
    Hq, Hkv, D = 4, 2, 64
    desc = AF.attn_desc(Hq, Hkv, D)
    for what in ("length 0", "length over", "page", "chunk longer than its sequence", "negative chunk"):
        c = Cache([20, 40, 10], Hkv, D, seed=3)
        offs = None
        if what == "length 0":
            c.ld[1] = 0
        elif what == "length over":
            c.ld[1] = 16 * c.table.shape[1] + 1
        elif what == "page":
            c.td[1, 2] = c.total
        elif what == "chunk longer than its sequence":
            offs = torch.tensor([0, 1, 42, 43], dtype=torch.int32, device=DEV)
        else:
            offs = torch.tensor([0, 5, 2, 3], dtype=torch.int32, device=DEV)
        T = 3 if offs is None else 43
        qkv = torch.randn(T, (Hq + 2 * Hkv) * D, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
        q = torch.zeros(T, Hq, D, dtype=torch.bfloat16, device=DEV)
        ctx.rope_append_bounds(desc, qkv, c.kv, c.bounds, q, None, None, 1e-6, 1e4, q_offsets=offs)
        assert ctx.device_status() == AF.ERR_BOUNDS, what
        bad = torch.from_numpy(c.table[1, :3].astype(np.int64))
        assert torch.equal(bits(c.kd)[bad], bits(c.k)[bad]) and (c.codes.cpu()[bad] == 55).all(), what
        ok = int(c.table[2, 0])
        assert not torch.equal(bits(c.kd)[ok], bits(c.k)[ok]), what          # the others were appended


# --------------------------------------------------------------------------- bounds of a cache
@pytest.mark.parametrize("Hkv,D,lens", [(2, 64, [1, 15, 16, 17, 200]), (8, 128, [333]), (1, 128, [7, 64]), (3, 64, [100, 2])])
def test_page_bounds_matches_the_definition(ctx, Hkv, D, lens):
    c = Cache(lens, Hkv, D, seed=sum(lens))
    k = c.k
    k[c.table[0, 0], 0, 0, 3] = float("nan")                                 # among others that are numbers, or alone
    k[c.table[0, 0], 0, 0, 9] = float("inf")
    k[c.table[-1, 0], -1, 0, 40] = -float("inf")
    k[c.table[-1, 0], 0, :, 32:] = 0.0                                        # a block of zeros
    k[c.table[-1, 0], 0, 0, 33] = -0.0
    k[c.table[-1, 0], -1, 0, :32] = 1e-39                                     # subnormal
    k[c.table[-1, 0], -1, 1:, :32] = 3e37
    c.put()
    desc = AF.attn_desc(Hkv, Hkv, D)
    ctx.page_bounds(desc, c.kv, c.bounds, len(lens))
    assert ctx.device_status() == AF.OK
    codes, scales = c.want_bounds(f64(c.k))
    np.testing.assert_array_equal(c.codes.cpu().numpy(), codes)
    np.testing.assert_array_equal(c.scales.cpu().numpy(), scales)
    # only pages with tokens from first_token on
    c.put()
    first = torch.tensor([min(n - 1, 16 * (i + 1)) for i, n in enumerate(lens)], dtype=torch.int32)
    ctx.page_bounds(desc, c.kv, c.bounds, len(lens), first.to(DEV))
    codes, scales = c.want_bounds(f64(c.k), first=first.tolist())
    np.testing.assert_array_equal(c.codes.cpu().numpy(), codes)
    np.testing.assert_array_equal(c.scales.cpu().numpy(), scales)


def test_page_bounds_lengths_out_of_range_and_bad_pages(ctx):
    c = Cache([20, 40, 10], 2, 64, seed=4)
    c.ld[1] = 0                                                              # an empty sequence is no error here
    ctx.page_bounds(AF.attn_desc(2, 2, 64), c.kv, c.bounds, 3)
    assert ctx.device_status() == AF.OK
    codes, _ = c.want_bounds(f64(c.k), lens=[20, 0, 10])
    np.testing.assert_array_equal(c.codes.cpu().numpy(), codes)
    c.put()
    c.td[0, 1] = -1
    c.ld[1] = 100000                                                         # clamped to the page table's width
    c.td[1, 2] = c.total + 5
    ctx.page_bounds(AF.attn_desc(2, 2, 64), c.kv, c.bounds, 3)
    assert ctx.device_status() == AF.ERR_BOUNDS
    codes2, scales2 = c.codes.cpu().numpy(), c.scales.cpu().numpy()
    for p in (c.table[0, 1], c.table[1, 2]):
        assert (codes2[p] == 55).all() and (scales2[p] == 200).all()
    np.testing.assert_array_equal(codes2[c.table[2, 0]], codes[c.table[2, 0]])


# --------------------------------------------------------------------------- selection
def run_select(ctx, c, q, Hq, top, sink, window, offs=None):
    rows = q.shape[0]
    lst = torch.full((rows, c.Hkv, top), -2, dtype=torch.int32, device=DEV)
    cnt = torch.full((rows, c.Hkv), -2, dtype=torch.int32, device=DEV)
    od = None if offs is None else torch.from_numpy(np.asarray(offs, dtype=np.int32)).to(DEV)
    ctx.page_select(AF.attn_desc(Hq, c.Hkv, c.D), q.to(DEV), c.kv, c.bounds, top, lst, cnt, sink_pages=sink, window_pages=window, q_offsets=od)
    return lst.cpu().numpy(), cnt.cpu().numpy()


SELECT = [  # Hq, Hkv, D, lens, top, sink, window, new
    (8, 2, 64, [1, 16, 17, 64, 65, 80, 81, 300], 4, 1, 1, None),
    (8, 1, 128, [2000, 333, 16], 10, 0, 1, None),
    (2, 2, 128, [1000], 7, 2, 5, None),                     # nothing but the forced pages
    (4, 2, 64, [1000, 17 * 16, 18 * 16 + 1], 17, 3, 2, None),
    (16, 8, 128, [4100, 2049, 257 * 16], 64, 1, 2, None),
    (64, 8, 128, [900], 1, 0, 1, None),                     # the own page alone
    (4, 4, 64, [40, 700, 90], 3, 1, 1, [3, 5, 0]),
    (8, 1, 128, [21 * 16, 35], 20, 1, 4, [40, 7]),          # rows on both sides of "all pages"
]


@pytest.mark.parametrize("Hq,Hkv,D,lens,top,sink,window,new", SELECT)
def test_selection_is_the_definition_bit_for_bit(ctx, Hq, Hkv, D, lens, top, sink, window, new):
    c = Cache(lens, Hkv, D, seed=top + D)
    ctx.page_bounds(AF.attn_desc(Hq, Hkv, D), c.kv, c.bounds, len(lens))
    offs = None if new is None else np.concatenate([[0], np.cumsum(new)])
    rows = len(lens) if new is None else int(offs[-1]) + 3
    q = torch.randn(rows, Hq, D, generator=torch.Generator().manual_seed(9)).to(torch.bfloat16)
    got = run_select(ctx, c, q, Hq, top, sink, window, offs)
    assert ctx.device_status() == AF.OK
    want = PO.page_select(f64(q), c.codes.cpu().numpy(), c.scales.cpu().numpy(), c.table, lens, top, sink, window, offs)
    np.testing.assert_array_equal(got[1], want[1])
    np.testing.assert_array_equal(got[0], want[0])


GROUPS = [  # Hq, Hkv, D, lens, top, sink, window, new, padding rows
    (16, 8, 64, [500, 333, 700, 64, 1200], 9, 1, 2, [4, 4, 4, 4, 4], 0),
    (8, 8, 128, [900, 400], 12, 0, 1, [16, 16], 0),             # groups of eight, one page more for the later rows
    (8, 8, 128, [400, 300, 257], 16, 2, 2, [11, 11, 11], 0),    # a prime number of rows per sequence
    (8, 4, 64, [600, 90, 17, 450, 800, 33], 5, 1, 1, [9, 1, 0, 20, 7, 13], 5),      # groups across sequences and padding
    (8, 8, 64, [40, 500, 35], 4, 1, 1, [9, 9, 9], 0),           # rows that see everything beside rows that choose
    (8, 8, 64, [300, 200, 250], 3, 1, 2, [8, 8, 8], 0),         # nothing but the forced pages
    (16, 8, 128, [200 + 31 * i for i in range(13)], 6, 1, 1, [6] * 13, 0),          # more than the GPU holds with eight warps each
    (8, 8, 64, [150 + 31 * i for i in range(17)], 6, 1, 1, [1 + i % 7 for i in range(17)], 3),
]


@pytest.mark.parametrize("Hq,Hkv,D,lens,top,sink,window,new,pad", GROUPS)
def test_selection_of_neighbouring_rows(ctx, Hq, Hkv, D, lens, top, sink, window, new, pad):
    """Enough (row, head) pairs that rows of a sequence are scored together."""
    c = Cache(lens, Hkv, D, seed=top + D, max_pages=600)
    ctx.page_bounds(AF.attn_desc(Hq, Hkv, D), c.kv, c.bounds, len(lens))
    offs = np.concatenate([[0], np.cumsum(new)])
    rows = int(offs[-1]) + pad
    assert rows * Hkv > 148 and rows >= 3 * len(lens)
    q = torch.randn(rows, Hq, D, generator=torch.Generator().manual_seed(9)).to(torch.bfloat16)
    got = run_select(ctx, c, q, Hq, top, sink, window, offs)
    assert ctx.device_status() == AF.OK
    want = PO.page_select(f64(q), c.codes.cpu().numpy(), c.scales.cpu().numpy(), c.table, lens, top, sink, window, offs)
    np.testing.assert_array_equal(got[1], want[1])
    np.testing.assert_array_equal(got[0], want[0])
    # a sequence shorter than its rows is reported; the others are as they were
    c.ld[1] = new[1] - 1
    if new[1] > 1:
        bad = run_select(ctx, c, q, Hq, top, sink, window, offs)
        assert ctx.device_status() == AF.ERR_BOUNDS
        others = np.r_[0:offs[1], offs[2]:rows]
        np.testing.assert_array_equal(bad[0][others], want[0][others])
        assert (bad[1][offs[1]] == 0).all() and (bad[0][offs[1]] == -1).all()


SPREAD = [  # Hq, Hkv, D, lens, top, sink, window, new, padding rows, page table width
    (8, 4, 64, [300 + 37 * i for i in range(14)], 7, 1, 1, [5] * 14, 0, 100),                # four rows' pairs of heads in one MMA; groups < SMs
    (4, 4, 128, [100 + 97 * i for i in range(13)], 5, 0, 2, [7] * 13, 0, 100),               # a head per row
    (64, 8, 128, [250 + 53 * i for i in range(22)], 6, 1, 1, [3] * 22, 0, 100),              # more groups than SMs, 2 CTAs on one
    (32, 8, 64, [60 + 11 * i for i in range(45)], 5, 1, 2, [2] * 45, 0, 60),                 # 3 CTAs
    (8, 8, 128, [40 + 17 * i for i in range(60)], 4, 1, 1, [2] * 60, 0, 70),                 # 4 CTAs
    (16, 8, 64, [90 + 13 * i for i in range(40)], 4, 1, 1, [7] * 40, 0, 60),                 # 4 CTAs of seven rows, a warp each
    (16, 8, 128, [40 + 31 * i for i in range(23)], 6, 1, 1, [1 + 5 * i % 9 for i in range(23)], 3, 60),     # uneven numbers of rows
    (32, 8, 128, [500, 3000, 33000, 90], 30, 1, 2, [8, 8, 8, 8], 0, 2100),                   # clusters, long rows
    (16, 8, 64, [2000 + 900 * i for i in range(7)], 20, 1, 2, [5] * 7, 0, 2100),             # of seven CTAs
    (16, 8, 64, [2000 + 900 * i for i in range(7)], 20, 1, 2, [5] * 7, 0, 700),              # of four
    (8, 8, 64, [9000, 40, 12000], 40, 2, 2, [3, 9, 5], 2, 2500),                             # clusters across sequences
    (8, 8, 64, [100 + 7 * i for i in range(30)], 5, 1, 1, [8] * 30, 0, 6000),                # scores that need two CTAs' shared memory
    (8, 8, 64, [90000, 50], 60, 1, 2, [8, 8], 0, 30000),                                     # eight
    (8, 8, 64, [70000, 50], 60, 1, 2, [4, 4], 0, 60000),                                     # more than there are
]


@pytest.mark.parametrize("Hq,Hkv,D,lens,top,sink,window,new,pad,width", SPREAD)
def test_selection_of_neighbouring_rows_however_they_are_spread(ctx, Hq, Hkv, D, lens, top, sink, window, new, pad, width):
    """Few and many groups, short and long tables: one CTA per group or several, of 8 or 16 warps, with and without a crowd."""
    c = Cache(lens, Hkv, D, seed=top + D, max_pages=width)
    ctx.page_bounds(AF.attn_desc(Hq, Hkv, D), c.kv, c.bounds, len(lens))
    offs = np.concatenate([[0], np.cumsum(new)])
    rows = int(offs[-1]) + pad
    assert rows >= 2 * len(lens)
    q = torch.randn(rows, Hq, D, generator=torch.Generator().manual_seed(width)).to(torch.bfloat16)
    codes, scales = c.codes.cpu().numpy(), c.scales.cpu().numpy()
    for _ in range(2):
        got = run_select(ctx, c, q, Hq, top, sink, window, offs)
        assert ctx.device_status() == AF.OK
        want = PO.page_select(f64(q), codes, scales, c.table, lens, top, sink, window, offs)
        n = int(offs[-1])
        np.testing.assert_array_equal(got[1][:n], want[1][:n])
        np.testing.assert_array_equal(got[0][:n], want[0][:n])
        assert (got[0][n:] == -2).all() and (got[1][n:] == -2).all()
        # the same with crowds of equal scores: every page's bounds one of two
        two = [(codes[c.table[0, 0]].copy(), scales[c.table[0, 0]].copy()), (codes[c.table[0, 1]].copy(), scales[c.table[0, 1]].copy())]
        for i in range(c.total):
            codes[i], scales[i] = two[i % 3 == 0]
        c.codes.copy_(torch.from_numpy(codes))
        c.scales.copy_(torch.from_numpy(scales))


def test_selection_ties_and_odd_queries(ctx):
    lens = [50 * 16 - 3] * 6
    c = Cache(lens, 2, 128, seed=1)
    g = torch.Generator().manual_seed(3)
    # few distinct codes: many equal scores
    c.codes.copy_(torch.randint(-1, 2, c.codes.shape, generator=g).to(torch.int8))
    c.codes[:, :, :, 1] = -1
    c.codes[:, :, 4:] = 1
    c.scales.copy_(torch.randint(126, 128, c.scales.shape, generator=g).to(torch.uint8))
    q = torch.randn(6, 8, 128, generator=g).to(torch.bfloat16)
    q[0] = 0.0
    q[1, :, :120] = 0.0
    q[2, 0] = float("nan")
    q[3, 1, 5] = float("inf")
    q[4] = 1e-30
    q[5, :, 7] = 2e38
    got = run_select(ctx, c, q, 8, 23, 2, 3)
    want = PO.page_select(f64(q), c.codes.cpu().numpy(), c.scales.cpu().numpy(), c.table, lens, 23, 2, 3)
    np.testing.assert_array_equal(got[0], want[0])
    np.testing.assert_array_equal(got[1], want[1])


def test_selection_from_bounds_that_nobody_made(ctx):
    """Any bytes as bounds: the lists are still lists of the sequence's pages."""
    lens = [3000, 90, 16 * 40]
    c = Cache(lens, 2, 64, seed=2)
    g = torch.Generator().manual_seed(8)
    q = (torch.randn(3, 4, 64, generator=g) * torch.exp(20 * torch.randn(3, 4, 64, generator=g))).to(torch.bfloat16)
    q[0, 0, :3] = torch.tensor([float("nan"), float("inf"), -float("inf")])
    for scales in ((0, 256), (250, 256), (0, 2), (255, 256)):
        c.codes.copy_(torch.randint(-128, 128, c.codes.shape, generator=g).to(torch.int8))
        c.scales.copy_(torch.randint(*scales, c.scales.shape, generator=g).to(torch.uint8))
        for top in (7, 39):
            lst, cnt = run_select(ctx, c, q, 4, top, 1, 2)
            assert ctx.device_status() == AF.OK
            for b, n in enumerate(lens):
                pages = (n + 15) // 16
                assert (cnt[b] == min(top, pages)).all()
                for h in range(2):
                    got = lst[b, h, :cnt[b, h]]
                    assert (np.diff(got) > 0).all() and got[0] >= 0 and got[-1] == pages - 1 and (lst[b, h, cnt[b, h]:] == -1).all()


@pytest.mark.parametrize("n_pages,rows", [(129, 1), (1024, 1), (5003, 2), (60001, 1)])
def test_selection_over_long_caches(ctx, n_pages, rows):
    """Every cluster size; at 60001 pages the scores no longer fit one CTA's shared memory.  Pages are shared, so scores repeat."""
    Hq, Hkv, D, pool = 8, 2, 64, 700
    g = torch.Generator().manual_seed(n_pages)
    table = torch.randint(0, pool, (rows, n_pages), generator=g, dtype=torch.int32)
    lens = torch.tensor([n_pages * 16 - 5 - 3 * i for i in range(rows)], dtype=torch.int32)
    k = torch.zeros(pool, Hkv, 16, D, dtype=torch.bfloat16, device=DEV)
    kv = AF.make_kv(k, k, table.to(DEV), lens.to(DEV))
    codes, scales = AF.empty_page_bounds(pool, Hkv, D, DEV)
    codes.copy_(torch.randint(-127, 128, codes.shape, generator=g).to(torch.int8))
    scales.copy_(torch.randint(120, 128, scales.shape, generator=g).to(torch.uint8))
    q = torch.randn(rows, Hq, D, generator=g).to(torch.bfloat16)
    for top in (5, 100, min(4000, n_pages - 1)):
        lst = torch.full((rows, Hkv, top), -2, dtype=torch.int32, device=DEV)
        cnt = torch.full((rows, Hkv), -2, dtype=torch.int32, device=DEV)
        ctx.page_select(AF.attn_desc(Hq, Hkv, D), q.to(DEV), kv, AF.make_page_bounds(codes, scales), top, lst, cnt, sink_pages=1, window_pages=2)
        want = PO.page_select(f64(q), codes.cpu().numpy(), scales.cpu().numpy(), table.numpy(), lens.tolist(), top, 1, 2)
        np.testing.assert_array_equal(lst.cpu().numpy(), want[0])
        np.testing.assert_array_equal(cnt.cpu().numpy(), want[1])
    assert ctx.device_status() == AF.OK


def test_selection_bad_inputs_are_reported(ctx):
    c = Cache([500, 400, 300], 2, 64, seed=8)
    ctx.page_bounds(AF.attn_desc(4, 2, 64), c.kv, c.bounds, 3)
    q = torch.randn(3, 4, 64, generator=torch.Generator().manual_seed(9)).to(torch.bfloat16)
    want, _ = run_select(ctx, c, q, 4, 6, 1, 1)
    assert ctx.device_status() == AF.OK
    c.ld[1] = 0
    got, cnt = run_select(ctx, c, q, 4, 6, 1, 1)
    assert ctx.device_status() == AF.ERR_BOUNDS
    assert (cnt[1] == 0).all() and (got[1] == -1).all()
    np.testing.assert_array_equal(got[[0, 2]], want[[0, 2]])
    c.ld[1] = 400
    c.td[1, 3] = 1 << 30
    got, cnt = run_select(ctx, c, q, 4, 6, 1, 1)
    assert ctx.device_status() == AF.ERR_BOUNDS
    np.testing.assert_array_equal(got[[0, 2]], want[[0, 2]])


# --------------------------------------------------------------------------- attention
def check_attention(out, lse, want_out, want_lse, slack, D):
    """out: one rounding to bf16; before it, in 32 bits: a score is D products and adds and a scaling, each within 2^-23 of
    sum |q_d K_d| * scale (which moves p by that much, above and below the line); an exponential, the two-part P (2^-16) and
    a sum over the tokens, with one more rescaling per page and join."""
    mag, num, absv = slack
    score = (D + 8) * 2.0 ** -23 * mag
    rel = 2 * score + 2.0 ** -16 + (2 * num + 64) * 2.0 ** -23
    assert (np.abs(f64(out) - want_out) <= HALF_STEP * np.abs(want_out) + rel[..., None] * absv).all()
    if lse is not None:
        empty = np.isinf(want_lse)
        got = f64(lse)
        assert (got[empty] == -np.inf).all()
        tol = score + (2 * num + 64) * 2.0 ** -23 + 4 * 2.0 ** -23 * np.abs(np.where(empty, 0, want_lse))
        assert (np.abs(got[~empty] - want_lse[~empty]) <= tol[~empty]).all()


def random_lists(lens, Hkv, top, seed, offs=None, own=True):
    rng = np.random.default_rng(seed)
    rows = PO.rows_of(lens, offs)
    lst = np.full((len(rows), Hkv, top), -1, dtype=np.int32)
    cnt = np.zeros((len(rows), Hkv), dtype=np.int32)
    for r, b, pos in rows:
        n = pos // 16 + 1
        for g in range(Hkv):
            take = rng.permutation(n)[:int(rng.integers(0, min(n, top) + 1))]
            if own and len(take) and n - 1 not in take:
                take[0] = n - 1
            lst[r, g, :len(take)] = rng.permutation(take)                    # any order
            cnt[r, g] = len(take)
    return lst, cnt


ATTEND = [  # Hq, Hkv, D, lens, top, new
    (8, 2, 64, [1, 15, 16, 17, 40, 300], 5, None),
    (8, 1, 128, [2000], 90, None),
    (64, 8, 128, [700, 1, 33], 33, None),
    (2, 2, 128, [300] * 70, 7, None),
    (32, 8, 128, [150 + i for i in range(130)], 3, None),                    # enough (row, head) pairs for one CTA each
    (4, 1, 64, [5000, 4999], 300, None),
    (16, 4, 64, [40, 700, 9], 12, [4, 7, 0]),
    (12, 3, 128, [65], 4, [33]),
]


ATTEND += [  # (row, head) pairs that take one CTA more per SM
    (8, 8, 128, [40 + 9 * i for i in range(41)], 9, None),
    (8, 8, 64, [33 + 5 * i for i in range(65)], 9, None),
    (16, 8, 128, [200 + i for i in range(81)], 5, None),
]


@pytest.mark.parametrize("Hq,Hkv,D,lens,top,new", ATTEND)
def test_attention_matches_the_definition(ctx, Hq, Hkv, D, lens, top, new):
    c = Cache(lens, Hkv, D, seed=top)
    offs = None if new is None else np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    lst, cnt = random_lists(lens, Hkv, top, seed=D, offs=offs)
    T = lst.shape[0]
    pad = 0 if new is None else 2
    lst = np.concatenate([lst, np.full((pad, Hkv, top), 77, np.int32)])
    cnt = np.concatenate([cnt, np.full((pad, Hkv), 3, np.int32)])
    q = torch.randn(T + pad, Hq, D, generator=torch.Generator().manual_seed(11)).to(torch.bfloat16)
    out = torch.full((T + pad, Hq, D), 9.5, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((T + pad, Hq), 9.5, device=DEV)
    od = None if offs is None else torch.from_numpy(offs).to(DEV)
    args = (AF.attn_desc(Hq, Hkv, D), q.to(DEV), c.kv, torch.from_numpy(lst).to(DEV), torch.from_numpy(cnt).to(DEV), out)
    ctx.attn_decode_pages(*args, lse, q_offsets=od)
    assert ctx.device_status() == AF.OK
    want = PO.attn_pages(f64(q), f64(c.k), f64(c.v), c.table, lens, lst, cnt, offs)
    check_attention(out[:T], lse[:T], want[0][:T], want[1][:T], [s[:T] for s in want[2]], D)
    assert (out[T:] == 9.5).all() and (lse[T:] == 9.5).all()
    again = torch.empty_like(out)
    ctx.attn_decode_pages(*args[:-1], again, q_offsets=od)                   # without lse; the same bits again
    assert torch.equal(bits(again[:T]), bits(out[:T]))


def test_attention_scale_and_large_scores(ctx):
    """Scores of some hundreds: every weight but a few underflows."""
    c = Cache([400, 90], 2, 128, seed=2)
    c.k.mul_(12.0)
    c.put()
    lst, cnt = random_lists([400, 90], 2, 20, seed=1)
    q = (torch.randn(2, 8, 128, generator=torch.Generator().manual_seed(4)) * 4).to(torch.bfloat16)
    out = torch.empty(2, 8, 128, dtype=torch.bfloat16, device=DEV)
    lse = torch.empty(2, 8, device=DEV)
    ctx.attn_decode_pages(AF.attn_desc(8, 2, 128, 0.25), q.to(DEV), c.kv, torch.from_numpy(lst).to(DEV), torch.from_numpy(cnt).to(DEV), out, lse)
    want = PO.attn_pages(f64(q), f64(c.k), f64(c.v), c.table, [400, 90], lst, cnt, sm_scale=0.25)
    check_attention(out, lse, *want, 128)


def test_attention_repeated_page_counts_twice_and_bad_entries_are_left_out(ctx):
    c = Cache([100, 60], 1, 64, seed=6)
    q = torch.randn(2, 4, 64, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16)
    desc = AF.attn_desc(4, 1, 64)
    run = lambda l, n: (ctx.attn_decode_pages(desc, q.to(DEV), c.kv, torch.tensor(l, dtype=torch.int32, device=DEV),  # noqa: E731
                                              torch.tensor(n, dtype=torch.int32, device=DEV), out, lse), ctx.device_status())[1]
    out = torch.empty(2, 4, 64, dtype=torch.bfloat16, device=DEV)
    lse = torch.empty(2, 4, device=DEV)
    both = [[[2, 2, 6, 0]], [[3, 0, 3, 3]]]
    assert run(both, [[3], [4]]) == AF.OK
    want = PO.attn_pages(f64(q), f64(c.k), f64(c.v), c.table, [100, 60], np.array(both), np.array([[3], [4]]))
    check_attention(out, lse, *want, 64)
    bad = [[[2, -1, 6, 7]], [[4, 1 << 20, -5, 100]]]                          # page 6 holds the last token of row 0; row 1 has 0 .. 3
    assert run(bad, [[4], [4]]) == AF.ERR_BOUNDS
    want = PO.attn_pages(f64(q), f64(c.k), f64(c.v), c.table, [100, 60], np.array(bad), np.array([[4], [4]]))
    check_attention(out, lse, *want, 64)
    assert (f64(out)[1] == 0).all()
    assert run(both, [[-3], [400]]) == AF.OK                                  # counts are clamped to [0, top_pages]
    assert (f64(out)[0] == 0).all() and (f64(lse)[0] == -np.inf).all()
    c.td[0, 2] = c.total
    assert run(both, [[3], [4]]) == AF.ERR_BOUNDS
    c.td[0, 2] = int(c.table[0, 2])
    c.ld[0] = 0
    assert run(both, [[3], [4]]) == AF.ERR_BOUNDS
    assert (f64(out)[0] == 0).all() and (f64(out)[1] != 0).any()


# --------------------------------------------------------------------------- together, as a decode step
def test_all_pages_listed_agrees_with_dense_attention(ctx):
    lens = [1, 17, 300, 64, 999]
    Hq, Hkv, D = 16, 2, 128
    c = Cache(lens, Hkv, D, seed=12)
    desc = AF.attn_desc(Hq, Hkv, D)
    ctx.page_bounds(desc, c.kv, c.bounds, len(lens))
    q = torch.randn(len(lens), Hq, D, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16)
    lst = torch.empty(len(lens), Hkv, 63, dtype=torch.int32, device=DEV)
    cnt = torch.empty(len(lens), Hkv, dtype=torch.int32, device=DEV)
    out, dense = torch.empty_like(q, device=DEV), torch.empty_like(q, device=DEV)
    lse, lse_d = torch.empty(len(lens), Hq, device=DEV), torch.empty(len(lens), Hq, device=DEV)
    qd = q.to(DEV)
    ctx.page_select(desc, qd, c.kv, c.bounds, 63, lst, cnt)
    ctx.attn_decode_pages(desc, qd, c.kv, lst, cnt, out, lse)
    ctx.attn_decode(desc, qd, c.kv, dense, lse_d)
    assert ctx.device_status() == AF.OK
    assert cnt.cpu()[:, 0].tolist() == [(n + 15) // 16 for n in lens]
    want, want_lse = O.attn_decode(u16(q), u16(c.k), u16(c.v), np.where(c.table < 0, 0, c.table), c.lens)[:2]
    _, _, slack = PO.attn_pages(f64(q), f64(c.k), f64(c.v), c.table, lens, lst.cpu().numpy(), cnt.cpu().numpy())
    check_attention(out, lse, want, want_lse, slack, D)
    assert (lse - lse_d).abs().max() < 1e-3


def layer_front(ctx, cfg, w, desc, x, xn, qkv):
    ctx.add_rmsnorm(x, None, w["ln_attn"], cfg.rms_eps, None, xn)
    ctx.linear(xn, w["qkv"], qkv)


@pytest.mark.parametrize("graph", [False, True])
def test_decode_steps_of_a_layer_with_sparse_attention(ctx, graph):
    """norm -> QKV -> append with bounds -> selection -> attention -> W_o, three tokens in a row on a cache that prefill filled,
    eagerly and as one captured and replayed graph; every operator against its definition on what it read."""
    cfg = IN.LayerConfig(31, "sparse-step", 3, 8, 2, 64, 256, 384, len_dist="uniform", len_lo=100, len_hi=400, rope_theta=1.0e4)
    Hq, Hkv, D, B, H = 8, 2, 64, 3, 256
    lens = np.array([150, 16 * 20, 333], dtype=np.int32)
    c = Cache(lens + 3, Hkv, D, seed=21, poison=False)
    w = {k: (t.to(DEV) if t is not None else None) for k, t in vars(IN.make_decoder_weights(cfg)).items()}
    desc = AF.attn_desc(Hq, Hkv, D)
    c.ld.copy_(torch.from_numpy(lens))
    ctx.page_bounds(desc, c.kv, c.bounds, B)                                 # the cache came from somewhere else
    top = 8
    x = torch.zeros(B, H, dtype=torch.bfloat16, device=DEV)
    xn, o = torch.empty_like(x), torch.empty_like(x)
    qkv = torch.empty(B, (Hq + 2 * Hkv) * D, dtype=torch.bfloat16, device=DEV)
    q = torch.empty(B, Hq, D, dtype=torch.bfloat16, device=DEV)
    a = torch.empty_like(q)
    lst = torch.empty(B, Hkv, top, dtype=torch.int32, device=DEV)
    cnt = torch.empty(B, Hkv, dtype=torch.int32, device=DEV)
    lse = torch.empty(B, Hq, device=DEV)

    def step():
        c.ld.add_(1)
        layer_front(ctx, cfg, w, desc, x, xn, qkv)
        ctx.rope_append_bounds(desc, qkv, c.kv, c.bounds, q, w["q_norm"], w["k_norm"], cfg.rms_eps, cfg.rope_theta)
        ctx.page_select(desc, q, c.kv, c.bounds, top, lst, cnt)
        ctx.attn_decode_pages(desc, q, c.kv, lst, cnt, a, lse)
        ctx.linear(a.view(B, Hq * D), w["o"], o)

    g = torch.Generator().manual_seed(2)
    side = torch.cuda.Stream()
    if graph:
        # the un-captured warm-up that the library asks for, on scratch copies of what it changes
        kb, vb, cb, sb = c.kd.clone(), c.vd.clone(), c.codes.clone(), c.scales.clone()
        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        for t, s in ((c.kd, kb), (c.vd, vb), (c.codes, cb), (c.scales, sb)):
            t.copy_(s)
        c.ld.copy_(torch.from_numpy(lens))
        cg = torch.cuda.CUDAGraph()
        with torch.cuda.graph(cg, stream=side):
            step()
    k, v = f64(c.kd).copy(), f64(c.vd).copy()
    for t in range(1, 4):
        x.copy_(torch.randn(B, H, generator=g).to(torch.bfloat16))
        torch.cuda.synchronize()
        if graph:
            cg.replay()
        else:
            with torch.cuda.stream(side):                                    # not the tensors' own stream
                step()
        torch.cuda.synchronize()
        now = lens + t
        want_q, size = PO.rope_append(f64(qkv), k, v, c.table, now, Hq, Hkv, f64(w["q_norm"]), f64(w["k_norm"]), float(np.float32(cfg.rms_eps)), cfg.rope_theta)
        assert (np.abs(f64(q) - want_q) <= HALF_STEP * np.abs(want_q) + (D + 16) * 2.0 ** -23 * size).all()
        np.testing.assert_array_equal(f64(c.kd), k)
        np.testing.assert_array_equal(f64(c.vd), v)
        codes, scales = c.want_bounds(k, lens=now)
        used = np.concatenate([c.table[b, :(now[b] + 15) // 16] for b in range(B)])
        np.testing.assert_array_equal(c.codes.cpu().numpy()[used], codes[used])
        np.testing.assert_array_equal(c.scales.cpu().numpy()[used], scales[used])
        want = PO.page_select(f64(q), codes, scales, c.table, now, top, 1, 2)
        np.testing.assert_array_equal(lst.cpu().numpy(), want[0])
        att = PO.attn_pages(f64(q), k, v, c.table, now, *want)
        check_attention(a, lse, *att, D)
        assert (np.abs(f64(o) - f64(a).reshape(B, -1) @ f64(w["o"]).T) <= HALF_STEP * np.abs(f64(o)) + 512 * 2.0 ** -23 * (np.abs(f64(a)).reshape(B, -1) @ np.abs(f64(w["o"])).T)).all()
    assert ctx.device_status() == AF.OK


def test_prefill_chunk_then_drafted_rows(ctx):
    """A prompt appended in two chunks, then four drafted tokens per sequence selected and attended to at once: every row
    sees its own past only, and agrees with the same token decoded alone."""
    Hq, Hkv, D, m = 8, 2, 128, 4
    lens = np.array([130, 97], dtype=np.int32)
    c = Cache(lens, Hkv, D, seed=30)
    desc = AF.attn_desc(Hq, Hkv, D)
    g = torch.Generator().manual_seed(6)
    qkv = torch.randn(int(lens.sum()), (Hq + 2 * Hkv) * D, generator=g).to(torch.bfloat16).to(DEV)
    parts = [qkv[:130], qkv[130:]]
    q = torch.empty(qkv.shape[0], Hq, D, dtype=torch.bfloat16, device=DEV)
    done = np.zeros(2, dtype=np.int64)
    for part in (np.array([60, 1]), np.array([66, 92]), np.array([4, 4])):
        rows = torch.cat([parts[b][done[b]:done[b] + part[b]] for b in range(2)]).contiguous()
        done += part
        c.ld.copy_(torch.from_numpy(done.astype(np.int32)))
        off = torch.tensor([0, part[0], part.sum()], dtype=torch.int32, device=DEV)
        qs = torch.empty(rows.shape[0], Hq, D, dtype=torch.bfloat16, device=DEV)
        ctx.rope_append_bounds(desc, rows, c.kv, c.bounds, qs, None, None, 1e-6, 1e6, q_offsets=off)
    top = 5
    new = lambda *s, dt=torch.int32: torch.empty(*s, dtype=dt, device=DEV)  # noqa: E731
    lst, cnt, out = new(2 * m, Hkv, top), new(2 * m, Hkv), new(2 * m, Hq, D, dt=torch.bfloat16)
    ctx.page_select(desc, qs, c.kv, c.bounds, top, lst, cnt, q_offsets=off)
    ctx.attn_decode_pages(desc, qs, c.kv, lst, cnt, out, q_offsets=off)
    kh, vh = f64(c.kd), f64(c.vd)
    want = PO.page_select(f64(qs), c.codes.cpu().numpy(), c.scales.cpu().numpy(), c.table, lens, top, 1, 2, [0, m, 2 * m])
    np.testing.assert_array_equal(lst.cpu().numpy(), want[0])
    att = PO.attn_pages(f64(qs), kh, vh, c.table, lens, *want, [0, m, 2 * m])
    check_attention(out, None, *att, D)
    for i in range(m):
        c.ld.copy_(torch.from_numpy(lens - (m - 1 - i)))
        one, n1, o1 = new(2, Hkv, top), new(2, Hkv), new(2, Hq, D, dt=torch.bfloat16)
        pick = qs[[i, m + i]].contiguous()
        ctx.page_select(desc, pick, c.kv, c.bounds, top, one, n1)
        ctx.attn_decode_pages(desc, pick, c.kv, one, n1, o1)
        assert torch.equal(one.cpu(), lst.cpu()[[i, m + i]])
        assert torch.equal(bits(o1), bits(out[[i, m + i]]))
    assert ctx.device_status() == AF.OK


TINY_MOE = IN.LayerConfig(33, "sparse-moe", 6, 8, 2, 64, 256, 384, num_experts=4, top_k=2, len_dist="uniform", len_lo=16, len_hi=600,
                          rms_eps=1e-5, qk_norm=False)
SPARSE_DENSE = IN.LayerConfig(34, "sparse-dense", 7, 16, 2, 128, 512, 640, len_dist="uniform", len_lo=1, len_hi=900)


class Layers:
    """`n` decoder layers of one configuration with a cache, key bounds and weights each."""

    def __init__(self, cfg, n):
        self.cfg, self.n = cfg, n
        kvh = IN.make_paged_kv(cfg)
        self.kvh = kvh
        self.table, self.lens = kvh.page_table.to(DEV), kvh.seq_lens.to(DEV)
        self.attn = AF.attn_desc(cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim)
        self.w, self.descs, self.kvs, self.caches, self.bounds = [], [], [], [], []
        for l in range(n):
            w = {k: (None if t is None else t.to(DEV)) for k, t in vars(IN.make_decoder_weights(cfg, l)).items()}
            layer = AF.layer_desc(self.attn, cfg.hidden, cfg.inter, w["o"], w["gate"], w["up"], w["down"], cfg.num_experts, cfg.top_k, w["router"])
            k, v = kvh.k_cache.to(DEV, copy=True), kvh.v_cache.to(DEV, copy=True)
            self.w.append(w)
            self.descs.append(AF.decoder_desc(layer, w["qkv"], w["ln_attn"], w["ln_ffn"], w["q_norm"], w["k_norm"], cfg.rms_eps, cfg.rope_theta))
            self.caches.append((k, v))
            self.kvs.append(AF.make_kv(k, v, self.table, self.lens, kvh.seq_lens))
            self.bounds.append(AF.make_page_bounds(*AF.empty_page_bounds(k.shape[0], cfg.num_kv_heads, cfg.head_dim, DEV)))
        self.x = IN.make_hidden(cfg).to(DEV)

    def reset(self, ctx):
        for (k, v), kv, b in zip(self.caches, self.kvs, self.bounds):
            k.copy_(self.kvh.k_cache)
            v.copy_(self.kvh.v_cache)
            ctx.page_bounds(self.attn, kv, b, self.cfg.batch)


def rows_apart(a, b):
    """Largest difference of a row over its largest value."""
    a, b = f64(a), f64(b)
    return (np.abs(a - b).max(-1) / np.abs(b).max(-1)).max()


@pytest.mark.parametrize("cfg", [SPARSE_DENSE, TINY_MOE], ids=lambda c: c.name)
@pytest.mark.parametrize("depth", [1, 2])
def test_sparse_decoder_layers_with_every_page_are_the_dense_ones(cfg, depth):
    L = Layers(cfg, 2)
    top = int((int(L.kvh.seq_lens.max()) + 15) // 16)
    ctx = AF.Context(0, AF.decoder_sparse_workspace_bytes(L.descs[0], cfg.batch, top))
    try:
        dense, sparse = torch.empty_like(L.x), torch.empty_like(L.x)
        L.reset(ctx)
        ctx.decoder_layers(L.descs, L.kvs, L.x, dense, depth)
        caches = [(k.clone(), v.clone()) for k, v in L.caches]
        L.reset(ctx)
        ctx.decoder_layers_sparse(L.descs, L.kvs, L.bounds, top, L.x, sparse, microbatch_depth=depth)
        assert ctx.device_status() == AF.OK
        # two chains of the same bf16 roundings (some twenty a layer, each off by at most 2^-8 of its row's largest value, and
        # adding up like independent ones): as far apart as the chain is from its definition elsewhere in these tests
        assert rows_apart(sparse, dense) <= 2e-2
        for (k, v), (kd, vd) in zip(L.caches, caches):
            assert rows_apart(k, kd) <= 2e-2 and rows_apart(v, vd) <= 2e-2
        # the bounds of every page are those of the cache as it now is
        for (k, _), kv, b in zip(L.caches, L.kvs, L.bounds):
            fresh = AF.make_page_bounds(*AF.empty_page_bounds(k.shape[0], cfg.num_kv_heads, cfg.head_dim, DEV))
            ctx.page_bounds(L.attn, kv, fresh, cfg.batch)
            assert all(torch.equal(x, y) for x, y in zip(b._keep, fresh._keep))
    finally:
        ctx.close()


@pytest.mark.parametrize("cfg", [SPARSE_DENSE, TINY_MOE], ids=lambda c: c.name)
def test_sparse_decoder_layer_is_its_operators_in_turn(cfg):
    L = Layers(cfg, 1)
    B, H, Hq, Hkv, D = cfg.batch, cfg.hidden, cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim
    top, w = 5, L.w[0]
    ctx = AF.Context(0, AF.decoder_sparse_workspace_bytes(L.descs[0], B, top))
    try:
        got = torch.empty_like(L.x)
        L.reset(ctx)
        ctx.decoder_layers_sparse(L.descs, L.kvs, L.bounds, top, L.x, got, sink_pages=0, window_pages=2)
        after = [t.clone() for t in (*L.caches[0], *L.bounds[0]._keep)]
        L.reset(ctx)
        new = lambda *s, dt=torch.bfloat16: torch.empty(*s, dtype=dt, device=DEV)  # noqa: E731
        xn, qkv, q, a, o, h1, y, out = new(B, H), new(B, (Hq + 2 * Hkv) * D), new(B, Hq, D), new(B, Hq, D), new(B, H), new(B, H), new(B, H), new(B, H)
        lst, cnt = new(B, Hkv, top, dt=torch.int32), new(B, Hkv, dt=torch.int32)
        layer_front(ctx, cfg, w, L.attn, L.x, xn, qkv)
        ctx.rope_append_bounds(L.attn, qkv, L.kvs[0], L.bounds[0], q, w["q_norm"], w["k_norm"], cfg.rms_eps, cfg.rope_theta)
        ctx.page_select(L.attn, q, L.kvs[0], L.bounds[0], top, lst, cnt, sink_pages=0, window_pages=2)
        ctx.attn_decode_pages(L.attn, q, L.kvs[0], lst, cnt, a)
        ctx.linear(a.view(B, -1), w["o"], o)
        ctx.add_rmsnorm(L.x, o, w["ln_ffn"], cfg.rms_eps, h1, xn)
        if cfg.num_experts:
            ctx.ffn_moe(xn, w["gate"], w["up"], w["down"], cfg.top_k, y, w_router=w["router"])
        else:
            ctx.ffn_dense(xn, w["gate"], w["up"], w["down"], y)
        ctx.add_rmsnorm(h1, y, None, 0.0, out, None)
        assert ctx.device_status() == AF.OK
        assert (cnt.max() == top) and int(L.kvh.seq_lens.max()) > 16 * top        # something had to be chosen
        assert rows_apart(got, out) <= 2e-2
        for x, z in zip(after, (*L.caches[0], *L.bounds[0]._keep)):
            assert torch.equal(x, z)                                              # the same kernels on the same qkv
    finally:
        ctx.close()


def test_sparse_decoder_layers_refusals():
    cfg = SPARSE_DENSE
    L = Layers(cfg, 1)
    ctx = AF.Context(0, AF.decoder_sparse_workspace_bytes(L.descs[0], cfg.batch, 4))
    try:
        out = torch.empty_like(L.x)
        run = lambda top, bounds=None, **kw: ctx.decoder_layers_sparse(L.descs, L.kvs, bounds or L.bounds, top, L.x, out, **kw)  # noqa: E731
        small = AF.Context(0, 1 << 20)
        with pytest.raises(AF.AflexError) as e:
            small.decoder_layers_sparse(L.descs, L.kvs, L.bounds, 4, L.x, out)
        assert e.value.status == AF.ERR_WORKSPACE
        small.close()
        for f, status in [(lambda: run(2), AF.ERR_INVALID_ARG), (lambda: run(4, window_pages=0), AF.ERR_INVALID_ARG),
                          (lambda: run(4, bounds=[AF.KeyBounds(None, None)]), AF.ERR_INVALID_ARG), (lambda: run(4, microbatch_depth=99), AF.ERR_INVALID_ARG)]:
            with pytest.raises(AF.AflexError) as e:
                f()
            assert e.value.status == status
        assert ctx.launch_count() == 0
        L.reset(ctx)
        run(4)
        assert ctx.device_status() == AF.OK
    finally:
        ctx.close()


def test_two_streams_at_once(ctx):
    """The calls keep nothing in the context's workspace: two streams may run them at the same time."""
    made = []
    for seed, lens in ((40, [900, 333, 64]), (41, [1500, 20])):
        Hq, Hkv, D = 16, 4, 128
        c = Cache(lens, Hkv, D, seed=seed)
        q = torch.randn(len(lens), Hq, D, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)
        B = len(lens)
        new = lambda *s, dt=torch.int32: torch.zeros(*s, dtype=dt, device=DEV)  # noqa: E731
        made.append((c, lens, q, q.to(DEV), new(B, Hkv, 12), new(B, Hkv), new(B, Hq, D, dt=torch.bfloat16), new(B, Hq, dt=torch.float32)))
    desc = AF.attn_desc(16, 4, 128)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, (c, lens, _, qd, lst, cnt, out, lse) in zip(streams, made):
            ctx.page_bounds(desc, c.kv, c.bounds, len(lens), stream=s)
            ctx.page_select(desc, qd, c.kv, c.bounds, 12, lst, cnt, stream=s)
            ctx.attn_decode_pages(desc, qd, c.kv, lst, cnt, out, lse, stream=s)
    torch.cuda.synchronize()
    for c, lens, q, _, lst, cnt, out, lse in made:
        want = PO.page_select(f64(q), c.codes.cpu().numpy(), c.scales.cpu().numpy(), c.table, lens, 12, 1, 2)
        np.testing.assert_array_equal(lst.cpu().numpy(), want[0])
        check_attention(out, lse, *PO.attn_pages(f64(q), f64(c.k), f64(c.v), c.table, lens, *want), 128)
    assert ctx.device_status() == AF.OK


def test_row_offsets_that_name_few_rows(ctx):
    """A batch padded to a fixed number of rows and sequences, as a captured step has it: empty sequences, and rows behind the last."""
    Hq, Hkv, D = 8, 2, 64
    lens = [100, 40, 0, 0]
    c = Cache(lens, Hkv, D, seed=50)
    desc = AF.attn_desc(Hq, Hkv, D)
    ctx.page_bounds(desc, c.kv, c.bounds, 4)
    offs = torch.tensor([0, 1, 2, 2, 2], dtype=torch.int32, device=DEV)
    g = torch.Generator().manual_seed(1)
    qkv = torch.randn(4, (Hq + 2 * Hkv) * D, generator=g).to(torch.bfloat16)
    full = lambda *s, dt: torch.full(s, 7, dtype=dt, device=DEV)  # noqa: E731
    q, out, lse = full(4, Hq, D, dt=torch.bfloat16), full(4, Hq, D, dt=torch.bfloat16), full(4, Hq, dt=torch.float32)
    lst, cnt = full(4, Hkv, 3, dt=torch.int32), full(4, Hkv, dt=torch.int32)
    ctx.rope_append_bounds(desc, qkv.to(DEV), c.kv, c.bounds, q, None, None, 1e-6, 1e4, q_offsets=offs)
    ctx.page_select(desc, q, c.kv, c.bounds, 3, lst, cnt, sink_pages=0, q_offsets=offs)
    ctx.attn_decode_pages(desc, q, c.kv, lst, cnt, out, lse, q_offsets=offs)
    assert ctx.device_status() == AF.OK
    for t in (q, out, lse, lst, cnt):
        assert (t[2:] == 7).all() and not (t[:2] == 7).all()
    want = PO.page_select(f64(q), c.codes.cpu().numpy(), c.scales.cpu().numpy(), c.table, lens, 3, 0, 2, offs.tolist())
    np.testing.assert_array_equal(lst[:2].cpu().numpy(), want[0][:2])
    att = PO.attn_pages(f64(q), f64(c.kd), f64(c.vd), c.table, lens, lst.cpu().numpy(), cnt.cpu().numpy(), offs.tolist())
    check_attention(out[:2], lse[:2], att[0][:2], att[1][:2], [s[:2] for s in att[2]], D)
    # nothing at all
    offs.zero_()
    ctx.rope_append_bounds(desc, qkv.to(DEV), c.kv, c.bounds, q.fill_(3), None, None, 1e-6, 1e4, q_offsets=offs)
    ctx.page_select(desc, q, c.kv, c.bounds, 3, lst.fill_(3), cnt, q_offsets=offs)
    ctx.attn_decode_pages(desc, q, c.kv, lst, cnt, out.fill_(3), lse, q_offsets=offs)
    assert ctx.device_status() == AF.OK
    assert (q == 3).all() and (lst == 3).all() and (out == 3).all()


def test_heads_of_every_group_size_and_a_large_pool_index(ctx):
    """Pages far into the pools: element offsets beyond 32 bits."""
    Hkv, D, pool = 8, 128, 140_000                                           # 140,000 pages x 8 heads x 16 x 128 elements > 2^31
    k = torch.zeros(pool, Hkv, 16, D, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    pages = [pool - 1, pool - 77, 3]
    g = torch.Generator().manual_seed(5)
    k[pages] = torch.randn(3, Hkv, 16, D, generator=g).to(torch.bfloat16).to(DEV)
    v[pages] = torch.randn(3, Hkv, 16, D, generator=g).to(torch.bfloat16).to(DEV)
    codes, scales = AF.empty_page_bounds(pool, Hkv, D, DEV)
    bounds = AF.make_page_bounds(codes, scales)
    kv = AF.make_kv(k, v, torch.tensor([pages], dtype=torch.int32, device=DEV), torch.tensor([47], dtype=torch.int32, device=DEV))
    small_k, small_v, table = f64(k[pages]), f64(v[pages]), np.array([[0, 1, 2]])
    for G in (1, 2, 4, 8):
        Hq = G * Hkv
        desc = AF.attn_desc(Hq, Hkv, D)
        qkv = torch.randn(1, (Hq + 2 * Hkv) * D, generator=g).to(torch.bfloat16)
        q = torch.empty(1, Hq, D, dtype=torch.bfloat16, device=DEV)
        ctx.page_bounds(desc, kv, bounds, 1)
        ctx.rope_append_bounds(desc, qkv.to(DEV), kv, bounds, q, None, None, 1e-6, 1e4)
        PO.rope_append(f64(qkv), small_k, small_v, table, [47], Hq, Hkv, None, None, 1e-6, 1e4)
        np.testing.assert_array_equal(f64(k[pages]), small_k)
        sc, ss = codes[pages].cpu().numpy(), scales[pages].cpu().numpy()
        for i, n in enumerate((16, 16, 15)):
            for h in range(Hkv):
                want = PO.page_bounds(small_k[i, h, :n])
                np.testing.assert_array_equal(sc[i, h], want[0])
                np.testing.assert_array_equal(ss[i, h], want[1])
        lst = torch.empty(1, Hkv, 2, dtype=torch.int32, device=DEV)
        cnt = torch.empty(1, Hkv, dtype=torch.int32, device=DEV)
        out, lse = torch.empty_like(q), torch.empty(1, Hq, device=DEV)
        ctx.page_select(desc, q, kv, bounds, 2, lst, cnt, sink_pages=0, window_pages=1)
        want = PO.page_select(f64(q), sc, ss, table, [47], 2, 0, 1)
        np.testing.assert_array_equal(lst.cpu().numpy(), want[0])
        ctx.attn_decode_pages(desc, q, kv, lst, cnt, out, lse)
        check_attention(out, lse, *PO.attn_pages(f64(q), small_k, small_v, table, [47], *want), D)
    assert ctx.device_status() == AF.OK
