"""Attention over listed pages where scores are far below zero, infinite or no number inside the attended tokens."""
import numpy as np
import pytest
import torch

from paper_2608_01891_b200 import aflex as AF
from tests.helpers import f64
from tests.test_gpu_pages import Cache, ctx, DEV, HALF_STEP  # noqa: F401

pytestmark = pytest.mark.gpu

SHAPES = [  # Hq, Hkv, D, sequences, pages: one CTA per pair, or a cluster
    (8, 2, 64, 2, 40),
    (8, 1, 128, 1, 3),
    (4, 4, 128, 100, 9),
    (64, 8, 128, 1, 90),
]


def attend(ctx, c, q, Hq, pages):  # noqa: F811
    rows = q.shape[0]
    lst = torch.arange(pages, dtype=torch.int32, device=DEV).expand(rows, c.Hkv, pages).contiguous()
    cnt = torch.full((rows, c.Hkv), pages, dtype=torch.int32, device=DEV)
    out = torch.full((rows, Hq, c.D), 9.5, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((rows, Hq), 9.5, device=DEV)
    c.put()
    ctx.attn_decode_pages(AF.attn_desc(Hq, c.Hkv, c.D), q.to(DEV), c.kv, lst, cnt, out, lse)
    assert ctx.device_status() == AF.OK
    return f64(out), f64(lse)


def check_mean(out, lse, v, score, Hq):
    """out is the plain mean of the values v [rows][Hkv][tokens][D], lse = score + ln tokens: one rounding to bf16, before it a weight
    of exactly 1 per token in two bf16 parts, sums and a division in 32 bits; lse is a product of three factors and a sum in 32 bits."""
    rows, Hkv, n, D = v.shape
    want, size = (np.repeat(x, Hq // Hkv, axis=1) for x in (v.mean(2), np.abs(v).mean(2)))
    assert (np.abs(out - want) <= HALF_STEP * np.abs(want) + (2 * n + 64) * 2.0 ** -23 * size).all()
    want_lse = score + np.log(n)
    assert (np.abs(lse - want_lse) <= 4 * 2.0 ** -23 * abs(want_lse) + 64 * 2.0 ** -23).all()


def values(c, first, last):
    """The values of the tokens of pages [first, last) of every sequence, [rows][Hkv][tokens][D]."""
    v = f64(c.v)[c.table[:, first:last]]                                    # [rows][pages][Hkv][16][D]
    return v.transpose(0, 2, 1, 3, 4).reshape(v.shape[0], c.Hkv, -1, c.D)


@pytest.mark.parametrize("Hq,Hkv,D,B,pages", SHAPES)
def test_scores_far_below_zero_are_scores(ctx, Hq, Hkv, D, B, pages):  # noqa: F811
    """Every score -2^112 D / sqrt(D), which 32 bits hold; then the same with half of the pages at twice that, which weigh nothing."""
    c = Cache([16 * pages] * B, Hkv, D, seed=pages)
    q = torch.full((B, Hq, D), 2.0 ** 56, dtype=torch.bfloat16)
    score = -2.0 ** 112 * np.sqrt(D)
    c.k.fill_(-2.0 ** 56)
    check_mean(*attend(ctx, c, q, Hq, pages), values(c, 0, pages), score, Hq)
    for lo, hi in ((0, pages // 2), (pages // 2, pages)):                    # the heavier pages first and last
        c.k.fill_(-2.0 ** 57)
        for b in range(B):
            c.k[c.table[b, lo:hi]] = -2.0 ** 56
        check_mean(*attend(ctx, c, q, Hq, pages), values(c, lo, hi), score, Hq)


@pytest.mark.parametrize("Hq,Hkv,D,B,pages", SHAPES)
def test_infinite_scores_and_no_numbers(ctx, Hq, Hkv, D, B, pages):  # noqa: F811
    inf, nan = float("inf"), float("nan")
    c = Cache([16 * pages] * B, Hkv, D, seed=pages + 1)
    q = torch.ones(B, Hq, D, dtype=torch.bfloat16)
    # a score of -infinity weighs nothing, wherever it stands
    for lo, hi in ((0, 1), (pages - 1, pages), (1, pages - 1)):
        c.k.fill_(0.5)
        for b in range(B):
            others = [i for i in range(pages) if not lo <= i < hi]
            c.k[c.table[b, others], :, :, 5] = -inf
        check_mean(*attend(ctx, c, q, Hq, pages), values(c, lo, hi), 0.5 * np.sqrt(D), Hq)
    # nothing but -infinity: as with nothing to attend to
    c.k[..., 5] = -inf
    out, lse = attend(ctx, c, q, Hq, pages)
    assert (out == 0).all() and (lse == -np.inf).all()
    # +infinity or no number anywhere: no number, in the heads that see it and in no others
    for bad, where in ((inf, 0), (nan, pages - 1), (nan, 0), (inf, pages // 2)):
        c.k.fill_(0.5)
        c.k[c.table[0, where], Hkv - 1, 3, 2] = bad
        out, lse = attend(ctx, c, q, Hq, pages)
        sees = np.zeros((B, Hq), dtype=bool)
        sees[0, (Hkv - 1) * (Hq // Hkv):] = True
        assert np.isnan(out[sees]).all() and np.isnan(lse[sees]).all()
        assert np.isfinite(out[~sees]).all() and np.isfinite(lse[~sees]).all()
    c.k.fill_(0.5)
    q[0, 1, 7] = nan
    out, lse = attend(ctx, c, q, Hq, pages)
    sees = np.zeros((B, Hq), dtype=bool)
    sees[0, 1] = True
    assert np.isnan(out[sees]).all() and np.isnan(lse[sees]).all()
    assert np.isfinite(out[~sees]).all() and np.isfinite(lse[~sees]).all()
