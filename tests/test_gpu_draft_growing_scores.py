"""Attention of drafted tokens where the scores outgrow what was seen before, again and again along the cache: the running references move at
chosen tokens (in every part of a step of 128, and several times in one), for lines of one warp at different ones.  And bits of a line do not
depend on whether another line's references moved."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as DO
from paper_2608_01891_b200 import aflex as AF
from test_gpu_draft import DEV, FORMATS, TYPES, Cache, check_attention, ctx, f64, offsets_of  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu
JUMPS = [(5, 40, 70, 100, 130, 190, 200, 260, 300, 383), (0, 127, 128, 255), (64, 65, 66, 192, 395, 399), (300, )]


def grown(fmt, Hkv, D, n):
    """A cache of one sequence of n tokens whose KV head g has channel 0 growing by 24 at every token of JUMPS[g], above random ones."""
    c = Cache([n], Hkv, D, fmt, seed=11)
    gen = torch.Generator().manual_seed(12)
    for g in range(Hkv):
        level = torch.zeros(n)
        for t in JUMPS[g % len(JUMPS)]:
            level[t:] += 24
        k = 0.5 * torch.randn(n, D, generator=gen)
        k[:, 0] = level
        for t in range(n):
            page, slot, x = int(c.table[0, t // 16]), t % 16, k[t].to(torch.bfloat16)
            if fmt == "bf16":
                c.tensors[0][page, g, slot] = x
            else:
                code, scale = DO.quantise(f64(x), fmt)
                c.tensors[0][page, g, slot] = torch.from_numpy(code).float().to(TYPES[fmt])
                c.tensors[2][page, g, slot] = float(scale)
    c.put()
    return c


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("Hq,Hkv,D,m", [(4, 4, 64, 1), (32, 4, 128, 1), (16, 4, 64, 3), (16, 4, 128, 6), (32, 4, 64, 20), (32, 4, 128, 40)])
def test_references_follow_growing_scores(ctx, fmt, Hq, Hkv, D, m):  # noqa: F811
    n = 400
    c = grown(fmt, Hkv, D, n)
    gen = torch.Generator().manual_seed(13)
    q = torch.randn(m, Hq, D, generator=gen)
    q[:, :, 0] = 8.0 * torch.randn(m, Hq, generator=gen)                   # (of either sign: some lines' scores grow by 17 a jump, some fall)
    q = q.to(torch.bfloat16).to(DEV)
    out, lse = torch.zeros_like(q), torch.zeros(m, Hq, device=DEV)
    offs = offsets_of([m])
    ctx.attn_draft(AF.attn_desc(Hq, Hkv, D), q, c.cache, out, lse, draft=AF.draft_rows(torch.from_numpy(offs).to(DEV)))
    assert ctx.device_status() == AF.OK
    check_attention(out, lse, q, c, offs, None, m, 2.0 ** -17 if fmt == "bf16" else 2.0 ** -12)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,m", [(64, 20), (128, 6), (128, 40)])
def test_a_line_does_not_depend_on_the_others_scores(ctx, fmt, D, m):  # noqa: F811
    """Every second line's queries exchanged for ones with scores that grow: the other lines come out the same, bit for bit."""
    Hq, Hkv, n = 8, 2, 400
    c = grown(fmt, Hkv, D, n)
    gen = torch.Generator().manual_seed(14)
    calm, wild = torch.randn(m, Hq, D, generator=gen), torch.randn(m, Hq, D, generator=gen)
    calm[:, :, 0] = 0
    wild[:, :, 0] = 8
    mixed = calm.clone()
    mixed[:, 1::2] = wild[:, 1::2]
    got = []
    for q in (calm, mixed):
        q = q.to(torch.bfloat16).to(DEV)
        out, lse = torch.zeros_like(q), torch.zeros(m, Hq, device=DEV)
        ctx.attn_draft(AF.attn_desc(Hq, Hkv, D), q, c.cache, out, lse, draft=AF.draft_rows(torch.from_numpy(offsets_of([m])).to(DEV)))
        assert ctx.device_status() == AF.OK
        got.append((out, lse))
    assert torch.equal(got[0][0][:, 0::2], got[1][0][:, 0::2]) and torch.equal(got[0][1][:, 0::2], got[1][1][:, 0::2])
    assert not torch.equal(got[0][0][:, 1::2], got[1][0][:, 1::2])
