"""Attention of drafted tokens and the operators around it where one value decides: references that move twice in a step of the tensor-core kernel."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as DO
from paper_2608_01891_b200 import aflex as AF
from test_gpu_draft import DEV, FORMATS, TYPES, Cache, check_attention, ctx, f64, offsets_of  # noqa: F401 (fixtures)

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
