"""Selection of pages where many candidates share the interval of scores that holds the last page to keep, for rows that one warp
selects for (five to eight rows of a sequence, more groups of them than the GPU has SMs) and for rows with more warps."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as PO
from paper_2608_01891_b200 import aflex as AF
from tests.helpers import f64
from tests.test_gpu_pages import Cache, ctx, DEV  # noqa: F401

pytestmark = pytest.mark.gpu

CROWDS = [  # Hq, Hkv, D, sequences, rows of each, pages, top, sink, window
    (8, 8, 64, 30, 8, 60, 52, 1, 2),            # 240 groups: two CTAs per SM, 57 candidates of which 49 are kept
    (16, 8, 128, 24, 5, 60, 50, 0, 2),          # 192 groups
    (8, 8, 64, 45, 6, 64, 60, 1, 1),            # 360 groups: three
    (8, 8, 128, 60, 7, 40, 37, 0, 1),           # 480 groups: four
    (8, 8, 64, 20, 8, 400, 150, 1, 2),          # a crowd that is divided again first
    (32, 8, 128, 19, 5, 300, 47, 2, 3),
    (8, 8, 64, 10, 8, 60, 52, 1, 2),            # 80 groups: more warps per row
    (8, 8, 64, 60, 1, 60, 52, 1, 2),            # a CTA per row and head
]


def last_interval(scores, keep):
    """(candidates, still to be kept) in that of the 256 equal intervals of the scores which holds the keep-th highest."""
    s = scores.astype(np.float64)
    per = 256.0 / max(s.max() - s.min(), 1e-30)
    i = np.clip(np.floor((s - s.min()) * per), 0, 255).astype(int)
    n = np.bincount(i, minlength=256)[::-1]
    above = np.cumsum(n) - n
    k = np.nonzero((above < keep) & (above + n >= keep))[0][0]
    return int(n[k]), int(keep - above[k])


@pytest.mark.parametrize("bounds", ["equal", "one page far above the others"])
@pytest.mark.parametrize("Hq,Hkv,D,seqs,each,pages,top,sink,window", CROWDS)
def test_selection_out_of_a_crowd(ctx, Hq, Hkv, D, seqs, each, pages, top, sink, window, bounds):  # noqa: F811
    lens = [16 * pages - 3] * seqs
    c = Cache(lens, Hkv, D, seed=pages + D)
    ctx.page_bounds(AF.attn_desc(Hq, Hkv, D), c.kv, c.bounds, seqs)
    if bounds == "equal":
        c.codes.zero_()
        c.scales.fill_(127)
    else:
        far = torch.from_numpy(c.table[:, sink + 3].astype(np.int64)).to(DEV)        # 2^12 times as large as it was
        c.scales[far] += 12
    rows = seqs * each
    offs = None if each == 1 else np.arange(seqs + 1) * each
    q = torch.randn(rows, Hq, D, generator=torch.Generator().manual_seed(each)).to(torch.bfloat16)
    codes, scales = c.codes.cpu().numpy(), c.scales.cpu().numpy()
    want = PO.page_select(f64(q), codes, scales, c.table, lens, top, sink, window, offs)
    # the case is the one it is meant to be: more members than a warp has lanes, and the last to keep behind the first 32 of them
    keep, crowded = top - sink - window, 0
    for r in range(0, rows, 7):
        pg = c.table[r // each, sink:pages - window]
        members, need = last_interval(PO.page_scores(f64(q)[r, :Hq // Hkv], codes[pg, 0], scales[pg, 0]), keep)
        crowded += members > 32 and need > 32
    assert crowded > 0
    guard = 64                                                                       # words behind the lists and the counts
    lst = torch.full((rows * Hkv * top + guard,), -2, dtype=torch.int32, device=DEV)
    cnt = torch.full((rows * Hkv + guard,), -2, dtype=torch.int32, device=DEV)
    n, m = rows * Hkv * top, rows * Hkv
    ctx.page_select(AF.attn_desc(Hq, Hkv, D), q.to(DEV), c.kv, c.bounds, top, lst[:n].view(rows, Hkv, top), cnt[:m].view(rows, Hkv),
                    sink_pages=sink, window_pages=window, q_offsets=None if offs is None else torch.from_numpy(offs.astype(np.int32)).to(DEV))
    assert ctx.device_status() == AF.OK
    np.testing.assert_array_equal(cnt[:m].view(rows, Hkv).cpu().numpy(), want[1])
    np.testing.assert_array_equal(lst[:n].view(rows, Hkv, top).cpu().numpy(), want[0])
    assert (lst[n:] == -2).all() and (cnt[m:] == -2).all()
