"""Operators on caches of 16 or 8 bits and drafted tokens: what the host checks of calls that the tests beside this one do not make (no GPU)."""
import ctypes

import pytest
import torch

from paper_2608_01891_b200 import aflex as AF
from test_host_launches import P, ctx, host  # noqa: F401 (fixtures)


def lens_cache(fmt, lens, pages=10):
    kv = AF.KV(P, P, 100, P, pages, P, ctypes.cast((ctypes.c_int32 * len(lens))(*lens), ctypes.c_void_p) if lens else None)
    return AF.Cache(kv, fmt, None if fmt == AF.CACHE_BF16 else P, None if fmt == AF.CACHE_BF16 else P)


@pytest.mark.parametrize("to", [AF.CACHE_INT8, AF.CACHE_E4M3, AF.CACHE_BF16])
def test_a_conversion_knows_empty_sequences(host, ctx, to):  # noqa: F811
    """Lengths of 0 are allowed, on the host as on the device; the destination's are not looked at."""
    desc = AF.attn_desc(8, 2, 64)
    fmt = AF.CACHE_INT8 if to == AF.CACHE_BF16 else AF.CACHE_BF16
    for src, dst, want in (([3, 0, 160], [], AF.OK), ([0, 0, 0], [], AF.OK), ([3, 1, 160], [0, -5, 9999], AF.OK), ([3, -1, 160], [], AF.ERR_INVALID_ARG),
                           ([3, 0, 161], [], AF.ERR_INVALID_ARG)):
        a, b = lens_cache(fmt, src), lens_cache(to, dst)
        host.host_forget()
        assert host.aflex_cache_convert(ctx._h, desc, a, b, 3, None, None) == want, (src, host.aflex_last_error(ctx._h))
        assert host.host_launch_count() == (want == AF.OK)
        assert want == AF.OK or b"seq_lens_host[" in host.aflex_last_error(ctx._h)


def test_rows_of_an_unknown_number_of_sequences_are_refused():
    """A Draft made by hand holds the address of its offsets, not how many there are: taken for one row per sequence, they would be read past their end."""
    class Stream:
        cuda_stream = 0

    c = AF.Context.__new__(AF.Context)
    c._lib, c._h, c.device = AF.load_library(), None, -1
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)  # noqa: E731
    k, v, ks, vs = AF.empty_cache(6, 2, 64, torch.int8, device="cpu")
    lens, table = z(8, dt=torch.int32), z(8, 4, dt=torch.int32)
    cache, desc, q, qkv = AF.make_cache(k, v, table, lens, ks, vs), AF.attn_desc(8, 2, 64), z(8, 8, 64), z(8, 12 * 64)
    offsets = torch.tensor([0, 5, 8], dtype=torch.int32)
    layer = AF.decoder_desc(AF.layer_desc(desc, 256, 512, q, q, q, q), q, q, q, None, None, 1e-6, 1e4)
    x = z(8, 256)
    for draft, error in ((AF.Draft(offsets.data_ptr(), None, None, 0), AssertionError), (AF.Draft(None, None, None, 0), AF.AflexError),
                         (AF.draft_rows(offsets), AF.AflexError)):                        # (AflexError: the library refuses, for want of a context)
        for call in (lambda: c.cache_append(desc, qkv, cache, q, None, None, 1e-6, 1e4, draft=draft, stream=Stream),
                     lambda: c.attn_draft(desc, q, cache, q, draft=draft, stream=Stream),
                     lambda: c.draft_layers([layer], [cache], x, x, draft=draft, stream=Stream)):
            with pytest.raises(error):
                call()
