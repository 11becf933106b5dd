"""Operators on caches of 16 or 8 bits and drafted tokens: what the host checks of calls that the tests beside this one do not make (no GPU)."""
import ctypes

import pytest

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
