"""Operators on caches of 16 or 8 bits and on drafted tokens: what they launch, where, and on which stream, on the stand-in for the CUDA
runtime of test_host_launches.py (no GPU)."""
import ctypes

import pytest

from paper_2608_01891_b200 import aflex as AF
from test_host_launches import KV, P, ctx, decoder, host  # noqa: F401 (fixtures)

CACHE = {"bf16": AF.Cache(KV, AF.CACHE_BF16, None, None), "int8": AF.Cache(KV, AF.CACHE_INT8, P, P), "e4m3": AF.Cache(KV, AF.CACHE_E4M3, P, P)}
ENTRIES = ["cache_append", "cache_convert", "attn_draft", "cache_accept", "draft_layers"]


def call(lib, ctx, name, fmt, batch=3, rows=15, Hq=8, Hkv=2, D=64, caches=2, stream=None):
    d, c, dr = AF.attn_desc(Hq, Hkv, D), CACHE[fmt], AF.Draft(P, P, P, 1)
    if name == "cache_append":
        return lib.aflex_cache_append(ctx._h, d, P, c, batch, dr, rows, None, None, 1e-6, 1e4, P, stream)
    if name == "cache_convert":
        other = AF.Cache(AF.KV(2 * P, 2 * P, 100, P, 10, P, None), AF.CACHE_INT8 if fmt == "bf16" else AF.CACHE_BF16, *((P, P) if fmt == "bf16" else (None, None)))
        return lib.aflex_cache_convert(ctx._h, d, c, other, batch, None, stream)
    if name == "attn_draft":
        return lib.aflex_attn_draft(ctx._h, d, P, c, batch, dr, rows, P, P, stream)
    if name == "cache_accept":
        return lib.aflex_cache_accept(ctx._h, d, (AF.Cache * caches)(*[c] * caches), caches, batch, P, P, 4, P, stream)
    layers = [decoder(1024, Hq=Hq, Hkv=Hkv, D=D), decoder(64, experts=4, Hq=Hq, Hkv=Hkv, D=D)]
    return lib.aflex_draft_layers(ctx._h, (AF.DecoderDesc * 2)(*layers), (AF.Cache * 2)(c, c), 2, P, batch, dr, rows, P, stream)


@pytest.mark.parametrize("fmt", list(CACHE))
@pytest.mark.parametrize("name", ENTRIES)
def test_launches_go_to_the_contexts_device_and_stream_and_the_callers_device_comes_back(host, name, fmt):  # noqa: F811
    c = AF.Context(1, 1 << 30)
    host.host_set_device(0)
    host.host_forget()
    try:
        assert call(host, c, name, fmt, stream=0x77) == AF.OK, host.aflex_last_error(c._h)
        n = host.host_launch_count()
        assert n > 0 and all(host.host_launch_device(i) == 1 and host.host_launch_stream(i) == 0x77 for i in range(n))
        assert host.host_device() == 0
    finally:
        c.close()


@pytest.mark.parametrize("caches, launches", [(1, 1), (64, 1), (65, 2), (130, 3)])
def test_up_to_64_caches_are_compacted_by_one_launch(host, ctx, caches, launches):  # noqa: F811
    assert call(host, ctx, "cache_accept", "int8", caches=caches) == AF.OK
    assert host.host_launch_count() == launches


@pytest.mark.parametrize("rows, batch, Hq, Hkv, D, kernel", [
    (4, 4, 8, 1, 64, "attn_draft_kernel"),               # one token per sequence, 8 lines: a tile of 8
    (12, 4, 8, 2, 128, "attn_draft_kernel"),             # 12 lines
    (32, 1, 8, 8, 128, "attn_draft_kernel"),             # 32 lines of heads of 128
    (33, 1, 8, 8, 128, "attn_draft_wide_kernel"),
    (48, 1, 8, 8, 64, "attn_draft_kernel"),              # 48 of 64
    (49, 1, 8, 8, 64, "attn_draft_wide_kernel"),
])
@pytest.mark.parametrize("fmt", list(CACHE))
def test_the_kernel_follows_the_lines_of_an_average_sequence(host, ctx, fmt, rows, batch, Hq, Hkv, D, kernel):  # noqa: F811
    assert call(host, ctx, "attn_draft", fmt, batch=batch, rows=rows, Hq=Hq, Hkv=Hkv, D=D) == AF.OK
    assert [host.host_launch_name(i).decode().count(kernel) for i in range(host.host_launch_count())] == [1]


@pytest.mark.parametrize("fmt", list(CACHE))
def test_draft_layers_append_and_attend_once_per_layer(host, ctx, fmt):  # noqa: F811
    assert call(host, ctx, "draft_layers", fmt) == AF.OK
    names = [host.host_launch_name(i).decode() for i in range(host.host_launch_count())]
    for kernel in ("cache_append_kernel", "attn_draft"):
        assert sum(kernel in n for n in names) == 2
    assert not any("rope_append_kernel" in n or "attn_decode" in n for n in names)
