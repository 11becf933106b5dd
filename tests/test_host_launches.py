"""What the entry points launch, and with which addresses, on a stand-in for the CUDA runtime (host_runtime.cpp): the library's own
objects, no GPU.  What only shows when kernels of two streams overlap, or with a second GPU, is decided here on the host."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2608_01891_b200 import aflex as AF
from paper_2608_01891_b200 import build as B

HERE = os.path.dirname(os.path.abspath(__file__))
P = 0x600000000000                          # an address that nothing follows


class SelectArgs(ctypes.Structure):
    """The argument of the page selection kernels, up to its outputs."""
    _fields_ = ([(n, ctypes.c_uint64) for n in ("q", "codes", "scales", "page_table", "seq_lens", "q_offsets")]
                + [(n, ctypes.c_int) for n in ("batch", "rows", "max_pages", "Hq", "Hkv", "G")] + [("num_pages", ctypes.c_longlong)]
                + [(n, ctypes.c_int) for n in ("top", "sink", "window", "cluster", "group", "stride", "row_warps")]
                + [("list", ctypes.c_uint64), ("count", ctypes.c_uint64)])


class AttendArgs(ctypes.Structure):
    """The argument of the kernel of attention over listed pages, up to its outputs."""
    _fields_ = ([(n, ctypes.c_uint64) for n in ("q", "k_cache", "v_cache", "page_table", "seq_lens", "q_offsets", "list", "count")]
                + [(n, ctypes.c_int) for n in ("batch", "rows", "max_pages", "Hq", "Hkv", "G", "top", "cluster")] + [("num_pages", ctypes.c_longlong)]
                + [("scale_log2", ctypes.c_float), ("out", ctypes.c_uint64), ("lse", ctypes.c_uint64)])


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    """The library on the stand-in, in the place of the real one."""
    B.build()
    objs = [os.path.join(B.HERE, "build", s + ".o") for s in B.SOURCES]
    if not all(os.path.exists(o) for o in objs):
        B.build(force=True)
    tmp = tmp_path_factory.mktemp("host")
    so, exports = str(tmp / "libaflex_host.so"), tmp / "exports"
    exports.write_text("{ global: aflex_*; host_*; local: *; };")
    cuda = os.path.join(os.path.dirname(os.path.dirname(B.NVCC)), "include")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", cuda, "-o", so, *objs, os.path.join(HERE, "host_runtime.cpp"),
                    f"-Wl,--version-script={exports}", "-Wl,--no-undefined"], check=True)
    mp = pytest.MonkeyPatch()
    mp.setattr(AF, "LIB_PATH", so)
    mp.setattr(AF, "_lib", None)
    lib = AF.load_library()
    lib.host_launch_name.restype = ctypes.c_char_p
    lib.host_launch_arg.restype = lib.host_launch_stream.restype = ctypes.c_void_p
    yield lib
    mp.undo()


@pytest.fixture
def ctx(host):
    host.host_set_device(0)
    c = AF.Context(0, 1 << 30)
    host.host_forget()
    yield c
    c.close()


def decoder(inter, experts=0, Hq=8, Hkv=2, D=64, hidden=256):
    attn = AF.attn_desc(Hq, Hkv, D)
    layer = AF.LayerDesc(attn, hidden, inter, experts, 2 if experts else 0, P, P, P, P, P if experts else None)
    return AF.DecoderDesc(layer, P, P, P, None, None, 1e-6, 1e4)


KV = AF.KV(P, P, 100, P, 10, P, None)


def run_sparse(lib, ctx, layers, batch, top, depth):
    """-> [(kernel name, device, stream, arguments of selection and attention, else None)]"""
    lib.host_forget()
    n = len(layers)
    bounds = (AF.KeyBounds * n)(*[AF.KeyBounds(P, P)] * n)
    st = lib.aflex_decoder_layers_sparse(ctx._h, (AF.DecoderDesc * n)(*layers), (AF.KV * n)(*[KV] * n), bounds, AF.PagePolicy(top, 1, 2), n, P, batch,
                                         depth, None, P, None)
    assert st == AF.OK, lib.aflex_last_error(ctx._h)
    out = []
    for i in range(lib.host_launch_count()):
        name = lib.host_launch_name(i).decode()
        kind = SelectArgs if "page_select" in name else AttendArgs if "attn_decode_pages" in name else None
        arg = kind.from_buffer_copy(ctypes.string_at(lib.host_launch_arg(i), ctypes.sizeof(kind))) if kind else None
        out.append((name, lib.host_launch_device(i), lib.host_launch_stream(i), arg))
    return out


def list_places(launched, batch, top, Hkv=2):
    """(start, end) of the page lists and of the counts of every selection, and whether its arguments are what they should be."""
    args = [a for *_, a in launched if isinstance(a, SelectArgs)]
    assert args and all(a.top == top and a.Hkv == Hkv and a.rows == a.batch and a.rows <= batch for a in args)
    return [(a.list, a.list + 4 * a.rows * Hkv * top) for a in args] + [(a.count, a.count + 4 * a.rows * Hkv) for a in args]


@pytest.mark.parametrize("depth", [1, 2])
@pytest.mark.parametrize("order", ["dense, MoE", "MoE, dense", "dense, MoE, dense"])
def test_page_lists_lie_in_no_layers_scratch(host, ctx, depth, order):
    """Layers with another FFN beside them have larger or smaller FFN scratch, which is used on another stream while the next layer's
    lists are written.  A layer alone has its lists behind its scratch: in a chain every list has to lie behind every layer's."""
    batch, top = 24, 5
    kinds = {"dense": decoder(8192), "MoE": decoder(64, experts=4)}
    alone = {}
    for k, d in kinds.items():
        alone[k] = min(a for a, _ in list_places(run_sparse(host, ctx, [d], batch, top, depth), batch, top))
    assert alone["dense"] > alone["MoE"] + 100000                  # (the case tells the two apart)
    chain = [kinds[k] for k in order.split(", ")]
    launched = run_sparse(host, ctx, chain, batch, top, depth)
    assert all(a >= max(alone.values()) for a, _ in list_places(launched, batch, top))
    # and a workspace of the size that the library asks for holds them
    small = AF.Context(0, max(AF.decoder_sparse_workspace_bytes(d, batch, top) for d in chain))
    try:
        assert all(host.host_allocated(ctypes.c_uint64(a), ctypes.c_uint64(b))
                   for a, b in list_places(run_sparse(host, small, chain, batch, top, depth), batch, top))
    finally:
        small.close()


@pytest.mark.parametrize("inter", [1024, 64])
def test_rows_of_a_microbatch_lie_apart_from_the_others_in_every_layer(host, ctx, inter):
    """Attention output of A_{l+1,i} is written while F_{l,j} reads that of its own rows (the output projection is part of the FFN's
    kernel), so no layer, however wide its heads together, may have a microbatch's rows where another layer has another one's."""
    batch, depth = 12, 3
    chain = [decoder(inter, Hq=4, Hkv=2), decoder(inter, Hq=16, Hkv=2), decoder(inter, Hq=8, Hkv=8, D=128), decoder(inter, Hq=4, Hkv=4)]
    args = [a for *_, a in run_sparse(host, ctx, chain, batch, 5, depth) if isinstance(a, AttendArgs)]
    assert len(args) == depth * len(chain)
    assert all(a.Hq == d.layer.attn.num_q_heads and a.rows == batch // depth for a, d in zip(args, [d for d in chain for _ in range(depth)]))
    for of in (lambda a: a.q, lambda a: a.out):
        rows = [[] for _ in range(depth)]
        for i, (a, d) in enumerate(zip(args, [d for d in chain for _ in range(depth)])):
            rows[i % depth].append((of(a), of(a) + 2 * a.rows * a.Hq * d.layer.attn.head_dim))
        for i in range(depth):
            for j in range(i):
                assert all(b0 <= a1 or b1 <= a0 for a0, b0 in rows[i] for a1, b1 in rows[j])


@pytest.mark.parametrize("depth", [1, 2])
@pytest.mark.parametrize("name", ["rope_append_bounds", "page_bounds", "page_select", "attn_decode_pages", "decoder_layers_sparse"])
def test_launches_go_to_the_contexts_device_and_the_callers_comes_back(host, name, depth):
    """The page-sparse entry points, called with another device current than the context's."""
    ctx = AF.Context(1, 1 << 30)
    host.host_set_device(0)
    host.host_forget()
    try:
        d, kv, b, a = AF.attn_desc(8, 2, 64), ctypes.byref(KV), ctypes.byref(AF.KeyBounds(P, P)), AF.PagePolicy(5, 1, 2)
        rows = 6 * depth
        if name == "rope_append_bounds":
            st = host.aflex_rope_append_bounds(ctx._h, d, P, kv, b, rows, None, rows, None, None, 1e-6, 1e4, P, None)
        elif name == "page_bounds":
            st = host.aflex_page_bounds(ctx._h, d, kv, b, rows, None, None)
        elif name == "page_select":
            st = host.aflex_page_select(ctx._h, d, P, kv, b, a, rows, None, rows, P, P, None)
        elif name == "attn_decode_pages":
            st = host.aflex_attn_decode_pages(ctx._h, d, P, kv, P, P, 5, rows, None, rows, P, None, None)
        else:
            st = AF.OK
            run_sparse(host, ctx, [decoder(1024), decoder(64, experts=4)], rows, 5, depth)
        assert st == AF.OK
        n = host.host_launch_count()
        assert n > 0 and all(host.host_launch_device(i) == 1 for i in range(n))
        assert host.host_device() == 0
    finally:
        ctx.close()


def test_no_more_listed_pages_than_32_bit_counters_take(host, ctx):
    """Lists of more than 2^26 pages (as many as a sequence can have) are refused before anything is launched: counters of list
    entries, stepping by a block of threads, would wrap near 2^31."""
    most, d, kv, b = 1 << 26, AF.attn_desc(8, 2, 64), ctypes.byref(KV), ctypes.byref(AF.KeyBounds(P, P))
    select = lambda top: host.aflex_page_select(ctx._h, d, P, kv, b, AF.PagePolicy(top, 1, 2), 3, None, 3, P, P, None)  # noqa: E731
    attend = lambda top: host.aflex_attn_decode_pages(ctx._h, d, P, kv, P, P, top, 3, None, 3, P, None, None)  # noqa: E731
    layers = lambda top: host.aflex_decoder_layers_sparse(  # noqa: E731
        ctx._h, (AF.DecoderDesc * 1)(decoder(64)), (AF.KV * 1)(KV), b, AF.PagePolicy(top, 1, 2), 1, P, 3, 1, None, P, None)
    for call in (select, attend, layers):
        for top in (most + 1, 2147483647, 2147483647 - 4):
            assert call(top) == AF.ERR_UNSUPPORTED
    assert host.host_launch_count() == 0
    assert select(most) == AF.OK and attend(most) == AF.OK
    assert layers(most) == AF.ERR_WORKSPACE
    assert AF.decoder_sparse_workspace_bytes(decoder(64), 3, most + 1) == 0 < AF.decoder_sparse_workspace_bytes(decoder(64), 3, most)


def test_sparse_layers_check_the_hidden_states_and_offsets_before_the_library_sees_them():
    """As the operators do: a tensor of another type or size would be read or written past its end."""
    class Stream:
        cuda_stream = 0

    ctx = AF.Context.__new__(AF.Context)
    ctx._lib, ctx._h, ctx.device = AF.load_library(), None, -1
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)  # noqa: E731
    k = z(6, 2, 16, 64)
    i32 = torch.int32
    kv = AF.make_kv(k, k, z(3, 4, dt=i32), z(3, dt=i32))
    bounds = AF.make_page_bounds(*AF.empty_page_bounds(6, 2, 64, device="cpu"))
    x = z(3, 256)
    call = lambda x_in=x, x_out=x, **kw: ctx.decoder_layers_sparse([decoder(64)], [kv], [bounds], 5, x_in, x_out, stream=Stream, **kw)  # noqa: E731
    with pytest.raises(AF.AflexError):                                 # all as it should be: it is the library that refuses (no context)
        call()
    with pytest.raises(AF.AflexError):
        call(microbatch_depth=2, mb_offsets=[0, 1, 3])
    for kw in (dict(x_in=x.float()), dict(x_out=x.half()), dict(x_in=z(3, 248), x_out=z(3, 248)), dict(x_out=z(2, 256)), dict(x_out=z(3, 128)),
               dict(x_in=z(3 * 256)), dict(microbatch_depth=2, mb_offsets=[0, 3])):
        with pytest.raises(AssertionError):
            call(**kw)
