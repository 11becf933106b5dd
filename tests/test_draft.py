"""Caches of 16 or 8 bits and drafted tokens without a GPU: the plain definitions on hand-computed cases, the tree helper, and every refusal
of the entry points.  Refusals are decided on the host before anything is enqueued, so a zeroed block of memory stands for the context (the
checks read nothing of it and write only its error string)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import draft_oracle as DO
from paper_2608_01891_b200 import aflex as AF


# --------------------------------------------------------------------------- the definitions, by hand
def test_quantisation_by_hand():
    x = np.zeros((4, 64))
    x[0, :4] = [127.0, -63.5, 0.5, 1.5]                 # scale 1: halves to even
    x[1, 0] = np.inf
    x[2, 5] = 2.0 ** -100
    codes, scale = DO.quantise(x, "int8")
    assert scale[0] == 1.0 and codes[0, :4].tolist() == [127, -64, 0, 2]
    assert np.isnan(scale[1]) and not codes[1].any()
    assert scale[2] == scale[3] == 2.0 ** -64 and not codes[2].any()
    x[0, 0] = 448.0
    codes, scale = DO.quantise(x, "e4m3")
    assert abs(scale[0] - 1) < 1e-6 and codes[0, 0] == 448 and codes[0, 1] == -64


@pytest.mark.parametrize("fmt,step", [("int8", 0.5), ("e4m3", 2.0 ** -4)])
def test_codes_are_near(fmt, step):
    x = DO.to_bf16(np.random.default_rng(0).standard_normal((200, 128)) * np.exp(np.random.default_rng(1).standard_normal((200, 1)) * 5))
    codes, scale = DO.quantise(x, fmt)
    assert np.abs(codes).max() <= DO.TOP[fmt]
    err = np.abs(codes * scale[:, None] - x)
    # half a step of a whole number, or of an e4m3 value (2^-10 where it is subnormal), and the scale's roundings
    bound = scale[:, None] * step if fmt == "int8" else np.maximum(np.abs(x) * step, scale[:, None] * 2.0 ** -10)
    assert (err <= bound * (1 + 1e-5)).all()


def test_e4m3_rounding_is_the_types():
    x = np.concatenate([np.random.default_rng(0).standard_normal(5000) * 100, np.linspace(-0.02, 0.02, 999), [0.0, 448, -448, 2.0 ** -10, 3 * 2.0 ** -10]])
    x = np.clip(x, -448, 448).astype(np.float32)
    assert (DO.to_e4m3(x) == torch.from_numpy(x).to(torch.float8_e4m3fn).float().numpy()).all()


def test_attention_of_one_token_is_its_value():
    k, v = np.random.default_rng(0).standard_normal((2, 3, 2, 16, 64))
    out, lse, *_ = DO.attend(np.ones((1, 4, 64)), k, v, np.array([[2]]), [1], None, None)
    assert np.allclose(out[0, 0], v[2, 0, 0]) and np.allclose(lse[0, 3], k[2, 1, 0].sum() / 8)


def test_tree_rows():
    mask, depth = AF.tree_rows([[-1, 0, 0, 2], [], [-1, -1]])
    assert mask.view(-1).tolist() == [1, 3, 5, 13, 1, 2] and depth.tolist() == [0, 1, 1, 2, 0, 0]
    mask, depth = AF.tree_rows([list(range(-1, 69))])
    assert mask.shape == (70, 3) and depth[-1] == 69
    assert mask[69].tolist() == [-1, -1, 63] and mask[31].tolist() == [-1, 0, 0] and mask[30].tolist() == [2 ** 31 - 1, 0, 0]
    for bad in ([0], [-2], [-1, 1], [-1, 0, 5]):
        with pytest.raises(ValueError):
            AF.tree_rows([bad])


# --------------------------------------------------------------------------- refusals
class Fake:
    """Arguments that pass every check (the pointers are never followed), and a stand-in for the context."""

    def __init__(self):
        self.ctx = ctypes.create_string_buffer(1 << 16)
        self.mem = torch.zeros(4096, dtype=torch.uint8)
        self.p = (self.mem.data_ptr() + 15) // 16 * 16
        self.desc = AF.attn_desc(8, 2, 64)
        self.kv = AF.KV(self.p, self.p, 100, self.p, 10, self.p, None)
        self.cache = AF.Cache(self.kv, AF.CACHE_INT8, self.p, self.p)
        self.bf16 = AF.Cache(self.kv, AF.CACHE_BF16, None, None)
        layer = AF.LayerDesc(self.desc, 256, 512, 0, 0, self.p, self.p, self.p, self.p, None)
        self.layer = AF.DecoderDesc(layer, self.p, self.p, self.p, None, None, 1e-6, 1e4)

    def call(self, name, **kw):
        lib, p = AF.load_library(), self.p
        a = dict(ctx=ctypes.addressof(self.ctx), desc=self.desc, cache=self.cache, src=self.bf16, batch=3, rows=3, draft=None, eps=1e-6, theta=1e4, q=p, out=p,
                 n=1, base=p, path=p, stride=4, count=p, layer=self.layer)
        a.update(kw)
        ref = lambda s: None if s is None else ctypes.byref(s)  # noqa: E731
        d, c, dr = ref(a["desc"]), ref(a["cache"]), ref(a["draft"])
        if name == "append":
            return lib.aflex_cache_append(a["ctx"], d, a["q"], c, a["batch"], dr, a["rows"], None, None, a["eps"], a["theta"], a["out"], None)
        if name == "convert":
            return lib.aflex_cache_convert(a["ctx"], d, ref(a["src"]), c, a["batch"], None, None)
        if name == "attend":
            return lib.aflex_attn_draft(a["ctx"], d, a["q"], c, a["batch"], dr, a["rows"], a["out"], None, None)
        if name == "accept":
            return lib.aflex_cache_accept(a["ctx"], d, c, a["n"], a["batch"], a["base"], a["path"], a["stride"], a["count"], None)
        return lib.aflex_draft_layers(a["ctx"], ref(a["layer"]), c, a["n"], a["q"], a["batch"], dr, a["rows"], a["out"], None)

    def changed(self, cache=None, **kw):
        c = AF.Cache.from_buffer_copy(cache or self.cache)
        for k, v in kw.items():
            setattr(c if k in ("format", "k_scales", "v_scales") else c.kv, k, v)
        return c


OPS = ["append", "convert", "attend", "accept", "layers"]


@pytest.mark.parametrize("name", OPS)
def test_common_refusals(name):
    f = Fake()
    bad, un = AF.ERR_INVALID_ARG, AF.ERR_UNSUPPORTED
    cases = [(dict(ctx=None), bad), (dict(cache=None), bad), (dict(batch=0, rows=0), bad), (dict(batch=70000, rows=70000), un),
             (dict(cache=f.changed(format=3)), bad), (dict(cache=f.changed(format=-1)), bad),
             (dict(cache=f.changed(k_scales=None)), bad), (dict(cache=f.changed(v_scales=None)), bad), (dict(cache=f.changed(v_scales=f.p + 4)), bad),
             (dict(cache=f.changed(f.bf16, k_scales=f.p)), bad),
             (dict(cache=f.changed(k_cache=None)), bad), (dict(cache=f.changed(v_cache=f.p + 8)), bad), (dict(cache=f.changed(page_table=None)), bad),
             (dict(cache=f.changed(num_pages=0)), bad), (dict(cache=f.changed(max_pages_per_seq=0)), bad),
             (dict(cache=f.changed(max_pages_per_seq=(1 << 26) + 1)), un), (dict(cache=f.changed(num_pages=1 << 27)), un)]
    if name != "layers":
        cases += [(dict(desc=None), bad), (dict(desc=AF.attn_desc(8, 3, 64)), bad), (dict(desc=AF.attn_desc(8, 2, 96)), un),
                  (dict(desc=AF.attn_desc(32, 2, 64)), un), (dict(desc=AF.AttnDesc(8, 2, 64, 32, 0.0)), un)]
    for kw, want in cases:
        assert f.call(name, **kw) == want, kw


@pytest.mark.parametrize("name", ["append", "attend", "layers"])
def test_refusals_of_rows(name):
    f = Fake()
    offs = AF.Draft(f.p, None, None, 0)
    for kw in (dict(rows=0), dict(rows=4), dict(rows=4, draft=AF.Draft(None, f.p, None, 0)), dict(rows=0, draft=offs), dict(rows=-1, draft=offs),
               dict(draft=AF.Draft(f.p, None, f.p, 0)), dict(draft=AF.Draft(f.p, None, f.p, -1)), dict(draft=AF.Draft(f.p, None, f.p, (1 << 20) + 1))):
        assert f.call(name, **kw) == AF.ERR_INVALID_ARG, kw
    for kw in (dict(q=None), dict(out=None), dict(q=f.p + 2), dict(out=f.p + 8)):
        assert f.call(name, **kw) == AF.ERR_INVALID_ARG, kw


def test_other_refusals():
    f = Fake()
    for kw in (dict(theta=0.0), dict(theta=float("nan")), dict(eps=-1.0)):
        assert f.call("append", **kw) == AF.ERR_INVALID_ARG
    assert f.call("convert", src=None) == AF.ERR_INVALID_ARG
    assert f.call("convert", src=f.cache) == AF.ERR_UNSUPPORTED
    assert f.call("convert", cache=f.bf16) == AF.ERR_UNSUPPORTED
    assert f.call("convert", src=f.changed(f.bf16, seq_lens=None)) == AF.ERR_INVALID_ARG
    for kw in (dict(n=0), dict(base=None), dict(path=None), dict(count=None), dict(stride=0)):
        assert f.call("accept", **kw) == AF.ERR_INVALID_ARG
    lib = AF.load_library()
    two = (AF.Cache * 2)(f.cache, f.bf16)
    assert lib.aflex_cache_accept(ctypes.addressof(f.ctx), f.desc, two, 2, 3, f.p, f.p, 4, f.p, None) == AF.ERR_UNSUPPORTED
    assert f.call("layers", n=0) == AF.ERR_INVALID_ARG
    d = AF.DecoderDesc.from_buffer_copy(f.layer)
    d.w_qkv = None
    assert f.call("layers", layer=d) == AF.ERR_INVALID_ARG
    assert AF.attn_draft_workspace_bytes(AF.attn_desc(8, 2, 96)) == 0 < AF.attn_draft_workspace_bytes(f.desc)
    assert AF.draft_workspace_bytes(f.layer, 0) == 0 < AF.draft_workspace_bytes(f.layer, 3)


def test_the_binding_checks_tensors_before_the_library_sees_them():
    """A tensor of another type, size or device would be read or written past its end."""
    class Stream:
        cuda_stream = 0

    ctx = AF.Context.__new__(AF.Context)
    ctx._lib, ctx._h, ctx.device = AF.load_library(), None, -1
    i32, bf = torch.int32, torch.bfloat16
    z = lambda *s, dt=bf: torch.zeros(*s, dtype=dt)  # noqa: E731
    k, v, ks, vs = AF.empty_cache(6, 2, 64, torch.int8, device="cpu")
    table, lens = z(3, 4, dt=i32), z(3, dt=i32)
    cache = AF.make_cache(k, v, table, lens, ks, vs)
    for a in ((k, v, table, lens), (k, v, table, lens, ks, None), (k.float(), v.float(), table, lens), (k, v[:5], table, lens, ks, vs), (k, v, table, lens, ks, vs[:5]),
              (k, v, table, lens, ks, vs.double()), (z(6, 2, 16, 64), z(6, 2, 16, 64), table, lens, ks, vs), (k, v, table.long(), lens, ks, vs)):
        with pytest.raises(AssertionError):
            AF.make_cache(*a)
    desc = AF.attn_desc(8, 2, 64)
    other = AF.attn_desc(8, 4, 64)
    q, qkv, lse, norm = z(3, 8, 64), z(3, 12 * 64), z(3, 8, dt=torch.float32), z(64)
    dr = AF.draft_rows(torch.tensor([0, 2, 3, 3], dtype=i32), z(3, dt=i32), z(3, 1, dt=i32))
    append = lambda qkv=qkv, q=q, c=cache, d=desc, w=norm, dr=dr: ctx.cache_append(d, qkv, c, q, w, w, 1e-6, 1e4, draft=dr, stream=Stream)  # noqa: E731
    attend = lambda q=q, out=q, c=cache, d=desc, lse=lse, dr=dr: ctx.attn_draft(d, q, c, out, lse, draft=dr, stream=Stream)  # noqa: E731
    accept = lambda base=lens, path=table, n=lens, c=cache, d=desc, b=3: ctx.cache_accept(d, [c], b, base, path, n, stream=Stream)  # noqa: E731
    convert = lambda c=cache, d=desc, b=3, first=lens: ctx.cache_convert(d, c, c, b, first, stream=Stream)  # noqa: E731
    for call in (append, attend, accept, convert):                     # all as it should be: it is the library that refuses (no context)
        with pytest.raises(AF.AflexError):
            call()
    short = AF.draft_rows(torch.tensor([0, 2, 3, 3], dtype=i32), z(2, dt=i32), None)
    narrow = AF.draft_rows(torch.tensor([0, 2, 3, 3], dtype=i32), None, z(2, 1, dt=i32))
    many = AF.draft_rows(torch.tensor([0, 1, 2, 3, 3], dtype=i32))
    for call, kws in ((append, (dict(qkv=qkv.float()), dict(qkv=z(3, 11 * 64)), dict(q=z(2, 8, 64)), dict(d=other), dict(w=z(32)), dict(dr=short), dict(dr=narrow), dict(dr=many))),
                      (attend, (dict(q=q.float()), dict(out=z(2, 8, 64)), dict(lse=z(3, 8)), dict(d=other), dict(dr=short), dict(dr=narrow), dict(dr=many))),
                      (accept, (dict(base=lens.long()), dict(base=lens[:2]), dict(path=lens), dict(path=table[:2]), dict(n=lens[:2]), dict(d=other), dict(b=4))),
                      (convert, (dict(d=other), dict(b=4), dict(first=lens[:2])))):
        for kw in kws:
            with pytest.raises(AssertionError):
                call(**kw)
    for a in ((lens.long(),), (table,), (lens, lens.long()), (lens, None, lens), (lens, None, table.long())):
        with pytest.raises(AssertionError):
            AF.draft_rows(*a)
