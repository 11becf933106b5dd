"""Page-sparse decode attention without a GPU: the plain definitions on hand-computed cases, and every refusal of the entry
points.  Refusals are decided on the host before anything is enqueued, so a zeroed block of memory stands for the context
(the checks read nothing of it and write only its error string)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import pages_oracle as PO
from paper_2608_01891_b200 import aflex as AF


# --------------------------------------------------------------------------- the definitions, by hand
def test_exponent_is_the_smallest_that_fits():
    for a, e in [(127.0, 0), (127.5, 1), (128.0, 1), (254.0, 1), (254.5, 2), (63.5, -1), (64.0, 0), (1.0, -6), (0.0, -60), (np.inf, 50),
                 (2.0 ** -70, -60), (127 * 2.0 ** 50, 50), (127 * 2.0 ** 51, 50)]:
        assert PO.exponent(a) == e, a


def test_bounds_round_outwards_and_ignore_nan():
    k = np.zeros((3, 64))
    k[:, 0] = [1.0, -127.5, 3.0]           # block 0: largest magnitude 127.5 -> scale 2
    k[:, 1] = [0.3, 0.2, 0.1]
    k[:, 2] = np.nan
    k[:, 3] = [np.nan, -5.0, -7.0]
    codes, scales = PO.page_bounds(k)
    assert scales.tolist() == [128, 67]
    assert codes[0, 0, :4].tolist() == [2, 1, 0, -2] and codes[0, 1, :4].tolist() == [-64, 0, 0, -4]


def test_score_bounds_every_product_and_ties_go_to_the_lower_page():
    rng = np.random.default_rng(3)
    keys = PO.to_bf16(rng.standard_normal((5, 16, 64)) * np.exp(rng.standard_normal(64)))
    q = np.clip(np.rint(rng.standard_normal((2, 64)) * 40), -127, 127)
    q[:, ::32] = 127                         # whole numbers of which each block's largest is 127: quantised without loss
    made = [PO.page_bounds(k) for k in keys]
    codes, scales = np.stack([m[0] for m in made]), np.stack([m[1] for m in made])
    s = PO.page_scores(q, codes, scales)
    for i in range(5):
        assert s[i] * (1 + 1e-6) >= (keys[i] @ q.T).max()
    lst, cnt = PO.page_select(q[None], np.zeros((9, 1, 8, 2, 8), np.int8), np.full((9, 1, 2), 127, np.uint8),
                              np.arange(9)[None], [9 * 16 - 3], 5, 1, 2)
    assert lst[0, 0].tolist() == [0, 1, 2, 7, 8] and cnt[0, 0] == 5


def test_attention_of_one_token_is_its_value():
    k, v = np.random.default_rng(0).standard_normal((2, 3, 2, 16, 64))
    out, lse, _ = PO.attn_pages(np.ones((1, 4, 64)), k, v, np.array([[2]]), [1], np.zeros((1, 2, 1), int), np.ones((1, 2), int))
    assert np.allclose(out[0, 0], v[2, 0, 0]) and np.allclose(lse[0, 3], k[2, 1, 0].sum() / 8)


# --------------------------------------------------------------------------- refusals
class Fake:
    """Arguments that pass every check (the pointers are never followed), and a stand-in for the context."""

    def __init__(self):
        self.ctx = ctypes.create_string_buffer(1 << 16)
        self.mem = torch.zeros(4096, dtype=torch.uint8)
        self.p = (self.mem.data_ptr() + 15) // 16 * 16
        self.desc = AF.attn_desc(8, 2, 64)
        self.kv = AF.KV(self.p, self.p, 100, self.p, 10, self.p, None)
        self.bounds = AF.KeyBounds(self.p, self.p)
        self.policy = AF.PagePolicy(4, 1, 1)

    def call(self, name, **kw):
        lib, p = AF.load_library(), self.p
        a = dict(ctx=ctypes.addressof(self.ctx), desc=self.desc, kv=self.kv, bounds=self.bounds, policy=self.policy, batch=3, offs=None,
                 rows=3, eps=1e-6, theta=1e4, q=p, out=p, list=p, count=p, top=4)
        a.update(kw)
        ref = lambda s: None if s is None else ctypes.byref(s)  # noqa: E731
        d, kv, b, pol = ref(a["desc"]), ref(a["kv"]), ref(a["bounds"]), ref(a["policy"])
        if name == "rope_append_bounds":
            return lib.aflex_rope_append_bounds(a["ctx"], d, a["q"], kv, b, a["batch"], a["offs"], a["rows"], None, None, a["eps"], a["theta"], a["out"], None)
        if name == "page_bounds":
            return lib.aflex_page_bounds(a["ctx"], d, kv, b, a["batch"], None, None)
        if name == "page_select":
            return lib.aflex_page_select(a["ctx"], d, a["q"], kv, b, pol, a["batch"], a["offs"], a["rows"], a["list"], a["count"], None)
        return lib.aflex_attn_decode_pages(a["ctx"], d, a["q"], kv, a["list"], a["count"], a["top"], a["batch"], a["offs"], a["rows"], a["out"], None, None)


ALL = ("rope_append_bounds", "page_bounds", "page_select", "attn_decode_pages")
INV, UNS = AF.ERR_INVALID_ARG, AF.ERR_UNSUPPORTED


def _kv(f, **kw):
    kv = AF.KV(f.p, f.p, 100, f.p, 10, f.p, None)
    for k, v in kw.items():
        setattr(kv, k, v)
    return kv


@pytest.mark.parametrize("name", ALL)
def test_common_refusals(name):
    f = Fake()
    assert f.call(name, ctx=None) == INV
    assert f.call(name, desc=None) == INV and f.call(name, kv=None) == INV
    for field in ("k_cache", "v_cache", "page_table", "seq_lens"):
        assert f.call(name, kv=_kv(f, **{field: None})) == INV
    assert f.call(name, kv=_kv(f, k_cache=f.p + 2)) == INV
    assert f.call(name, kv=_kv(f, num_pages=0)) == INV and f.call(name, kv=_kv(f, max_pages_per_seq=0)) == INV
    assert f.call(name, batch=0) == INV and f.call(name, batch=65536, rows=65536) == UNS
    assert f.call(name, kv=_kv(f, num_pages=1 << 27)) == UNS
    for d, st in [(AF.attn_desc(8, 3, 64), INV), (AF.attn_desc(0, 0, 64), INV), (AF.attn_desc(8, 2, 96), UNS), (AF.attn_desc(24, 8, 64), UNS),
                  (AF.attn_desc(16, 1, 64), UNS), (AF.AttnDesc(8, 2, 64, 32, 0.0), UNS)]:
        assert f.call(name, desc=d) == st
    host = (ctypes.c_int32 * 3)(5, 0, 7)
    assert f.call(name, kv=_kv(f, seq_lens_host=ctypes.addressof(host))) == INV
    host[1] = 161
    assert f.call(name, kv=_kv(f, seq_lens_host=ctypes.addressof(host))) == INV
    if name != "attn_decode_pages":
        assert f.call(name, bounds=None) == INV
        assert f.call(name, bounds=AF.KeyBounds(None, f.p)) == INV and f.call(name, bounds=AF.KeyBounds(f.p, None)) == INV
        assert f.call(name, bounds=AF.KeyBounds(f.p + 8, f.p)) == INV
    if name != "page_bounds":
        assert f.call(name, q=None) == INV and f.call(name, q=f.p + 4) == INV
        assert f.call(name, rows=0, offs=f.p) == INV and f.call(name, rows=-1, offs=f.p) == INV
        assert f.call(name, rows=4) == INV                        # without q_offsets there is one row per sequence


def test_particular_refusals():
    f = Fake()
    assert f.call("rope_append_bounds", out=None) == INV and f.call("rope_append_bounds", theta=0.0) == INV
    assert f.call("rope_append_bounds", eps=-1.0) == INV and f.call("rope_append_bounds", theta=float("nan")) == INV
    for pol in [(4, -1, 1), (4, 1, 0), (4, 3, 2), (0, 0, 1), (2147483647, 2147483647, 2147483647)]:
        assert f.call("page_select", policy=AF.PagePolicy(*pol)) == INV, pol
    assert f.call("page_select", policy=None) == INV
    assert f.call("page_select", list=None) == INV and f.call("page_select", count=None) == INV
    assert f.call("page_select", kv=_kv(f, max_pages_per_seq=393217)) == UNS
    for name in ALL:
        assert f.call(name, kv=_kv(f, max_pages_per_seq=(1 << 26) + 1)) == UNS
    assert f.call("attn_decode_pages", list=None) == INV and f.call("attn_decode_pages", count=None) == INV
    assert f.call("attn_decode_pages", top=0) == INV and f.call("attn_decode_pages", out=None) == INV


@pytest.mark.skipif(torch.cuda.is_available(), reason="the arguments are made up")
@pytest.mark.parametrize("name", ALL)
def test_good_arguments_pass_the_checks_and_fail_loudly_without_a_gpu(name):
    assert Fake().call(name) == AF.ERR_CUDA


def test_binding_checks_tensors_before_the_library_sees_them():
    """Shapes and types of every tensor argument; a wrong one never reaches a kernel."""
    ctx = AF.Context.__new__(AF.Context)
    ctx._lib, ctx._h, ctx.device = AF.load_library(), None, 0
    bf, i32 = torch.bfloat16, torch.int32
    z = lambda *s, dt=bf: torch.zeros(*s, dtype=dt)  # noqa: E731
    desc = AF.attn_desc(8, 2, 64)
    k = z(6, 2, 16, 64)
    kv = AF.make_kv(k, k, z(3, 4, dt=i32), z(3, dt=i32))
    bounds = AF.make_page_bounds(*AF.empty_page_bounds(6, 2, 64, device="cpu"))
    q, lst, cnt, offs = z(3, 8, 64), z(3, 2, 5, dt=i32), z(3, 2, dt=i32), z(4, dt=i32)
    qkv = z(3, 12 * 64)
    bad = [
        lambda: ctx.rope_append_bounds(desc, z(3, 11 * 64), kv, bounds, q, None, None, 1e-6, 1e4),
        lambda: ctx.rope_append_bounds(desc, qkv.float(), kv, bounds, q, None, None, 1e-6, 1e4),
        lambda: ctx.rope_append_bounds(desc, qkv, kv, bounds, z(2, 8, 64), None, None, 1e-6, 1e4),
        lambda: ctx.rope_append_bounds(desc, qkv, kv, bounds, q, z(32), None, 1e-6, 1e4),
        lambda: ctx.rope_append_bounds(desc, z(4, 12 * 64), kv, bounds, z(4, 8, 64), None, None, 1e-6, 1e4),       # four sequences
        lambda: ctx.rope_append_bounds(desc, qkv, kv, bounds, q, None, None, 1e-6, 1e4, q_offsets=offs.long()),
        lambda: ctx.rope_append_bounds(AF.attn_desc(8, 2, 128), z(3, 12 * 128), kv, bounds, z(3, 8, 128), None, None, 1e-6, 1e4),
        lambda: ctx.page_bounds(desc, kv, bounds, 4),
        lambda: ctx.page_bounds(desc, kv, AF.make_page_bounds(*AF.empty_page_bounds(5, 2, 64, device="cpu")), 3),
        lambda: ctx.page_bounds(desc, kv, bounds, 3, first_token=z(2, dt=i32)),
        lambda: ctx.page_select(desc, q, kv, bounds, 6, lst, cnt),
        lambda: ctx.page_select(desc, q, kv, bounds, 5, lst.long(), cnt),
        lambda: ctx.page_select(desc, q, kv, bounds, 5, lst, z(3, 1, dt=i32)),
        lambda: ctx.page_select(desc, q.half(), kv, bounds, 5, lst, cnt),
        lambda: ctx.attn_decode_pages(desc, q, kv, lst, cnt, z(3, 7, 64)),
        lambda: ctx.attn_decode_pages(desc, z(2, 8, 64), kv, lst, cnt, q),
        lambda: ctx.attn_decode_pages(desc, q, kv, lst, cnt, q, z(3, 8)),
        lambda: ctx.attn_decode_pages(desc, q, kv, lst.transpose(0, 1).contiguous(), cnt, q),
        lambda: ctx.attn_decode_pages(desc, q, kv, lst, cnt, q),                                                   # not on the device
    ]
    for i, f in enumerate(bad):
        with pytest.raises(AssertionError):
            f()
            print(i)


def test_binding_checks_where_every_tensor_lies():
    """A tensor on another device than the context's (here: one that says so) is refused before the library sees its address."""
    class Elsewhere(torch.Tensor):
        def get_device(self):
            return 7

    class Stream:
        cuda_stream = 0

    ctx = AF.Context.__new__(AF.Context)
    ctx._lib, ctx._h, ctx.device = AF.load_library(), None, -1
    bf, i32 = torch.bfloat16, torch.int32
    z = lambda *s, dt=bf: torch.zeros(*s, dtype=dt)  # noqa: E731
    desc = AF.attn_desc(8, 2, 64)
    k = z(6, 2, 16, 64)
    cache = dict(k_cache=k, v_cache=k, page_table=z(3, 4, dt=i32), seq_lens=z(3, dt=i32))
    codes, scales = AF.empty_page_bounds(6, 2, 64, device="cpu")
    kv, bounds = AF.make_kv(**cache), AF.make_page_bounds(codes, scales)
    far_kv = AF.make_kv(**{n: t.as_subclass(Elsewhere) for n, t in cache.items()})
    far_bounds = AF.make_page_bounds(codes.as_subclass(Elsewhere), scales.as_subclass(Elsewhere))
    offs = z(4, dt=i32)
    calls = {
        "rope_append_bounds": dict(qkv=z(3, 12 * 64), kv=kv, bounds=bounds, q_out=z(3, 8, 64), w_q_norm=z(64), w_k_norm=z(64), rms_eps=1e-6,
                                   rope_theta=1e4, q_offsets=offs),
        "page_bounds": dict(kv=kv, bounds=bounds, batch=3, first_token=z(3, dt=i32)),
        "page_select": dict(q=z(3, 8, 64), kv=kv, bounds=bounds, top_pages=5, page_list=z(3, 2, 5, dt=i32), page_count=z(3, 2, dt=i32),
                            q_offsets=offs),
        "attn_decode_pages": dict(q=z(3, 8, 64), kv=kv, page_list=z(3, 2, 5, dt=i32), page_count=z(3, 2, dt=i32), out=z(3, 8, 64),
                                  lse=z(3, 8, dt=torch.float32), q_offsets=offs),
    }
    for name, args in calls.items():
        call = getattr(ctx, name)
        with pytest.raises(AF.AflexError):                       # all where it should be: it is the library that refuses (no context)
            call(desc, **args, stream=Stream)
        for arg, value in args.items():
            far = {"kv": far_kv, "bounds": far_bounds}.get(arg, value.as_subclass(Elsewhere) if isinstance(value, torch.Tensor) else None)
            if far is not None:
                with pytest.raises(AssertionError, match="context's device"):
                    call(desc, **{**args, arg: far}, stream=Stream)
    split_kv = AF.make_kv(**{**cache, "page_table": cache["page_table"].as_subclass(Elsewhere)})
    split_bounds = AF.make_page_bounds(codes, scales.as_subclass(Elsewhere))
    for args in (dict(kv=split_kv, bounds=bounds), dict(kv=kv, bounds=split_bounds)):
        with pytest.raises(AssertionError, match="context's device"):
            ctx.page_bounds(desc, batch=3, stream=Stream, **args)


def test_binding_checks_shapes():
    codes, scales = AF.empty_page_bounds(6, 2, 64, device="cpu")
    assert codes.shape == (6, 2, 8, 2, 8) and scales.shape == (6, 2, 2)
    AF.make_page_bounds(codes, scales)
    with pytest.raises(AssertionError):
        AF.make_page_bounds(codes, scales[:, :, :1])
    with pytest.raises(AssertionError):
        AF.make_page_bounds(codes.to(torch.uint8), scales)
