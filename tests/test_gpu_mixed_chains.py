"""Chains whose layers are not of one kind: dense and MoE FFNs, and attention of different shapes, in the decoder chains."""
import numpy as np
import pytest
import torch

from paper_2608_01891_b200 import aflex as AF
from paper_2608_01891_b200 import inputs as IN
from tests.helpers import f64
from tests.test_gpu_pages import DEV, rows_apart

pytestmark = pytest.mark.gpu

BATCH = 24


def shape(cfg_id, name, inter, experts=0, Hq=8, Hkv=2, D=64, **kw):
    return IN.LayerConfig(cfg_id, name, BATCH, Hq, Hkv, D, 512, inter, num_experts=experts, top_k=2 if experts else 0, len_lo=1, len_hi=900,
                          **{"rope_theta": 1.0e4, **kw})


DENSE, MOE = shape(61, "wide-dense", 8192), shape(62, "small-moe", 128, 4, qk_norm=False)


class Chain:
    """Layers of the given configurations on sequences of the same lengths, each with a cache, a page table and key bounds of its own."""

    def __init__(self, cfgs):
        self.cfgs = cfgs
        self.lens = torch.from_numpy(IN.make_seq_lens(cfgs[0]).astype(np.int32))
        self.lens_d = self.lens.to(DEV)
        self.x = IN.make_hidden(cfgs[0]).to(DEV)
        self.descs, self.attns, self.stored, self.caches, self.tables, self.codes, self.keep = [], [], [], [], [], [], []
        for l, cfg in enumerate(cfgs):
            w = {k: (None if t is None else t.to(DEV)) for k, t in vars(IN.make_decoder_weights(cfg, l)).items()}
            attn = AF.attn_desc(cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim)
            layer = AF.layer_desc(attn, cfg.hidden, cfg.inter, w["o"], w["gate"], w["up"], w["down"], cfg.num_experts, cfg.top_k, w["router"])
            self.descs.append(AF.decoder_desc(layer, w["qkv"], w["ln_attn"], w["ln_ffn"], w["q_norm"], w["k_norm"], cfg.rms_eps, cfg.rope_theta))
            kvh = IN.make_paged_kv(cfg, self.lens.numpy())
            self.keep.append(w)
            self.attns.append(attn)
            self.stored.append((kvh.k_cache, kvh.v_cache))
            self.caches.append((kvh.k_cache.to(DEV), kvh.v_cache.to(DEV)))
            self.tables.append(kvh.page_table.to(DEV))
            self.codes.append(AF.empty_page_bounds(kvh.num_pages, cfg.num_kv_heads, cfg.head_dim, DEV))
        self.bounds = [AF.make_page_bounds(*c) for c in self.codes]

    def kvs(self, r0=0, r1=BATCH):
        return [AF.make_kv(k, v, t[r0:r1], self.lens_d[r0:r1]) for (k, v), t in zip(self.caches, self.tables)]

    def reset(self, ctx):
        for (k, v), (k0, v0), a, kv, b in zip(self.caches, self.stored, self.attns, self.kvs(), self.bounds):
            k.copy_(k0)
            v.copy_(v0)
            ctx.page_bounds(a, kv, b, BATCH)

    def state(self):
        return [t.clone() for c in (*self.caches, *self.codes) for t in c]


@pytest.mark.parametrize("cfgs", [(DENSE, MOE), (MOE, DENSE), (DENSE, MOE, MOE, DENSE, DENSE)], ids=lambda c: "-".join(x.name for x in c))
def test_sparse_chain_of_dense_and_moe_layers_in_microbatches(cfgs):
    """Two microbatches on two streams, against each of them alone on one: the same kernels on the same rows, so the same bits."""
    c, top = Chain(cfgs), 6
    ctx = AF.Context(0, max(AF.decoder_sparse_workspace_bytes(d, BATCH, top) for d in c.descs))
    try:
        assert (int(c.lens.max()) + 15) // 16 > top
        half = BATCH // 2
        want = torch.empty_like(c.x)
        c.reset(ctx)
        for r0 in (0, half):
            ctx.decoder_layers_sparse(c.descs, c.kvs(r0, r0 + half), c.bounds, top, c.x[r0:r0 + half], want[r0:r0 + half])
        after = c.state()
        assert torch.isfinite(want).all()
        for _ in range(10):
            got = torch.zeros_like(want)
            c.reset(ctx)
            ctx.decoder_layers_sparse(c.descs, c.kvs(), c.bounds, top, c.x, got, microbatch_depth=2)
            assert ctx.device_status() == AF.OK
            assert torch.equal(got, want)
            assert all(torch.equal(a, b) for a, b in zip(c.state(), after))
    finally:
        ctx.close()


@pytest.mark.parametrize("depth", [1, 2])
def test_sparse_chain_of_dense_and_moe_layers_is_the_dense_chain_with_every_page(depth):
    c = Chain((DENSE, MOE, DENSE))
    top = (int(c.lens.max()) + 15) // 16
    ctx = AF.Context(0, max(AF.decoder_sparse_workspace_bytes(d, BATCH, top) for d in c.descs))
    try:
        dense, sparse = torch.empty_like(c.x), torch.empty_like(c.x)
        c.reset(ctx)
        ctx.decoder_layers(c.descs, c.kvs(), c.x, dense, depth)
        c.reset(ctx)
        ctx.decoder_layers_sparse(c.descs, c.kvs(), c.bounds, top, c.x, sparse, microbatch_depth=depth)
        assert ctx.device_status() == AF.OK
        # two chains of the same bf16 roundings: some twenty a layer, each off by at most 2^-8 of its row's largest value and adding up
        # like independent ones, in each of the two chains: sqrt(2 x 3 x 20) 2^-8 = 4.3e-2
        assert rows_apart(sparse, dense) <= 4.3e-2 and np.isfinite(f64(dense)).all()
    finally:
        ctx.close()


NARROW, WIDE, LARGE = shape(63, "narrow", 1408), shape(64, "wide", 1408, Hq=16), shape(65, "large-heads", 1408, Hq=8, Hkv=8, D=128)
NARROW_MOE = shape(66, "narrow-moe", 192, 4, Hq=4, Hkv=4)
ATTENTION_MIXES = [(NARROW, WIDE), (LARGE, NARROW, NARROW), (NARROW, NARROW_MOE, LARGE)]


@pytest.mark.parametrize("sparse", [False, True], ids=["dense", "sparse"])
@pytest.mark.parametrize("depth", [1, 2])
@pytest.mark.parametrize("cfgs", ATTENTION_MIXES, ids=lambda c: "-".join(x.name for x in c))
def test_chain_of_layers_with_different_heads_is_its_layers_in_turn(cfgs, depth, sparse):
    c = Chain(cfgs)
    top = (int(c.lens.max()) + 15) // 16
    ctx = AF.Context(0, 1 << 28)
    try:
        def run(layers, x, y):
            part = lambda t: [t[l] for l in layers]  # noqa: E731
            if sparse:
                ctx.decoder_layers_sparse(part(c.descs), part(c.kvs()), part(c.bounds), top, x, y, microbatch_depth=depth)
            else:
                ctx.decoder_layers(part(c.descs), part(c.kvs()), x, y, depth)

        got, want = torch.empty_like(c.x), c.x.clone()
        c.reset(ctx)
        for l in range(len(cfgs)):
            run([l], want, want)
        after = c.state()
        c.reset(ctx)
        run(range(len(cfgs)), c.x, got)
        assert ctx.device_status() == AF.OK
        # two chains of the same bf16 roundings, as above: sqrt(2 x 3 x 20) 2^-8
        assert rows_apart(got, want) <= 4.3e-2 and np.isfinite(f64(want)).all()
        n = 2 * len(cfgs)                                                       # keys and values
        assert all(rows_apart(a, b) <= 4.3e-2 for a, b in zip(c.state()[:n], after[:n]))
    finally:
        ctx.close()


@pytest.mark.parametrize("cfgs", ATTENTION_MIXES, ids=lambda c: "-".join(x.name for x in c))
def test_sparse_chain_of_layers_with_different_heads_in_microbatches(cfgs):
    """Two microbatches on two streams, against each of them alone on one."""
    c, top, half = Chain(cfgs), 6, BATCH // 2
    ctx = AF.Context(0, 1 << 28)
    try:
        want = torch.empty_like(c.x)
        c.reset(ctx)
        for r0 in (0, half):
            ctx.decoder_layers_sparse(c.descs, c.kvs(r0, r0 + half), c.bounds, top, c.x[r0:r0 + half], want[r0:r0 + half])
        after = c.state()
        for _ in range(10):
            got = torch.zeros_like(want)
            c.reset(ctx)
            ctx.decoder_layers_sparse(c.descs, c.kvs(), c.bounds, top, c.x, got, microbatch_depth=2)
            assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(c.state(), after))
        assert ctx.device_status() == AF.OK
    finally:
        ctx.close()


@pytest.mark.parametrize("cfgs", ATTENTION_MIXES, ids=lambda c: "-".join(x.name for x in c))
def test_prefill_chain_of_layers_with_different_heads_is_its_layers_in_turn(cfgs):
    c = Chain(cfgs)
    new = [int(n) // 2 + 1 for n in c.lens.tolist()]
    offs = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32)
    x = torch.randn(int(offs[-1]), cfgs[0].hidden, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
    ctx = AF.Context(0, 1 << 30)
    try:
        got, want = torch.empty_like(x), x.clone()
        c.reset(ctx)
        for d, kv in zip(c.descs, c.kvs()):
            ctx.prefill_layers([d], [kv], want, offs.to(DEV), offs, want)
        after = c.state()
        c.reset(ctx)
        ctx.prefill_layers(c.descs, c.kvs(), x, offs.to(DEV), offs, got)
        assert ctx.device_status() == AF.OK
        # the same kernels in the same order; between two layers the chain normalises the sum before it is rounded
        assert rows_apart(got, want) <= 4.3e-2 and np.isfinite(f64(want)).all()
        n = 2 * len(cfgs)
        assert all(rows_apart(a, b) <= 4.3e-2 for a, b in zip(c.state()[:n], after[:n]))
    finally:
        ctx.close()


@pytest.mark.parametrize("depth", [1, 2])
@pytest.mark.parametrize("cfgs", ATTENTION_MIXES, ids=lambda c: "-".join(x.name for x in c))
def test_pair_of_contexts_on_layers_with_different_heads_is_its_layers_in_turn(cfgs, depth):
    """(Every layer hands rounded hidden states over, so the chain and its layers alone launch the same kernels on the same rows.)"""
    c = Chain(cfgs)
    ca, cf = AF.Context(0, 1 << 28), AF.Context(0, 1 << 28)
    try:
        got, want = torch.zeros_like(c.x), c.x.clone()
        c.reset(ca)
        for d, kv in zip(c.descs, c.kvs()):
            AF.af_decoder_layers(ca, cf, [d], [kv], want, want, depth)
        torch.cuda.synchronize()
        after = c.state()
        c.reset(ca)
        AF.af_decoder_layers(ca, cf, c.descs, c.kvs(), c.x, got, depth)
        torch.cuda.synchronize()
        assert ca.device_status() == AF.OK and cf.device_status() == AF.OK
        assert torch.equal(got, want) and torch.isfinite(got).all()
        n = 2 * len(cfgs)
        assert all(torch.equal(a, b) for a, b in zip(c.state()[:n], after[:n]))
    finally:
        ca.close()
        cf.close()
