"""A decode step with its attention: pages given out, keys and values stored,
attention, MoE layers, over the blocks of a generation, with a fork and a
compaction on the way.  Every layer's attention must match the 64-bit
definition on what the cache holds, the step captured in one graph must equal
the eager one on every replay, and a cache whose pages moved must give the
same results.  Marked ``gpu``."""
import math

import pytest
import torch

import attention_ref as R
from dmoe_synth import get_config, make_inputs
from paper_2605_30876_amd.attention import AttentionLayer, BlockAttention, PagedCache, Rope
from paper_2605_30876_amd.layer import MoELayer, decode_step, pack_weights

pytestmark = pytest.mark.gpu

L, HEADS, KV, DIM, PAGE = 3, 8, 2, 64, 32


class Model:
    def __init__(self, name, routing, seqs=None, heads=HEADS, kv=KV, dim=DIM):
        cfg = get_config(name)
        self.cfg = cfg = cfg if seqs is None else cfg.with_(name=f"{name}_{seqs}", NB=seqs)
        self.routing, self.n, self.bs, self.T = routing, cfg.NB, cfg.bs, cfg.NB * cfg.bs
        ds = [make_inputs(cfg, seed=2, layer=l, device="cuda") for l in range(L)]
        self.w = [pack_weights(d) for d in ds]
        dt = torch.float32 if cfg.dtype == "f32" else torch.bfloat16
        self.m = [MoELayer(cfg.H, cfg.E, cfg.I, cfg.I_s, cfg.k, cfg.NB, cfg.bs, dtype=dt, device="cuda") for _ in range(L)]
        self.xs = [ds[0]["x"]] + [torch.empty_like(ds[0]["x"]) for _ in range(L - 1)]
        self.cache = PagedCache(L, 12 * self.n, PAGE, kv, dim, self.n + 1, 6, dtype=dt)
        self.att = BlockAttention(self.cache, heads, self.n, self.bs, self.T, mask_block=self.bs, rope=Rope(dim // 2))
        g = torch.Generator(device="cuda").manual_seed(5)
        new = lambda *s: torch.randn(*s, generator=g, device="cuda").mul_(1 / math.sqrt(s[1])).to(dt)  # noqa: E731
        self.al = [AttentionLayer(self.att, l, {"wq": 3 * new(heads * dim, cfg.H), "wk": new(kv * dim, cfg.H), "wv": new(kv * dim, cfg.H),
                                                "wo": new(cfg.H, heads * dim)}) for l in range(L)]
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.slots, self.i32 = i32(list(range(self.n))), i32
        self.att.begin(i32([i * self.bs for i in range(self.n + 1)]), self.slots)

    def step(self):
        return decode_step(self.m, self.w, self.xs, self.routing, attention=self.al)

    def check_attention(self):
        """Every layer's attention output against the definition on the cache's contents."""
        c = self.cache
        lens, table = c.lens.tolist(), c.table.cpu()
        for l, a in enumerate(self.al):
            kp, vp = c.k[l].cpu().view(-1), c.v[l].cpu().view(-1)
            q, o = (t.cpu().view(self.T, HEADS, DIM) for t in (a.q, a.o))
            for i, s in enumerate(self.slots.tolist()):
                pos = torch.arange(lens[s])
                ka, va = R.places(c.dtype, PAGE, KV, DIM, pos, table[s][pos // PAGE])
                rows = slice(i * self.bs, (i + 1) * self.bs)
                ref = R.attention(q[rows], kp[ka], vp[va], R.ends(range(lens[s] - self.bs, lens[s]), lens[s], self.bs), 1 / math.sqrt(DIM))
                tol, _ = R.bounds(c.dtype, DIM, lens[s], *ref)
                assert bool(((o[rows].double() - ref[0]).abs() <= tol).all()), f"layer {l}, sequence {i}"


@pytest.mark.parametrize("name,routing,seqs", [("small_bf16", "block", None), ("small_bf16", "topp", 1), ("small_f32", "token", None)])
def test_generation(gpu_lib, name, routing, seqs):
    if name == "small_f32":
        torch.backends.cuda.matmul.allow_tf32 = False
    m = Model(name, routing, seqs)
    g = torch.Generator(device="cuda").manual_seed(7)
    length = 0
    for block in range(3):
        length += m.bs
        m.cache.resize(m.slots, m.i32([length] * m.n))
        for _ in range(2):  # the block denoised over two steps: its keys and values are stored again
            m.xs[0].copy_(torch.randn(m.xs[0].shape, generator=g, device="cuda"))
            y = m.step()
            torch.cuda.synchronize()
            assert int(m.cache.status[0]) == 0 and torch.isfinite(y).all()
            m.check_attention()
    # the last sequence forked at the last finished block, its parent freed, the fork decoded in its place
    last = m.n - 1
    before, o_before = m.step().clone(), [a.o.clone() for a in m.al]
    m.cache.fork(m.i32([m.n]), m.i32([last]), m.i32([length - m.bs]), m.i32([length]))
    m.cache.free(m.i32([last]))
    m.cache.compact()
    m.slots[last] = m.n
    assert int(m.cache.status[0]) == 0 and int(m.cache.lens[m.n]) == length
    after = m.step()
    torch.cuda.synchronize()
    assert all(torch.equal(a.o, b) for a, b in zip(m.al, o_before)) and torch.equal(after, before)
    m.check_attention()


@pytest.mark.parametrize("name,heads,kv,dim", [("small_bf16", HEADS, KV, DIM), ("decode_b1", 16, 4, 128)])
def test_captured_step_equals_eager(gpu_lib, name, heads, kv, dim):
    """The projections are library products of these sizes: what they record in a graph is replayed here too."""
    m = Model(name, "block", 1, heads, kv, dim)
    e = Model(name, "block", 1, heads, kv, dim)
    for x in (m, e):
        x.cache.resize(x.slots, x.i32([x.bs] * x.n))
        x.step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.step()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            y = m.step()
    torch.cuda.current_stream().wait_stream(side)
    gen = torch.Generator(device="cuda").manual_seed(9)
    for rep, length in enumerate((m.bs, m.bs, 2 * m.bs, 5 * m.bs, 3 * m.bs)):
        x0 = torch.randn(m.xs[0].shape, generator=gen, device="cuda")
        for x in (m, e):
            x.cache.resize(x.slots, x.i32([length] * x.n))
            x.xs[0].copy_(x0)
            # keys and values of tokens that no step stored: the same in both
            x.cache.k.nan_to_num_(0.0), x.cache.v.nan_to_num_(0.0)
        if rep == 0:
            e.cache.k.copy_(m.cache.k), e.cache.v.copy_(m.cache.v)
        y.zero_()
        torch.cuda.synchronize()
        g.replay()
        want = e.step()
        torch.cuda.synchronize()
        assert torch.equal(y, want), f"replay {rep}"
        assert torch.equal(m.cache.k, e.cache.k) and torch.equal(m.cache.v, e.cache.v)
    del g


def test_attention_layers_are_checked(gpu_lib):
    m = Model("small_bf16", "block", 1)
    with pytest.raises(ValueError):
        decode_step(m.m, m.w, m.xs, "block", attention=m.al[:2])
    with pytest.raises(ValueError):
        AttentionLayer(m.att, 0, {**m.al[0].w, "wk": m.al[0].w["wq"]})
