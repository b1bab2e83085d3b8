"""Attention over caches of few bits against the 64-bit definition on what
their codes stand for: formats and types, head layouts, lengths from nothing
to many key tiles, every kernel form, masks that leave rows empty, what lies in
masked places, strides, streams, graphs, moved pages, and a decode run with its
cache in few bits.  Marked ``gpu``.

Codes are exact in the products, so the bounds are those of a plain cache (attention_ref.bounds), but for fp32
rows: their queries and probabilities are multiplied in three parts, which makes three terms of each in the
float32 sums."""
import math

import pytest
import torch

import attention_ref as R
import quant_ref as Q
from dmoe_synth import get_config, make_inputs
from paper_2605_30876_amd.attention import AttentionLayer, BlockAttention, PagedCache, Rope
from paper_2605_30876_amd.layer import MoELayer, decode_step, pack_weights

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
FORMATS = ["fp8", "fp4", "fp8_fp4"]


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Setup:
    """A batch over a cache whose unused bytes are 255 (NaN in both formats), pages in random order."""

    def __init__(self, fmt, dtype, heads, kv_heads, dim, page, lens, new, mask, seed=0, layers=1, extra_rows=2, slack=3, scale=None, capacity=0):
        g = torch.Generator().manual_seed(seed)
        self.fmt, self.dtype, self.dim, self.lens, self.new, self.mask, self.page, self.kv = fmt, dtype, dim, lens, new, mask, page, kv_heads
        self.bits = Q.BITS[fmt]
        n = len(lens)
        held = [-(-x // page) for x in lens]
        pages = sum(held) + slack
        ids = torch.randperm(pages, generator=g).tolist()
        self.slots = torch.randperm(n + 2, generator=g)[:n].tolist()
        width = max(max(held + [0]) + 1, capacity // page)
        self.table = torch.full((n + 2, width), -1, dtype=torch.int32)
        all_lens, at = torch.full((n + 2,), 3, dtype=torch.int32), 0
        for s, h, m in zip(self.slots, held, lens):
            self.table[s, :h] = torch.tensor(ids[at:at + h], dtype=torch.int32)
            all_lens[s], at = m, at + h
        self.pools = [torch.full((layers, pages, Q.page_bytes(b, page, kv_heads, dim)), 255, dtype=torch.uint8) for b in self.bits]
        self.k, self.v = [], []
        for i, m in enumerate(lens):
            rows = [torch.randn(layers, m, kv_heads, dim, generator=g), torch.randn(layers, m, kv_heads, dim, generator=g) + 0.25]
            got = []
            for w in range(2):
                codes, scales = Q.quantise(rows[w], self.bits[w])
                got.append(Q.values(codes, scales, self.bits[w])[..., :dim])
                pos = torch.arange(m)
                for l in range(layers):
                    if m:
                        Q.put(self.pools[w][l].view(-1), self.bits[w], page, dim, pos, self.table[self.slots[i]][pos // page], codes[l], scales[l])
            self.k.append(got[0])
            self.v.append(got[1])
        off = [0]
        for x in new:
            off.append(off[-1] + x)
        self.off, rows = off, off[-1] + extra_rows
        self.q = (1.5 * torch.randn(layers, max(rows, 1), heads, dim, generator=g)).to(dtype)
        self.scale = 1.0 / math.sqrt(dim) if scale is None else scale
        self.cache = PagedCache(layers, pages, page, kv_heads, dim, n + 2, width, dtype=dtype, k=self.pools[0].cuda(), v=self.pools[1].cuda(),
                                table=self.table.cuda(), lens=all_lens.cuda(), format=fmt)
        self.qd = self.q.cuda()
        self.att = BlockAttention(self.cache, heads, n, max(new + [1]), self.q.shape[1], mask_block=mask, scale=scale)
        self.offd, self.slotsd = i32(off), i32(self.slots)

    def run(self, layer=0):
        out = torch.full(self.q.shape[1:], 7.0, dtype=self.dtype, device="cuda")
        lse = torch.full(self.q.shape[1:3], 7.0, device="cuda")
        self.att.begin(self.offd, self.slotsd)
        self.att.plan()
        self.att.attend(layer, self.qd[layer], out, lse)
        torch.cuda.synchronize()
        return out.cpu(), lse.cpu()

    def reference(self, i, layer=0):
        m, n = self.lens[i], self.new[i]
        rows = slice(self.off[i], self.off[i + 1])
        ref = R.attention(self.q[layer, rows], self.k[i][layer], self.v[i][layer], R.ends(range(m - n, m), m, self.mask), self.scale)
        parts = 3 if self.dtype == F32 else 1
        return rows, ref, R.bounds(self.dtype, parts * self.dim, parts * max(m, 1), *ref)

    def check(self, out, lse, layer=0, skip=()):
        for i in range(len(self.lens)):
            if i in skip:
                continue
            rows, ref, (tol, ltol) = self.reference(i, layer)
            err, lerr = (out[rows].double() - ref[0]).abs(), (lse[rows].double() - ref[1]).abs()
            assert bool((err <= tol).all()), (i, float((err / tol).max()))
            empty = ref[1] == -math.inf
            assert bool((lse[rows][empty] == -math.inf).all()) and bool((lerr[~empty] <= ltol[~empty]).all())
        assert bool((out[self.off[-1]:] == 7).all()) and bool((lse[self.off[-1]:] == 7).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,kv,dim,page,lens,new,mask", [
    (1, 1, 64, 32, [1], [1], 0),                               # one token that sees itself
    (4, 4, 32, 32, [5, 40], [5, 8], 8),
    (8, 2, 128, 32, [100, 33, 64], [1, 1, 1], 1),              # single tokens
    (6, 3, 80, 64, [70, 200], [32, 7], 32),                    # an odd head dimension
    (5, 1, 96, 96, [300, 0, 31], [9, 0, 31], 1),               # a sequence with nothing, pages of an odd number of tiles
    (16, 2, 64, 32, [130], [24], 8),                           # 192 rows of a kv head
    (4, 2, 256, 32, [90, 20], [20, 3], 0),
    (2, 1, 192, 64, [150], [150], 1),                          # a whole prompt, causal
    (3, 3, 8, 32, [64, 65], [1, 40], 1),
    (32, 1, 40, 32, [50], [3], 1),
    (7, 7, 128, 160, [161, 3], [2, 5], 32),                    # more new tokens than the sequence has: rows that see nothing
])
def test_against_the_definition(gpu_lib, fmt, dtype, heads, kv, dim, page, lens, new, mask):
    s = Setup(fmt, dtype, heads, kv, dim, page, lens, new, mask)
    s.check(*s.run())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 192, 256])
@pytest.mark.parametrize("group,new,lens", [(1, 20, [700, 90]), (2, 32, [500, 64]), (4, 40, [1200, 45])])
def test_every_form(gpu_lib, fmt, dtype, dim, group, new, lens):
    """32, 64 and 128 rows to a workgroup, split along the keys and joined; room for sequences long enough that 128 rows are taken."""
    s = Setup(fmt, dtype, 2 * group, 2, dim, 32, lens, [new, min(new, lens[1])], 32, capacity=1 << 17 if group == 4 else 0)
    s.check(*s.run())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("mask", [0, 1, 32])
def test_many_rows(gpu_lib, fmt, dtype, mask):
    """More than a workgroup's rows, several stages, ranges that end within a stage."""
    s = Setup(fmt, dtype, 4, 1, 64, 32, [461, 333], [150, 100], mask, capacity=1 << 17)
    s.check(*s.run())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype,dim", [(BF16, 128), (F32, 64)])
def test_long_sequences(gpu_lib, fmt, dtype, dim):
    s = Setup(fmt, dtype, 4, 2, dim, 128, [9000, 1, 4097], [1, 1, 1], 1)
    s.check(*s.run())


def spoil(s, which, i, token, head, value):
    """A token's scale byte of head `head` made `value`, all groups."""
    pos = torch.tensor([token])
    _, st = Q.places(s.bits[which], s.page, s.kv, s.dim, pos, s.table[s.slots[i]][pos // s.page])
    (s.cache.k, s.cache.v)[which].view(s.cache.k.shape[0], -1)[0, st[0, head].cuda()] = value


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,capacity,dim", [(2, 0, 64), (8, 0, 64), (8, 1 << 17, 64), (8, 1 << 17, 192), (8, 1 << 17, 256), (2, 0, 96)])
def test_what_rows_do_not_see(gpu_lib, fmt, dtype, heads, capacity, dim):
    """Values and keys that are NaN or infinite reach the rows that see them, and no others: the rows before keep their results."""
    s = Setup(fmt, dtype, heads, 2, dim, 32, [90], [40], 1, capacity=capacity)
    clean, clean_lse = s.run()
    s.check(clean, clean_lse)
    spoil(s, 1, 0, 70, 0, 255)       # a value of kv head 0 becomes NaN
    spoil(s, 1, 0, 75, 0, 254)       # and one beyond bf16: infinite, if it is not 0
    spoil(s, 0, 0, 80, 1, 255)       # a key of kv head 1
    out, lse = s.run()
    g = heads // 2
    for t in range(40):
        pos = 50 + t
        for h in range(heads):
            hit = pos >= (70 if h < g else 80)
            if hit:
                assert bool(out[t, h].isnan().any())
            else:  # other code paths run, their sums may be ordered otherwise
                rows, ref, (tol, ltol) = s.reference(0)
                assert bool(((out[t, h].double() - ref[0][t, h]).abs() <= tol[t, h]).all()), (t, h)
                assert abs(float(lse[t, h]) - float(ref[1][t, h])) <= float(ltol[t, h])
    # only its value is NaN: the log-sum-exp is every row's
    rows, ref, (tol, ltol) = s.reference(0)
    assert bool(((lse[:40, :g].double() - ref[1][:, :g]).abs() <= ltol[:, :g]).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("capacity,dim", [(0, 64), (1 << 14, 64), (1 << 14, 128), (1 << 14, 256)])
def test_what_few_rows_do_not_see(gpu_lib, fmt, dtype, capacity, dim):
    """As above with 16 rows or fewer to a workgroup, of four waves and, where sequences may be long, of eight."""
    s = Setup(fmt, dtype, 2, 2, dim, 32, [900, 30], [12, 3], 1, capacity=capacity)
    s.check(*s.run())
    spoil(s, 1, 0, 893, 0, 255)
    spoil(s, 0, 0, 895, 1, 255)
    out, lse = s.run()
    rows, ref, (tol, ltol) = s.reference(0)
    for t in range(12):
        for h, first in ((0, 893), (1, 895)):
            if 888 + t >= first:
                assert bool(out[t, h].isnan().any())
            else:
                assert bool(((out[t, h].double() - ref[0][t, h]).abs() <= tol[t, h]).all()), (t, h)
    assert bool(((lse[:12, 0].double() - ref[1][:, 0]).abs() <= ltol[:, 0]).all())
    rows, ref, (tol, ltol) = s.reference(1)
    assert bool(((out[rows].double() - ref[0]).abs() <= tol).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("group", [1, 2, 4])
def test_pages_that_are_not_there(gpu_lib, fmt, group):
    """Ids outside the pool are never followed: no key is seen there."""
    s = Setup(fmt, BF16, 2 * group, 2, 64, 32, [200, 70], [32, 32], 0, capacity=1 << 17)
    slot = s.slots[0]
    s.cache.table[slot, 1], s.cache.table[slot, 4] = -1, s.cache.n_pages
    out, lse = s.run()
    keep = torch.tensor([t for t in range(200) if t // 32 not in (1, 4)])
    ref = R.attention(s.q[0, :32], s.k[0][0][keep], s.v[0][0][keep], [len(keep)] * 32, s.scale)
    tol, ltol = R.bounds(BF16, 64, 200, *ref)
    assert bool(((out[:32].double() - ref[0]).abs() <= tol).all()) and bool(((lse[:32].double() - ref[1]).abs() <= ltol).all())
    s.check(out, lse, skip=(0,))


@pytest.mark.parametrize("group", [1, 2, 4])
def test_a_plan_holds_while_pages_move(gpu_lib, group):
    s = Setup("fp8_fp4", BF16, 2 * group, 2, 96, 32, [300, 150], [32, 20], 32, slack=40, capacity=1 << 17)
    s.cache.refs.zero_()
    ids = s.cache.table[s.cache.table >= 0].long()
    s.cache.refs[ids] = 1
    s.att.begin(s.offd, s.slotsd)
    s.att.plan()
    s.cache.compact()
    out, lse = torch.full_like(s.qd[0], 7.0), torch.full(s.qd.shape[1:3], 7.0, device="cuda")
    s.att.attend(0, s.qd[0], out, lse)
    s.check(out.cpu(), lse.cpu())


def test_strides_streams_and_no_lse(gpu_lib):
    """Columns of wider tensors, another stream, no log-sum-exp; a slot that was refused is left alone."""
    s = Setup("fp4", BF16, 8, 2, 64, 32, [90, 100], [32, 32], 32)
    wide_q = torch.zeros(s.q.shape[1], 3 * 512, dtype=BF16, device="cuda")
    wide_o = torch.full_like(wide_q, 7.0)
    q, o = (t[:, 512:1024].unflatten(1, (8, 64)) for t in (wide_q, wide_o))
    q.copy_(s.qd[0])
    s.att.begin(s.offd, s.slotsd)
    s.cache.refused[s.slots[1]] = 5
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    s.att.plan(side)
    s.att.attend(0, q, o, stream=side)
    side.synchronize()
    rows, ref, (tol, _) = s.reference(0)
    assert bool(((o[:32].cpu().double() - ref[0]).abs() <= tol).all())
    assert bool((wide_o[:, :512] == 7).all()) and bool((wide_o[:, 1024:] == 7).all()) and bool((o[32:] == 7).all())


def test_results_repeat(gpu_lib):
    s = Setup("fp4", BF16, 16, 4, 128, 64, [5000, 700, 3000], [32, 32, 1], 32)
    first = s.run()
    s.check(*first)
    for _ in range(3):
        again = s.run()
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_far_into_a_large_pool(gpu_lib):
    """Offsets beyond 32 bits: pages behind more than 4 GiB of others."""
    kv, dim, page = 8, 256, 1024
    size = Q.page_bytes(4, page, kv, dim)
    pages = (1 << 32) // size + 4
    cache = PagedCache(1, pages, page, kv, dim, 1, 2, table=i32([[pages - 1, pages - 2]]), lens=i32([page + 40]), format="fp4")
    g = torch.Generator().manual_seed(1)
    n = page + 40
    k, v, q = torch.randn(n, kv, dim, generator=g).to(BF16), torch.randn(n, kv, dim, generator=g).to(BF16), torch.randn(n, kv, dim, generator=g).to(BF16)
    att = BlockAttention(cache, kv, 1, n, n, mask_block=0)
    att.begin(i32([0, n]))
    att.append(0, k.cuda(), v.cuda())
    out = att_last(cache, q[-2:].cuda(), 0)
    ref = R.attention(q[-2:], Q.held(k, 4), Q.held(v, 4), [n, n], 1 / math.sqrt(dim))
    tol, _ = R.bounds(BF16, dim, n, *ref)
    assert bool(((out.cpu().double() - ref[0]).abs() <= tol).all())


def att_last(cache, q, layer, mask=0):
    """Attention of a sequence's last rows."""
    att = BlockAttention(cache, q.shape[1], 1, q.shape[0], q.shape[0], mask_block=mask)
    att.begin(i32([0, q.shape[0]]))
    att.plan()
    return att.attend(layer, q)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("name,dtype", [("small_bf16", BF16), ("tiny_f32", F32)])
def test_a_decode_run(gpu_lib, fmt, name, dtype):
    """Blocks of a generation with the cache in few bits, as decode_step runs them: pages given out, a block denoised twice (its keys
    stored again), attention, MoE layers; a fork on the way.  Every layer's attention is the definition's on what the
    cache holds, read back; one captured step replays to the eager one's bits as lengths grow."""
    cfg = get_config(name)
    L, heads, kv, dim = 2, 4, 2, 64
    ds = [make_inputs(cfg, seed=2, layer=l, device="cuda") for l in range(L)]
    w = [pack_weights(d) for d in ds]
    T = cfg.NB * cfg.bs
    m = [MoELayer(cfg.H, cfg.E, cfg.I, cfg.I_s, cfg.k, cfg.NB, cfg.bs, dtype=dtype, device="cuda") for _ in range(L)]
    xs = [ds[0]["x"]] + [torch.empty_like(ds[0]["x"]) for _ in range(L - 1)]
    cache = PagedCache(L, 16 * cfg.NB, 32, kv, dim, cfg.NB + 1, 8, dtype=dtype, format=fmt)
    att = BlockAttention(cache, heads, cfg.NB, cfg.bs, T, mask_block=cfg.bs, rope=Rope(dim // 2))
    g = torch.Generator(device="cuda").manual_seed(5)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda").mul_(1 / math.sqrt(s[1])).to(dtype)  # noqa: E731
    al = [AttentionLayer(att, l, {"wq": 3 * new(heads * dim, cfg.H), "wk": new(kv * dim, cfg.H), "wv": new(kv * dim, cfg.H),
                                  "wo": new(cfg.H, heads * dim)}) for l in range(L)]
    slots = list(range(cfg.NB))
    off, slot_t = i32([i * cfg.bs for i in range(cfg.NB + 1)]), i32(slots)
    att.begin(off, slot_t)
    graph, y = None, None
    for step in range(6):
        if step == 3:  # the first sequence goes on as a copy of itself, which shares its full pages
            n = int(cache.lens[0])
            cache.fork(i32([cfg.NB]), i32([0]), i32([n]))
            slot_t[0] = cfg.NB
        if step % 2 == 0:
            cache.resize(slot_t, cache.lens[slot_t.long()] + cfg.bs)
        xs[0].copy_(torch.randn(xs[0].shape, generator=g, device="cuda").to(dtype))
        assert int(cache.status) == 0
        eager = decode_step(m, w, xs, "block", attention=al).clone()
        seen = [(a.q.clone(), a.o.clone()) for a in al]
        if graph is None:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                y = decode_step(m, w, xs, "block", attention=al)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, eager)
        lens = cache.lens.tolist()
        for l, (q, o) in enumerate(seen):
            for i, s in enumerate(slot_t.tolist()):
                n = lens[s]
                k, v = (torch.zeros(n, kv, dim, dtype=dtype, device="cuda") for _ in range(2))
                cache.read(l, i32([0, n]), k, v, slots=i32([s]))
                rows = slice(i * cfg.bs, (i + 1) * cfg.bs)
                ref = R.attention(q.view(T, heads, dim)[rows].cpu(), k.cpu(), v.cpu(), R.ends(range(n - cfg.bs, n), n, cfg.bs), 1 / math.sqrt(dim))
                parts = 3 if dtype == F32 else 1
                tol, _ = R.bounds(dtype, parts * dim, parts * n, *ref)
                assert bool(((o.view(T, heads, dim)[rows].cpu().double() - ref[0]).abs() <= tol).all()), (step, l, i)
