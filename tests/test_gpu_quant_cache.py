"""Keys and values quantised as they are cached, and read back, against the
plain definition: every stored byte, every value, what has no place, pages
that are shared, copied and moved, strides, streams and graphs.  Marked ``gpu``.

What the cache holds is a decision (which code, which scale), so it is
compared bit for bit: the definition's products by a power of two are exact, and a rotated key is rounded
from 64 bits (off by some 2^-50 of it), which would have to lie that near to a border of two float32s to
come out otherwise."""
import math

import pytest
import torch

import attention_ref as R
import quant_ref as Q
from paper_2605_30876_amd.attention import BlockAttention, PagedCache, Rope

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
FORMATS = ["fp8", "fp4", "fp8_fp4"]


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def rows_of(dtype, T, heads, dim, g, special=True):
    """Normal rows of channels of several sizes; with groups of what is hard to quantise in front."""
    x = torch.randn(T, heads, dim, generator=g) * torch.exp(torch.randn(heads, dim, generator=g))
    if special and dim >= 32:
        n = 0
        for a in (0.0, 7.0, 6.9, 464.0, 448.0, 1e-38, 2.0 ** -108, 3e38, 2.0 ** -133):  # maxima at and about the borders of scales
            for s in (1.0, 1.0 + 2 ** -7, 1.0 - 2 ** -8):
                x[n % T, n // T % heads, :32] *= min(a * s, 3.3e38) / x[n % T, n // T % heads, :32].abs().max()
                n += 1
        if T >= 8:
            x[3, 0, :32] = torch.tensor([0.25, -0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -7.0, 0.0, -0.0, 0.26, 0.24, 6.0, 4.0] * 2)
            x[4, 0, :32] = torch.arange(32) * 17.0 - 63  # ties of 8-bit codes
            x[5, 0, 5], x[6, 0, 1], x[7, 0, 31] = math.nan, math.inf, -math.inf
    return x.to(dtype)


class Store:
    def __init__(self, fmt, dtype, heads, kv, dim, page, lens, new, rope=None, layers=2, seed=0, width=0, special=True):
        g = torch.Generator().manual_seed(seed)
        n = len(lens)
        held = [-(-x // page) for x in lens]
        pages = sum(held) + 2
        ids = torch.randperm(pages, generator=g).tolist()
        self.slots = torch.randperm(n + 1, generator=g)[:n].tolist()
        table = torch.full((n + 1, max(held) + 1), -1, dtype=torch.int32)
        all_lens, at = torch.zeros(n + 1, dtype=torch.int32), 0
        for s, h, m in zip(self.slots, held, lens):
            table[s, :h] = torch.tensor(ids[at:at + h], dtype=torch.int32)
            all_lens[s], at = m, at + h
        self.bits, self.fmt, self.dtype, self.dim, self.page, self.kv, self.table, self.lens, self.new = Q.BITS[fmt], fmt, dtype, dim, page, kv, table, lens, new
        pool = [torch.randint(0, 256, (layers, pages, Q.page_bytes(b, page, kv, dim)), generator=g, dtype=torch.uint8) for b in self.bits]
        self.pools = [x.clone() for x in pool]
        self.cache = PagedCache(layers, pages, page, kv, dim, n + 1, table.shape[1], dtype=dtype, k=pool[0].cuda(), v=pool[1].cuda(),
                                table=table.cuda(), lens=all_lens.cuda(), format=fmt)
        self.off = [0]
        for x in new:
            self.off.append(self.off[-1] + x)
        self.T = self.off[-1] + 2
        self.k, self.v = rows_of(dtype, self.T, kv, dim, g, special), rows_of(dtype, self.T, kv, dim, g, special)
        self.q = torch.randn(self.T, heads, dim, generator=g).to(dtype)
        self.att = BlockAttention(self.cache, heads, n, max(new + [1]), self.T, rope=rope)
        self.att.begin(i32(self.off), i32(self.slots))
        self.offd, self.slotsd = i32(self.off), i32(self.slots)

    def positions(self, i):
        return torch.arange(self.lens[i] - self.new[i], self.lens[i])

    def expect(self, layer, f=None, scale=1.0, inter=False):
        """The pools after an append, and the rows as they are held then (None where a token has no place)."""
        k = self.k.double()
        rows = [torch.zeros(self.T, self.kv, self.dim, dtype=torch.float64) for _ in range(2)]
        for i, s in enumerate(self.slots):
            pos, at = self.positions(i), torch.arange(self.off[i], self.off[i + 1])
            keep = pos >= 0
            pos, at = pos[keep], at[keep]
            if len(pos) == 0:
                continue
            page = self.table[s][pos // self.page]
            keys = self.k[at] if f is None else R.rotate(self.k[at], pos, f, scale, inter).float().to(self.dtype)
            for which, x in enumerate((keys, self.v[at])):
                codes, scales = Q.quantise(x, self.bits[which])
                rows[which][at] = Q.values(codes, scales, self.bits[which])[..., :self.dim]
                Q.put(self.pools[which][layer].view(-1), self.bits[which], self.page, self.dim, pos, page, codes, scales)
        return rows


def same(a, b):
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kv,dim,page,lens,new", [
    (2, 128, 32, [40], [8]), (1, 64, 64, [1], [1]), (3, 80, 32, [33, 100, 7], [33, 2, 7]), (2, 32, 32, [64, 31], [64, 1]),
    (1, 256, 32, [50], [50]), (2, 96, 96, [200, 5], [130, 5]), (1, 8, 32, [10, 40], [10, 20]), (1, 192, 32, [9, 0, 90], [9, 0, 3]),
    (2, 40, 64, [3], [9])])  # the last: more new tokens than the sequence has
def test_every_stored_byte(gpu_lib, fmt, dtype, kv, dim, page, lens, new):
    s = Store(fmt, dtype, kv, kv, dim, page, lens, new)
    rows = s.expect(1)
    s.att.append(1, s.k.cuda(), s.v.cuda())
    for got, want, what in ((s.cache.k, s.pools[0], "keys"), (s.cache.v, s.pools[1], "values")):
        off = torch.nonzero(got.cpu() != want)
        assert len(off) == 0, (what, [(i.tolist(), int(got.cpu()[tuple(i)]), int(want[tuple(i)])) for i in off[:8]])
    out = [torch.full((s.T, kv, dim), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    s.cache.read(1, s.offd, *out, slots=s.slotsd)
    for x, want in zip(out, rows):
        assert same(x[:s.off[-1]].cpu().double(), want[:s.off[-1]]) and bool((x[s.off[-1]:] == 7).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim,rot,inter,scaling,start", [
    (128, 128, False, "none", 0), (128, 64, False, "yarn", 100000), (64, 64, True, "ntk", 5000), (80, 50, True, "linear", 1 << 20),
    (96, 24, False, "none", 300), (256, 256, False, "none", 0), (40, 6, False, "none", 12), (64, 34, True, "none", 7)])
def test_rotated_keys(gpu_lib, fmt, dtype, dim, rot, inter, scaling, start):
    factor = 1.0 if scaling == "none" else 8.0
    rope = Rope(rot, interleaved=inter, scaling=scaling, factor=factor)
    page = 32 if start < 1000 else 1024
    s = Store(fmt, dtype, 4, 2, dim, page, [start + 40, start + 3], [40, 3], rope, special=False)
    rows = s.expect(0, rope.turns.cpu().tolist(), float(torch.tensor(rope.scale)), inter)
    q_out = torch.zeros_like(s.q).cuda()
    s.att.append(0, s.k.cuda(), s.v.cuda(), q=s.q.cuda(), q_out=q_out)
    assert torch.equal(s.cache.k.cpu(), s.pools[0]) and torch.equal(s.cache.v.cpu(), s.pools[1])
    out = [torch.zeros(s.T, 2, dim, dtype=dtype, device="cuda") for _ in range(2)]
    s.cache.read(0, s.offd, *out, slots=s.slotsd, max_tokens=40)
    assert all(same(x.cpu().double(), want) for x, want in zip(out, rows))
    # Queries are turned in float32: (cos, sin) off by 2^-22, one product of two fused with the sum (2^-23), one rounding
    # to the type, of at most 2 scale max|x| in size.  (Equal bits to a plain cache's append would ask for the same product fused.)
    f, scale = rope.turns.cpu().tolist(), float(torch.tensor(rope.scale))
    for i in range(2):
        at = slice(s.off[i], s.off[i + 1])
        want = R.rotate(s.q[at], s.positions(i), f, scale, inter)
        size = 2 * scale * s.q[at].double().abs().amax(-1, keepdim=True)
        assert bool(((q_out[at].cpu().double() - want).abs() <= (2.0 ** -22 + 2.0 ** -23 + R.EPS[dtype]) * size).all())
        assert torch.equal(q_out[at, :, rot:].cpu(), s.q[at, :, rot:])
    assert bool((q_out[s.off[-1]:] == 0).all())


@pytest.mark.parametrize("fmt,inter", [("fp8", False), ("fp8", True), ("fp4", True)])
def test_keys_are_rounded_twice(gpu_lib, fmt, inter):
    """From 64 bits to float32 and from there to bf16: keys of which float32 lies in the middle of two bf16s and 64 bits do
    not, where the other bf16 has another code."""
    rope = Rope(128, interleaved=inter)
    f = rope.turns.cpu().tolist()
    g = torch.Generator().manual_seed(3)
    k = torch.randn(4000, 8, 128, generator=g).to(BF16)
    y = R.rotate(k, torch.arange(4000), f, 1.0, inter)
    near = y.float().to(BF16)
    below = (y.float().view(torch.int32) >> 16).to(torch.int16)
    straight = torch.where(y.abs() > y.float().double().abs(), below + 1, below).view(BF16)  # of ties
    tie = (y.float().view(torch.int32) & 0xffff == 0x8000) & (y != y.float().double())
    rows = [(t, h) for t, h, e in tie.nonzero().tolist()]
    twice = torch.stack([near[t, h] for t, h in rows])
    once = torch.stack([torch.where(tie[t, h], straight[t, h], near[t, h]) for t, h in rows])
    hard = [r for r, a, b in zip(rows, twice, once) if not torch.equal(Q.held(a, Q.BITS[fmt][0]), Q.held(b, Q.BITS[fmt][0]))]
    assert len(hard) >= 1, "the definition itself has to tell them apart"
    s = Store(fmt, BF16, 1, 1, 128, 1024, [t + 1 for t, _ in hard], [1] * len(hard), rope, special=False)
    for i, (t, h) in enumerate(hard):
        s.k[i, 0] = k[t, h]
    s.expect(0, f, 1.0, inter)
    s.att.append(0, s.k.cuda(), s.v.cuda())
    assert torch.equal(s.cache.k.cpu(), s.pools[0]) and torch.equal(s.cache.v.cpu(), s.pools[1])


def fill(cache, tokens, g, slots=None):
    """Every slot of a cache filled with rows of so many tokens; returns what each holds, [layers][slot]."""
    n = len(tokens)
    slots = list(range(n)) if slots is None else slots
    off = [0]
    for t in tokens:
        off.append(off[-1] + t)
    att = BlockAttention(cache, cache.n_kv_heads, n, max(tokens), off[-1])
    att.begin(i32(off), i32(slots))
    rows = torch.randn(cache.n_layers, 2, off[-1], cache.n_kv_heads, cache.head_dim, generator=g).to(cache.dtype)
    for l in range(cache.n_layers):
        att.append(l, rows[l, 0].cuda(), rows[l, 1].cuda())
    bits = Q.BITS.get(cache.format)
    hold = lambda x, w: x.double() if bits is None else Q.held(x, bits[w])  # noqa: E731
    return [[[hold(rows[l, w, a:b], w) for w in range(2)] for a, b in zip(off[:-1], off[1:])] for l in range(cache.n_layers)]


@pytest.mark.parametrize("fmt", ["plain"] + FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kv,dim,page", [(2, 64, 32), (3, 80, 64), (1, 128, 96), (2, 8, 32), (1, 256, 32)])
def test_windows(gpu_lib, fmt, dtype, kv, dim, page):
    """Windows from any token on: whole, empty, across tiles and pages, past the end, the same slot twice; the last tokens by
    default, also more of them than there are; keys or values alone; columns of a wider tensor."""
    g = torch.Generator().manual_seed(3)
    tokens = [150, 1, 97]
    cache = PagedCache(2, 12, page, kv, dim, 4, 6, dtype=dtype, format=fmt)
    cache.resize(i32([0, 1, 2]), i32(tokens))
    held = fill(cache, tokens, g)
    slots, starts, counts = [0, 2, 0, 1, 2, 3, 0, 9, 1], [0, 31, 149, 0, 90, 0, 40, 0, 1], [150, 40, 1, 1, 20, 4, 0, 5, 3]
    off = [0]
    for c in counts:
        off.append(off[-1] + c)
    T = off[-1] + 3
    # the last tokens, as many as each sequence has at most
    last = [-1 if s > 2 else tokens[s] - c for s, c in zip(slots, counts)]
    for begin, given in ((starts, i32(starts)), (last, None)):
        wide = torch.full((T, 3, kv, dim), 7.0, dtype=dtype, device="cuda")
        k, v = wide[:, 0], wide[:, 2]
        cache.read(1, i32(off), k=k, v=v, slots=i32(slots), starts=given, max_tokens=150)
        got = wide.cpu().double()
        assert bool((got[:, 1] == 7).all()) and bool((got[off[-1]:] == 7).all())
        for i, (s, a) in enumerate(zip(slots, begin)):
            for w in range(2):
                x = got[off[i]:off[i + 1], 2 * w]
                if s > 3:  # a slot that the cache does not have: rows of no sequence
                    assert bool((x == 7).all())
                    continue
                m = tokens[s] if s < 3 else 0
                for j in range(counts[i]):
                    there = 0 <= a + j < m
                    assert same(x[j], held[1][s][w][a + j] if there else torch.zeros(kv, dim, dtype=torch.float64)), (i, w, j)
    for w in range(2):
        one = torch.full((T, kv, dim), 7.0, dtype=dtype, device="cuda")
        cache.read(1, i32(off), **{"kv"[w]: one}, slots=i32(slots), max_tokens=150)
        assert torch.equal(one, wide[:, 2 * w])


@pytest.mark.parametrize("fmt", ["plain"] + FORMATS)
def test_tokens_of_no_page(gpu_lib, fmt):
    """Ids outside the pool, a refused slot and rows beyond max_tokens."""
    g = torch.Generator().manual_seed(4)
    cache = PagedCache(1, 6, 32, 2, 64, 3, 4, format=fmt)
    cache.resize(i32([0, 1]), i32([90, 40]))
    held = fill(cache, [90, 40], g)
    before = cache.k.clone(), cache.v.clone()
    cache.table[0, 1] = 6
    cache.table[0, 2] = -7
    cache.resize(i32([1]), i32([1000]))  # lacks room: the slot is marked
    assert cache.refused.tolist()[1] != 0
    k, v = (torch.full((130, 2, 64), 7.0, dtype=BF16, device="cuda") for _ in range(2))
    cache.read(0, i32([0, 90, 130]), k, v)
    for w, x in enumerate((k.cpu().double(), v.cpu().double())):
        assert same(x[:32], held[0][0][w][:32]) and bool((x[32:90] == 0).all()) and bool((x[90:] == 7).all())
    x = torch.full((90, 2, 64), 7.0, dtype=BF16, device="cuda")
    cache.read(0, i32([0, 90]), x, starts=i32([0]), max_tokens=20)
    assert same(x[:20].cpu().double(), held[0][0][0][:20]) and bool((x[20:] == 7).all())
    # nothing is stored where there is no page
    att = BlockAttention(cache, 2, 2, 90, 130)
    att.begin(i32([0, 90, 130]))
    att.append(0, torch.ones(130, 2, 64, dtype=BF16, device="cuda"), torch.ones(130, 2, 64, dtype=BF16, device="cuda"))
    own = int(cache.table[0, 0])
    for x, old in ((cache.k, before[0]), (cache.v, before[1])):
        assert torch.equal(torch.cat((x[:, :own], x[:, own + 1:]), 1), torch.cat((old[:, :own], old[:, own + 1:]), 1))


@pytest.mark.parametrize("fmt", FORMATS)
def test_pages_move(gpu_lib, fmt):
    """A fork shares and copies pages, a compaction moves them: what every slot holds stays."""
    g = torch.Generator().manual_seed(5)
    cache = PagedCache(3, 20, 32, 2, 80, 5, 8, format=fmt)
    cache.resize(i32([0, 1, 2]), i32([100, 40, 70]))
    held = fill(cache, [100, 40, 70], g)
    cache.fork(i32([3, 4]), i32([0, 2]), i32([50, 70]), i32([60, 90]))
    cache.free(i32([1]))
    cache.compact()
    assert int(cache.status) == 0
    for slot, of, n in ((0, 0, 100), (2, 2, 70), (3, 0, 50), (4, 2, 70)):
        for l in range(3):
            k, v = (torch.zeros(n, 2, 80, dtype=BF16, device="cuda") for _ in range(2))
            cache.read(l, i32([0, n]), k, v, slots=i32([slot]), starts=i32([0]))
            assert all(same(x.cpu().double(), held[l][of][w][:n]) for w, x in enumerate((k, v)))


def test_streams_and_graphs(gpu_lib):
    """Stored and read on a stream that is not the current one; captured once, replayed as lengths and rows change."""
    cache = PagedCache(1, 8, 32, 2, 128, 1, 8, format="fp8_fp4")
    rope = Rope(64)
    att = BlockAttention(cache, 4, 1, 8, 8, rope=rope)
    off, slot, lens = i32([0, 8]), i32([0]), i32([0])
    att.begin(off, slot)
    x, y, q = (torch.zeros(8, h, 128, dtype=BF16, device="cuda") for h in (2, 2, 4))
    q_out, k, v = torch.zeros_like(q), torch.zeros_like(x), torch.zeros_like(x)

    def step(stream=None):
        att.append(0, x, y, q, q_out, stream=stream)
        cache.read(0, off, k, v, slots=slot, stream=stream)

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    g = torch.Generator().manual_seed(6)
    for turn in range(5):
        lens.fill_(8 * turn + 8)
        cache.resize(slot, lens)
        for t in (x, y, q):
            t.copy_(torch.randn(t.shape, generator=g))
        torch.cuda.synchronize()
        if turn == 0:
            step(side)
            side.synchronize()
        elif turn == 1:
            with torch.cuda.graph(graph):
                step()
            graph.replay()
        else:
            graph.replay()
        torch.cuda.synchronize()
        pos = torch.arange(8 * turn, 8 * turn + 8)
        keys = R.rotate(x.cpu(), pos, rope.turns.cpu().tolist()).float().to(BF16)
        assert same(k.cpu().double(), Q.held(keys, 8)) and same(v.cpu().double(), Q.held(y.cpu(), 4))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("inter,rot", [(False, 64), (True, 50), (False, 36), (False, 0)])
def test_columns_of_one_tensor_in_place(gpu_lib, dtype, inter, rot):
    """Queries turned in place beside their keys and values, enough rows that a workgroup takes several heads, the last one
    fewer: the bits of a call with tensors of their own, and nothing else touched."""
    new, heads, kv, dim = [600, 0, 333], 12, 3, 64
    T, n = sum(new) + 2, len(new)
    g = torch.Generator().manual_seed(9)
    wide = torch.randn(T, heads + 2 * kv, dim, generator=g).to(dtype).cuda()
    before = wide.clone()
    got = []
    for fused in (False, True):
        cache = PagedCache(1, 64, 32, kv, dim, n, 24, dtype=dtype, format="fp8_fp4")
        cache.resize(i32(list(range(n))), i32([x + 70 for x in new]))
        att = BlockAttention(cache, heads, n, max(new), T, rope=Rope(rot, interleaved=inter) if rot else None)
        att.begin(i32([0, 600, 600, 933]))
        x = wide if fused else before.clone()
        q, k, v = x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:]
        if fused:
            att.append(0, k, v, q)
            got.append((cache.k, cache.v, q))
        else:
            q_out = before[:, :heads].clone()
            att.append(0, k.contiguous(), v.contiguous(), q.contiguous(), q_out)
            got.append((cache.k, cache.v, q_out))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert torch.equal(wide[:, heads:], before[:, heads:]) and torch.equal(wide[-2:], before[-2:])
    assert rot == 0 or not torch.equal(wide[:, :heads], before[:, :heads])


def test_far_into_a_large_pool(gpu_lib):
    """Offsets beyond 32 bits: a page behind more than 4 GiB of others."""
    kv, dim, page = 8, 256, 1024
    size = Q.page_bytes(8, page, kv, dim)
    pages = (1 << 32) // size + 3
    cache = PagedCache(1, pages, page, kv, dim, 1, 2, format="fp8", table=i32([[pages - 1, pages - 2]]), lens=i32([page + 5]))
    held = fill(cache, [page + 5], torch.Generator().manual_seed(7))
    k, v = (torch.zeros(page + 5, kv, dim, dtype=BF16, device="cuda") for _ in range(2))
    cache.read(0, i32([0, page + 5]), k, v)
    assert all(same(x.cpu().double(), held[0][0][w]) for w, x in enumerate((k, v)))
    assert bool((cache.k[0, :4] == 0).all())


def test_many_sequences(gpu_lib):
    """More sequences than a wave counts at once, of uneven lengths, some without tokens."""
    n = 150
    g = torch.Generator().manual_seed(8)
    tokens = [int(t) for t in torch.randint(0, 80, (n,), generator=g)]
    cache = PagedCache(1, 3 * n, 32, 1, 64, n, 3, format="fp4")
    cache.resize(i32(list(range(n))), i32(tokens))
    held = fill(cache, tokens, g)
    off = [0]
    for t in tokens:
        off.append(off[-1] + t)
    k, v = (torch.full((off[-1] + 1, 1, 64), 7.0, dtype=BF16, device="cuda") for _ in range(2))
    cache.read(0, i32(off), k, v)
    for w, x in enumerate((k.cpu().double(), v.cpu().double())):
        assert bool((x[-1] == 7).all())
        for i, t in enumerate(tokens):
            assert same(x[off[i]:off[i + 1]], held[0][i][w]), i
