"""Calls of the attention's objects as a program makes them: on another stream than the current one, with batches that
shrink, plans that outlive a compaction, updates that are refused, several hundred sequences, pages of every size.
Marked ``gpu``."""
import math

import pytest
import torch

import attention_ref as R
from paper_2605_30876_amd import lib
from paper_2605_30876_amd.attention import AttentionLayer, BlockAttention, PagedCache, Rope
from paper_2605_30876_amd.layer import decode_step
from test_gpu_attention import FORMS, Setup, _form, _poison
from test_gpu_decode_attention import L, Model

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _busy():
    """Keeps the current stream occupied for a while (at most a second) without the host's waiting."""
    torch.cuda.synchronize()
    torch.cuda._sleep(50_000_000)


def test_free_on_another_stream(gpu_lib):
    """What free() makes for its call is made on the call's stream: the current one is behind."""
    cache = PagedCache(1, 64, 32, 1, 32, 8, 8)
    slots, side = i32(list(range(8))), torch.cuda.Stream()
    cache.resize(slots, i32([40] * 8))
    blocks = [torch.full_like(slots, 7) for _ in range(32)]  # what an allocation on the current stream finds in its memory
    torch.cuda.synchronize()
    del blocks
    _busy()
    cache.free(slots, stream=side)
    side.synchronize()
    assert cache.lens.tolist() == [0] * 8 and int(cache.status[0]) == 0 and int(cache.refs.sum()) == 0


def _pending(like, n=24):
    """Tensors that are read on the current stream once it gets to it, and whose memory is free to the allocator."""
    xs = [torch.full_like(like, 3.0) for _ in range(n)]
    _busy()
    ys = [x.clone() for x in xs]
    del xs
    return ys


def test_attend_on_another_stream_allocates_there(gpu_lib):
    s = Setup(BF16, 8, 2, 64, 32, [500], [8], 8, seed=8)
    want, _ = s.run()
    side = torch.cuda.Stream()
    ys = _pending(s.qd[0])
    got = s.att.attend(0, s.qd[0], stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert all(bool((y == 3.0).all()) for y in ys)
    assert torch.equal(got[:8].cpu(), want[:8])


def test_a_larger_workspace_is_allocated_on_the_calls_stream(gpu_lib):
    """An update of more entries than the cache has slots (refused: some come twice) needs a workspace of its own."""
    cache = PagedCache(1, 64, 32, 1, 32, 4, 128)
    n, side = 3000, torch.cuda.Stream()
    slots, lens = i32([i % 4 for i in range(n)]), i32([1] * n)
    before = cache._ws[-1].numel()
    nbytes = lib.dmoe_cache_update_workspace_size(n, cache.max_pages, cache.n_pages)
    assert nbytes > before
    ys = _pending(torch.empty((nbytes // 4,), device="cuda"))
    cache.resize(slots, lens, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert all(bool((y == 3.0).all()) for y in ys)
    assert int(cache.status[0]) == -1 and cache.lens.tolist() == [0] * 4


class Half:
    """One layer's attention half over two sequences of up to eight new tokens."""

    def __init__(self, dtype=BF16, n=2, new=8, H=96, heads=4, kv=2, dim=32):
        g = torch.Generator(device="cuda").manual_seed(11)
        mat = lambda *s: torch.randn(*s, generator=g, device="cuda").mul_(1 / math.sqrt(s[1])).to(dtype)  # noqa: E731
        self.cache = PagedCache(1, 20, 32, kv, dim, n, 4, dtype=dtype)
        self.T, self.slots = n * new, i32(list(range(n)))
        self.cache.resize(self.slots, i32([40 + 3 * i for i in range(n)]))
        self.cache.k.zero_(), self.cache.v.fill_(0.5)
        self.att = BlockAttention(self.cache, heads, n, new, self.T, mask_block=new, rope=Rope(dim))
        self.w = {"wq": mat(heads * dim, H), "wk": mat(kv * dim, H), "wv": mat(kv * dim, H), "wo": mat(H, heads * dim)}
        self.layer = AttentionLayer(self.att, 0, self.w)
        self.off = i32([new * i for i in range(n + 1)])
        self.x = mat(self.T, H)

    def step(self, layer=None):
        self.att.begin(self.off, self.slots)
        self.att.plan()
        return (layer or self.layer)(self.x).clone()


@pytest.mark.parametrize("how", ["fewer rows", "no such slot", "a graph"])
def test_rows_that_dropped_out_keep_nothing(gpu_lib, how):
    """A full batch, then a smaller one: rows of no sequence are the input, as in a layer that has done nothing before."""
    h = Half()
    full = h.step()
    assert not torch.equal(full[8:], h.x[8:])
    if how == "a graph":
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            h.step()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                y = h.step()
        torch.cuda.current_stream().wait_stream(side)
    for off, slots in (([0, 8, 8], [0, 1]), ([0, 8, 16], [0, 1]), ([0, 5, 5], [0, 1]), ([0, 8, 16], [0, 9 if how == "no such slot" else 1])):
        h.off.copy_(torch.tensor(off, dtype=torch.int32))
        h.slots.copy_(torch.tensor(slots, dtype=torch.int32))
        torch.cuda.synchronize()
        if how == "a graph":
            g.replay()
            torch.cuda.synchronize()
            got = y.clone()
        else:
            got = h.step()
        want = h.step(AttentionLayer(h.att, 0, h.w))
        assert torch.equal(got, want)
        used = 8 if slots[1] == 9 else off[2]
        assert torch.equal(got[used:], h.x[used:])


def test_a_new_cache_holds_zeros(gpu_lib):
    """Tokens that are given room but never stored are attended to like any others: not whatever the memory held."""
    c = PagedCache(2, 8, 32, 2, 64, 1, 8)
    blocks = [torch.full_like(c.k, float("nan")) for _ in range(16)]
    del blocks, c
    c = PagedCache(2, 8, 32, 2, 64, 1, 8)
    assert (c.k == 0).all() and (c.v == 0).all()


@pytest.mark.parametrize("form", list(FORMS))
def test_a_plan_outlives_a_compaction(gpu_lib, form):
    """A plan goes by offsets, slots and lengths: pages that move after it was made are found where they are."""
    s = _form(form, 24, slack=60)
    n = s.cache.n_pages
    held = s.cache.table[s.cache.table >= 0].long()
    s.cache.refs[held] = 1
    out, lse = s.run()
    s.check(out, lse)
    s.att.plan()
    counts = torch.zeros(2, dtype=torch.int32, device="cuda")
    s.cache.compact(counts=counts)
    live, moved = counts.tolist()
    assert live == held.numel() and moved > 4
    s.cache.k[:, live:n] = float("nan")
    s.cache.v[:, live:n] = float("nan")
    again, lse2 = torch.full_like(out, 7.0, device="cuda"), torch.full_like(lse, 7.0, device="cuda")
    s.att.attend(0, s.qd[0], again, lse2)
    assert torch.equal(again.cpu(), out) and torch.equal(lse2.cpu(), lse)
    # and pages taken away after the plan are not followed
    s.cache.table.fill_(-1)
    s.att.attend(0, s.qd[0], again, lse2)
    rows = slice(0, s.off[-1])
    assert (again[rows] == 0).all() and (lse2[rows] == -math.inf).all()


def test_attend_needs_a_plan_of_its_batch(gpu_lib):
    s = Setup(BF16, 4, 2, 64, 32, [60, 50], [6, 2], 0)
    s.att.begin(s.offd, s.slotsd)
    with pytest.raises(RuntimeError, match="plan"):
        s.att.attend(0, s.qd[0])
    want, _ = s.run()
    s.att.begin(s.offd, s.slotsd)
    with pytest.raises(RuntimeError, match="plan"):
        s.att.attend(0, s.qd[0])
    s.att.plan()
    assert torch.equal(s.att.attend(0, s.qd[0])[:8].cpu(), want[:8])


def _stored(cache):
    return cache.k.clone(), cache.v.clone()


@pytest.mark.parametrize("pages", [6, 9000])
def test_a_refused_update_leaves_its_slots_alone(gpu_lib, pages):
    """A sequence that was not given the room it asked for: a later call on another slot does not hide it, and nothing
    is stored over what it shares with others."""
    cache = PagedCache(1, pages, 32, 1, 32, 4, 8)
    cache.k.zero_(), cache.v.zero_()
    if pages > 6:
        cache.refs[6:] = 1  # taken by others
    cache.resize(i32([0]), i32([96]))
    cache.fork(i32([1]), i32([0]), i32([96]))  # all three pages shared
    cache.resize(i32([3]), i32([33]))
    seen = torch.zeros(3, dtype=torch.int32, device="cuda")
    cache.resize(i32([1, 2]), i32([104, 100]), status=seen[0:1])  # five pages, of which there is one
    cache.resize(i32([3]), i32([40]), status=seen[1:2])
    assert seen.tolist() == [4, 0, 0] and cache.refused.tolist() == [0, 4, 4, 0]
    att = BlockAttention(cache, 2, 2, 8, 16, mask_block=8)
    att.begin(i32([0, 8, 16]), i32([1, 3]))
    kv, q = torch.ones(16, 1, 32, device="cuda").to(BF16), torch.ones(16, 2, 32, device="cuda").to(BF16)
    before = _stored(cache)
    att.append(0, kv, kv, q)
    ka, va = R.places(BF16, 32, 1, 32, torch.arange(32, 40), cache.table[3, 1].cpu().expand(8))
    for was, now, at in zip(before, _stored(cache), (ka, va)):
        was.view(-1)[at.cuda()] = 1.0  # the other sequence's
        assert torch.equal(was, now)
    out = torch.full_like(q, 7.0)
    att.plan()
    att.attend(0, q, out)
    assert (out[:8] == 7.0).all() and (out[8:] != 7.0).all()
    # the same request with room for it
    cache.resize(i32([1]), i32([104]), status=seen[2:3])
    assert seen.tolist() == [4, 0, 0] and cache.refused.tolist() == [0, 0, 4, 0]
    before = _stored(cache)
    att.append(0, kv, kv, q)
    ka, va = R.places(BF16, 32, 1, 32, torch.arange(96, 104), cache.table[1, 3].cpu().expand(8))
    for was, now, at in zip(before, _stored(cache), (ka, va)):
        was.view(-1)[at.cuda()] = 1.0
        assert torch.equal(was, now)


def test_a_wrong_update_marks_the_slots_it_names(gpu_lib):
    cache = PagedCache(1, 6, 32, 1, 32, 4, 8)
    cache.resize(i32([0, 1]), i32([40, 40]))
    cache.resize(i32([0, 9, -3, 2]), i32([50, 1, 1, 8]))
    assert cache.refused.tolist() == [-1, 0, -1, 0] and cache.lens.tolist() == [40, 40, 0, 0]
    cache.resize(i32([0, 2]), i32([50, 8]))
    assert cache.refused.tolist() == [0, 0, 0, 0] and cache.lens.tolist() == [50, 40, 8, 0]
    cache.table[1, 1] = 99
    cache.free(i32([1]))
    assert cache.refused.tolist() == [0, -1, 0, 0]


@pytest.mark.parametrize("attended", [False, True])
@pytest.mark.parametrize("residual", ["step", "stream"])
@pytest.mark.parametrize("name", ["small_bf16", "small_f32"])
def test_the_residual_of_a_step(gpu_lib, name, residual, attended):
    """Layer l+1's input: the step's input plus y, or the layer's own input (with its attention) plus y, rounded once."""
    m = Model(name, "block")
    m.cache.resize(m.slots, m.i32([m.bs] * m.n))
    y = decode_step(m.m, m.w, m.xs, "block", attention=m.al if attended else None, residual=residual)
    assert torch.equal(y, m.m[-1].y) and torch.isfinite(y).all()
    for l in range(L - 1):
        base = m.xs[0] if residual == "step" else m.al[l].out if attended else m.xs[l]
        assert torch.equal(m.xs[l + 1], (base.float() + m.m[l].y.float()).to(base.dtype)), f"layer {l}"
    with pytest.raises(ValueError):
        decode_step(m.m, m.w, m.xs, "block", residual="layer")


def test_unsorted_offsets_stay_within_the_plan(gpu_lib):
    """Every second sequence claims all rows: 2^31 row tiles, of which the plan has places for 2^20 and a few."""
    T, n, heads = 1 << 17, 4096, 1024
    cache = PagedCache(1, 4, 32, 1, 8, 4, 2)
    cache.lens.fill_(40)
    cache.table[:, 0], cache.table[:, 1] = 1, 2
    att = BlockAttention(cache, heads, n, T, T, mask_block=1)
    att.begin(i32([0, T] * (n // 2) + [0]), i32([i % 4 for i in range(n)]))
    att.plan()
    n_items, n_merges = att._plan[:2].tolist()
    assert T * heads // 128 <= n_items <= T * heads // 128 + n and n_merges == 0
    assert 4 + 16 * n_items <= att._plan.numel()
    slot, row0, rows, length, first, all_rows, kt0, kt1 = att._plan[4:4 + 16 * n_items].view(-1, 16)[:, :8].unbind(1)
    assert ((slot >= 0) & (slot < 4) & (row0 == 0) & (rows == T) & (length == 40)).all()
    assert ((all_rows == T * heads) & (first >= 0) & (first < all_rows) & (first % 128 == 0)).all()
    assert ((kt0 >= 0) & (kt0 <= kt1) & (kt1 <= 2)).all()


@pytest.mark.parametrize("page", [96, 160])
@pytest.mark.parametrize("form", ["two_halves", "two_halves_f32", "one_128", "one_256", "one_f32", "sixty_four", "sixty_four_f32", "thirty_two",
                                  "thirty_two_f32_256"])
def test_pages_whose_tiles_are_no_power_of_two(gpu_lib, form, page):
    dtype, heads, kv, dim, _, n, capacity = FORMS[form]
    new = [40, 33, 0, 21, 1, 40, 9, 2, 0][:n]
    if form.startswith("thirty_two"):
        new = [min(x, 32 * kv // heads) for x in new]
    s = Setup(dtype, heads, kv, dim, page, [333, 64, 0, 900, 33, 159, 5, 0, 97][:n], new, 24, seed=page, capacity=capacity)
    s.check(*s.run())


@pytest.mark.parametrize("dtype,heads,kv,dim", [(BF16, 96, 2, 64), (BF16, 1024, 1, 8), (F32, 17, 1, 32), (BF16, 57, 3, 40)])
def test_many_heads_of_a_group(gpu_lib, dtype, heads, kv, dim):
    s = Setup(dtype, heads, kv, dim, 32, [70, 1, 0, 33], [2, 1, 0, 2], 1, seed=heads)
    s.check(*s.run())


@pytest.mark.parametrize("heads,kv,new", [(2, 2, 1), (16, 2, 5), (8, 1, 9)])
def test_plans_of_several_passes(gpu_lib, heads, kv, new):
    """600 sequences: more row tiles than the plan has threads, and more sequences than it keeps."""
    lens = [(5 * i * i) % 97 for i in range(600)]
    s = Setup(BF16, heads, kv, 32, 32, lens, [min(x, i % (new + 1)) for i, x in enumerate(lens)], 1, seed=3)
    s.check(*s.run())


def _append_case(dtype, heads, kv, dim, page, lens, new, rot, inter, seed):
    """Stores a batch and compares with the definition; every element of the pool and of q_out."""
    g = torch.Generator().manual_seed(seed)
    n, dp = len(lens), R.padded(dim)
    width = max(-(-m // page) for m in lens) + 1
    pages = sum(-(-m // page) for m in lens) + 2
    ids, at = torch.randperm(pages, generator=g).int(), 0
    table = torch.full((n, width), -1, dtype=torch.int32)
    for i, m in enumerate(lens):
        h = -(-m // page)
        table[i, :h] = ids[at:at + h]
        at += h
    cache = PagedCache(1, pages, page, kv, dim, n, width, dtype=dtype, table=table.cuda(), lens=i32(lens))
    cache.k.fill_(77.0), cache.v.fill_(77.0)
    off = [0]
    for x in new:
        off.append(off[-1] + x)
    T = off[-1] + 3
    q, k, v = (torch.randn(T, h, dim, generator=g).to(dtype) for h in (heads, kv, kv))
    att = BlockAttention(cache, heads, n, max(new), T, rope=Rope(rot, interleaved=inter))
    att.begin(i32(off))
    q_out = torch.full((T, heads, dim), 7.0, dtype=dtype, device="cuda")
    att.append(0, k.cuda(), v.cuda(), q.cuda(), q_out)
    want_k = torch.full((pages * page * kv * dp,), 77.0, dtype=torch.float64)
    want_v, want_q = want_k.clone(), torch.full((T, heads, dim), 7.0, dtype=torch.float64)
    f, pad = R.turns(rot)[0], (0, dp - dim)
    rows = torch.cat([torch.arange(b - min(m, x), b) for m, x, b in zip(lens, new, off[1:])])
    pos = torch.cat([torch.arange(m - min(m, x), m) for m, x in zip(lens, new)])
    seq = torch.cat([torch.full((min(m, x),), i) for i, (m, x) in enumerate(zip(lens, new))])
    ka, va = R.places(dtype, page, kv, dp, pos, table[seq, pos // page])
    want_q[rows] = R.rotate(q[rows], pos, f, 1.0, inter)
    want_k[ka] = torch.nn.functional.pad(R.rotate(k[rows], pos, f, 1.0, inter), pad)
    want_v[va] = torch.nn.functional.pad(v[rows].double(), pad)
    # cos and sin 2^-22, two products and a sum 2^-23, the rounding to the type, of at most twice the largest value
    tol = (2.0 ** -22 + 2.0 ** -23 + R.EPS[dtype]) * 2
    assert torch.equal(cache.v.cpu().view(-1).double(), want_v)
    assert bool(((cache.k.cpu().view(-1).double() - want_k).abs() <= tol * float(k.abs().max())).all())
    assert torch.equal(cache.k.cpu().view(-1) == 77.0, want_k == 77.0)
    assert bool(((q_out.cpu().double() - want_q).abs() <= tol * float(q.abs().max())).all())
    assert torch.equal(q_out[off[-1]:].cpu(), torch.full((3, heads, dim), 7.0, dtype=dtype))


@pytest.mark.parametrize("dtype,heads,kv,dim,rot,inter", [(BF16, 2, 1, 64, 64, False), (F32, 3, 3, 40, 22, False), (BF16, 7, 1, 32, 16, True),
                                                          (BF16, 29, 1, 256, 128, False)])
def test_append_counts_its_tiles(gpu_lib, dtype, heads, kv, dim, rot, inter):
    """One long sequence among many short ones: the tiles there are, found by counting, 64 sequences at a time."""
    lens = [(11 * i) % 70 for i in range(131)]
    new = [min(x, i % 4) for i, x in enumerate(lens)]
    lens[97], new[97] = 700, 650
    lens[3], new[3] = 2, 5  # more new tokens than the sequence has
    _append_case(dtype, heads, kv, dim, 32, lens, new, rot, inter, 17)


@pytest.mark.parametrize("dtype,heads,kv,dim,rot,inter", [(BF16, 20, 2, 128, 128, False), (BF16, 26, 1, 8, 8, True), (F32, 11, 11, 64, 64, True),
                                                          (BF16, 10, 5, 80, 36, False), (F32, 37, 1, 24, 24, False)])
def test_append_of_many_tokens(gpu_lib, dtype, heads, kv, dim, rot, inter):
    """Enough tokens for several heads to a workgroup, the last group not full."""
    lens = [2500, 40, 1900, 0, 999]
    _append_case(dtype, heads, kv, dim, 64, lens, [2500, 33, 1700, 0, 1], rot, inter, 23)


@pytest.mark.parametrize("dtype,T,heads,dim,rot,inter", [(BF16, 4100, 13, 64, 64, False), (BF16, 5003, 7, 128, 64, True), (F32, 4100, 13, 32, 22, False),
                                                         (BF16, 9000, 5, 8, 8, False), (F32, 4097, 11, 64, 64, False)])
def test_rotation_of_many_rows(gpu_lib, dtype, T, heads, dim, rot, inter):
    """Enough rows for several heads to a workgroup, the last group not full."""
    g = torch.Generator().manual_seed(T)
    x = torch.randn(T, heads, dim, generator=g).to(dtype)
    pos = torch.randint(0, 100_000, (T,), generator=g, dtype=torch.int32)
    out = torch.full((T + 1, heads, dim), 7.0, dtype=dtype, device="cuda")
    Rope(rot, interleaved=inter).apply(x.cuda(), pos.cuda(), out=out[:T])
    want = R.rotate(x, pos, R.turns(rot)[0], 1.0, inter)
    tol = (2.0 ** -22 + 2.0 ** -23 + R.EPS[dtype]) * 2 * float(x.abs().max())
    assert bool(((out[:T].cpu().double() - want).abs() <= tol).all()) and (out[T:] == 7.0).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf"), torch.finfo(BF16).min])
@pytest.mark.parametrize("dtype,new", [(BF16, 8), (BF16, 40), (F32, 8)])
@pytest.mark.parametrize("which", ["k", "v"])
def test_values_of_masked_places_reach_the_rows_that_see_them(gpu_lib, dtype, new, value, which):
    """The counterpart of masked places that do not matter: the rows behind the first such token differ."""
    s = Setup(dtype, 4, 2, 64, 32, [150], [new], 1, seed=3)
    before, lse0 = s.run()
    first = 150 - new + new // 2
    _poison(s, 0, list(range(first, 150)), value, which)
    out, lse = s.run()
    rows = slice(new // 2, new)
    if which == "v":
        assert torch.equal(lse[rows], lse0[rows]) and (out[rows] != before[rows]).all()
    else:  # the keys' scores are not numbers, or beyond all others, or below them
        assert (lse[rows] != lse0[rows]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_single_tokens_of_an_attention_layer(gpu_lib, dtype):
    """Autoregressive steps of three sequences: every step's new row against the definition on the cache's contents."""
    h = Half(dtype, n=3, new=1)
    for step in range(3):
        h.cache.resize(h.slots, i32([41 + 3 * i + 15 * step for i in range(3)]))
        h.cache.k.nan_to_num_(0.0), h.cache.v.nan_to_num_(0.0)  # tokens that no step stored
        h.step()
        c, o, q = h.cache, h.layer.o.cpu().view(3, 4, 32), h.layer.q.cpu().view(3, 4, 32)
        for i, m in enumerate(c.lens.tolist()):
            pos = torch.arange(m)
            ka, va = R.places(dtype, 32, 2, 32, pos, c.table[i].cpu()[pos // 32])
            ref = R.attention(q[i:i + 1], c.k.cpu().view(-1)[ka], c.v.cpu().view(-1)[va], torch.tensor([m]), 1 / math.sqrt(32))
            tol, _ = R.bounds(dtype, 32, m, *ref)
            assert bool(((o[i:i + 1].double() - ref[0]).abs() <= tol).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_columns_of_one_tensor(gpu_lib, dtype):
    """Inputs and outputs side by side in one wider tensor share rows' span and no element."""
    s = Setup(dtype, 6, 2, 72, 32, [90, 40], [33, 2], 8, seed=6)
    want, _ = s.run()
    T, W = s.q.shape[1], 6 * 72
    wide = torch.full((T, 3 * W + 8), 3.0, dtype=dtype, device="cuda")
    part = lambda at: wide[:, at:at + W].view(T, 6, 72)  # noqa: E731
    part(8).copy_(s.qd[0])
    part(8 + W).fill_(7.0)
    s.att.attend(0, part(8), part(8 + W))
    assert torch.equal(part(8 + W).cpu(), want) and torch.equal(part(8), s.qd[0])
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    rope = Rope(72)
    turned = rope.apply(s.qd[0].clone(), pos)
    assert torch.equal(rope.apply(part(8), pos, out=part(8 + 2 * W)), turned)
    kv = torch.randn(T, 2, 72, device="cuda").to(dtype)
    s.att.append(0, kv, kv, part(8), part(8 + W))
    used = s.off[-1]
    assert torch.equal(part(8 + W)[:used], s.qd[0][:used]) and torch.equal(part(8 + 2 * W), turned) and (wide[:, :8] == 3.0).all()
    for at in (16, W, 8):
        with pytest.raises(lib.DmoeError, match="overlap"):
            s.att.attend(0, part(8), part(at))


def test_weights_that_an_attention_layer_does_not_use(gpu_lib):
    """A layer's whole set of weights may be passed, whatever else it holds."""
    h = Half()
    want = h.step()
    more = {"bias": None, "norm": torch.ones(4, device="cuda", requires_grad=True), **h.w}
    assert torch.equal(h.step(AttentionLayer(h.att, 0, more)), want)


@pytest.mark.parametrize("where", ["current", "other"])
def test_no_workspace_is_made_during_a_capture(gpu_lib, where):
    """Whether the call is on the stream that captures or on another: memory is not allocated outside the graph's pool."""
    cache = PagedCache(1, 64, 32, 1, 32, 4, 128)
    slots, lens, side = i32([i % 4 for i in range(3000)]), i32([1] * 3000), torch.cuda.Stream()
    g, n = torch.cuda.CUDAGraph(), len(cache._ws)
    x = torch.zeros(4, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        with pytest.raises(RuntimeError, match="workspace"):
            cache.resize(slots, lens, stream=side if where == "other" else None)
        x.add_(1.0)
    g.replay()
    torch.cuda.synchronize()
    assert len(cache._ws) == n and (x == 1.0).all() and cache.lens.tolist() == [0] * 4
