"""Attention over caches of few bits, and of none, where the other tests do not go: 16 rows or fewer at every width of a head,
rows whose scores are all -inf, what the bytes of codes and scales stand for, results that repeat.  Marked ``gpu``."""
import math

import pytest
import torch

import attention_ref as R
import quant_ref as Q
from paper_2605_30876_amd.attention import BlockAttention, PagedCache, Rope
from test_gpu_quant_attention import BF16, F32, FORMATS, Setup, i32, spoil

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [8, 32, 64, 80, 96, 128, 160, 192, 256])
@pytest.mark.parametrize("capacity", [0, 1 << 14])
@pytest.mark.parametrize("group,new", [(1, [12, 3]), (4, [4, 1])])
def test_few_rows_of_every_width(gpu_lib, fmt, dtype, dim, capacity, group, new):
    """16 rows of a kv head to a workgroup of four waves and, where sequences may be long, of eight, split along the keys or not."""
    s = Setup(fmt, dtype, 2 * group, 2, dim, 32, [900, 30], new, 1, capacity=capacity)
    s.check(*s.run())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("capacity", [0, 1 << 14])
@pytest.mark.parametrize("dim", [32, 80, 96, 192])
def test_what_few_rows_of_other_widths_do_not_see(gpu_lib, fmt, dtype, capacity, dim):
    s = Setup(fmt, dtype, 2, 2, dim, 32, [900, 30], [12, 3], 1, capacity=capacity)
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


@pytest.mark.parametrize("fmt", ["plain"] + FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("group,new,capacity", [(1, 3, 0), (1, 3, 1 << 14), (1, 24, 0), (4, 12, 0), (4, 40, 0), (4, 40, 1 << 17)])
@pytest.mark.parametrize("lens", [[40, 60], [900, 60]])
def test_rows_whose_scores_are_all_minus_infinity(gpu_lib, fmt, dtype, group, new, capacity, lens):
    """They are 0 with log-sum-exp -inf, also where they see values that are not finite, in every form and joined from pieces;
    the rows beside them are the definition's."""
    kv, dim, heads = 2, 64, 2 * group
    g = torch.Generator().manual_seed(11)
    width = max(max(lens) // 32 + 2, capacity // 32)
    cache = PagedCache(1, sum(lens) // 32 + 8, 32, kv, dim, 2, width, dtype=dtype, format=fmt)
    cache.resize(i32([0, 1]), i32(lens))
    k, v = (torch.randn(sum(lens), kv, dim, generator=g) for _ in range(2))
    k[:, :, 0] = 2.0 + k[:, :, 0].abs()  # never rounded to 0: largest of its group, or a quarter of it at least
    k[:, :, 1:32] = k[:, :, 1:32].clamp(-2, 2)
    v[7, 0, 3] = math.inf
    v[20, 1, 40] = math.nan
    fill = BlockAttention(cache, kv, 2, max(lens), sum(lens))
    fill.begin(i32([0, lens[0], sum(lens)]))
    fill.append(0, k.to(dtype).cuda(), v.to(dtype).cuda())
    q = torch.randn(2 * new, heads, dim, generator=g)
    q[::2] = 0.0
    q[::2, :, 0] = -3e38
    q = q.to(dtype)
    att = BlockAttention(cache, heads, 2, new, 2 * new)
    att.begin(i32([0, new, 2 * new]))
    att.plan()
    lse = torch.full((2 * new, heads), 7.0, device="cuda")
    out = att.attend(0, q.cuda(), lse=lse).cpu()
    assert bool((out[::2] == 0).all()) and bool((lse[::2] == -math.inf).all())
    held = [torch.zeros(sum(lens), kv, dim, dtype=dtype, device="cuda") for _ in range(2)]
    cache.read(0, i32([0, lens[0], sum(lens)]), *held)
    held = [x.cpu() for x in held]
    parts = 3 if dtype == F32 and fmt != "plain" else 1
    for i, at in enumerate((slice(0, lens[0]), slice(lens[0], sum(lens)))):
        rows = torch.arange(i * new, (i + 1) * new)
        rows = rows[rows % 2 == 1]
        # a sum with a NaN is NaN, which the bounds leave out: the first sequence's values of the elements that are finite
        vv = held[1][at].clone()
        bad = ~vv.isfinite().all(0)
        vv[:, bad] = 0
        ref = R.attention(q[rows], held[0][at], vv, [lens[i]] * len(rows), 1 / math.sqrt(dim))
        tol, ltol = R.bounds(dtype, parts * dim, parts * lens[i], *ref)
        bad = bad.repeat_interleave(group, 0)[None].expand(len(rows), -1, -1)
        err = (out[rows].double() - ref[0]).abs()
        assert bool((err[~bad] <= tol[~bad]).all()) and bool((~out[rows][bad].isfinite()).all())
        assert bool(((lse[rows].cpu().double() - ref[1]).abs() <= ltol).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_results_repeat_in_every_form(gpu_lib, fmt, dtype):
    for group, new, lens, capacity in ((2, 1, [3000, 70], 0), (2, 1, [3000, 70], 1 << 14), (2, 20, [3000, 70], 0), (4, 32, [2000, 64], 0),
                                       (4, 40, [2000, 64], 1 << 17)):
        s = Setup(fmt, dtype, 2 * group, 2, 128, 32, lens, [new, new], 32, capacity=capacity)
        first = s.run()
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(first, s.run()))


@pytest.mark.parametrize("fmt,bits", [("fp8", 8), ("fp4", 4)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_what_every_byte_stands_for(gpu_lib, fmt, bits, dtype):
    """Every code at every scale byte, also those that are never stored, in arrays that were given: code times scale, rounded to bf16."""
    dim, n = 256, 256
    codes = (torch.arange(dim) % (1 << bits)).repeat(n, 1, 1)
    scales = torch.arange(n)[:, None, None].expand(n, 1, dim // 32)
    pool = torch.zeros(Q.page_bytes(bits, n, 1, dim), dtype=torch.uint8)
    Q.put(pool, bits, n, dim, torch.arange(n), torch.zeros(n), codes, scales)
    given = [pool.view(1, 1, -1).cuda() for _ in range(2)]
    cache = PagedCache(1, 1, n, 1, dim, 1, 1, dtype=dtype, k=given[0], v=given[1], table=i32([[0]]), lens=i32([n]), format=fmt)
    got = [torch.full((n, 1, dim), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    cache.read(0, i32([0, n]), *got)
    want = Q.values(codes, scales, bits).to(BF16).to(dtype)
    for x in got:
        assert bool(((x.cpu() == want) | (x.cpu().isnan() & want.isnan())).all())


@pytest.mark.parametrize("fmt", ["plain"] + FORMATS)
def test_a_bound_of_any_size(gpu_lib, fmt):
    """An upper bound of a read's tokens may be any number that is large enough."""
    cache = PagedCache(1, 4, 32, 2, 64, 1, 4, format=fmt)
    cache.resize(i32([0]), i32([70]))
    att = BlockAttention(cache, 2, 1, 70, 70)
    att.begin(i32([0, 70]))
    x = torch.randn(70, 2, 64, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    att.append(0, x, x)
    got = [torch.zeros_like(x) for _ in range(3)]
    for y, most in zip(got, (None, 70, 1 << 40)):
        cache.read(0, i32([0, 70]), y, max_tokens=most)
    assert bool((got[0] != 0).any()) and torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


@pytest.mark.parametrize("fmt", ["plain"] + FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_one_row_of_any_stride(gpu_lib, fmt, dtype):
    """The distance between rows of a tensor that has one row says nothing: views [1, heads, dim] of heads that lie one after
    another are taken like any others."""
    heads, kv, dim = 4, 2, 64
    g = torch.Generator().manual_seed(2)
    rows = [torch.randn(h, 1, dim, generator=g).to(dtype).cuda() for h in (kv, kv, heads)]
    rope, got = Rope(dim), []
    for flip in (False, True):
        new = lambda h: torch.zeros(h, 1, dim, dtype=dtype, device="cuda").transpose(0, 1) if flip else torch.zeros(1, h, dim, dtype=dtype, device="cuda")  # noqa: E731
        k, v, q = (x.clone().transpose(0, 1) if flip else x.transpose(0, 1).clone(memory_format=torch.contiguous_format) for x in rows)
        assert q.stride(0) == (dim if flip else heads * dim)
        cache = PagedCache(1, 2, 32, kv, dim, 1, 2, dtype=dtype, format=fmt)
        cache.resize(i32([0]), i32([3]))
        att = BlockAttention(cache, heads, 1, 1, 1, rope=rope)
        att.begin(i32([0, 1]))
        q_out, out, k_out, v_out, turned = new(heads), new(heads), new(kv), new(kv), new(heads)
        att.append(0, k, v, q, q_out)
        att.plan()
        att.attend(0, q_out, out)
        cache.read(0, i32([0, 1]), k_out, v_out)
        rope.apply(q, i32([7]), turned)
        got.append((cache.k, cache.v, q_out, out, att.attend(0, q_out), k_out, v_out, turned))
    assert all(bool((x != 0).any()) and torch.equal(x, y) for x, y in zip(*got))
