"""CPU checks of caches of few bits: the plain definition by hand, sizes, the
Python objects' arrays, and refusals before anything is launched."""
import ctypes
import itertools
import math

import numpy as np
import pytest
import torch

import quant_ref as Q
from paper_2605_30876_amd import lib
from paper_2605_30876_amd.attention import BlockAttention, PagedCache

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="host-validation tests run without a GPU")

_HOST = np.zeros(1 << 16, dtype=np.float32)  # stands in for device memory, never dereferenced
BAD, NO = lib.DMOE_ERR_INVALID_ARG, lib.DMOE_ERR_UNSUPPORTED
FORMATS = ["fp8", "fp4", "fp8_fp4"]


@pytest.fixture(scope="module")
def L():
    return lib.load()


@pytest.fixture(scope="module")
def p():
    a = _HOST
    return a.ctypes.data + (-a.ctypes.data) % 16


def cache(p, **over):
    c = lib.dmoe_cache(p, p, p, p, p, lib.DMOE_BF16, 2, 10, 32, 2, 64, 4, 8, None, lib.DMOE_KV_FP4)
    for k, v in over.items():
        setattr(c, k, v)
    return c


def batch(p, **over):
    b = lib.dmoe_batch(p, None, 2, 16, 8)
    for k, v in over.items():
        setattr(b, k, v)
    return b


def status(L, name, *args):
    st = getattr(L, name)(*args)
    assert st == lib.DMOE_OK or L.dmoe_last_error().decode().startswith(name)
    return st


def test_the_reference_by_hand():
    """A group whose largest element is 7 keeps scale 1 and holds it as 6; one just above takes 2; ties go to the even code."""
    x = torch.zeros(3, 32)
    x[0, :8] = torch.tensor([7.0, 5.0, 2.5, -0.25, 0.75, 1.25, 3.5, -6.5])
    x[1, 0] = 7.0 + 2 ** -20
    x[2, 0], x[2, 1] = math.inf, 1.0
    codes, scales = Q.quantise(x, 4)
    assert scales[:, 0].tolist() == [127, 128, 255]
    held = Q.held(x, 4)
    assert held[0, :8].tolist() == [6.0, 4.0, 2.0, 0.0, 1.0, 1.0, 4.0, -6.0] and held[1, 0] == 8.0 and held[2].isnan().all()
    assert codes[0, 3] == 8 and codes[0, 8] == 0 and codes[1, 0] == 6
    x = torch.zeros(2, 32)
    x[0, :5] = torch.tensor([464.0, 1.0625, -1.1875, 2 ** -10, 3 * 2 ** -10])
    x[1, 0] = 465.0
    codes, scales = Q.quantise(x, 8)
    assert scales[:, 0].tolist() == [127, 128]
    assert Q.held(x, 8)[0, :5].tolist() == [448.0, 1.0, -1.25, 0.0, 2 ** -8] and Q.held(x, 8)[1, 0] == 480  # 232.5 lies above the middle of 224 and 240
    assert Q.scale_byte(0.0, 4) == 17 and Q.scale_byte(3.4e38, 4) == 252 and Q.scale_byte(3.4e38, 8) == 246
    assert all(Q.code(m, b) == i for b in (4, 8) for i, m in enumerate(Q.magnitudes(b)))


def test_places_are_apart():
    """Every byte of a page is one pair's or one code's, one scale's, or one of a row of scales that is not used."""
    for bits in (4, 8):
        for dim in (8, 64, 80, 136, 256):
            page, heads = 64, 3
            pos = torch.arange(2 * page)
            at, st = Q.places(bits, page, heads, dim, pos, pos // page)
            if bits == 4:
                assert (at[..., 0::2] == at[..., 1::2]).all()
                at = at[..., 0::2]
            used = torch.cat((at.reshape(-1), st.reshape(-1)))
            size = Q.page_bytes(bits, page, heads, dim)
            assert used.unique().numel() == used.numel() and int(used.max()) < 2 * size
            w, sb, tile = Q.layout(bits, dim)
            assert used.numel() == 2 * size - 2 * page * heads * (sb - Q.padded(dim) // 32)


def test_sizes():
    for name in FORMATS:
        f, (bk, bv) = lib.KV_FORMAT[name], Q.BITS[name]
        for dt in (lib.DMOE_BF16, lib.DMOE_F32):
            for dim in (8, 64, 80, 136, 256):
                assert lib.dmoe_cache_key_page_bytes(dt, f, 64, 3, dim) == Q.page_bytes(bk, 64, 3, dim)
                assert lib.dmoe_cache_value_page_bytes(dt, f, 64, 3, dim) == Q.page_bytes(bv, 64, 3, dim)
    for size in (lib.dmoe_cache_key_page_bytes, lib.dmoe_cache_value_page_bytes):
        assert size(lib.DMOE_BF16, 0, 64, 3, 80) == lib.dmoe_cache_page_bytes(lib.DMOE_BF16, 64, 3, 80)
        for bad in ((5, 1, 32, 1, 64), (1, 4, 32, 1, 64), (1, -1, 32, 1, 64), (1, 1, 31, 1, 64), (1, 1, 32, 0, 64), (1, 1, 32, 1, 63)):
            assert size(*bad) == 0


def test_read_refusals(L, p):
    def call(c=None, layer=0, b=None, starts=p, k=p, ks=128, v=p + (1 << 16), vs=128):
        return status(L, "dmoe_cache_read", cache(p) if c is None else c, layer, batch(p) if b is None else b, starts, k, ks, v, vs, None)

    for over in (dict(layer=-1), dict(layer=2), dict(k=None, v=None), dict(ks=64), dict(vs=130), dict(k=p + 8), dict(v=p + 2), dict(v=p),
                 dict(v=p + 16), dict(starts=p + 2), dict(c=cache(p, format=4)), dict(c=cache(p, format=-1)), dict(c=cache(p, k=None)),
                 dict(c=cache(p, head_dim=12)), dict(b=batch(p, q_offsets=None)), dict(b=batch(p, T=0)), dict(b=batch(p, n_seqs=5)),
                 dict(ks=1 << 32)):
        assert call(**over) == BAD, over
    assert call(b=batch(p, T=(1 << 26) + 1)) == NO and call(c=cache(p, n_slots=70000)) == NO


@pytest.mark.parametrize("name", ["dmoe_cache_append", "dmoe_attention_plan", "dmoe_attention", "dmoe_cache_copy_pages", "dmoe_cache_update", "dmoe_cache_compact"])
def test_unknown_formats_are_refused(L, p, name):
    rot = lib.dmoe_rotary(None, 0, 0, 1.0)
    for fmt in (-1, 4, 7):
        c = cache(p, format=fmt)
        args = {"dmoe_cache_append": [c, 0, batch(p), p, 128, p, 128, None, 0, None, 0, 0, rot, None],
                "dmoe_attention_plan": [c, batch(p), 4, 0, p, 1 << 40, None],
                "dmoe_attention": [c, 0, batch(p), 4, 0, p, 256, 1.0, p, 1 << 40, p + (1 << 17), 256, None, p, 1 << 40, None],
                "dmoe_cache_copy_pages": [c, p, 1, None], "dmoe_cache_update": [c, p, None, None, p, 1, None, p, 1 << 40, None],
                "dmoe_cache_compact": [c, p, p, None, p, 1 << 40, None]}[name]
        assert status(L, name, *args) == BAD and "format" in L.dmoe_last_error().decode()


def test_cache_objects():
    for name in FORMATS:
        bk, bv = Q.BITS[name]
        c = PagedCache(2, 3, 64, 2, 80, 1, 1, device="cpu", format=name)
        assert c.k.dtype == c.v.dtype == torch.uint8 and c.c.format == lib.KV_FORMAT[name] and c.format == name
        assert c.k.shape == (2, 3, Q.page_bytes(bk, 64, 2, 80)) and c.v.shape == (2, 3, Q.page_bytes(bv, 64, 2, 80))
        given = PagedCache(2, 3, 64, 2, 80, 1, 1, device="meta", format=name, k=c.k, v=c.v)
        assert given.k is c.k and given.device.type == "cpu"
    assert PagedCache(1, 2, 32, 1, 64, 1, 1, device="cpu").c.format == lib.DMOE_KV_PLAIN
    with pytest.raises(ValueError, match="format"):
        PagedCache(1, 2, 32, 1, 64, 1, 1, device="cpu", format="int4")
    for k in (torch.zeros(1, 2, 32 * 64, dtype=torch.bfloat16), torch.zeros(1, 2, 7, dtype=torch.uint8)):
        with pytest.raises(ValueError):
            PagedCache(1, 2, 32, 1, 64, 1, 1, device="cpu", format="fp4", k=k)


def test_read_objects():
    c = PagedCache(1, 2, 32, 1, 64, 2, 1, device="cpu", format="fp4")
    off, x = torch.tensor([0, 4], dtype=torch.int32), torch.zeros(4, 1, 64, dtype=torch.bfloat16)
    for bad in (dict(), dict(k=x.float()), dict(k=x[:, :, :32]), dict(k=x, v=x[:3]), dict(k=x, slots=off.long()), dict(k=x, starts=off[:0]),
                dict(k=x.transpose(0, 2).contiguous().transpose(0, 2))):
        with pytest.raises(ValueError):
            c.read(0, off, **bad)
    with pytest.raises(ValueError):
        c.read(0, off[:1], k=x)
    with pytest.raises(ValueError):
        c.read(0, off.long(), k=x)
    with pytest.raises(RuntimeError, match="gradient"):
        c.read(0, off, k=x.clone().requires_grad_(True))
    with pytest.raises(ValueError, match="GPU"):
        c.read(0, off, k=x)
    att = BlockAttention(c, 2, 1, 1, 1)
    att.begin(off)
    with pytest.raises(ValueError):  # rows are of the cache's dtype, not of its pages'
        att.append(0, x.to(torch.uint8), x)


@pytest.mark.parametrize("format", [lib.DMOE_KV_PLAIN, lib.DMOE_KV_FP8, lib.DMOE_KV_FP4, lib.DMOE_KV_FP8_FP4])
@pytest.mark.parametrize("dtype", [lib.DMOE_BF16, lib.DMOE_F32])
def test_sizes_told_are_the_sizes_needed(L, p, format, dtype):
    """What the size functions tell, which do not know a cache's format or capacity, is enough for the tiles that a batch is
    cut into, whatever they are.  (Nothing is launched: there is no GPU.)"""
    wrong = []
    for seqs, new, group, kv, dim, pages in itertools.product([1, 2, 40], [1, 8, 20, 32, 500], [1, 2, 3, 4, 16], [1, 2, 8], [64, 256], [8, 1 << 12]):
        T, heads = seqs * new, group * kv
        c, b = cache(p, format=format, dt=dtype, n_kv_heads=kv, head_dim=dim, n_slots=seqs, max_pages=pages), batch(p, n_seqs=seqs, T=T, max_new=new)
        ints = L.dmoe_attention_plan_ints(seqs, T, new, heads, kv)
        ws = L.dmoe_attention_workspace_size(dtype, seqs, T, new, heads, kv, dim)
        out = p + T * heads * dim * 4  # behind the queries
        got = [status(L, "dmoe_attention_plan", ctypes.byref(c), b, heads, 32, p, ints, None),
               status(L, "dmoe_attention", ctypes.byref(c), 0, b, heads, 32, p, heads * dim, 1.0, p, ints, out, heads * dim, None, p, ws, None)]
        wrong += [(seqs, new, group, kv, dim, pages, L.dmoe_last_error().decode())] if BAD in got or NO in got else []
    assert not wrong, wrong[:3]
