"""CPU checks of the attention section of the C ABI: sizes, the rotation's
frequencies, and the refusal of invalid arguments on the host before anything
is launched."""
import math

import numpy as np
import pytest
import torch

import attention_ref as R
from paper_2605_30876_amd import lib
from paper_2605_30876_amd.attention import BlockAttention, PagedCache

# These calls pass host addresses as "device" pointers; validation must reject
# them before any launch.  Never run them where a GPU could execute a launch.
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="host-validation tests run without a GPU")

_HOST = np.zeros(1 << 16, dtype=np.float32)  # stands in for device memory, never dereferenced
BAD, NO = lib.DMOE_ERR_INVALID_ARG, lib.DMOE_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def L():
    return lib.load()


@pytest.fixture(scope="module")
def p():
    a = _HOST
    return a.ctypes.data + (-a.ctypes.data) % 16


def cache(p, **over):
    c = lib.dmoe_cache(p, p, p, p, p, lib.DMOE_BF16, 2, 10, 32, 2, 64, 4, 8)
    for k, v in over.items():
        setattr(c, k, v)
    return c


def status(L, name, *args):
    st = getattr(L, name)(*args)
    msg = L.dmoe_last_error().decode()
    assert st == lib.DMOE_OK or msg.startswith(name), msg
    return st


BAD_CACHES = [dict(k=None), dict(v=None), dict(table=None), dict(lens=None), dict(dt=7), dict(n_layers=0), dict(n_pages=0), dict(page_tokens=16),
              dict(page_tokens=48), dict(page_tokens=2048), dict(n_kv_heads=0), dict(n_kv_heads=257), dict(head_dim=0), dict(head_dim=12),
              dict(head_dim=264), dict(n_slots=0), dict(max_pages=0), dict(max_pages=1 << 27)]
BAD_BATCHES = [dict(q_offsets=None), dict(n_seqs=0), dict(T=0), dict(max_new=0), dict(n_seqs=5)]


def batch(p, **over):
    b = lib.dmoe_batch(p, None, 2, 16, 8)
    for k, v in over.items():
        setattr(b, k, v)
    return b


def calls(p):
    """name -> a call that is valid but for what `over` and the arguments change (never made as it is)."""
    rot = lib.dmoe_rotary(p, 64, 0, 1.0)
    big = 1 << 40
    return {
        "dmoe_cache_append": lambda c, b, **o: [c, o.get("layer", 0), b, o.get("k", p), o.get("ks", 128), o.get("v", p), o.get("vs", 128),
                                                o.get("q", p), o.get("qs", 256), o.get("q_out", p), o.get("os", 256), o.get("heads", 4),
                                                o.get("rope", rot), None],
        "dmoe_attention_plan": lambda c, b, **o: [c, b, o.get("heads", 4), o.get("mask", 0), o.get("plan", p), o.get("ints", big), None],
        "dmoe_attention": lambda c, b, **o: [c, o.get("layer", 0), b, o.get("heads", 4), o.get("mask", 0), o.get("q", p), o.get("qs", 256),
                                             o.get("scale", 1.0), o.get("plan", p), o.get("ints", big), o.get("out", p + (1 << 17)), o.get("os", 256),
                                             o.get("lse"), o.get("ws", p), o.get("ws_bytes", big), None],
    }


@pytest.mark.parametrize("name", ["dmoe_cache_append", "dmoe_attention_plan", "dmoe_attention"])
def test_caches_and_batches(L, p, name):
    f = calls(p)[name]
    assert status(L, name, *f(None, batch(p))) == BAD
    for over in BAD_CACHES:
        assert status(L, name, *f(cache(p, **over), batch(p))) == BAD, over
    assert status(L, name, *f(cache(p, n_slots=70000), batch(p))) == NO
    for over in BAD_BATCHES:
        assert status(L, name, *f(cache(p), batch(p, **over))) == BAD, over
    assert status(L, name, *f(cache(p), batch(p, slots=p, n_seqs=5000))) == NO
    assert status(L, name, *f(cache(p), batch(p, T=(1 << 26) + 1))) == NO
    assert status(L, name, *f(cache(p), batch(p, T=1 << 26), heads=32, qs=2048, os=2048)) == NO
    assert status(L, name, *f(cache(p), batch(p), heads=3)) == BAD
    assert status(L, name, *f(cache(p), batch(p), heads=0)) == BAD
    assert status(L, name, *f(cache(p), batch(p), heads=2 * 1025, qs=2 * 1025 * 64, os=2 * 1025 * 64)) == NO


def test_append_refusals(L, p):
    name, f = "dmoe_cache_append", calls(p)["dmoe_cache_append"]
    rot = lambda **o: lib.dmoe_rotary(o.get("turns", p), o.get("rot", 64), 0, o.get("scale", 1.0))  # noqa: E731
    for over in (dict(layer=-1), dict(layer=2), dict(k=None), dict(v=None), dict(k=p + 2), dict(ks=64), dict(ks=130), dict(vs=0), dict(q=None),
                 dict(q_out=None), dict(qs=192), dict(os=260), dict(q_out=p + 8), dict(q_out=p + 16), dict(os=512), dict(ks=1 << 32),
                 dict(rope=rot(rot=3)), dict(rope=rot(rot=0)), dict(rope=rot(rot=66)), dict(rope=rot(scale=math.inf)), dict(rope=rot(turns=p + 4))):
        assert status(L, name, *f(cache(p), batch(p), **over)) == BAD, over


def test_attention_refusals(L, p):
    name, f = "dmoe_attention", calls(p)["dmoe_attention"]
    ints = lib.dmoe_attention_plan_ints(2, 16, 8, 4, 2)
    ws = lib.dmoe_attention_workspace_size(lib.DMOE_BF16, 2, 16, 8, 4, 2, 64)
    for over in (dict(layer=2), dict(q=None), dict(out=None), dict(plan=None), dict(ws=None), dict(mask=-1), dict(scale=0.0), dict(scale=-1.0),
                 dict(scale=math.nan), dict(scale=math.inf), dict(qs=250), dict(os=8), dict(out=p), dict(out=p + 64), dict(lse=p + 2), dict(plan=p + 8),
                 dict(ws=p + 8), dict(ints=ints - 1), dict(ws_bytes=ws - 1)):
        assert status(L, name, *f(cache(p), batch(p), **over)) == BAD, over
    name, f = "dmoe_attention_plan", calls(p)["dmoe_attention_plan"]
    for over in (dict(plan=None), dict(plan=p + 8), dict(mask=-1), dict(ints=ints - 1)):
        assert status(L, name, *f(cache(p), batch(p), **over)) == BAD, over


def test_rope_refusals(L, p):
    rot = lib.dmoe_rotary(p, 64, 0, 1.0)

    def call(x=p, xs=256, out=p, os=256, dt=lib.DMOE_BF16, T=4, heads=4, dim=64, pos=p, rope=rot):
        return status(L, "dmoe_rope", x, xs, out, os, dt, T, heads, dim, pos, rope, 0, None)

    for over in (dict(x=None), dict(out=None), dict(pos=None), dict(rope=lib.dmoe_rotary(None, 64, 0, 1.0)), dict(dt=3), dict(T=0), dict(heads=0),
                 dict(dim=60), dict(dim=512), dict(xs=128), dict(xs=257), dict(os=512), dict(out=p + 32), dict(x=p + 8), dict(pos=p + 1),
                 dict(rope=lib.dmoe_rotary(p, 128, 0, 1.0)), dict(rope=lib.dmoe_rotary(p, 5, 0, 1.0))):
        assert call(**over) == BAD, over
    assert call(T=(1 << 26) + 1) == NO and call(heads=65536, xs=1 << 23, os=1 << 23) == NO


def test_page_refusals(L, p):
    ws = lib.dmoe_cache_update_workspace_size(3, 8, 10)

    def update(c=None, dst=p, src=p, keep=p, lens=p, n=3, st=p, w=p, nbytes=ws):
        return status(L, "dmoe_cache_update", cache(p) if c is None else c, dst, src, keep, lens, n, st, w, nbytes, None)

    for over in (dict(c=cache(p, refs=None)), dict(dst=None), dict(lens=None), dict(n=0), dict(w=None), dict(w=p + 4), dict(nbytes=ws - 1),
                 dict(dst=p + 1), dict(src=p + 2), dict(st=p + 3)):
        assert update(**over) == BAD, over
    assert update(n=4097, nbytes=1 << 40) == NO
    assert update(c=cache(p, max_pages=1 << 22), n=4096, nbytes=1 << 60) == BAD
    cw = lib.dmoe_cache_compact_workspace_size(10)

    def compact(c=None, t=p, r=p, n=p, w=p, nbytes=cw):
        return status(L, "dmoe_cache_compact", cache(p) if c is None else c, t, r, n, w, nbytes, None)

    for over in (dict(c=cache(p, refs=None)), dict(t=None), dict(r=None), dict(w=None), dict(nbytes=cw - 1), dict(t=p + 4), dict(r=p + 4)):
        assert compact(**over) == BAD, over
    for args in ((cache(p, k=None), p, 1), (cache(p), None, 1), (cache(p), p, 0), (cache(p), p + 2, 1)):
        assert status(L, "dmoe_cache_copy_pages", *args, None) == BAD


def test_sizes():
    for dt, e in ((lib.DMOE_BF16, 2), (lib.DMOE_F32, 4)):
        for dim in (8, 64, 80, 136, 256):
            assert lib.dmoe_cache_page_bytes(dt, 64, 3, dim) == 64 * 3 * R.padded(dim) * e
    for bad in ((5, 32, 1, 64), (1, 31, 1, 64), (1, 32, 0, 64), (1, 32, 1, 63)):
        assert lib.dmoe_cache_page_bytes(*bad) == 0
    assert lib.dmoe_attention_plan_ints(0, 1, 1, 4, 2) == 0 and lib.dmoe_attention_plan_ints(1, 1, 1, 3, 2) == 0
    assert lib.dmoe_attention_plan_ints(5000, 1, 1, 4, 2) == 0 and lib.dmoe_attention_plan_ints(1, 1 << 30, 1, 4, 2) == 0
    assert lib.dmoe_attention_workspace_size(lib.DMOE_BF16, 1, 1, 1, 4, 2, 63) == 0
    assert lib.dmoe_cache_update_workspace_size(0, 1, 1) == 0 and lib.dmoe_cache_compact_workspace_size(0) == 0
    # the plan holds an item per row tile and what splitting may add, whatever the batch
    small, large = (lib.dmoe_attention_plan_ints(n, 4096, 4096 // n, 16, 4) for n in (1, 64))
    assert 0 < small <= large


@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("linear", 2.0), ("ntk", 8.0), ("yarn", 4.0), ("yarn", 1.0)])
@pytest.mark.parametrize("rot,base", [(2, 10000.0), (6, 500000.0), (64, 10000.0), (128, 1e6), (254, 10000.0)])
def test_turns(rot, base, scaling, factor):
    got, scale = lib.dmoe_rope_turns(rot, base, scaling, factor, 4096)
    want, ws = R.turns(rot, base, scaling, factor, 4096)
    assert len(got) == rot // 2 and abs(scale - ws) < 1e-6
    assert all(abs(a - b) <= 1e-14 * abs(b) for a, b in zip(got, want))
    assert got == sorted(got, reverse=True)


def test_turns_by_hand():
    """rot 4, base 10000: one radian and a hundredth per position."""
    got, scale = lib.dmoe_rope_turns(4, 10000.0, "none", 1.0, 0)
    assert scale == 1.0 and abs(got[0] * 2 * math.pi - 1.0) < 1e-15 and abs(got[1] * 2 * math.pi - 0.01) < 1e-16


def test_turns_refusals():
    for args in ((3, 1e4, "none", 1.0, 0), (0, 1e4, "none", 1.0, 0), (4, 1.0, "none", 1.0, 0), (4, math.nan, "none", 1.0, 0), (4, 1e4, "none", 2.0, 0),
                 (4, 1e4, "linear", 0.5, 0), (4, 1e4, "yarn", 2.0, 0), (4, 1e4, "linear", math.inf, 0)):
        with pytest.raises(lib.DmoeError):
            lib.dmoe_rope_turns(*args)


def test_cache_object_refuses_wrong_arrays():
    with pytest.raises(ValueError):
        PagedCache(1, 2, 48, 1, 64, 1, 1, device="cpu")
    with pytest.raises(TypeError):
        PagedCache(1, 2, 32, 1, 64, 1, 1, dtype=torch.float16, device="cpu")
    with pytest.raises(ValueError):
        PagedCache(1, 2, 32, 1, 64, 1, 1, device="cpu", k=torch.zeros(1, 2, 7, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        PagedCache(1, 2, 32, 1, 64, 1, 1, device="cpu", table=torch.zeros(1, 1, dtype=torch.int64))
    c = PagedCache(1, 2, 32, 1, 64, 1, 1, device="cpu")
    one = torch.zeros(1, dtype=torch.int32)
    for call in (lambda: c.resize(one, one), c.compact, lambda: c.copy_pages(one.expand(1, 2).contiguous())):
        with pytest.raises(ValueError, match="GPU"):
            call()
    att = BlockAttention(c, 2, 1, 1, 1)
    att.begin(torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="GPU"):
        att.plan()
    assert c.c.n_pages == 2 and c.table.tolist() == [[-1]] and c.k.shape == (1, 2, 32 * 64)


def test_the_reference_bookkeeping_by_hand():
    """Two sequences share a prefix of one and a half pages; the second's half is a copy; compaction closes the hole."""
    m = R.Pages(8, 32, 3, 4)
    assert m.update([0], [48]) == (0, []) and m.table[0] == [0, 1, -1, -1]
    assert m.update([1], [70], [0], [48]) == (0, [(1, 2)]) and m.table[1] == [0, 2, 3, -1] and m.refs[:4] == [2, 1, 1, 1]
    assert m.update([0], [0]) == (0, []) and m.refs[:4] == [1, 0, 1, 1]
    assert m.compact() == (3, [(3, 1)]) and m.table[1] == [0, 2, 1, -1]
    assert m.update([2], [32 * 4], None, None) == (0, []) and m.update([0], [64]) == (1, [])


def test_the_reference_attention_by_hand():
    """Two keys with scores 0 and ln 3: weights 1/4 and 3/4; the row before them sees nothing."""
    q, k = torch.tensor([[[1.0, 0.0]], [[1.0, 0.0]]]), torch.tensor([[[0.0, 5.0]], [[math.log(3.0), 1.0]]])
    v = torch.tensor([[[4.0, 0.0]], [[0.0, 8.0]]])
    out, lse, _, _ = R.attention(q, k, v, R.ends([-1, 1], 2, 1), 1.0)
    assert torch.allclose(out[1, 0], torch.tensor([1.0, 6.0], dtype=torch.float64)) and abs(float(lse[1, 0]) - math.log(4.0)) < 1e-6
    assert (out[0] == 0).all() and float(lse[0, 0]) == -math.inf
    assert R.ends([0, 31, 32, 40], 41, 32).tolist() == [32, 32, 41, 41] and R.ends([3], 5, 0).tolist() == [5]


@pytest.mark.parametrize("rot", [2, 8, 64])
@pytest.mark.parametrize("base,original,slow", [(10000.0, 4.0, True), (1.5, 6.0, True), (10000.0, 6.2, True), (2.0, 4096.0, False), (1.1, 300.0, False),
                                                (10000.0, 1e30, False)])
def test_yarn_ramps_beyond_the_pairs(rot, base, original, slow):
    """All pairs slow (under one turn in `original` positions): all interpolated; all fast (over 32): all kept."""
    plain, _ = lib.dmoe_rope_turns(rot, base, "none", 1.0, 0)
    assert all(f * original < 1 if slow else f * original > 32 for f in plain)
    got, _ = lib.dmoe_rope_turns(rot, base, "yarn", 8.0, original)
    want = [f / 8 for f in plain] if slow else plain
    assert all(abs(a - b) <= 1e-15 * b for a, b in zip(got, want))


def test_scales_beyond_float32_are_refused(L, p):
    """The kernels' scores are in units of log 2: scale * log2(e) has to be a float32 too."""
    name, f = "dmoe_attention", calls(p)["dmoe_attention"]
    for scale in (3e38, 2.4e38):
        assert status(L, name, *f(cache(p), batch(p), scale=scale, ints=0)) == BAD and "scale" in L.dmoe_last_error().decode(), scale
    for scale in (2.3e38, 1e-40):  # what is refused then is the plan
        assert status(L, name, *f(cache(p), batch(p), scale=scale, ints=0)) == BAD and "plan" in L.dmoe_last_error().decode(), scale
