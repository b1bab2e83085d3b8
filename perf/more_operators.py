"""Operators on a key/value cache held in 8 or 4 bits, as cases that can be timed and compared: keys and values quantised as they
are written, read back, and attended to.

Kinds of case:
  store    the new tokens of every sequence: queries rotated, keys rotated and quantised into the cache, values quantised; then
           the same tokens read back as the cache holds them (what a chunk's own attention has to see for its result to be the
           one that later steps would give)
  read     tokens of every sequence read back: whole sequences, or windows of them (a prefix handed on, a cache moved)
  attend   attention of the new tokens over the cache, for ``layers`` layers that share one plan (a decode step plans once)

Common fields: dtype (of rows: queries, new keys and values, results); format: "plain" (the cache holds dtype), "fp8", "fp4", or
"fp8_fp4" (keys fp8, values fp4); heads, kv_heads, dim (per head); page (tokens per page); seqs; new (new tokens per sequence; of a
read: tokens of a window, 0: all); ctx (cached tokens in front of them; of a read: tokens of a sequence); ragged: "no", "len" (1 to
ctx cached tokens) or "all" (also 1 to new new ones); mask (0: every key of the sequence, 1: causal, n: blocks of n tokens see
each other and everything before); graph: captured once and replayed, as a decode loop does.  Lengths go by the case alone, values
by the seed.

Values in few bits.  32 consecutive elements of a token's head share a scale 2^(b - 127), b a byte; an element is an 8-bit float of
4 exponent and 3 fraction bits (largest 448) or a 4-bit one of 2 and 1 (0, 0.5, 1, 1.5, 2, 3, 4, 6).  b is the smallest, not below 17,
at which no element is off by more than half a step: the largest of them is at most 464 (7) times the scale; not above 246 (252),
so that every value fits bf16.  A group with an element that is not finite has b = 255 and is NaN.  A key is rotated in 64 bits and rounded
once to dtype before.  A page holds, per kv head and tile of 32 tokens (head dimension padded to dp), chunks of 16 bytes, 32 elements
(4 bits; element 2i in the low half of byte i) or 16 (8 bits), [chunk][32 tokens][16 bytes], then the scales, [32 tokens][sb], sb the least
power of two that holds dp/32.  A plain cache is that of `perf/operators.py`.
"""
import math
import random

import torch

own = False
DEV = "cuda"
FORMATS = {"plain": (0, 0), "fp8": (8, 8), "fp4": (4, 4), "fp8_fp4": (8, 4)}  # bits of keys and of values


def _case(name, kind, format="fp4", dtype="bf16", heads=16, kv_heads=4, dim=128, page=32, seqs=1, new=32, ragged="no", ctx=1024,
          mask=32, rot=64, inter=False, scaling="none", factor=1.0, layers=1, graph=False):
    return {"name": name, "kind": kind, "format": format, "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "page": page, "seqs": seqs, "new": new, "ragged": ragged, "ctx": ctx, "mask": mask, "rot": rot, "inter": inter,
            "scaling": scaling, "factor": factor, "layers": layers, "graph": graph}


def listed():
    return [
        # a decode step of one sequence: one block of 32 tokens into eight layers' caches, half of each head rotated
        _case("store_block_fp4_x8", "store", layers=8, graph=True),
        # prompts of several users, ragged, far behind the trained length; keys in 8 bits, values in 4
        _case("store_prompts_fp8_fp4", "store", "fp8_fp4", heads=32, kv_heads=8, seqs=6, new=4096, ragged="all", ctx=200000, rot=128,
              inter=True, scaling="yarn", factor=8.0),
        # full-precision rows, an odd head dimension, an odd number of rotated pairs
        _case("store_odd_f32_fp8", "store", "fp8", "f32", heads=12, kv_heads=6, dim=80, seqs=3, new=1000, ragged="all", ctx=3000, rot=50),
        # whole sequences handed on to something that reads rows
        _case("read_whole_fp4", "read", seqs=48, kv_heads=8, new=0, ragged="len", ctx=8192, page=64),
        # short windows of many sequences, some running past the end, of a cache that holds bf16
        _case("read_windows_plain", "read", "plain", seqs=40, kv_heads=4, dim=96, new=20, ragged="all", ctx=2000, layers=2),
        # the smallest call: full-precision rows, two short sequences, a few heads
        _case("attend_tiny_f32_fp4", "attend", dtype="f32", heads=4, kv_heads=4, dim=64, seqs=2, new=8, ctx=100, mask=8, graph=True),
        # a decode step of one sequence: one block of 32 tokens over 4096 cached ones, eight layers
        _case("attend_block_fp8_x8", "attend", "fp8", ctx=4096, layers=8, graph=True),
        # sixteen sequences decoded together, ragged; keys in 8 bits, values in 4
        _case("attend_block_b16_fp8_fp4", "attend", "fp8_fp4", seqs=16, ctx=8192, ragged="len"),
        # single tokens of 64 sequences, ragged: the cache is read once
        _case("attend_token_b64_fp4", "attend", heads=32, kv_heads=8, seqs=64, new=1, ctx=16384, ragged="len", mask=1, page=64),
        # one token over a long document, one sequence
        _case("attend_token_long_fp4", "attend", heads=32, kv_heads=8, new=1, ctx=131000, mask=1, page=128),
        # a prompt's last chunk over what is cached of it, block-causal: the compute-heavy end
        _case("attend_chunk_fp4", "attend", seqs=1, new=4096, ctx=12288),
        # full-precision rows, an odd head dimension, causal
        _case("attend_mid_f32_fp8", "attend", "fp8", "f32", heads=12, kv_heads=6, dim=80, seqs=4, new=100, ragged="all", ctx=2000, mask=1),
    ]


# ---- draws ------------------------------------------------------------------

def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    kv = rng.choice([1, 2, 3, 4, 8])
    heads = kv * rng.choice([1, 2, 4, 5, 8])
    dim = rng.choice([32, 64, 80, 96, 128, 128, 192, 256])
    kind = rng.choice(["store", "store", "read", "attend", "attend", "attend"])
    scaling = rng.choice(["none", "linear", "ntk", "yarn"])
    rot = max(4, rng.choice([dim, dim // 2, 2 * rng.randint(1, dim // 2)]))
    base = dict(dtype=dtype, format=rng.choice(["fp4", "fp4", "fp8", "fp8_fp4"]), heads=heads, kv_heads=kv, dim=dim,
                page=rng.choice([32, 32, 64, 128]), rot=rot, inter=rng.random() < 0.5, scaling=scaling,
                factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 32.0]), ragged=rng.choice(["no", "len", "all"]))
    while True:
        if kind == "store":
            seqs = _log_int(rng, 1, 64)
            c = _case("", kind, seqs=seqs, new=_log_int(rng, 1, 8192 // seqs), ctx=_log_int(rng, 1, 200000), **base)
            c["graph"] = seqs * c["new"] <= 256
            if seqs * c["new"] * (heads + 2 * kv) * dim <= 16384 * 48 * 128:
                break
        elif kind == "read":
            base["format"] = rng.choice(["plain", "fp8", "fp4", "fp8_fp4"])
            seqs, ctx = _log_int(rng, 1, 128), _log_int(rng, 1, 32768)
            c = _case("", kind, seqs=seqs, new=rng.choice([0, _log_int(rng, 1, ctx)]), ctx=ctx, **base)
            if seqs * ctx * kv * dim <= 3e8:
                break
        else:
            seqs, ctx = _log_int(rng, 1, 128), _log_int(rng, 1, 65536)
            new = rng.choice([1, 1, 8, 24, 32, 32, _log_int(rng, 1, 2048)])
            c = _case("", kind, seqs=seqs, new=new, ctx=ctx, mask=rng.choice([0, 1, 8, 32, 32]), **base)
            c["graph"] = seqs * new <= 64 and ctx <= 4096
            pairs = seqs * new * (ctx + new)
            # plain scores and their fp32 keys have to fit
            if (pairs * heads * dim <= (2e10 if dtype == "f32" else 1.2e11) and seqs * (ctx + new) * kv * dim <= 7e8
                    and pairs * heads <= 1.5e9):
                break
    del c["name"]
    return c


# ---- inputs -----------------------------------------------------------------

def _gen(seed, *key):
    g = torch.Generator(device=DEV)
    v = seed
    for x in key:
        v = (v * 1000003 + x + 12345) & 0x7FFFFFFFFFFF
    g.manual_seed(v)
    return g


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _dp(c):
    return next(d for d in (32, 64, 96, 128, 192, 256) if d >= c["dim"])


def _layout(c, bits):
    """Chunks of a tile, elements of a chunk, scale bytes of a token, bytes of a tile."""
    dp = _dp(c)
    n, w = dp * bits // 128, 128 // bits
    sb = 1
    while sb < dp // 32:
        sb *= 2
    return n, w, sb, n * 512 + 32 * sb


def _tables(c):
    """Values of the codes, and the scales, by byte."""
    small = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    wide = [math.ldexp(8 + x % 8, x // 8 - 10) if x >= 8 else math.ldexp(x, -9) for x in range(127)] + [math.nan]
    return {4: torch.tensor(small + [-x for x in small], device=DEV), 8: torch.tensor(wide + [-x for x in wide], device=DEV),
            "scale": torch.tensor([2.0 ** (b - 127) for b in range(255)] + [math.nan], device=DEV),
            "inverse": torch.tensor([2.0 ** (127 - b) for b in range(255)] + [0.0], device=DEV)}


def _quantise(t, x, bits):
    """x [..., dp] in 32 bits as bytes of codes [..., dp * bits / 8] and of scales [..., dp / 32]."""
    g = x.unflatten(-1, (-1, 32))
    top = g.abs().amax(-1)
    m, e = torch.frexp(top)
    b = e + torch.where(m > (0.875 if bits == 4 else 0.90625), 1, 0) + (124 if bits == 4 else 118)
    b = torch.where(top > 0, b.clamp(17, 252 if bits == 4 else 246), 17)
    b = torch.where(torch.isfinite(top), b, 255)
    y = torch.where((b < 255)[..., None], g.abs() * t["inverse"][b][..., None], 0.0)
    if bits == 4:
        step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
        y = (torch.round(y / step) * step).clamp(max=6.0)
        code = torch.where(y < 2, 2 * y, torch.where(y < 4, y + 2, y / 2 + 4)).int()
    else:
        step = t["scale"][(torch.frexp(y)[1] - 1).clamp(min=-6) + 124]
        y = (torch.round(y / step) * step).clamp(max=448.0)
        e = torch.frexp(y)[1] - 1
        code = torch.where(y < 2 ** -6, y * 512, (e + 7) * 8 + y * t["scale"][(130 - e.clamp(min=-6))] - 8).int()
    code = (code + torch.where(torch.signbit(g), 1 << (bits - 1), 0)).flatten(-2)
    if bits == 4:
        code = code[..., 0::2] + 16 * code[..., 1::2]
    return code.to(torch.uint8), b.to(torch.uint8)


def _values(t, codes, scales, bits):
    """What bytes of codes [..., dp * bits / 8] and of scales [..., dp / 32] stand for, in 32 bits."""
    i = codes.int()
    if bits == 4:
        i = torch.stack((i & 15, i >> 4), -1).flatten(-2)
    return (t[bits][i].unflatten(-1, (-1, 32)) * t["scale"][scales.int()][..., None]).flatten(-2)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _lengths(c):
    """New tokens and lengths (the new tokens included) of every sequence, and the first token read, by the case alone."""
    r = random.Random(str(sorted((k, v) for k, v in c.items() if k not in ("name", "graph"))))
    n, m, first = [], [], []
    for i in range(c["seqs"]):
        old = r.choice([_log_int(r, 1, c["ctx"]), r.randint(1, c["ctx"])]) if c["ragged"] != "no" else c["ctx"]
        if c["kind"] == "read":
            m.append(old)
            n.append(old if c["new"] == 0 else r.randint(1, c["new"]) if c["ragged"] == "all" else c["new"])
            first.append(0 if c["new"] == 0 else r.randint(0, old - 1))
        else:
            n.append(r.randint(1, c["new"]) if c["ragged"] == "all" else c["new"])
            m.append(n[-1] + old)
            first.append(old)
    if c["ragged"] == "all" and c["seqs"] > 2:
        n[1] = 0  # a sequence that waits
        first[1] = m[1] if c["kind"] != "read" else 0
    return n, m, first


def _pages(c, m, lows):
    """Page tables over a pool in random order, with pages from the one that holds token `low` on."""
    r = random.Random(len(m) * 1000 + sum(m))
    p = c["page"]
    held = [(a // p, -(-b // p)) for a, b in zip(lows, m)]
    total = sum(hi - lo for lo, hi in held)
    ids = list(range(total + 3))
    r.shuffle(ids)
    width = max(hi for _, hi in held) + 1
    rows, at = [], 0
    for lo, hi in held:
        rows.append([-1] * lo + ids[at:at + hi - lo] + [-1] * (width - hi))
        at += hi - lo
    slots = list(range(len(m) + 1))
    r.shuffle(slots)
    slots = slots[:len(m)]
    table, lens = [[-1] * width for _ in range(len(m) + 1)], [0] * (len(m) + 1)
    for s, row, b in zip(slots, rows, m):
        table[s], lens[s] = row, b
    return _ints(table), _ints(lens), _ints(slots), total + 3


def _pool(c, t, bits, pages, g, keys):
    """Pages of values as a model leaves them: normal, a key's channels of several sizes."""
    L, K, dp = c["layers"], c["kv_heads"], _dp(c)
    if bits == 0:
        return torch.empty((L, pages, K * c["page"] * dp), dtype=_dtype(c), device=DEV).normal_(generator=g)
    n, w, sb, size = _layout(c, bits)
    tiles = c["page"] // 32
    out = torch.zeros((L, pages, K, tiles, size), dtype=torch.uint8, device=DEV)
    std = torch.empty((K, 1, 1, dp), device=DEV).normal_(generator=g).mul_(0.5 if keys else 0.0).exp_()
    some = max(1, int(1.5e8 / (K * c["page"] * dp)))
    for l in range(L):
        for a in range(0, pages, some):
            x = torch.empty((min(some, pages - a), K, tiles, 32, dp), device=DEV).normal_(generator=g).mul_(std)
            x[..., c["dim"]:] = 0
            codes, scales = _quantise(t, x, bits)
            out[l, a:a + some, ..., :n * 512] = codes.unflatten(-1, (n, 16)).transpose(-3, -2).flatten(-3)
            out[l, a:a + some, ..., n * 512:].unflatten(-1, (32, sb))[..., :dp // 32] = scales
    return out.view(L, pages, -1)


def _graphed(s):
    """The pass as a HIP graph, captured after one run on a stream of its own."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _pass(s)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s["result"] = _pass(s)
    return g


def prepare(case, seed):
    c = dict(case)
    s = {"case": c, "graph": None, "tables": _tables(c)}
    g = _gen(seed, 1)
    n, m, first = _lengths(c)
    lows = first if c["kind"] == "store" else [0] * len(m)
    s["table"], s["lens"], s["slots"], pages = _pages(c, m, lows)
    off = [0]
    for a in n:
        off.append(off[-1] + a)
    s["off"], s["first"], s["used"], s["longest"], s["most"] = _ints(off), _ints(first), off[-1], max(m), max(max(n), 1)
    rows = off[-1] + (3 if c["ragged"] == "all" else 0)  # rows behind the last sequence stay as they are
    L, H, K, D = c["layers"], c["heads"], c["kv_heads"], c["dim"]
    bk, bv = FORMATS[c["format"]]
    if c["kind"] == "store":  # only what is written is read
        s["k"], s["v"] = (torch.zeros((L, pages, K * (c["page"] // 32) * _layout(c, b)[3]), dtype=torch.uint8, device=DEV) for b in (bk, bv))
    else:
        s["k"], s["v"] = (_pool(c, s["tables"], b, pages, g, b is bk) for b in (bk, bv))
    fill = lambda h, std: torch.empty((L, rows, h, D), dtype=_dtype(c), device=DEV).normal_(0.0, std, generator=g)  # noqa: E731
    if c["kind"] != "read":
        s["q"] = fill(H, 2.0)
        s["q_out"] = torch.zeros_like(s["q"])
    if c["kind"] == "store":
        std = torch.empty((K, D), device=DEV).normal_(generator=g).mul_(0.5).exp_().to(_dtype(c))
        s["k_new"], s["v_new"] = fill(K, 1.0) * std, fill(K, 1.0)
    if c["kind"] == "attend":
        s["lse"] = torch.zeros((L, rows, H), dtype=torch.float32, device=DEV)
    else:
        s["k_out"], s["v_out"] = (torch.zeros((L, rows, K, D), dtype=_dtype(c), device=DEV) for _ in range(2))
    if c["graph"]:
        s["graph"] = _graphed(s)
    return s


def run(state):
    if state["graph"] is not None:
        state["graph"].replay()
        return state["result"]
    return _pass(state)


def _pass(s):
    return (_OWN if own else _PLAIN)[s["case"]["kind"]](s)


# ---- the framework's calls --------------------------------------------------

def _cache(s):
    from paper_2605_30876_amd.attention import PagedCache

    c = s["case"]
    return PagedCache(c["layers"], s["k"].shape[1], c["page"], c["kv_heads"], c["dim"], s["table"].shape[0], s["table"].shape[1],
                      dtype=_dtype(c), device=DEV, k=s["k"], v=s["v"], table=s["table"], lens=s["lens"], format=c["format"])


def _attention(s):
    if "own" not in s:
        from paper_2605_30876_amd.attention import BlockAttention, Rope

        c = s["case"]
        rope = Rope(c["rot"], base=10000.0, interleaved=c["inter"], scaling=c["scaling"], factor=c["factor"], original=4096, device=DEV)
        s["own"] = BlockAttention(_cache(s), c["heads"], c["seqs"], s["most"], s["q"].shape[1], mask_block=c["mask"],
                                  rope=rope if c["kind"] == "store" else None)
    s["own"].begin(s["off"], s["slots"])
    return s["own"]


def _own_store(s):
    a = _attention(s)
    for l in range(s["case"]["layers"]):
        a.append(l, s["k_new"][l], s["v_new"][l], q=s["q"][l], q_out=s["q_out"][l])
        a.cache.read(l, s["off"], k=s["k_out"][l], v=s["v_out"][l], slots=s["slots"], max_tokens=s["most"])
    return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}


def _own_read(s):
    if "own" not in s:
        s["own"] = _cache(s)
    for l in range(s["case"]["layers"]):
        s["own"].read(l, s["off"], k=s["k_out"][l], v=s["v_out"][l], slots=s["slots"], starts=s["first"], max_tokens=s["most"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_attend(s):
    a = _attention(s)
    a.plan()
    for l in range(s["case"]["layers"]):
        a.attend(l, s["q"][l], out=s["q_out"][l], lse=s["lse"][l])
    return {"out": s["q_out"], "lse": s["lse"]}


_OWN = {"store": _own_store, "read": _own_read, "attend": _own_attend}


# ---- plain forms ------------------------------------------------------------

def _turns(c):
    """Turns per position of every pair, in 64 bits, and the factor of the rotated values (a 32-bit number)."""
    r, base, f, orig = c["rot"], 10000.0, c["factor"], 4096
    i = torch.arange(r // 2, dtype=torch.float64, device=DEV)
    if c["scaling"] == "ntk":
        base *= f ** (r / (r - 2)) if r > 2 else 1.0
    turns = base ** (-2.0 * i / r) / (2.0 * math.pi)
    if c["scaling"] == "linear":
        turns = turns / f
    if c["scaling"] != "yarn":
        return turns, 1.0
    lo, hi = (r * math.log(orig / (b * 2.0 * math.pi)) / (2.0 * math.log(base)) for b in (32.0, 1.0))
    lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), r - 1)
    if hi > lo:
        ramp = ((i - lo) / (hi - lo)).clamp(0.0, 1.0)
    else:  # every pair is slow, or every pair is fast
        ramp = torch.full_like(i, 1.0 if hi <= 0 else 0.0)
    return turns / f * ramp + turns * (1.0 - ramp), torch.tensor(0.1 * math.log(f) + 1.0).item()


def _rotate(c, x, pos):
    """x [T, heads, dim] with its first rot elements rotated, in x's precision; angles in 64 bits."""
    turns, scale = _turns(c)
    a = pos.double()[:, None] * turns
    a = (a - torch.floor(a)) * (2.0 * math.pi)
    cos, sin = (torch.cos(a) * scale).to(x.dtype)[:, None], (torch.sin(a) * scale).to(x.dtype)[:, None]
    r = c["rot"]
    x1, x2 = (x[..., 0:r:2], x[..., 1:r:2]) if c["inter"] else (x[..., :r // 2], x[..., r // 2:r])
    y1, y2 = x1 * cos - x2 * sin, x2 * cos + x1 * sin
    y = torch.stack((y1, y2), -1).flatten(-2) if c["inter"] else torch.cat((y1, y2), -1)
    return torch.cat((y, x[..., r:]), -1)


def _rows(s):
    """Sequence, cache slot and position of every row in use."""
    t = torch.arange(s["used"], device=DEV)
    seq = torch.searchsorted(s["off"].long(), t, right=True) - 1
    return seq, s["slots"].long()[seq], s["first"].long()[seq] + t - s["off"].long()[seq]


def _places(c, bits, page, pos):
    """Places in one layer's pool of tokens [T]: of their codes [T, kv_heads, bytes] and scales [T, kv_heads, dp / 32]."""
    n, _, sb, size = _layout(c, bits)
    hk, p = c["kv_heads"], c["page"]
    r = (pos % 32)[:, None, None]
    at = (page[:, None, None] * hk + torch.arange(hk, device=DEV)[None, :, None]) * (p // 32 * size) + (pos % p // 32)[:, None, None] * size
    i = torch.arange(n * 16, device=DEV)[None, None]
    return at + (i // 16 * 32 + r) * 16 + i % 16, at + n * 512 + r * sb + torch.arange(_dp(c) // 32, device=DEV)[None, None]


def _plain_places(c, page, pos, values):
    """Places in one layer's pool of a plain cache of the tokens' keys (or values): [T, kv_heads, dim]."""
    e, dp, hk, p = 4 if c["dtype"] == "f32" else 8, _dp(c), c["kv_heads"], c["page"]
    d = torch.arange(c["dim"], device=DEV)[None, None]
    r = (pos % 32)[:, None, None]
    at = (page[:, None, None] * hk + torch.arange(hk, device=DEV)[None, :, None]) * (p * dp) + (pos % p // 32)[:, None, None] * (32 * dp)
    if not values:
        return at + ((d // (2 * e) * 2 + d // e % 2) * 32 + r) * e + d % e
    return at + ((d // 32 * (16 // e) + r // (2 * e)) * 2 + r // 4 % 2) * 32 * e + d % 32 * e + r % (2 * e) // 8 * 4 + r % 4


def _fetch(s, which):
    """Every row in use as the cache holds it: [layers, T, kv_heads, dim]; 0 where its sequence has no such token."""
    c, bits = s["case"], FORMATS[s["case"]["format"]][which]
    _, slot, pos = _rows(s)
    has = pos < s["lens"].long()[slot]
    pos = torch.where(has, pos, 0)
    page, pool = s["table"].long()[slot, pos // c["page"]], s["kv"[which]].view(c["layers"], -1)
    if bits == 0:
        x = pool[:, _plain_places(c, page, pos, which == 1)]
    else:
        codes, scales = _places(c, bits, page, pos)
        x = _values(s["tables"], pool[:, codes], pool[:, scales], bits)[..., :c["dim"]]
    return torch.where(has[None, :, None, None], x, 0.0)


def _plain_read(s):
    for which, name in enumerate(("k_out", "v_out")):
        s[name][:, :s["used"]] = _fetch(s, which).to(s[name].dtype)
    return {"k": s["k_out"], "v": s["v_out"]}


def _plain_store(s):
    c = s["case"]
    _, slot, pos = _rows(s)
    u, L = s["used"], c["layers"]
    page = s["table"].long()[slot, pos // c["page"]]
    turn = lambda t, kind: _rotate(c, t[:, :u].transpose(0, 1).reshape(u, -1, c["dim"]).to(kind), pos).view(u, L, -1, c["dim"]).transpose(0, 1)  # noqa: E731
    s["q_out"][:, :u] = turn(s["q"], torch.float32).to(_dtype(c))
    # in 64 bits, so that a key next to the border of two codes takes the one it is nearer to
    for which, x in enumerate((turn(s["k_new"], torch.float64).to(_dtype(c)), s["v_new"][:, :u])):
        bits = FORMATS[c["format"]][which]
        codes_at, scales_at = _places(c, bits, page, pos)
        codes, scales = _quantise(s["tables"], torch.nn.functional.pad(x.float(), (0, _dp(c) - c["dim"])), bits)
        pool = s["kv"[which]].view(L, -1)
        pool[:, codes_at.view(-1)] = codes.reshape(L, -1)
        pool[:, scales_at.view(-1)] = scales.reshape(L, -1)
    return {"q": s["q_out"], **_plain_read(s)}


def _plain_attend(s):
    c = s["case"]
    n, hk, g, D, L, p = c["seqs"], c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"], c["layers"], c["page"]
    pages = -(-s["longest"] // p)
    tab = s["table"].long()[s["slots"].long(), :pages].clamp(min=0)
    J = pages * p
    kv = []
    for which, bits in enumerate(FORMATS[c["format"]]):
        # pages of every sequence, side by side, with tokens and elements in order: [L, n, hk, J, D]
        chunks, _, sb, size = _layout(c, bits)
        x = s["kv"[which]][:, tab].view(L, n, pages, hk, p // 32, size).transpose(2, 3)
        codes = x[..., :chunks * 512].unflatten(-1, (chunks, 32, 16)).transpose(-3, -2).flatten(-2)
        scales = x[..., chunks * 512:].unflatten(-1, (32, sb))[..., :_dp(c) // 32]
        kv.append(_values(s["tables"], codes, scales, bits)[..., :D].reshape(L, n, hk, J, D))
    k, v = kv
    lens, off, m = s["lens"].long()[s["slots"].long()], s["off"].long(), s["most"]
    i = torch.arange(m, device=DEV)[None]
    new = off[1:] - off[:-1]
    q = s["q"][:, (off[:-1, None] + i).clamp(max=s["q"].shape[1] - 1)].float()
    q = q.view(L, n, m, hk, g, D).permute(0, 1, 3, 2, 4, 5).reshape(L, n, hk, m * g, D)
    pos = (lens - new)[:, None] + i
    end = lens[:, None].expand(n, m)
    if c["mask"]:
        end = torch.minimum(end, (pos // c["mask"] + 1) * c["mask"])
    end = torch.where(pos < 0, 0, end)[:, None, :, None].expand(n, hk, m, g).reshape(n, hk, m * g, 1)
    out = (torch.arange(J, device=DEV) >= end)[None]
    x = torch.matmul(q, k.transpose(-1, -2)).mul_(1.0 / math.sqrt(D)).masked_fill_(out, -math.inf)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x, v) / torch.where(total > 0, total, 1.0)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)
    o = o.view(L, n, hk, m, g, D).permute(0, 1, 3, 2, 4, 5).reshape(L, n, m, hk * g, D)
    lse = lse.view(L, n, hk, m, g).permute(0, 1, 3, 2, 4).reshape(L, n, m, hk * g)
    seq, _, _ = _rows(s)
    t = torch.arange(s["used"], device=DEV) - off[seq]
    s["q_out"][:, :s["used"]] = o[:, seq, t].to(_dtype(c))
    s["lse"][:, :s["used"]] = lse[:, seq, t]
    return {"out": s["q_out"], "lse": s["lse"]}


_PLAIN = {"store": _plain_store, "read": _plain_read, "attend": _plain_attend}


# ---- the definitions in 64 bits ---------------------------------------------

def _angles(c, pos):
    """cos and sin [T, rot/2] times the scale, from the powers themselves."""
    r, f = c["rot"], c["factor"]
    base = 10000.0 * f ** (r / (r - 2.0)) if c["scaling"] == "ntk" and r > 2 else 10000.0
    inv = [1.0 / base ** (2.0 * i / r) for i in range(r // 2)]
    scale = 1.0
    if c["scaling"] == "linear":
        inv = [x / f for x in inv]
    elif c["scaling"] == "yarn":
        edge = [r * math.log(4096.0 / (2.0 * math.pi * b)) / (2.0 * math.log(base)) for b in (32.0, 1.0)]
        a, b = float(max(0, math.floor(edge[0]))), float(min(r - 1, math.ceil(edge[1])))
        slow = lambda i: min(1.0, max(0.0, (i - a) / (b - a))) if b > a else float(b <= 0.0)  # noqa: E731
        inv = [x * (1.0 - slow(i)) + x / f * slow(i) for i, x in enumerate(inv)]
        scale = torch.tensor(1.0 + 0.1 * math.log(f), dtype=torch.float32).double().item()
    a = pos.double()[:, None] * torch.tensor(inv, dtype=torch.float64, device=DEV)
    return torch.cos(a) * scale, torch.sin(a) * scale


def _exact_rotate(c, x, pos):
    cos, sin = _angles(c, pos)
    y = x.double().clone()
    for i in range(c["rot"] // 2):
        a, b = (2 * i, 2 * i + 1) if c["inter"] else (i, i + c["rot"] // 2)
        u, w = x[..., a].double(), x[..., b].double()
        y[..., a] = u * cos[:, i, None] - w * sin[:, i, None]
        y[..., b] = w * cos[:, i, None] + u * sin[:, i, None]
    return y


def _magnitudes(bits):
    """What a code without its sign stands for, in order."""
    if bits == 4:
        return [0.0, 0.5] + [(1 + f / 2) * 2.0 ** e for e in range(3) for f in range(2)]
    return [f / 8 * 2.0 ** -6 for f in range(8)] + [(1 + f / 8) * 2.0 ** e for e in range(-6, 9) for f in range(8)][:-1]


def _nearest(x, bits):
    """x [..., dim] in 64 bits as the nearest values that a cache holds, 32 elements to a scale."""
    dim = x.shape[-1]
    x = torch.nn.functional.pad(x, (0, -dim % 32)).unflatten(-1, (-1, 32))
    most, lim, high = (6.0, 7.0, 125.0) if bits == 4 else (448.0, 464.0, 119.0)
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top.clamp(min=1e-300) / lim))
    e = torch.where(torch.ldexp(torch.full_like(top, lim), e - 1) >= top, e - 1, e)  # the logarithm is rounded
    e = torch.where(torch.ldexp(torch.full_like(top, lim), e) < top, e + 1, e).clamp(-110.0, high)
    y = torch.ldexp(x.abs(), -e)
    table = torch.tensor(_magnitudes(bits), dtype=torch.float64, device=x.device)
    between = (table[1:] + table[:-1]) / 2
    i = torch.searchsorted(between, y.contiguous())  # a value between two codes: the lower one here
    odd = (i % 2 == 1) & (y == between[i.clamp(max=between.numel() - 1)])
    y = table[torch.where(odd, i + 1, i).clamp(max=table.numel() - 1)].clamp(max=most)
    return torch.copysign(torch.ldexp(y, e), x).flatten(-2)[..., :dim]


def _opened(s, which, layer):
    """A layer's pool as values in 64 bits: [pages, page tokens, kv_heads, dim]."""
    c, pool = s["case"], s["kv"[which]][layer]
    bits, P, K, tiles, dp = FORMATS[c["format"]][which], pool.shape[0], c["kv_heads"], c["page"] // 32, _dp(c)
    x = torch.zeros((P, K, tiles, 32, dp), dtype=torch.float64, device=DEV)
    if bits == 0:
        e = 4 if c["dtype"] == "f32" else 8
        pool = pool.view(P, K, tiles, 32 * dp)
        for r in range(32):
            for d in range(dp):
                if which == 0:
                    at = ((d // (2 * e) * 2 + d % (2 * e) // e) * 32 + r) * e + d % e
                else:
                    u = r % (2 * e)
                    at = d // 32 * 1024 + r // (2 * e) * (64 * e) + u % 8 // 4 * (32 * e) + d % 32 * e + u // 8 * 4 + u % 4
                x[:, :, :, r, d] = pool[..., at].double()
    else:
        pool = pool.view(P, K, tiles, -1)
        per = 128 // bits
        n = dp // per
        sign = [1.0, -1.0]
        table = torch.tensor([z * v for z in sign for v in (_magnitudes(bits) + [math.nan] * (bits // 8))], dtype=torch.float64, device=DEV)
        sb = (pool.shape[-1] - n * 512) // 32
        for d in range(dp):
            where = torch.arange(32, device=DEV) * 16 + d // per * 512 + d % per * bits // 8
            code = pool[..., where].long()
            if bits == 4:
                code = code >> 4 if d % 2 else code % 16
            power = pool[..., n * 512 + torch.arange(32, device=DEV) * sb + d // 32].double() - 127
            x[..., d] = torch.ldexp(table[code], power)
    return x[..., :c["dim"]].permute(0, 2, 3, 1, 4).reshape(P, c["page"], K, c["dim"])


def exact(case, seed):
    c = {**case, "graph": False}
    s = prepare(c, seed)
    L = c["layers"]
    off, slots, lens, first = (s[x].tolist() for x in ("off", "slots", "lens", "first"))
    bits = FORMATS[c["format"]]
    parts = [(a, b, slot, f) for a, b, slot, f in zip(off[:-1], off[1:], slots, first) if b > a]
    if c["kind"] == "store":
        q, k, v = (s[x].double() for x in ("q_out", "k_out", "v_out"))
        for a, b, slot, f in parts:
            pos = torch.arange(f, f + b - a, device=DEV)
            for l in range(L):
                q[l, a:b] = _exact_rotate(c, s["q"][l, a:b], pos)
                k[l, a:b] = _nearest(_exact_rotate(c, s["k_new"][l, a:b], pos).to(_dtype(c)).double(), bits[0])
                v[l, a:b] = _nearest(s["v_new"][l, a:b].double(), bits[1])
        return {"q": q, "k": k, "v": v}
    if c["kind"] == "read":
        out = []
        for which, name in enumerate(("k_out", "v_out")):
            x = s[name].double()
            for l in range(L):
                pool = _opened(s, which, l)
                for a, b, slot, f in parts:
                    m = min(b - a, lens[slot] - f)
                    t = torch.arange(f, f + m, device=DEV)
                    x[l, a:b] = 0
                    x[l, a:a + m] = pool[s["table"][slot].long()[t // c["page"]], t % c["page"]]
            out.append(x)
        return {"k": out[0], "v": out[1]}
    g, D = c["heads"] // c["kv_heads"], c["dim"]
    out, lse = s["q_out"].double(), s["lse"].double()
    for l in range(L):
        ks, vs = _opened(s, 0, l), _opened(s, 1, l)
        for a, b, slot, _ in parts:
            m = lens[slot]
            pos = torch.arange(m - (b - a), m, device=DEV)[:, None]
            j = torch.arange(m, device=DEV)
            page, at = s["table"][slot].long()[j // c["page"]], j % c["page"]
            see = (pos >= 0) & ((j // c["mask"] <= pos // c["mask"]) if c["mask"] else (j >= 0))
            for h in range(c["heads"]):
                k, v = ks[page, at, h // g], vs[page, at, h // g]
                z = (s["q"][l, a:b, h].double() @ k.t() / math.sqrt(D)).masked_fill(~see, -math.inf)
                lse[l, a:b, h] = torch.logsumexp(z, -1)
                out[l, a:b, h] = torch.nan_to_num(torch.softmax(z, -1)) @ v
    return {"out": out, "lse": lse}


def work(case):
    c = case
    b = 4 if c["dtype"] == "f32" else 2
    H, K, D, L = c["heads"], c["kv_heads"], c["dim"], c["layers"]
    # bytes of a token's head in the cache, keys and values together
    held = sum(D * x / 8 + -(-D // 32) if x else D * b for x in FORMATS[c["format"]])
    n, m, first = _lengths(c)
    t = sum(n)
    if c["kind"] == "store":  # rows in, queries out, codes out and in again, rows out
        return {"bytes": L * t * (2.0 * H * D * b + 4.0 * K * D * b + 2.0 * K * held), "flops": L * 3.0 * t * (H + K) * c["rot"]}
    if c["kind"] == "read":
        there = sum(max(0, min(x, y - f)) for x, y, f in zip(n, m, first))
        return {"bytes": L * K * (there * held + t * 2.0 * D * b), "flops": 0.0}
    pairs, keys = 0, 0
    for x, y in zip(n, m):
        w = c["mask"] or y
        ends = [min(y, (i // w + 1) * w) for i in range(y - x, y)]
        pairs += sum(ends)
        keys += max(ends, default=0)
    return {"bytes": L * (keys * K * held + t * H * (2.0 * D * b + 4)), "flops": L * 4.0 * pairs * H * D}
