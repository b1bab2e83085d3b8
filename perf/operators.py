"""Operators of a decode step around its MoE layers, as cases that can be timed and compared: rotary positions, attention of
new tokens over a paged cache, and the pages of that cache.

Kinds of case:
  rope     positions rotated into one tensor of heads (queries or keys before they are cached, or a gradient: ``inverse``)
  append   the new tokens of every sequence: queries rotated, keys rotated and stored in the cache, values stored
  attend   attention of the new tokens over the cache, for ``layers`` layers that share one plan (a decode step plans once)
  update   hypotheses of a search: children released, forked again from their parents, everything grown by ``grow`` tokens
  compact  live pages of a fragmented pool moved together, tables rewritten

Common fields: dtype; heads, kv_heads, dim (per head); page (tokens per page); seqs; new (new tokens per sequence); ctx (cached
tokens in front of them); ragged: "no", "len" (1 to ctx cached tokens) or "all" (also 1 to new new ones); mask (0: every key of
the sequence, 1: causal, n: blocks of n tokens see each other and everything before); graph: captured once and replayed, as
a decode loop does.  Lengths go by the case alone, values by the seed.

The cache keeps keys and values in the order in which matrix instructions read them.  A page holds, per kv head and tile of
32 tokens, 16-byte chunks of c values (8 bf16, 4 fp32), the head dimension padded to dp:
  keys    [dp/2c][2][32 tokens][c]: token r, dimension 2c*s + c*h + e  at [s][h][r][e]
  values  [dp/32][16/c][2][32 dimensions][c/4][4]: token 2c*s + 8j + 4h + t, dimension 32*b + r  at [b][s][h][r][j][t]
"""
import math
import random

import torch

own = False
DEV = "cuda"


def _case(name, kind, dtype="bf16", heads=16, kv_heads=4, dim=128, page=32, seqs=1, new=32, ragged="no", ctx=1024, mask=32,
          rot=64, inter=False, scaling="none", factor=1.0, layers=1, graph=False, **more):
    return {"name": name, "kind": kind, "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page,
            "seqs": seqs, "new": new, "ragged": ragged, "ctx": ctx, "mask": mask, "rot": rot, "inter": inter,
            "scaling": scaling, "factor": factor, "layers": layers, "graph": graph, **more}


def listed():
    return [
        # a decode step of one sequence: one block of 32 tokens into eight layers' caches, half of each head rotated
        _case("append_block_b1_x8", "append", layers=8, graph=True),
        # prompts of several users, ragged, far behind the trained length
        _case("append_prompts_far", "append", heads=32, kv_heads=8, seqs=6, new=4096, ragged="all", ctx=200000, rot=128, inter=True,
              scaling="yarn", factor=8.0),
        # queries rotated alone, fp32, positions to a million (a gradient on its way back)
        _case("rope_far_f32_inverse", "rope", "f32", heads=12, kv_heads=12, dim=96, seqs=1, new=4096, ctx=1000000, rot=48, inter=True,
              scaling="linear", factor=4.0, inverse=True),
        # the smallest call: fp32, two short sequences, a few heads
        _case("attend_tiny_f32", "attend", "f32", heads=4, kv_heads=4, dim=64, seqs=2, new=8, ctx=100, mask=8, graph=True),
        # a decode step of one sequence: one block of 32 tokens over 4096 cached ones, eight layers
        _case("attend_block_b1_x8", "attend", ctx=4096, layers=8, graph=True),
        # sixteen sequences decoded together, ragged
        _case("attend_block_b16", "attend", seqs=16, ctx=8192, ragged="len"),
        # single tokens of 64 sequences, ragged: the cache is read once
        _case("attend_token_b64", "attend", heads=32, kv_heads=8, seqs=64, new=1, ctx=16384, ragged="len", mask=1, page=64),
        # one token over a long document, one sequence
        _case("attend_token_long_b1", "attend", heads=32, kv_heads=8, new=1, ctx=131000, mask=1, page=128),
        # a prompt's last chunk over what is cached of it, block-causal: the compute-heavy end
        _case("attend_chunk", "attend", seqs=1, new=4096, ctx=12288),
        # full precision, an odd head dimension, causal
        _case("attend_mid_f32", "attend", "f32", heads=12, kv_heads=6, dim=80, seqs=4, new=100, ragged="all", ctx=2000, mask=1),
        # a search over four hypotheses of eight prompts: fork, copy the partial pages of every layer, grow
        _case("update_beams", "update", seqs=8, width=4, ctx=2000, grow=32, layers=19, spare=1.0),
        # a fragmented pool brought together
        _case("compact_pool", "compact", seqs=64, ctx=900, layers=12, live=0.5),
    ]


# ---- draws ------------------------------------------------------------------

def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def _heads(rng):
    kv = rng.choice([1, 2, 3, 4, 8])
    return kv * rng.choice([1, 2, 4, 5, 8]), kv


def draw(rng):
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    heads, kv = _heads(rng)
    dim = rng.choice([32, 64, 80, 96, 128, 128, 192, 256])
    page = rng.choice([32, 32, 64, 128])
    kind = rng.choice(["rope", "append", "append", "attend", "attend", "attend", "attend", "update", "compact"])
    scaling = rng.choice(["none", "linear", "ntk", "yarn"])
    rot = rng.choice([dim, dim // 2, 2 * rng.randint(1, dim // 2)])
    base = dict(dtype=dtype, heads=heads, kv_heads=kv, dim=dim, page=page, rot=max(4, rot), inter=rng.random() < 0.5,
                scaling=scaling, factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 32.0]), ragged=rng.choice(["no", "len", "all"]))
    while True:
        if kind == "rope":
            c = _case("", kind, seqs=1, new=_log_int(rng, 1, 8192), ctx=_log_int(rng, 1, 1000000), inverse=rng.random() < 0.5, **base)
            if c["new"] * heads * dim <= 4096 * 32 * 128:
                break
        elif kind == "append":
            seqs = _log_int(rng, 1, 64)
            c = _case("", kind, seqs=seqs, new=_log_int(rng, 1, 8192 // seqs), ctx=_log_int(rng, 1, 200000), **base)
            c["graph"] = seqs * c["new"] <= 256
            if seqs * c["new"] * (heads + 2 * kv) * dim <= 16384 * 48 * 128:
                break
        elif kind == "attend":
            seqs, ctx = _log_int(rng, 1, 128), _log_int(rng, 1, 65536)
            new = rng.choice([1, 1, 8, 24, 32, 32, _log_int(rng, 1, 2048)])
            c = _case("", kind, seqs=seqs, new=new, ctx=ctx, mask=rng.choice([0, 1, 8, 32, 32]), **base)
            c["graph"] = seqs * new <= 64 and ctx <= 4096
            pairs = seqs * new * (ctx + new)
            # plain scores and their fp32 keys have to fit; fp32 products cost sixteen times bf16 ones
            if (pairs * heads * dim <= (2e10 if dtype == "f32" else 1.2e11) and seqs * (ctx + new) * kv * dim <= 7e8
                    and pairs * heads <= 1.5e9):
                break
        elif kind == "update":
            c = _case("", kind, seqs=_log_int(rng, 1, 32), width=rng.randint(2, 8), ctx=_log_int(rng, 30, 8000),
                      grow=rng.choice([1, 8, 32, 100]), layers=rng.choice([1, 4, 19]), spare=rng.choice([1.0, 1.0, 1.0, 0.2]), **base)
            if _update_pages(c)[1] * _page_elems(c) * c["layers"] <= 6e8:
                break
        else:
            c = _case("", kind, seqs=_log_int(rng, 1, 256), ctx=_log_int(rng, 30, 8000), layers=rng.choice([1, 4, 19]),
                      live=rng.choice([0.1, 0.3, 0.5, 0.9]), **base)
            if c["seqs"] * c["ctx"] / c["live"] * kv * _dp(c) * c["layers"] <= 6e8:
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


def _chunk(c):
    return 4 if c["dtype"] == "f32" else 8


def _dp(c):
    return next(d for d in (32, 64, 96, 128, 192, 256) if d >= c["dim"])


def _page_elems(c):
    return c["kv_heads"] * c["page"] * _dp(c)


def _normal(shape, std, c, g, mean=0.0):
    return torch.empty(shape, dtype=_dtype(c), device=DEV).normal_(mean, std, generator=g)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _lengths(c):
    """New tokens and lengths (the new tokens included) of every sequence, by the case alone."""
    r = random.Random(str(sorted((k, v) for k, v in c.items() if k not in ("name", "graph"))))
    n, m = [], []
    for i in range(c["seqs"]):
        n.append(r.randint(1, c["new"]) if c["ragged"] == "all" else c["new"])
        m.append(n[-1] + (r.choice([_log_int(r, 1, c["ctx"]), r.randint(1, c["ctx"])]) if c["ragged"] != "no" else c["ctx"]))
    if c["ragged"] == "all" and c["seqs"] > 2:
        n[1] = 0  # a sequence that waits
    return n, m


def _tables(c, n, m, whole):
    """Page tables over a pool in random order; without `whole` only the pages that the new tokens lie in."""
    r = random.Random(len(m) * 1000 + sum(m))
    p = c["page"]
    held = [(0 if whole else (b - a) // p, -(-b // p)) for a, b in zip(n, m)]
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


def _update_pages(c):
    """Pages of a parent, and of the pool: what the pass needs, times `spare`, and the parents'."""
    p, final = c["page"], c["ctx"] + c["grow"]
    parent = -(-c["ctx"] // p)
    need = c["width"] * (-(-final // p) - c["ctx"] // p)
    return parent, c["seqs"] * parent + max(1, int(c["seqs"] * need * min(1.0, c["spare"])) + 2)


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
    s = {"case": c, "graph": None}
    g = _gen(seed, 1)
    if c["kind"] == "rope":
        t = c["new"]
        s["x"] = _normal((t, c["heads"], c["dim"]), 1.0, c, g)
        s["pos"] = torch.randint(0, c["ctx"] + 1, (t,), generator=g, device=DEV, dtype=torch.int32)
        s["out"] = torch.zeros_like(s["x"])
        return s
    if c["kind"] in ("append", "attend"):
        n, m = _lengths(c)
        s["table"], s["lens"], s["slots"], pages = _tables(c, n, m, c["kind"] == "attend")
        off = [0]
        for a in n:
            off.append(off[-1] + a)
        s["off"], s["used"], s["longest"], s["most"] = _ints(off), off[-1], max(m), max(max(n), 1)
        rows = off[-1] + (3 if c["ragged"] == "all" else 0)  # rows behind the last sequence stay as they are
        L, H, K, D = c["layers"], c["heads"], c["kv_heads"], c["dim"]
        s["k"] = _normal((L, pages, _page_elems(c)), 1.0, c, g)
        s["v"] = _normal((L, pages, _page_elems(c)), 1.0, c, g)
        s["q"] = _normal((L, rows, H, D), 2.0, c, g)
        s["q_out"] = torch.zeros_like(s["q"])
        if c["kind"] == "append":
            s["k_new"] = _normal((L, rows, K, D), 1.0, c, g)
            s["v_new"] = _normal((L, rows, K, D), 1.0, c, g)
        else:
            s["lse"] = torch.zeros((L, rows, H), dtype=torch.float32, device=DEV)
    elif c["kind"] == "update":
        p, w, n = c["page"], c["width"], c["seqs"]
        parent, pages = _update_pages(c)
        width = -(-(c["ctx"] + c["grow"]) // p)
        ids = torch.randperm(pages, generator=g, device=DEV).int()
        s["table"] = torch.full((n * w, width), -1, dtype=torch.int32, device=DEV)
        s["table"][:n, :parent] = ids[:n * parent].view(n, parent)
        s["lens"] = _ints([c["ctx"]] * n + [0] * (n * (w - 1)))
        s["refs"] = torch.zeros((pages,), dtype=torch.int32, device=DEV)
        s["refs"][ids[:n * parent].long()] = 1
        s["all"], s["base"] = _ints(list(range(n * w))), s["lens"].clone()
        kids = n * (w - 1)
        s["kids"], s["parents"] = _ints(list(range(n, n * w))), _ints([i % n for i in range(kids)])
        s["keep"], s["grown"] = _ints([c["ctx"]] * kids), _ints([c["ctx"] + c["grow"]] * kids)
        s["first"], s["first_grown"] = _ints(list(range(n))), _ints([c["ctx"] + c["grow"]] * n)
        s["status"] = torch.zeros((3,), dtype=torch.int32, device=DEV)
        s["k"] = _normal((c["layers"], pages, _page_elems(c)), 1.0, c, g)
        s["v"] = _normal((c["layers"], pages, _page_elems(c)), 1.0, c, g)
    else:
        p, n = c["page"], c["seqs"]
        lens = _lengths({**c, "new": 1, "ragged": "len"})[1]
        held = [-(-b // p) for b in lens]
        pages = max(sum(held), int(sum(held) / c["live"]))
        ids = torch.randperm(pages, generator=g, device=DEV).int()
        width, at = max(held) + 1, [0]
        for h in held:
            at.append(at[-1] + h)
        j, h = torch.arange(width, device=DEV)[None], _ints(held).long()[:, None]
        # every fourth sequence starts with half the pages of the one before it
        row = torch.arange(n, device=DEV)[:, None].expand(n, width)
        take = torch.minimum(h, h.roll(1)) // 2
        row = torch.where((row % 4 == 3) & (j < take), row - 1, row)
        idx = (_ints(at[:-1]).long()[row] + j).clamp(max=pages - 1)
        s["table"] = torch.where(j < h, ids[idx], torch.tensor(-1, dtype=torch.int32, device=DEV)).contiguous()
        s["lens"] = _ints(lens)
        s["refs"] = torch.zeros((pages + 1,), dtype=torch.int32, device=DEV)
        s["refs"].index_add_(0, torch.where(j < h, s["table"], pages).view(-1).long(), torch.ones(n * width, dtype=torch.int32, device=DEV))
        s["refs"] = s["refs"][:pages].clone()
        s["table_out"], s["refs_out"] = torch.zeros_like(s["table"]), torch.zeros_like(s["refs"])
        s["counts"] = torch.zeros((2,), dtype=torch.int32, device=DEV)
        s["k"] = _normal((c["layers"], pages, _page_elems(c)), 1.0, c, g)
        s["v"] = _normal((c["layers"], pages, _page_elems(c)), 1.0, c, g)
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
                      dtype=_dtype(c), device=DEV, k=s["k"], v=s["v"], table=s["table"], lens=s["lens"], refs=s.get("refs"))


def _rope(c):
    from paper_2605_30876_amd.attention import Rope

    return Rope(c["rot"], base=10000.0, interleaved=c["inter"], scaling=c["scaling"], factor=c["factor"], original=4096, device=DEV)


def _own_rope(s):
    if "own" not in s:
        s["own"] = _rope(s["case"])
    s["own"].apply(s["x"], s["pos"], out=s["out"], inverse=s["case"]["inverse"])
    return {"out": s["out"]}


def _attention(s):
    if "own" not in s:
        from paper_2605_30876_amd.attention import BlockAttention

        c = s["case"]
        s["own"] = BlockAttention(_cache(s), c["heads"], c["seqs"], s["most"], s["q"].shape[1], mask_block=c["mask"],
                                  rope=_rope(c) if c["kind"] == "append" else None)
    s["own"].begin(s["off"], s["slots"])
    return s["own"]


def _own_append(s):
    a = _attention(s)
    for l in range(s["case"]["layers"]):
        a.append(l, s["k_new"][l], s["v_new"][l], q=s["q"][l], q_out=s["q_out"][l])
    return {"q": s["q_out"], "k": s["k"], "v": s["v"]}


def _own_attend(s):
    a = _attention(s)
    a.plan()
    for l in range(s["case"]["layers"]):
        a.attend(l, s["q"][l], out=s["q_out"][l], lse=s["lse"][l])
    return {"out": s["q_out"], "lse": s["lse"]}


def _own_update(s):
    if "own" not in s:
        s["own"] = _cache(s)
    a = s["own"]
    a.update(s["all"], s["base"], status=s["status"][0:1])
    a.update(s["kids"], s["grown"], src=s["parents"], keep=s["keep"], status=s["status"][1:2])
    a.update(s["first"], s["first_grown"], status=s["status"][2:3])
    return {n: s[n] for n in ("table", "lens", "refs", "status", "k", "v")}


def _own_compact(s):
    if "own" not in s:
        s["own"] = _cache(s)
    s["own"].compact(table_out=s["table_out"], refs_out=s["refs_out"], counts=s["counts"])
    return {n: s[n] for n in ("table_out", "refs_out", "counts", "k", "v")}


_OWN = {"rope": _own_rope, "append": _own_append, "attend": _own_attend, "update": _own_update, "compact": _own_compact}


# ---- plain forms ------------------------------------------------------------

def _turns(c):
    """Turns per position of every pair, in 64 bits, and the factor of the rotated values."""
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
    ramp = ((i - lo) / (hi - lo if hi != lo else 0.001)).clamp(0.0, 1.0)
    return turns / f * ramp + turns * (1.0 - ramp), 0.1 * math.log(f) + 1.0


def _rotate(c, x, pos, inverse=False):
    """x [T, heads, dim] in fp32 with its first rot elements rotated; angles in 64 bits."""
    turns, scale = _turns(c)
    a = pos.double()[:, None] * turns
    a = (a - torch.floor(a)) * (2.0 * math.pi)
    cos, sin = (torch.cos(a) * scale).float()[:, None], (torch.sin(a) * scale).float()[:, None]
    if inverse:
        sin = -sin
    r = c["rot"]
    x1, x2 = (x[..., 0:r:2], x[..., 1:r:2]) if c["inter"] else (x[..., :r // 2], x[..., r // 2:r])
    y1, y2 = x1 * cos - x2 * sin, x2 * cos + x1 * sin
    y = torch.stack((y1, y2), -1).flatten(-2) if c["inter"] else torch.cat((y1, y2), -1)
    return torch.cat((y, x[..., r:]), -1)


def _plain_rope(s):
    c = s["case"]
    s["out"].copy_(_rotate(c, s["x"].float(), s["pos"], c["inverse"]).to(_dtype(c)))
    return {"out": s["out"]}


def _rows(s):
    """Sequence, cache slot and position of every row in use."""
    t = torch.arange(s["used"], device=DEV)
    seq = torch.searchsorted(s["off"].long(), t, right=True) - 1
    slot = s["slots"].long()[seq]
    return seq, slot, s["lens"].long()[slot] - s["off"].long()[seq + 1] + t


def _places(c, page, pos):
    """Places in one layer's pools of the keys and values of tokens [T]: [T, kv_heads, dp] each."""
    e, dp, hk, p = _chunk(c), _dp(c), c["kv_heads"], c["page"]
    d = torch.arange(dp, device=DEV)[None, None]
    r, tile = (pos % 32)[:, None, None], (pos % p // 32)[:, None, None]
    at = (page[:, None, None] * hk + torch.arange(hk, device=DEV)[None, :, None]) * (p * dp) + tile * (32 * dp)
    k = at + ((d // (2 * e) * 2 + d // e % 2) * 32 + r) * e + d % e
    v = at + ((d // 32 * (16 // e) + r // (2 * e)) * 2 + r // 4 % 2) * 32 * e + d % 32 * e + r % (2 * e) // 8 * 4 + r % 4
    return k, v


def _plain_append(s):
    c = s["case"]
    _, slot, pos = _rows(s)
    k_at, v_at = _places(c, s["table"].long()[slot, pos // c["page"]], pos)
    u, layers = s["used"], c["layers"]
    turned = [t[:, :u].transpose(0, 1).reshape(u, -1, c["dim"]).float() for t in (s["q"], s["k_new"])]
    q, k = (_rotate(c, t, pos).view(u, layers, -1, c["dim"]).transpose(0, 1).to(_dtype(c)) for t in turned)
    s["q_out"][:, :u] = q
    pad = (0, _dp(c) - c["dim"])
    s["k"].view(layers, -1)[:, k_at.view(-1)] = torch.nn.functional.pad(k, pad).reshape(layers, -1)
    s["v"].view(layers, -1)[:, v_at.view(-1)] = torch.nn.functional.pad(s["v_new"][:, :u], pad).reshape(layers, -1)
    return {"q": s["q_out"], "k": s["k"], "v": s["v"]}


def _plain_attend(s):
    c = s["case"]
    n, hk, g, D, e, dp, L, p = c["seqs"], c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"], _chunk(c), _dp(c), c["layers"], c["page"]
    pages = -(-s["longest"] // p)
    tab = s["table"].long()[s["slots"].long(), :pages].clamp(min=0)
    J = pages * p
    # pages of every sequence, side by side, with tokens and dimensions in order: [L, n, hk, J, D]
    k = s["k"][:, tab].view(L, n, pages, hk, p // 32, dp // (2 * e), 2, 32, e).permute(0, 1, 3, 2, 4, 7, 5, 6, 8)
    k = k.reshape(L, n, hk, J, dp)[..., :D].float()
    v = s["v"][:, tab].view(L, n, pages, hk, p // 32, dp // 32, 16 // e, 2, 32, e // 4, 4).permute(0, 1, 3, 2, 4, 6, 9, 7, 10, 5, 8)
    v = v.reshape(L, n, hk, J, dp)[..., :D].float()
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


def _plain_step(s, dst, new_len, src, keep, status):
    """One update: dst <- the first keep tokens of src, then room for new_len tokens."""
    p, table, refs, lens = s["case"]["page"], s["table"], s["refs"], s["lens"]
    dst, src, new_len = dst.long(), dst.long() if src is None else src.long(), new_len.long()
    n, w = dst.numel(), table.shape[1]
    keep = torch.minimum(lens[src].long(), new_len) if keep is None else keep.long()
    j = torch.arange(w, device=DEV)[None]
    rows, old = table[src].long(), table[dst].long()
    full, count = (keep // p)[:, None], (-(-new_len // p))[:, None]
    part = keep % p > 0
    shared, had = j < full, j < -(-lens[dst].long() // p)[:, None]
    after = refs.clone()
    after.index_add_(0, rows.clamp(min=0).view(-1), shared.view(-1).int())
    after.index_add_(0, old.clamp(min=0).view(-1), -had.view(-1).int())
    mine = torch.where(part, rows.gather(1, full.clamp(max=w - 1))[:, 0], 0)
    own_part = part & (src == dst)
    same = (mine[:, None] == mine[None]) & own_part[None]
    kept = own_part & (after[mine] == 0) & ~(same & torch.ones_like(same).tril(-1)).any(1)
    copied = part & ~kept
    after.index_add_(0, mine, part.int())
    fresh = ((j == full) & copied[:, None]) | ((j >= full + part[:, None]) & (j < count))
    free = torch.sort((after != 0).int(), stable=True).indices
    lacking = (fresh.sum() - (after == 0).sum()).clamp(min=0)
    rank = fresh.view(-1).cumsum(0).view(n, w) - 1
    given = free[rank.clamp(0, free.numel() - 1)]
    row = torch.where(shared, rows, torch.where((j == full) & kept[:, None], mine[:, None], torch.where(fresh, given, -1)))
    after.index_add_(0, mine, -copied.int())
    after.index_add_(0, given.view(-1), fresh.view(-1).int())
    ok = lacking == 0
    table[dst] = torch.where(ok, row, old).int()
    lens[dst] = torch.where(ok, new_len, lens[dst].long()).int()
    refs.copy_(torch.where(ok, after, refs))
    status.copy_(lacking.view(1))
    pick = torch.nonzero(copied & ok)[:, 0]
    to, of = given.gather(1, full.clamp(max=w - 1))[pick, 0], mine[pick]
    s["k"][:, to] = s["k"][:, of]
    s["v"][:, to] = s["v"][:, of]


def _plain_update(s):
    _plain_step(s, s["all"], s["base"], None, None, s["status"][0:1])
    _plain_step(s, s["kids"], s["grown"], s["parents"], s["keep"], s["status"][1:2])
    _plain_step(s, s["first"], s["first_grown"], None, None, s["status"][2:3])
    return {n: s[n] for n in ("table", "lens", "refs", "status", "k", "v")}


def _plain_compact(s):
    live = s["refs"] > 0
    n = live.sum()
    ids = torch.arange(live.numel(), device=DEV)
    holes, movers = torch.nonzero(~live & (ids < n))[:, 0], torch.nonzero(live & (ids >= n))[:, 0]
    moved = ids.clone()
    moved[movers] = holes
    s["refs_out"].zero_()
    s["refs_out"][moved[live]] = s["refs"][live]
    s["table_out"].copy_(torch.where(s["table"] >= 0, moved[s["table"].long().clamp(min=0)], -1))
    s["counts"].copy_(torch.stack((n, (live & (ids >= n)).sum())))
    s["k"][:, holes] = s["k"][:, movers]
    s["v"][:, holes] = s["v"][:, movers]
    return {n: s[n] for n in ("table_out", "refs_out", "counts", "k", "v")}


_PLAIN = {"rope": _plain_rope, "append": _plain_append, "attend": _plain_attend, "update": _plain_update, "compact": _plain_compact}


# ---- the definitions in 64 bits ---------------------------------------------

def _angles(c, pos):
    """cos and sin [T, rot/2] and the scale, from the powers themselves."""
    r, f = c["rot"], c["factor"]
    base = 10000.0 * f ** (r / (r - 2.0)) if c["scaling"] == "ntk" and r > 2 else 10000.0
    inv = [1.0 / base ** (2.0 * i / r) for i in range(r // 2)]
    scale = 1.0
    if c["scaling"] == "linear":
        inv = [x / f for x in inv]
    elif c["scaling"] == "yarn":
        edge = [r * math.log(4096.0 / (2.0 * math.pi * b)) / (2.0 * math.log(base)) for b in (32.0, 1.0)]
        a, b = float(max(0, math.floor(edge[0]))), float(min(r - 1, math.ceil(edge[1])))
        b = b if b != a else a + 0.001
        inv = [x * (1.0 - min(1.0, max(0.0, (i - a) / (b - a))) * (1.0 - 1.0 / f)) for i, x in enumerate(inv)]
        scale = 1.0 + 0.1 * math.log(f)
    a = pos.double()[:, None] * torch.tensor(inv, dtype=torch.float64, device=DEV)
    return torch.cos(a) * scale, torch.sin(a) * scale


def _exact_rotate(c, x, pos, sign=1.0):
    cos, sin = _angles(c, pos)
    y = x.double().clone()
    for i in range(c["rot"] // 2):
        a, b = (2 * i, 2 * i + 1) if c["inter"] else (i, i + c["rot"] // 2)
        u, w = x[..., a].double(), x[..., b].double()
        y[..., a] = u * cos[:, i, None] - sign * w * sin[:, i, None]
        y[..., b] = w * cos[:, i, None] + sign * u * sin[:, i, None]
    return y


def _spots(c, pages, lens, dim):
    """Places in one layer's pools of one kv head's tokens 0 .. lens-1 (head 0): two [lens, dim] index tensors."""
    e, dp, p = _chunk(c), _dp(c), c["page"]
    t, d = torch.arange(lens, device=DEV)[:, None], torch.arange(dim, device=DEV)[None]
    first = pages[t // p] * (c["kv_heads"] * p * dp) + t % p // 32 * (32 * dp)
    step, half = d // (2 * e), d % (2 * e) // e
    k = first + step * (64 * e) + half * (32 * e) + t % 32 * e + d % e
    u = t % 32 % (2 * e)
    v = first + d // 32 * 1024 + t % 32 // (2 * e) * (64 * e) + u % 8 // 4 * (32 * e) + d % 32 * e + u // 8 * 4 + u % 4
    return k, v


def exact(case, seed):
    c = {**case, "graph": False}
    s = prepare(c, seed)
    kind, p, L = c["kind"], c["page"], c["layers"]
    if kind == "rope":
        return {"out": _exact_rotate(c, s["x"], s["pos"], -1.0 if c["inverse"] else 1.0)}
    if kind in ("append", "attend"):
        off, slots, lens = s["off"].tolist(), s["slots"].tolist(), s["lens"].tolist()
    if kind == "append":
        q, k, v = s["q_out"].double(), s["k"].float(), s["v"].float()
        k = k.double().view(L, -1)
        v = v.double().view(L, -1)
        hk, dp = c["kv_heads"], _dp(c)
        for a, b, slot in zip(off[:-1], off[1:], slots):
            if a == b:
                continue
            m = lens[slot]
            pos = torch.arange(m - (b - a), m, device=DEV)
            ka, va = _spots(c, s["table"][slot].long(), m, dp)
            for l in range(L):
                q[l, a:b] = _exact_rotate(c, s["q"][l, a:b], pos)
                kr = torch.nn.functional.pad(_exact_rotate(c, s["k_new"][l, a:b], pos), (0, dp - c["dim"]))
                vr = torch.nn.functional.pad(s["v_new"][l, a:b].double(), (0, dp - c["dim"]))
                for h in range(hk):
                    k[l, (ka[pos] + h * p * dp).view(-1)] = kr[:, h].reshape(-1)
                    v[l, (va[pos] + h * p * dp).view(-1)] = vr[:, h].reshape(-1)
        return {"q": q, "k": k.view(s["k"].shape), "v": v.view(s["v"].shape)}
    if kind == "attend":
        g, D = c["heads"] // c["kv_heads"], c["dim"]
        out, lse = s["q_out"].double(), s["lse"].double()
        for a, b, slot in zip(off[:-1], off[1:], slots):
            if a == b:
                continue
            m = lens[slot]
            ka, va = _spots(c, s["table"][slot].long(), m, D)
            pos = torch.arange(m - (b - a), m, device=DEV)[:, None]
            j = torch.arange(m, device=DEV)[None]
            see = (pos >= 0) & ((j // c["mask"] <= pos // c["mask"]) if c["mask"] else (j >= 0))
            for l in range(L):
                for h in range(c["heads"]):
                    shift = h // g * p * _dp(c)
                    k, v = s["k"][l].view(-1)[ka + shift].double(), s["v"][l].view(-1)[va + shift].double()
                    z = (s["q"][l, a:b, h].double() @ k.t() / math.sqrt(D)).masked_fill(~see, -math.inf)
                    lse[l, a:b, h] = torch.logsumexp(z, -1)
                    out[l, a:b, h] = torch.nan_to_num(torch.softmax(z, -1)) @ v
        return {"out": out, "lse": lse}
    k, v = s["k"], s["v"]
    table, lens, refs = s["table"].tolist(), s["lens"].tolist(), s["refs"].tolist()
    moves = []
    if kind == "compact":
        n = sum(r > 0 for r in refs)
        holes = [i for i in range(n) if refs[i] == 0]
        to = {m: h for h, m in zip(holes, [i for i in range(n, len(refs)) if refs[i] > 0])}
        for m, h in to.items():
            refs[h], refs[m] = refs[m], 0
        table = [[to.get(x, x) for x in row] for row in table]
        moves.append((list(to.values()), list(to.keys())))
    else:
        said = []
        for dst, src, keep, size in ((s["all"], s["all"], None, s["base"]), (s["kids"], s["parents"], s["keep"], s["grown"]),
                                     (s["first"], s["first"], None, s["first_grown"])):
            said.append(_simulate(table, lens, refs, p, dst.tolist(), src.tolist(), None if keep is None else keep.tolist(), size.tolist(), moves))
    for to, of in moves:
        k[:, to], v[:, to] = k[:, of], v[:, of]
    if kind == "compact":
        return {"table_out": _ints(table), "refs_out": _ints(refs), "counts": _ints([n, len(moves[0][0])]), "k": k, "v": v}
    return {"table": _ints(table), "lens": _ints(lens), "refs": _ints(refs), "status": _ints(said), "k": k, "v": v}


def _simulate(table, lens, refs, p, dst, src, keep, size, moves):
    """One update on lists, entry by entry; the pages copied are added to `moves`.  Returns the pages lacking."""
    count = lambda n: -(-n // p)  # noqa: E731
    keep = [min(lens[a], n) for a, n in zip(src, size)] if keep is None else keep
    r = list(refs)
    for d, a, n in zip(dst, src, keep):
        for x in table[a][:n // p]:
            r[x] += 1
        for x in table[d][:count(lens[d])]:
            r[x] -= 1
    rows, wait = [], []
    held = list(r)  # a page that is copied from in this call is not handed out by it
    claimed = set()
    for d, a, n, m in zip(dst, src, keep, size):
        row = table[a][:n // p]
        if n % p:
            x = table[a][n // p]
            held[x] += 1
            if d == a and r[x] == 0 and x not in claimed:
                claimed.add(x)
                row = row + [x]
            else:
                row = row + [("copy", x)]
        rows.append(row + ["new"] * (count(m) - len(row)))
    free = [i for i, x in enumerate(held) if x == 0]
    need = sum(not isinstance(x, int) for row in rows for x in row)
    if need > len(free):
        return need - len(free)
    for x in claimed:
        r[x] = 1
    at, to, of = iter(free), [], []
    for d, m, row in zip(dst, size, rows):
        for i, x in enumerate(row):
            if not isinstance(x, int):
                row[i] = next(at)
                r[row[i]] = 1
                if x != "new":
                    to.append(row[i])
                    of.append(x[1])
        wait.append((d, m, row + [-1] * (len(table[d]) - len(row))))
    for d, m, row in wait:
        table[d], lens[d] = row, m
    refs[:] = r
    moves.append((to, of))
    return 0


def work(case):
    c = case
    b = 4 if c["dtype"] == "f32" else 2
    H, K, D, L = c["heads"], c["kv_heads"], c["dim"], c["layers"]
    page = 2.0 * _page_elems(c) * b * L                                      # keys and values of one page, every layer
    if c["kind"] == "rope":
        return {"bytes": c["new"] * (2.0 * H * D * b + 4), "flops": 3.0 * c["new"] * H * c["rot"]}
    if c["kind"] == "append":
        t = sum(_lengths(c)[0])
        return {"bytes": L * t * 2.0 * (H + 2 * K) * D * b, "flops": L * 3.0 * t * (H + K) * c["rot"]}
    if c["kind"] == "attend":
        n, m = _lengths(c)
        pairs, keys = 0, 0
        for x, y in zip(n, m):
            w = c["mask"] or y
            ends = [min(y, (i // w + 1) * w) for i in range(y - x, y)]
            pairs += sum(ends)
            keys += max(ends, default=0)
        t = sum(n)
        return {"bytes": L * (keys * 2.0 * K * D * b + t * H * (2.0 * D * b + 4)), "flops": L * 4.0 * pairs * H * D}
    if c["kind"] == "update":
        parent, pages = _update_pages(c)
        kids = c["seqs"] * (c["width"] - 1)
        copies = kids if c["ctx"] % c["page"] and c["spare"] >= 1.0 else 0
        cells = (3 * c["seqs"] * c["width"]) * (-(-(c["ctx"] + c["grow"]) // c["page"]))
        return {"bytes": copies * 2.0 * page + 8.0 * (cells + 3 * pages), "flops": 0.0}
    held = [-(-y // c["page"]) for y in _lengths({**c, "new": 1, "ragged": "len"})[1]]
    pages = max(sum(held), int(sum(held) / c["live"]))
    moved = sum(held) * (1.0 - sum(held) / pages)                            # live pages that lie behind the live ones' number
    return {"bytes": moved * 2.0 * page + 8.0 * (c["seqs"] * (max(held) + 1) + pages), "flops": 0.0}
