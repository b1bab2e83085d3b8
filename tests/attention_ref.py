"""Plain 64-bit definitions of the attention section of include/dmoe.h, on
the CPU and token by token where that is clearer: the cache's layout, the
visible keys, attention, rotation and the page bookkeeping."""
import math

import torch

EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}  # the largest rounding of a value, relative


def padded(dim):
    return next(d for d in (32, 64, 96, 128, 192, 256) if d >= dim)


def chunk(dtype):
    return 4 if dtype == torch.float32 else 8


def places(dtype, page, kv_heads, dim, pos, pages):
    """Places in one layer's pools of the keys and values of tokens at positions pos on pages: two [T, kv_heads, dim]."""
    c, dp = chunk(dtype), padded(dim)
    pos, pages = pos.view(-1, 1, 1), pages.view(-1, 1, 1).long()
    h, d = torch.arange(kv_heads).view(1, -1, 1), torch.arange(dim).view(1, 1, -1)
    tile = ((pages * kv_heads + h) * (page // 32) + pos % page // 32) * (32 * dp)
    r = pos % 32
    k = tile + ((d // (2 * c) * 2 + d % (2 * c) // c) * 32 + r) * c + d % c
    s, j, half, t = r // (2 * c), r % (2 * c) // 8, r % 8 // 4, r % 4
    v = tile + (((d // 32 * (16 // c) + s) * 2 + half) * 32 + d % 32) * c + 4 * j + t
    return k, v


def ends(positions, length, mask):
    """Keys that tokens at these positions see."""
    e = [0 if p < 0 else length if mask == 0 else min(length, (p // mask + 1) * mask) for p in positions]
    return torch.tensor(e)


def attention(q, k, v, end, scale):
    """q [n, H, D], k and v [J, K, D]; row i sees keys below end[i].  Returns out, lse, sum_j p_j |v_j| and the largest
    scale * sum_d |q_d k_jd| of a row (for bounds), all float64."""
    n, H, D = q.shape
    g = H // k.shape[1]
    q = q.double()
    out, size = torch.zeros(n, H, D, dtype=torch.float64), torch.zeros(n, H, D, dtype=torch.float64)
    lse, big = torch.full((n, H), -math.inf, dtype=torch.float64), torch.zeros(n, H, dtype=torch.float64)
    for h in range(H):
        kh, vh = k[:, h // g].double(), v[:, h // g].double()
        for i in range(n):
            e = int(end[i])
            if e == 0:
                continue
            s = scale * (kh[:e] @ q[i, h])
            m = s.max()
            p = torch.exp(s - m)
            lse[i, h] = m + torch.log(p.sum())
            p = p / p.sum()
            out[i, h], size[i, h] = p @ vh[:e], p @ vh[:e].abs()
            big[i, h] = scale * (kh[:e].abs() @ q[i, h].abs()).max()
    return out, lse, size, big


def bounds(dtype, D, J, out, lse, size, big):
    """How far the kernel's out and lse may be off.  Scores are float32 sums of D products: off by d = (D + 2) 2^-24 of
    sum |q k|, and by 2^-22 of their size from the scaling and the exponential's argument; that moves each probability by
    twice that, relative.  The probabilities' and the products' sums over J keys add (2 J + 8) 2^-24.  With bf16 each
    probability is rounded once (2^-8) before its product, and the result once."""
    d = ((D + 2) * 2.0 ** -24 + 2.0 ** -22) * big + 2.0 ** -22
    rel = 2 * d[..., None] + (2 * J + 8) * 2.0 ** -24
    if dtype == torch.bfloat16:
        rel = rel + EPS[dtype]
    b = rel * size
    b = b + EPS[dtype] * (out.abs() + b) + 1e-37
    return b, d + (2 * J + 8) * 2.0 ** -24 + 2.0 ** -22 * torch.nan_to_num(lse.abs(), posinf=0.0)


def turns(rot, base=10000.0, scaling="none", factor=1.0, original=4096):
    """Turns per position of every pair, and the scale."""
    if scaling == "ntk" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    f = [base ** (-2 * i / rot) / (2 * math.pi) for i in range(rot // 2)]
    if scaling == "linear":
        f = [x / factor for x in f]
    if scaling != "yarn":
        return f, 1.0
    lo, hi = (rot * math.log(original / (2 * math.pi * b)) / (2 * math.log(base)) for b in (32, 1))
    lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), rot - 1)
    width = hi - lo if hi != lo else 0.001
    ramp = [min(max((i - lo) / width, 0), 1) for i in range(rot // 2)]
    return [x / factor * r + x * (1 - r) for x, r in zip(f, ramp)], 0.1 * math.log(factor) + 1


def rotate(x, pos, f, scale=1.0, interleaved=False, inverse=False):
    """x [T, heads, D] with its first 2 len(f) elements rotated, float64."""
    y = x.double().clone()
    n = len(f)
    a = pos.double().view(-1, 1) * torch.tensor(f, dtype=torch.float64)
    a = (a - a.floor()) * (2 * math.pi)
    co, si = scale * torch.cos(a)[:, None], scale * torch.sin(a)[:, None] * (-1 if inverse else 1)
    one, two = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    u, w = x[..., one].double(), x[..., two].double()
    y[..., one], y[..., two] = u * co - w * si, w * co + u * si
    return y


class Pages:
    """The bookkeeping of dmoe_cache_update and dmoe_cache_compact on lists."""

    def __init__(self, n_pages, page, n_slots, max_pages):
        self.page, self.max_pages = page, max_pages
        self.table = [[-1] * max_pages for _ in range(n_slots)]
        self.lens, self.refs = [0] * n_slots, [0] * n_pages

    def update(self, dst, size, src=None, keep=None):
        """Returns (status, copies [(from, to)])."""
        p, up = self.page, lambda n: -(-n // self.page)
        src = dst if src is None else src
        slots = range(len(self.table))
        if len(set(dst)) < len(dst) or any(s not in slots for s in list(dst) + list(src)):
            return -1, []
        keep = [min(self.lens[s], n) for s, n in zip(src, size)] if keep is None else keep
        if any(not 0 <= n <= self.max_pages * p or not 0 <= m <= min(n, self.lens[s]) for n, m, s in zip(size, keep, src)):
            return -1, []
        refs = list(self.refs)
        for d, s, m in zip(dst, src, keep):
            for x in self.table[s][:m // p]:
                refs[x] += 1
            for x in self.table[d][:up(self.lens[d])]:
                refs[x] -= 1
        kept, busy, rows = set(), list(refs), []
        for d, s, m, n in zip(dst, src, keep, size):
            row = list(self.table[s][:m // p])
            if m % p:
                x = self.table[s][m // p]
                busy[x] += 1
                own = d == s and refs[x] == 0 and x not in kept
                if own:
                    kept.add(x)
                row.append(x if own else (x,))
            rows.append(row + [None] * (up(n) - len(row)))
        free = [i for i, r in enumerate(busy) if r == 0]
        need = sum(not isinstance(x, int) for row in rows for x in row)
        if need > len(free):
            return need - len(free), []
        for x in kept:
            refs[x] = 1
        copies = []
        for row in rows:
            for i, x in enumerate(row):
                if not isinstance(x, int):
                    row[i] = free.pop(0)
                    refs[row[i]] = 1
                    if x is not None:
                        copies.append((x[0], row[i]))
        for d, n, row in zip(dst, size, rows):
            self.table[d], self.lens[d] = row + [-1] * (self.max_pages - len(row)), n
        self.refs = refs
        return 0, copies

    def compact(self):
        """Returns (live pages, moves [(from, to)])."""
        n = sum(r > 0 for r in self.refs)
        moves = list(zip([i for i in range(n, len(self.refs)) if self.refs[i] > 0], [i for i in range(n) if self.refs[i] <= 0]))
        to = dict(moves)
        self.table = [[to.get(x, x) for x in row] for row in self.table]
        for a, b in moves:
            self.refs[b], self.refs[a] = self.refs[a], 0
        return n, moves
