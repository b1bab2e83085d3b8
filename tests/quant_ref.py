"""Plain definition of a cache of few bits (dmoe_kv_format of include/dmoe.h) in 64 bits on the CPU: codes by search among all
of them, places in a page by the header's formula."""
import math

import torch

from attention_ref import padded

BITS = {"fp8": (8, 8), "fp4": (4, 4), "fp8_fp4": (8, 4)}
LIMIT, LOWEST, HIGHEST = {4: 7.0, 8: 464.0}, 17, {4: 252, 8: 246}


def magnitudes(bits):
    """What the codes without a sign stand for, by code."""
    if bits == 4:
        return [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    return [c % 8 * 2.0 ** -9 if c < 8 else (1 + c % 8 / 8) * 2.0 ** (c // 8 - 7) for c in range(127)]


def scale_byte(top, bits):
    """The least byte at which an element of this magnitude is at most LIMIT times the scale."""
    if not math.isfinite(top):
        return 255
    b = LOWEST
    while b < HIGHEST[bits] and top > LIMIT[bits] * 2.0 ** (b - 127):
        b += 1
    return b


def code(y, bits):
    """The nearest code of a magnitude, ties to the even one, the largest beyond it."""
    table = magnitudes(bits)
    best = min(range(len(table)), key=lambda c: (abs(table[c] - y), c % 2))
    return best


def quantise(x, bits):
    """x [..., dim]: (codes [..., dp], scale bytes [..., dp / 32]), whole numbers."""
    dim = x.shape[-1]
    dp = padded(dim)
    flat = torch.nn.functional.pad(x.double(), (0, dp - dim)).reshape(-1, 32)
    top = torch.where(flat.isfinite(), flat.abs(), math.inf).amax(-1)
    scales = torch.tensor([scale_byte(float(t), bits) for t in top])
    table = torch.tensor(magnitudes(bits), dtype=torch.float64)
    y = flat.abs() * torch.pow(2.0, (127 - scales).double())[:, None]
    y = torch.where((scales == 255)[:, None], 0.0, y)
    away = (y[..., None] - table).abs()
    odd = torch.arange(table.numel()) % 2
    near = away == away.amin(-1, keepdim=True)
    codes = (near.int() * (4 - 2 * odd) * 1000 - torch.arange(table.numel())).argmax(-1)  # the nearest, the even one of two
    codes = codes + torch.where(torch.signbit(flat), 1 << (bits - 1), 0)
    codes = torch.where((scales == 255)[:, None], 0, codes)
    return codes.view(*x.shape[:-1], dp), scales.view(*x.shape[:-1], dp // 32)


def values(codes, scales, bits):
    """What codes [..., dp] and scale bytes [..., dp / 32] stand for, float64."""
    table = magnitudes(bits)
    table = table + [math.nan] * (128 - len(table) if bits == 8 else 0)
    table = torch.tensor(table + [-t for t in table], dtype=torch.float64)
    scale = torch.where(scales == 255, math.nan, torch.pow(2.0, (scales - 127).double()))
    return (table[codes].unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2)


def held(x, bits):
    """Rows [..., dim] as a cache of so many bits holds them, float64."""
    return values(*quantise(x, bits), bits)[..., :x.shape[-1]]


def layout(bits, dim):
    """Elements of a chunk, scale bytes of a token, bytes of a tile."""
    dp = padded(dim)
    w, sb = 128 // bits, 1
    while sb < dp // 32:
        sb *= 2
    return w, sb, dp // w * 512 + 32 * sb


def page_bytes(bits, page, kv_heads, dim):
    return kv_heads * (page // 32) * layout(bits, dim)[2]


def places(bits, page, kv_heads, dim, pos, pages):
    """Bytes of one layer's pool that hold tokens at positions pos on pages: of the codes [T, kv_heads, dp] and of the scales
    [T, kv_heads, dp / 32]."""
    w, sb, tile = layout(bits, dim)
    dp = padded(dim)
    pos, pages = pos.view(-1, 1, 1), pages.view(-1, 1, 1).long()
    at = ((pages * kv_heads + torch.arange(kv_heads).view(1, -1, 1)) * (page // 32) + pos % page // 32) * tile
    d, g = torch.arange(dp).view(1, 1, -1), torch.arange(dp // 32).view(1, 1, -1)
    return at + (d // w * 32 + pos % 32) * 16 + d % w * bits // 8, at + dp // w * 512 + pos % 32 * sb + g


def put(pool, bits, page, dim, pos, pages, codes, scales):
    """Writes tokens' codes [T, kv_heads, dp] and scales into a layer's pool (a flat uint8 tensor)."""
    at, st = places(bits, page, codes.shape[1], dim, pos, pages)
    if bits == 4:
        at, codes = at[..., 0::2], codes[..., 0::2] + 16 * codes[..., 1::2]
    pool[at.reshape(-1)] = codes.reshape(-1).to(torch.uint8)
    pool[st.reshape(-1)] = scales.reshape(-1).to(torch.uint8)


def get(pool, bits, page, kv_heads, dim, pos, pages):
    """Tokens of a layer's pool: [T, kv_heads, dim], float64."""
    at, st = places(bits, page, kv_heads, dim, pos, pages)
    codes = pool[at].long()
    if bits == 4:
        codes = torch.where(torch.arange(codes.shape[-1]) % 2 == 1, codes >> 4, codes & 15)
    return values(codes, pool[st].long(), bits)[..., :dim]
