"""Independent 64-bit oracle of the attention half of a decode step: rotary positions, the key/value cache's quantisation
and its byte layout (written from the text of include/lutgemm.h, place by place), attention.  Test infrastructure."""
import math

import numpy as np

BLOCK = 32


# ---- rotary positions --------------------------------------------------------------------------
def frequencies(rot, base=10000.0, scaling=0, factor=1.0, low=1.0, high=32.0, trained=0.0):
    """Radians a position, scaling 0..3: plain, linear, base, parts."""
    if scaling == 2 and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    f = np.array([base ** (-2.0 * i / rot) for i in range(rot // 2)])
    if scaling == 1:
        f = f / factor
    if scaling == 3:
        kept = np.clip((f * trained / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
        f = f * kept + f / factor * (1 - kept)
    return f


def rope(x, positions, turns, rot, neighbours=False, transpose=False, amplitude=1.0):
    """x [tokens][heads][dim]; turns: uint64 fractions of a turn a position.  The angle is exact: Python integers."""
    y = np.array(x, dtype=np.float64)
    for t, pos in enumerate(positions):
        for i in range(rot // 2):
            part = (int(pos) * int(turns[i])) % (1 << 64)
            angle = 2 * math.pi * (part / 2.0 ** 64)
            c, s = amplitude * math.cos(angle), amplitude * math.sin(-angle if transpose else angle)
            a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + rot // 2)
            xa, xb = x[t, :, a].astype(np.float64), x[t, :, b].astype(np.float64)
            y[t, :, a], y[t, :, b] = xa * c - xb * s, xa * s + xb * c
    return y


# ---- quantisation ------------------------------------------------------------------------------
def toward_zero_f16(x):
    """float64 >= 0 -> float16 rounded towards zero."""
    h = x.astype(np.float16)
    return np.where(h.astype(np.float64) > x, np.nextafter(h, np.float16(0)), h)


def quantise(x, bits, group):
    """x fp16 [..., dim] -> (codes uint8 or fp16, scale fp16, offset fp16), scales [..., dim / group]."""
    if bits == 16:
        return x.copy(), None, None
    g = x.reshape(*x.shape[:-1], -1, group).astype(np.float64)
    bad = ~np.isfinite(g).all(-1)
    g = np.where(bad[..., None], 0.0, g)
    low = g.min(-1)
    if bits == 8:
        scale = toward_zero_f16(np.abs(g).max(-1) / 127.0)
        u = np.rint(np.divide(g, scale[..., None].astype(np.float64), out=np.zeros_like(g), where=scale[..., None] > 0))
        u = np.clip(u, -127, 127) + 128
        offset = None
    else:
        scale = toward_zero_f16((g.max(-1) - low) / 15.0)
        offset = low.astype(np.float16)
        u = np.rint(np.divide(g - low[..., None], scale[..., None].astype(np.float64), out=np.zeros_like(g), where=scale[..., None] > 0))
        u = np.clip(u, 0, 15)
    scale = np.where(bad, np.float16(np.nan), scale).astype(np.float16)
    return u.reshape(x.shape).astype(np.uint8), scale, offset


def values(code, scale, offset, bits, group):
    """What the codes stand for: fp16, one rounding."""
    if bits == 16:
        return code
    u = code.reshape(*code.shape[:-1], -1, group).astype(np.float64)
    s = scale[..., None].astype(np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        v = s * (u - 128) if bits == 8 else s * u + offset[..., None].astype(np.float64)
        return v.astype(np.float16).reshape(code.shape)


# ---- layout ------------------------------------------------------------------------------------
def code_bytes(dim, bits):
    return BLOCK * dim * bits // 8


def scale_bytes(dim, bits, group):
    return 0 if bits == 16 else dim // group * BLOCK * (2 if bits == 8 else 4)


def block_bytes(dim, bits, group):
    return 2 * (code_bytes(dim, bits) + scale_bytes(dim, bits, group))


def pool_bytes(pages, page, heads, dim, bits, group):
    return pages * heads * (page // BLOCK) * block_bytes(dim, bits, group)


def put(pool, where, key, x, bits, group):
    """Write one position of one head.  where: (page, place in the page, head, page size, heads); x fp16 [dim]."""
    page, at, head, page_size, heads = where
    dim = x.shape[0]
    code, scale, offset = quantise(x, bits, group)
    base = ((page * heads + head) * (page_size // BLOCK) + at // BLOCK) * block_bytes(dim, bits, group)
    base += 0 if key else code_bytes(dim, bits) + scale_bytes(dim, bits, group)
    n = at % BLOCK
    for d in range(dim):
        c = d // 32
        if key:
            a, j, b, g, e = n // 8, n // 4 % 2, n % 4, d % 32 // 8, d % 8
            lane = 16 * g + 4 * a + b
        else:
            g, e, j, r = n // 8, n % 8, d % 32 // 16, d % 16
            lane = 16 * g + r
        if bits == 16:
            half = ((c * 2 + j) * 64 + lane) * 8 + e
            pool[base + 2 * half:base + 2 * half + 2] = np.frombuffer(code[d].tobytes(), np.uint8)
        elif bits == 8:
            pool[base + ((c * 64 + lane) * 2 + j) * 8 + e] = code[d]
        else:
            if key:
                nibble = e // 2 + 4 * (e % 2)
                byte, high = base + ((c * 64 + lane) * 2 + j) * 4 + nibble // 2, nibble % 2
            else:
                byte, high = base + (c * 64 + lane) * 8 + 4 * (e // 4) + (0, 2, 1, 3)[e % 4], j
            old = int(pool[byte])
            pool[byte] = (old & 0x0f) | (int(code[d]) << 4) if high else (old & 0xf0) | int(code[d])
    if bits != 16:
        base += code_bytes(dim, bits)
        for G in range(dim // group):
            if key:
                a, j, b = n // 8, n // 4 % 2, n % 4
                half = G * 32 + (4 * a + b) * 2 + j if bits == 8 else G * 64 + (4 * a + b) * 4 + 2 * j
                other = half + 1
            else:
                half = G * 32 + n if bits == 8 else G * 64 + n
                other = half + 32
            pool[base + 2 * half:base + 2 * half + 2] = np.frombuffer(scale[G].tobytes(), np.uint8)
            if bits == 4:
                pool[base + 2 * other:base + 2 * other + 2] = np.frombuffer(offset[G].tobytes(), np.uint8)


# ---- attention ---------------------------------------------------------------------------------
def attention(q, k, v, past, mask, scale):
    """One sequence.  q [tokens][q_heads][dim], k and v [positions][heads][dim] (positions = past + tokens), mask: ints or
    None.  Returns y and what error bounds need: sum of w |v|, and the largest sum of |q| |k| scale of a row."""
    tokens, q_heads, dim = q.shape
    heads = k.shape[1]
    y = np.zeros((tokens, q_heads, dim))
    mass = np.zeros((tokens, q_heads, dim))
    reach = 0.0
    for t in range(tokens):
        sees = np.ones(past + tokens, dtype=bool)
        word = (1 << (t + 1)) - 1 if mask is None else int(mask[t])
        for j in range(tokens):
            sees[past + j] = bool(word >> j & 1)
        if not sees.any():
            continue
        for h in range(q_heads):
            kk, vv = k[sees, h * heads // q_heads].astype(np.float64), v[sees, h * heads // q_heads].astype(np.float64)
            with np.errstate(invalid="ignore"):
                s = kk @ q[t, h].astype(np.float64) * scale
                reach = max(reach, float(np.nan_to_num(np.abs(kk) @ np.abs(q[t, h].astype(np.float64)), posinf=0, nan=0).max()) * abs(scale))
                w = np.exp(s - s.max())
                w /= w.sum()
                y[t, h] = w @ vv
                mass[t, h] = w @ np.abs(vv)
    return y, mass, reach
