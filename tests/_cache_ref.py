"""The 4-bit key/value cache in 64 bits, from include/mcd.h's description: byte by byte, numpy
only, sharing nothing with the library.  Test infrastructure."""
import numpy as np

PAGE = 64
LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def page_bytes(D):
    return 66 * D + 128


def bf16_round(x):
    """Nearest bfloat16 (ties to even) of float32 values, as float32; NaN stays."""
    u = np.asarray(x, np.float32).view(np.uint32)
    r = ((u.astype(np.uint64) + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32)
    return np.where(np.isnan(x), np.float32(np.nan), r.view(np.float32))


def code(x, scale):
    """e2m1 code of one number: nearest level of |x| / scale, ties to the even code."""
    with np.errstate(divide="ignore", invalid="ignore"):
        a = abs(float(x)) / float(scale) if scale > 0 else (np.inf if x != 0 else 0.0)
    d = np.abs(LEVELS - min(a, 100.0))
    near = np.flatnonzero(d == d.min())
    c = near[0] if len(near) == 1 else [i for i in near if i % 2 == 0][0]
    return int(c) | (8 if np.signbit(x) else 0)


def key_exponent(block):
    """Byte of 32 keys: the smallest b in 1..254 with max <= 7 * 2^(b - 127), 255 if not finite."""
    if not np.isfinite(block).all():
        return 255
    top = float(np.abs(block).max())
    b = 1
    while b < 254 and top > 7.0 * 2.0 ** (b - 127):
        b += 1
    return b


def value_scale(v):
    """bfloat16 scale of a token's values, as float."""
    if not np.isfinite(v).all():
        return float("nan")
    return float(bf16_round(np.float32(np.abs(v).max()) * np.float32(1.0 / 6.0)))


def put(page, D, t, k, v):
    """Token t (of its page) into page (uint8 [bytes] of one head): keys k, values v [D]."""
    nb = D // 32
    for b in range(nb):
        block = k[32 * b:32 * b + 32]
        e = key_exponent(block)
        page[64 * D + ((t % 16) * nb + b) * 4 + t // 16] = e
        for i in range(32):
            c = 0 if e == 255 else code(block[i], 2.0 ** (e - 127))
            set_nibble(page, (t * D + 32 * b + i), c)
    s = value_scale(v)
    for c in range(D):
        set_nibble(page, value_nibble(D, t, c), 0 if np.isnan(s) else code(v[c], s))
    bits = 0x7FC0 if np.isnan(s) else int(np.float32(s).view(np.uint32)) >> 16
    at = 66 * D + 2 * (t // 4 % 4 * 16 + t // 16 * 4 + t % 4)
    page[at], page[at + 1] = bits & 255, bits >> 8


def set_nibble(page, n, c):
    page[n // 2] = (page[n // 2] & (0xF0 if n % 2 == 0 else 0x0F)) | (c << 4 * (n % 2))


def value_nibble(D, t, c):
    """Index of the nibble (from the page's start) of channel c of token t's values."""
    h, j, g, i = t // 32, t // 16 % 2, t // 4 % 4, t % 4
    quarter, rest = divmod(c, D // 4)
    tile, low = divmod(rest, 4)
    m = quarter * 4 + low
    word = ((h * (D // 64) + tile // 4) * 64 + 16 * g + m) * 4 + tile % 4
    return 2 * 32 * D + 8 * word + 4 * j + i


def get(page, D, t):
    """Keys and values [D] (float64) of token t."""
    nb = D // 32
    nib = lambda n: (page[n // 2] >> 4 * (n % 2)) & 15  # noqa: E731
    val = lambda c: -LEVELS[c & 7] if c & 8 else LEVELS[c & 7]  # noqa: E731
    k = np.array([val(nib(t * D + c)) for c in range(D)])
    for b in range(nb):
        e = int(page[64 * D + ((t % 16) * nb + b) * 4 + t // 16])
        k[32 * b:32 * b + 32] *= np.nan if e == 255 else 2.0 ** (e - 127)
    at = 66 * D + 2 * (t // 4 % 4 * 16 + t // 16 * 4 + t % 4)
    bits = np.uint32((int(page[at]) | int(page[at + 1]) << 8) << 16)
    v = np.array([val(nib(value_nibble(D, t, c))) for c in range(D)])
    return k, v * float(bits.view(np.float32))


def decode_pages(pages, D):
    """Keys and values [n, Hkv, 64, D] of pages [n, Hkv, bytes], vectorised get()."""
    pages = np.asarray(pages)
    t, c = np.arange(PAGE)[:, None], np.arange(D)[None]
    nb = D // 32
    lut = np.concatenate([LEVELS, -LEVELS])
    kn = t * D + c
    k = lut[(pages[..., kn // 2] >> (4 * (kn % 2))) & 15]
    e = pages[..., 64 * D + ((t % 16) * nb + c // 32) * 4 + t // 16].astype(int)
    with np.errstate(invalid="ignore"):
        k = np.where(e == 255, np.nan, k * 2.0 ** (np.minimum(e, 254) - 127))
    h, j, g, i = t // 32, t // 16 % 2, t // 4 % 4, t % 4
    quarter, rest = c // (D // 4), c % (D // 4)
    word = ((h * (D // 64) + rest // 4 // 4) * 64 + 16 * g + quarter * 4 + rest % 4) * 4 \
        + rest // 4 % 4
    vn = 64 * D + 8 * word + 4 * j + i
    v = lut[(pages[..., vn // 2] >> (4 * (vn % 2))) & 15]
    at = 66 * D + 2 * (t // 4 % 4 * 16 + t // 16 * 4 + t % 4)
    bits = (pages[..., at].astype(np.uint32) | pages[..., at + 1].astype(np.uint32) << 8) << 16
    return k, v * bits.view(np.float32).astype(np.float64)


def attend(k, v, q, ctx, scale):
    """k, v [Hkv, L, D], q [n, Hq, D] in float64 -> out [n, Hq, D], lse [n, Hq], weight [Hkv, L]
    and sum of p |v| [n, Hq, D]."""
    H, L, D = k.shape
    n, Hq, _ = q.shape
    out, size = np.zeros((n, Hq, D)), np.zeros((n, Hq, D))
    lse, weight = np.full((n, Hq), -np.inf), np.zeros((H, L))
    for i in range(n):
        upto = min(max(ctx + i + 1, 0), L)
        if upto == 0:
            continue
        for a in range(Hq):
            h = a // (Hq // H)
            x = scale * (k[h, :upto] @ q[i, a])
            top = x.max()
            p = np.exp(x - top)
            lse[i, a] = top + np.log(p.sum())
            p /= p.sum()
            out[i, a] = p @ v[h, :upto]
            size[i, a] = p @ np.abs(v[h, :upto])
            weight[h, :upto] += p
    return out, lse, weight, size


def evict(w, keep, recent):
    """Positions kept of one head's weights w [n]."""
    n = len(w)
    if n <= keep:
        return np.arange(n)
    rank = np.where(np.isnan(w[:n - recent]), -np.inf, w[:n - recent])
    # NaN below every number, -infinity among them; equal weights by position
    order = np.lexsort((np.arange(n - recent), -rank, np.isnan(w[:n - recent])))
    return np.concatenate([np.sort(order[:keep - recent]), np.arange(n - recent, n)])
