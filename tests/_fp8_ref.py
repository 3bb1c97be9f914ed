"""The 8-bit float format, the products and AdamW from their definitions, in 64 bits on the CPU: what the library's
results are held against.  numpy only; no code of the library."""
import numpy as np

MOST = 448.0
F8 = None


def _table():
    """The 256 values of the codes: 1 sign, 4 exponent, 3 fraction bits, bias 7, no infinity."""
    global F8
    if F8 is None:
        v = []
        for c in range(256):
            e, m = (c >> 3) & 15, c & 7
            x = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
            v.append(float("nan") if c & 127 == 127 else (-x if c >> 7 else x))
        F8 = np.array(v)
    return F8


def values(codes):
    return _table()[np.asarray(codes, dtype=np.uint8)]


def nearest(x):
    """Codes of the 8-bit floats next to x (|x| <= 448), ties to the even code."""
    grid = _table()[:127]                              # ascending magnitudes
    a = np.abs(x)
    hi = np.searchsorted(grid, a).clip(0, 126)
    lo = (hi - 1).clip(0)
    dl, dh = a - grid[lo], grid[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return (code + 128 * np.signbit(x)).astype(np.uint8)


def exponent(amax):
    """The least e >= -127 with amax <= 448 2^e."""
    if amax == 0:
        return -127
    e = int(np.floor(np.log2(amax / MOST))) - 2
    while amax > MOST * 2.0 ** e:
        e += 1
    return max(e, -127)


def quantize(x, block=1):
    """(codes [R, pitch], bytes [ceil(R / block), pitch / 128]) of x [R, C] (exact values in 64 bits)."""
    x = np.asarray(x, dtype=np.float64)
    R, C = x.shape
    kb, rb = -(-C // 128), -(-R // block)
    codes, scale = np.zeros((R, 128 * kb), np.uint8), np.zeros((rb, kb), np.uint8)
    for i in range(rb):
        for j in range(kb):
            rows, cols = slice(block * i, min(R, block * (i + 1))), slice(128 * j, min(C, 128 * (j + 1)))
            t = x[rows, cols]
            if not np.isfinite(t).all():
                codes[rows, cols], scale[i, j] = 0x7F, 255
                continue
            e = exponent(np.abs(t).max())
            codes[rows, cols] = nearest(t * 2.0 ** -e)
            scale[i, j] = e + 127
    return codes, scale


def held(codes, scale, block, cols):
    """The values of a quantized matrix, [R, cols]."""
    s = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    s = np.repeat(np.repeat(s, block, 0)[:codes.shape[0]], 128, 1)
    return (values(codes) * s)[:, :cols]


def round_trip(x, block=1):
    return held(*quantize(x, block), block, x.shape[1])


def mix(x):
    x = np.asarray(x, dtype=np.uint64)
    m = np.uint64(0xFFFFFFFF)
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x9E3779B1)) & m
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0x93CD3A2D)) & m
    return x ^ (x >> np.uint64(16))


def random20(n, seed, step, tensor):
    """The 20 random bits of each element's two states."""
    m = np.uint64(0xFFFFFFFF)
    key = mix((mix((seed ^ (step * 0x6A09E667)) & 0xFFFFFFFF) + np.uint64(tensor)) & m)
    h = mix((np.arange(n, dtype=np.uint64) + key) & m)
    return h >> np.uint64(12), mix((h + np.uint64(1)) & m) >> np.uint64(12)


def adamw(p, g, m, v, lr, b1, b2, eps, decay, step, scale=1.0):
    """(p, m, v) after a step, in 64 bits."""
    g = g * scale
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    d = np.sqrt(v) / np.sqrt(1 - b2 ** step) + eps
    with np.errstate(invalid="ignore", divide="ignore"):
        return p * (1 - lr * decay) - lr / (1 - b1 ** step) * (m / d), m, v


def blocks(x):
    """x padded to whole blocks of 128, [blocks, 128]."""
    return np.pad(x, (0, -len(x) % 128)).reshape(-1, 128)


def stochastic(x, e, u, keep):
    """The code values (unscaled) that x 2^-e is rounded to: in magnitude the one below, or the one above where u is not
    below the distance to it in steps; past 448 it is 448.  keep: what is not zero does not become zero."""
    grid = _table()[:127]
    a = (np.abs(x) * 2.0 ** -e).clip(max=MOST)
    lo = np.searchsorted(grid, a, side="right") - 1
    hi = np.minimum(lo + 1, 126)
    part = np.where(hi > lo, (a - grid[lo]) / np.where(hi > lo, grid[hi] - grid[lo], 1.0), 0.0)
    got = np.where(part + u >= 1, grid[hi], grid[lo])
    if keep:
        got = np.where(x > 0, np.maximum(got, 2.0 ** -9), got)
    return np.copysign(got, x)
