"""CPU oracle of the 8-bit forms, the 8-bit linear layer and the batched Adam step, in float64 and by tables of the formats'
values (test infrastructure only).

Formats: e4m3 (bias 7, code 0x7f NaN, largest 448) and e5m2 (bias 15, 0x7c infinity, largest 57344).  A scale is 2^(byte - 127).
"""
import numpy as np

E4M3, E5M2 = 0, 1
LARGEST = {E4M3: 448.0, E5M2: 57344.0}


def code_values(fmt):
    """The value of each of the 256 codes."""
    exp_bits, man_bits, bias = ((4, 3, 7), (5, 2, 15))[fmt]
    out = np.empty(256)
    for code in range(256):
        e, m = (code >> man_bits) & ((1 << exp_bits) - 1), code & ((1 << man_bits) - 1)
        v = m * 2.0 ** (1 - bias - man_bits) if e == 0 else (1 + m / (1 << man_bits)) * 2.0 ** (e - bias)
        if fmt == E4M3 and (code & 0x7f) == 0x7f:
            v = np.nan
        if fmt == E5M2 and e == 31:
            v = np.inf if m == 0 else np.nan
        out[code] = -v if code & 0x80 else v
    return out


def _finite_codes(fmt):
    v = code_values(fmt)[:128]
    return v[np.isfinite(v)]                                        # ascending with the code


def encode_nearest(x, fmt):
    """Codes of the nearest values, ties to the even code; |x| at most the largest value."""
    x = np.asarray(x, dtype=np.float64)
    v = _finite_codes(fmt)
    mid = (v[:-1] + v[1:]) / 2
    lo = np.searchsorted(mid, np.abs(x), side="left")               # at a tie: the lower code
    tie = (lo < mid.size) & (np.abs(x) == mid[np.minimum(lo, mid.size - 1)])
    code = lo + (tie & (lo % 2 == 1))
    return (code | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def scale_byte(amax, fmt):
    """The smallest exponent (plus 127, at least 0) whose power of two brings amax to the format's range, by trying all of them."""
    amax = np.asarray(amax, dtype=np.float64)
    out = np.full(amax.shape, 255, dtype=np.int64)
    for b in range(254, -1, -1):
        out = np.where(amax <= LARGEST[fmt] * 2.0 ** (b - 127), b, out)
    return out


def _cut(n, size):
    return [(lo, min(lo + size, n)) for lo in range(0, n, size)]


def quantize(x, rows, cols, fmt):
    """(codes, scale bytes) of a matrix, one scale for each block of rows x cols; blocks that are not finite are NaN under byte 127."""
    x = np.asarray(x, dtype=np.float64)
    n, k = x.shape
    q = np.empty((n, k), dtype=np.uint8)
    amax = np.zeros((-(-n // rows), -(-k // cols)))
    with np.errstate(invalid="ignore"):
        padded = np.zeros((amax.shape[0] * rows, amax.shape[1] * cols))
        padded[:n, :k] = np.where(np.isfinite(x), np.abs(x), np.inf)
        amax = padded.reshape(amax.shape[0], rows, amax.shape[1], cols).max(axis=(1, 3))
    bad = ~np.isfinite(amax)
    s = np.where(bad, 127, scale_byte(np.where(bad, 0.0, amax), fmt))
    wide = lambda a: np.repeat(np.repeat(a, rows, 0)[:n], cols, 1)[:, :k]  # noqa: E731
    with np.errstate(invalid="ignore"):
        q = encode_nearest(np.where(wide(bad), 0.0, x) * 2.0 ** (127.0 - wide(s)), fmt)
    q[wide(bad)] = 0x7f
    return q, s.astype(np.uint8)


def dequantize(q, s, rows, cols, fmt):
    n, k = q.shape
    return code_values(fmt)[q] * 2.0 ** (np.repeat(np.repeat(s.astype(np.float64), rows, 0)[:n], cols, 1)[:, :k] - 127.0)


def mix(x):
    """32-bit hash behind the random bits of the Adam step."""
    x = np.asarray(x, dtype=np.uint64) & 0xFFFFFFFF
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x6A09E667)) & np.uint64(0xFFFFFFFF)
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0xBB67AE85)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def random_bits(seed, step, job, rows, cols):
    key = int(mix((seed + 0x9E3779B9 * step + 0xBB67AE85 * job) & 0xFFFFFFFF))
    h = mix(np.arange(rows * cols, dtype=np.uint64) + np.uint64(key)).reshape(rows, cols)
    return (h & np.uint64(0xFFFF)).astype(np.int64), (h >> np.uint64(16)).astype(np.int64)


def encode_randomly(y, random16, fmt):
    """Codes of magnitudes y (float32 values): the lower neighbour, or the upper one where the random bits, as a fraction of the
    distance between the two, carry y past it."""
    v = _finite_codes(fmt)
    # (below the smallest normal value y takes part with the last place it has after that value is added to it in float32)
    low = 2.0 ** (-6 if fmt == E4M3 else -14)
    y32 = np.asarray(y, dtype=np.float32)
    y = np.where(y32 < low, (y32 + np.float32(low)).astype(np.float64) - low, y32.astype(np.float64))
    lo = np.searchsorted(v, y, side="right") - 1
    step = np.where(lo + 1 < v.size, v[np.minimum(lo + 1, v.size - 1)] - v[lo], 1.0)
    return (lo + ((y - v[lo]) / step + random16 / 65536.0 >= 1.0)).astype(np.uint8)


def adam_moments(m, v, g, beta1, beta2):
    """New moments in float32, one rounding behind product and sum (the product of two float32 values is exact in float64)."""
    f = np.float32
    c1, c2 = f(1) - f(beta1), f(1) - f(beta2)
    a, b = (c1 * g).astype(f), ((c2 * g).astype(f) * g).astype(f)
    return ((np.float64(f(beta1)) * m + a.astype(np.float64)).astype(f), (np.float64(f(beta2)) * v + b.astype(np.float64)).astype(f))


def store_moments(m, v, seed, step, job):
    """(m codes, m scales, v codes, v scales) of float32 moments [rows, cols]."""
    rows, cols = m.shape
    rm, rv = random_bits(seed, step, job, rows, cols)
    out = []
    for x, random, fmt in ((m, rm, E4M3), (v, rv, E5M2)):
        q, s = np.empty((rows, cols), dtype=np.uint8), np.empty((rows, -(-cols // 128)), dtype=np.uint8)
        for j, (lo, hi) in enumerate(_cut(cols, 128)):
            part = x[:, lo:hi]
            bad = ~np.isfinite(part).all(1)
            byte = np.where(bad, 127, scale_byte(np.where(bad, 0.0, np.abs(np.nan_to_num(part)).max(1)), fmt))
            y = np.abs(np.where(bad[:, None], 0.0, part)) * 2.0 ** (127.0 - byte)[:, None]
            code = encode_randomly(y.astype(np.float32), random[:, lo:hi], fmt)
            if fmt == E5M2:
                code = np.maximum(code, (part > 0).astype(np.uint8))
            else:
                code = code | np.where(np.signbit(part), 0x80, 0).astype(np.uint8)
            q[:, lo:hi] = np.where(bad[:, None], 0x7f, code)
            s[:, j] = byte
        out += [q, s]
    return out
