"""Plain implementation of the 8-bit floats with a scale per block of 128 (64 bits, numpy), from the definitions in include/qgemm.h."""
import math

import numpy as np

BLOCK = 128
NUMBERS = np.array([f / 512 for f in range(8)] + [(8 + f) * 2.0 ** (e - 10) for e in range(1, 16) for f in range(8)][:-1])   # by code
MIDDLES = (NUMBERS[1:] + NUMBERS[:-1]) / 2


def up(x, m):
    return (x + m - 1) // m * m


def value(codes, byte):
    """What codes (uint8) stand for under scale bytes that broadcast with them."""
    codes, byte = np.asarray(codes), np.asarray(byte).astype(np.int64)
    size = np.append(NUMBERS, math.nan)[codes & 127]
    x = np.where(codes & 128, -size, size) * 2.0 ** (byte - 127.0)
    return np.where(byte == 255, math.nan, x)


def byte_of(amax):
    """Scale byte for the largest size of a block (an infinity or NaN among its numbers: amax is one)."""
    out = np.zeros(np.shape(amax), np.uint8)
    for at, a in np.ndenumerate(np.asarray(amax, np.float64)):
        if not math.isfinite(a):
            out[at] = 255
        elif a > 0:
            m, k = math.frexp(a)
            out[at] = max(0, (k - 9 if 2 * m <= 1.75 else k - 8) + 127)
    return out


def round_codes(y):
    """Nearest e4m3 codes of 64-bit numbers of at most 448 in size, ties to the even code."""
    v = np.abs(y)
    at = np.searchsorted(MIDDLES, v)                     # middles below v
    tie = (at < len(MIDDLES)) & (v == MIDDLES[np.minimum(at, len(MIDDLES) - 1)]) & (at % 2 == 1)
    return ((at + tie) | np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def top(x, axis):
    with np.errstate(invalid="ignore"):
        t = np.max(np.abs(x), axis=axis, initial=0.0)
    return t                                              # (numpy's max passes a NaN on)


def quantize(x):
    """x [T, K] (64 bits) -> (codes [T, K rounded up to 128], scale bytes [T, blocks]); codes of a NaN block are 0 here."""
    T, K = x.shape
    y = np.zeros((T, up(K, BLOCK)))
    y[:, :K] = x
    y = y.reshape(T, -1, BLOCK)
    byte = byte_of(top(y, 2))
    with np.errstate(invalid="ignore", over="ignore"):
        z = np.where(byte[..., None] == 255, 0.0, y * 2.0 ** (127.0 - byte[..., None].astype(np.float64)))
    return round_codes(z).reshape(T, -1), byte


def held(x):
    """What 8 bits keep of x [T, K]."""
    codes, byte = quantize(x)
    return value(codes, np.repeat(byte, BLOCK, 1))[:, :x.shape[1]]


def quantize_weight(b):
    """B [K, N] -> (codes of the same shape, scale bytes [K blocks, N blocks])."""
    K, N = b.shape
    y = np.zeros((up(K, BLOCK), up(N, BLOCK)))
    y[:K, :N] = b
    y = y.reshape(y.shape[0] // BLOCK, BLOCK, -1, BLOCK)
    byte = byte_of(top(y, (1, 3)))
    with np.errstate(invalid="ignore", over="ignore"):
        z = np.where(byte[:, None, :, None] == 255, 0.0, y * 2.0 ** (127.0 - byte[:, None, :, None].astype(np.float64)))
    return round_codes(z).reshape(up(K, BLOCK), up(N, BLOCK))[:K, :N], byte


def held_weight(b):
    codes, byte = quantize_weight(b)
    K, N = b.shape
    return value(codes, np.repeat(np.repeat(byte, BLOCK, 0)[:K], BLOCK, 1)[:, :N])


def unpack(data, k, n, gated):
    """The bytes of a packed matrix -> [(codes [kp, np], scale bytes [kp / 128, np / 128])] of B, or of gate and up; whole blocks, padding
    included."""
    kb = up(k, 128) // 128
    kb4 = up(kb, 4)
    groups = up(n, 128) // 32 if gated else up(n, 256) // 64
    size = groups * kb * 8192
    pieces = data[:size].reshape(groups, kb, 4, 2, 4, 16, 16)     # group, k block, fragment, half, 16 of K, slot, byte
    scales = data[size:size + groups * kb4 * 4].reshape(groups, kb4, 4)[:, :kb]
    out = []
    for which in range(2 if gated else 1):
        width = 32 if gated else 64
        codes = np.zeros((kb * 128, groups * width), np.uint8)
        byte = np.zeros((kb, groups * width), np.uint8)
        for j in range(which, 4, 2 if gated else 1):
            for slot in range(16):
                q, r = slot // 4, slot % 4
                col = np.arange(groups) * width + (8 * q + 4 * (j >> 1) + r if gated else 16 * q + 4 * j + r)
                codes[:, col] = pieces[:, :, j, :, :, slot].reshape(groups, -1).T
                byte[:, col] = scales[:, :, j].T
        assert (byte.reshape(kb, -1, 32) == byte.reshape(kb, -1, 32)[:, :, :1]).all()
        out.append((codes, byte))
    return out


def activate(kind, g):
    """(activation, slope) in 64 bits."""
    from scipy.special import erfc, expit
    if kind == "silu":
        return g * expit(g), expit(g) * (1 + g * expit(-g))
    if kind == "gelu":
        p = 0.5 * erfc(-g / math.sqrt(2))
        return g * p, p + g * np.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        r = 2 * math.sqrt(2 / math.pi)
        z = r * (g + 0.044715 * g ** 3)
        return g * expit(z), expit(z) + g * expit(z) * expit(-z) * r * (1 + 3 * 0.044715 * g * g)
    return np.maximum(g, 0), (g > 0).astype(float)


# ---- bounds.  A product of 8-bit numbers is exact in fp32.  Sums in fp32: at most `adds` roundings meet on the way of a product to the
# result, and each is at most one unit 2^-23 (the matrix cores need not round to nearest) of the partial sum, itself at most the mass
# sum |x||b|.  On the way: 128 of a block within the instructions, one for each block of K, 32 for joins.  Sums on the 8-bit cores also lose,
# of every eight products, less than 2^-13 of the leading bit of the largest each: 8 * 2^-13 of the largest, so at most 2^-10 of the mass.


def sum_bound(mass, K, wide):
    return mass * ((128 + (K + 127) // 128 + 32) * 2.0 ** -23 + (0.0 if wide else 2.0 ** -10))


STEP = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}   # half a step of a rounding, relative
TINY = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -25}  # and absolute, among subnormals


def rounding(x, dtype):
    name = str(dtype).replace("torch.", "")
    return STEP[name] * np.abs(x) + TINY[name]


def held_bound(h, err):
    """How far the 8-bit form of a number within err of h [T, K] may be from that of h: the codes are monotonic for a given scale, and the
    scale is that of amax - err or amax + err, or between."""
    T, K = h.shape
    pad = up(K, BLOCK) - K
    y, e = np.pad(h, ((0, 0), (0, pad))).reshape(T, -1, BLOCK), np.pad(err, ((0, 0), (0, pad))).reshape(T, -1, BLOCK)
    size = np.abs(y)
    low, high = byte_of((size - e).max(2).clip(0)), byte_of((size + e).max(2))
    base = held(h).reshape(T, K)
    worst = np.zeros((T, K))
    for byte in (low, high):
        scale = 2.0 ** (byte[..., None].astype(np.float64) - 127)
        for s in (-1, 1):
            z = np.clip((y + s * e) / scale, -448, 448)
            v = value(round_codes(z), np.broadcast_to(byte[..., None], z.shape)).reshape(T, -1)[:, :K]
            worst = np.maximum(worst, np.abs(v - base))
    return worst
