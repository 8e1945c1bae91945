"""Plain numpy implementations of the rotary positions, the 4-bit cache and its attention, from their definitions: the
quantization in fp32 operation for operation (one result is right), everything else in 64 bits."""
import math

import numpy as np


def frequencies(rot, base, scaling="plain", factor=1.0, low=1.0, high=32.0, context=0.0):
    i = np.arange(rot // 2, dtype=np.float64)
    f = base ** (-2 * i / rot)
    if scaling == "linear":
        return f / factor
    if scaling == "by_index":
        first, last = (rot * math.log(context / (2 * math.pi * t)) / (2 * math.log(base)) for t in (high, low))
        first, last = max(math.floor(first), 0), min(math.ceil(last), rot // 2 - 1)
        w = np.clip((i - first) / (max(last - first, 0.001)), 0, 1)
        return f * (1 - w) + f / factor * w
    if scaling == "by_turns":
        w = np.clip((high - context * f / (2 * math.pi)) / (high - low), 0, 1)
        return f * (1 - w) + f / factor * w
    return f


def turn(x, cos, sin, rot, interleaved, inverse=False):
    """fp32 x [..., D], cos and sin [..., rot / 2]: products and sums rounded to fp32 one by one."""
    x = x.astype(np.float32)
    y = x.copy()
    if interleaved:
        a, b = slice(0, rot, 2), slice(1, rot, 2)
    else:
        a, b = slice(0, rot // 2), slice(rot // 2, rot)
    s = -sin if inverse else sin
    with np.errstate(all="ignore"):
        y[..., a] = x[..., a] * cos - x[..., b] * s
        y[..., b] = x[..., b] * cos + x[..., a] * s
    return y


def quantize(x):
    """fp32 x [..., D] -> codes uint8 [..., D], words uint32 [...]."""
    x = x.astype(np.float32)
    zero, f15 = np.float32(0), np.float32(15)
    with np.errstate(all="ignore"):
        lo, hi = np.minimum(np.fmin.reduce(x, -1), zero), np.maximum(np.fmax.reduce(x, -1), zero)
        span = (hi - lo) * np.float32(1 / 15)
        poison = ~np.isfinite(x).all(-1) | ~np.isfinite(span)
        bits = span.view(np.uint32) & np.uint32(0xFFFFFFF0)
        none = bits < 0x00800000
        alpha = np.where(none | poison, np.uint32(0x3F800000), bits).astype(np.uint32).view(np.float32)
        inv = np.float32(1) / alpha
        theta = np.minimum(np.rint(-lo * inv), f15)[..., None]
        code = np.minimum(np.maximum(np.rint(x * inv[..., None]), -theta), f15 - theta) + theta
    dead = none | poison
    code = np.where(dead[..., None], 0, np.nan_to_num(code)).astype(np.uint8)
    word = np.where(poison, np.uint32(0x7FC00000), np.where(none, np.uint32(0), bits | np.nan_to_num(theta[..., 0]).astype(np.uint32)))
    return code, word.astype(np.uint32)


def worth(code, word):
    """fp32 values of codes [..., D] under words [...]."""
    alpha = (word & np.uint32(0xFFFFFFF0)).view(np.float32)
    theta = (word & np.uint32(15)).astype(np.int32)
    with np.errstate(all="ignore"):
        return alpha[..., None] * (code.astype(np.int32) - theta[..., None]).astype(np.float32)


class Cache:
    """The bytes of a cache, page by page as the layout has them."""

    def __init__(self, data, n_pages, heads, D, P):
        self.n, self.h, self.D, self.P = n_pages, heads, D, P
        self.data = np.ascontiguousarray(data).reshape(n_pages, heads, P * (D + 8))

    def token(self, slot):
        """(key codes, key words, value codes, value words) of one token: [heads, D] and [heads]."""
        page, at = divmod(int(slot), self.P)
        b, D, P = self.data[page], self.D, self.P
        kb = b[:, at * D // 2:(at + 1) * D // 2]
        kc = np.stack([kb & 15, kb >> 4], -1).reshape(self.h, D)
        vb = b[:, P * D // 2:P * D].reshape(self.h, P // 8, D // 4, 8, 2)[:, at // 8, :, at % 8]
        vc = np.stack([vb & 15, vb >> 4], -1).reshape(self.h, D)
        w = np.ascontiguousarray(b[:, P * D:]).view(np.uint32).reshape(self.h, P // 8, 2, 8)[:, at // 8, :, at % 8]
        return kc, w[:, 0], vc, w[:, 1]

    def put(self, slot, kc, kw, vc, vw):
        page, at = divmod(int(slot), self.P)
        b, D, P = self.data[page], self.D, self.P
        b[:, at * D // 2:(at + 1) * D // 2] = kc[:, 0::2] | kc[:, 1::2] << 4
        b[:, P * D // 2:P * D].reshape(self.h, P // 8, D // 4, 8, 2)[:, at // 8, :, at % 8] = \
            (vc[:, 0::2] | vc[:, 1::2] << 4).reshape(self.h, D // 4, 2)
        words = np.stack([kw, vw], -1).astype(np.uint32)
        for which in range(2):
            o = P * D + (at // 8) * 64 + which * 32 + (at % 8) * 4
            b[:, o:o + 4] = np.ascontiguousarray(words[:, which]).view(np.uint8).reshape(self.h, 4)

    def load(self, slots):
        """fp64 keys and values [tokens, heads, D]."""
        out = [self.token(s) for s in slots]
        if not out:
            z = np.zeros((0, self.h, self.D))
            return z, z
        k = np.stack([worth(t[0], t[1]) for t in out]).astype(np.float64)
        v = np.stack([worth(t[2], t[3]) for t in out]).astype(np.float64)
        return k, v


def attention(q, k, v, scale, causal):
    """q [n, Hq, D], k and v [m, Hkv, D] -> (output, sum p |v|, largest sum |q||k| scale), 64 bits; a row without keys is 0."""
    n, Hq, D = q.shape
    m, Hkv, _ = k.shape
    g = Hq // Hkv
    out, mass, size = np.zeros((n, Hq, D)), np.zeros((n, Hq, D)), 0.0
    for i in range(n):
        seen = min(m, max(0, m - n + i + 1)) if causal else m
        if seen == 0:
            continue
        for h in range(Hq):
            kk, vv = k[:seen, h // g], v[:seen, h // g]
            s = kk @ q[i, h] * scale
            size = max(size, float(np.max(np.abs(kk) @ np.abs(q[i, h]))) * abs(scale))
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h], mass[i, h] = p @ vv, p @ np.abs(vv)
    return out, mass, size
