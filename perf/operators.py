"""Rotary positions, the paged 4-bit key/value cache and the attention over it, as a serving program calls them.

Where `own` is false the operators run in their plain form, elementary torch operations in 32 bits; where it is true through
the library.  A cache is one uint8 buffer of pages; a page holds, for each KV head, `page` tokens as
    key codes    page x D/2 bytes      channel c of a token in byte c/2, the even channel in the low half
    value codes  page x D/2 bytes      [page/8][D/4][8 tokens] 16-bit words of four channels, the lowest in the low bits
    words        page x 8 bytes        [page/8][key, value][8 tokens] 32-bit words
and a word is the fp32 scale alpha of one token's key (or value) with its low four bits replaced by the zero point theta:
the channel is worth alpha * (code - theta).
"""
import math
import random

import torch

own = False
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # one generated token of 16 users: the queries alone, where the launch is everything
        {"name": "rope_decode_16x32x128", "kind": "rope", "T": 16, "H": 32, "D": 128, "rot": 128, "interleaved": False,
         "inverse": False, "dtype": "bf16", "packed": False, "max_pos": 8192},
        # a long prompt: query and key heads as they lie in the fused projection's rows
        {"name": "rope_prompt_8192x40x128", "kind": "rope", "T": 8192, "H": 40, "D": 128, "rot": 128, "interleaved": False,
         "inverse": False, "dtype": "bf16", "packed": True, "max_pos": 32768},
        # the gradient of a rotation of half the head, neighbouring channels in pairs, an odd number of tokens
        {"name": "rope_gradient_4099x16x64_f32", "kind": "rope", "T": 4099, "H": 16, "D": 64, "rot": 32, "interleaved": True,
         "inverse": True, "dtype": "f32", "packed": False, "max_pos": 8192},
        # a decode step of 64 users: rotate queries and keys, store keys and values
        {"name": "append_decode_64x8x128", "kind": "append", "T": 64, "Hq": 32, "Hkv": 8, "D": 128, "rot": 128,
         "interleaved": False, "dtype": "bf16", "page": 64, "max_pos": 8192, "runs": 64},
        # a prompt of 8192 tokens
        {"name": "append_prompt_8192x8x128", "kind": "append", "T": 8192, "Hq": 32, "Hkv": 8, "D": 128, "rot": 128,
         "interleaved": False, "dtype": "bf16", "page": 64, "max_pos": 32768, "runs": 1},
        # ragged prompts off the fp32 end of a quantized projection, small heads of which half is rotated, small pages
        {"name": "append_ragged_1531x4x64_f32", "kind": "append", "T": 1531, "Hq": 0, "Hkv": 4, "D": 64, "rot": 32,
         "interleaved": True, "dtype": "f32", "page": 16, "max_pos": 4096, "runs": 5},
        # one user, a short conversation: one generated token
        {"name": "decode_1x777", "kind": "attention", "B": 1, "S": 1, "L": 777, "Hq": 32, "Hkv": 8, "D": 128, "dtype": "bf16",
         "page": 16, "ragged": False},
        # a batch of 64 users with histories of up to 8192 tokens
        {"name": "decode_64x8192", "kind": "attention", "B": 64, "S": 1, "L": 8192, "Hq": 32, "Hkv": 8, "D": 128,
         "dtype": "bf16", "page": 64, "ragged": True},
        # one very long document, eight queries to each key
        {"name": "decode_1x131072", "kind": "attention", "B": 1, "S": 1, "L": 131072, "Hq": 64, "Hkv": 8, "D": 128,
         "dtype": "f16", "page": 128, "ragged": False},
        # a small fp32 model without shared heads
        {"name": "decode_32x2048_heads16x64_f32", "kind": "attention", "B": 32, "S": 1, "L": 2048, "Hq": 16, "Hkv": 16, "D": 64,
         "dtype": "f32", "page": 32, "ragged": True},
        # five drafted tokens of 16 users checked in one pass, wide heads
        {"name": "verify_16x5x4096_heads16x256", "kind": "attention", "B": 16, "S": 5, "L": 4096, "Hq": 16, "Hkv": 4, "D": 256,
         "dtype": "bf16", "page": 64, "ragged": True},
        # the last 512 tokens of four long prompts, read in pieces
        {"name": "chunk_4x512x8192", "kind": "attention", "B": 4, "S": 512, "L": 8192, "Hq": 32, "Hkv": 8, "D": 128,
         "dtype": "bf16", "page": 64, "ragged": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope", "append", "attention", "attention", "attention"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "rope":
        D = rng.choice([64, 80, 96, 128, 128, 192, 256])
        H = rng.choice([1, 2, 5, 8, 16, 32, 40])
        T = _log_int(rng, 1, 8192 * 40 * 128 // (H * D) if H * D > 2560 else 16384)
        return {"kind": kind, "T": T, "H": H, "D": D, "rot": rng.choice([D, D, D // 2, D // 4]),
                "interleaved": rng.random() < 0.4, "inverse": rng.random() < 0.3,
                "dtype": dtype if T * H * D < 1 << 23 else rng.choice(["bf16", "f16"]), "packed": rng.random() < 0.5,
                "max_pos": rng.choice([16384, 32768, 131072])}
    D = rng.choice([64, 128, 128, 256])
    page = rng.choice([16, 32, 64, 128, 256])
    if kind == "append":
        Hkv = rng.choice([1, 2, 4, 8])
        Hq = Hkv * rng.choice([0, 1, 4, 5, 8]) if Hkv * D <= 512 else Hkv * rng.choice([0, 1, 2, 4])
        T = _log_int(rng, 1, 8192 if dtype != "f32" and (2 * Hkv + 2 * Hq) * D <= 10240 else 2048)
        return {"kind": kind, "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "rot": rng.choice([D, D, D // 2]),
                "interleaved": rng.random() < 0.4, "dtype": dtype, "page": page, "max_pos": 32768,
                "runs": rng.choice([1, min(3, T), T]) if T <= 512 else rng.choice([1, 3])}
    Hkv = rng.choice([1, 2, 4, 8])
    g = rng.choice([1, 2, 4, 5, 7, 8, 16]) if Hkv <= 4 else rng.choice([1, 4, 8])
    shape = rng.choice(["decode", "decode", "verify", "chunk"])
    S = 1 if shape == "decode" else _log_int(rng, 2, 8) if shape == "verify" else _log_int(rng, 16, 512)
    L = _log_int(rng, max(S, 16), 131072 if shape == "decode" else 8192)
    # the cache's bytes, and the products, are at most the largest listed cases'
    most = min(64 * 8192 * 8 * 136 * 0.6 / (L * Hkv * (D + 8)), 4 * 512 * 8192 * 32 * 128 / (S * L * Hkv * g * D))
    B = _log_int(rng, 1, max(1, min(64, int(most))))
    return {"kind": kind, "B": B, "S": S, "L": L, "Hq": Hkv * g, "Hkv": Hkv, "D": D, "dtype": dtype, "page": page,
            "ragged": rng.random() < 0.7}


# ---- inputs -------------------------------------------------------------------------------------------------------------


def _lens(c):
    """(query tokens, keys) of every sequence: the longest whole, the others spread below it."""
    r = random.Random(1234)
    out = [(c["S"], c["L"])]
    for _ in range(c["B"] - 1):
        if c["ragged"]:
            s = c["S"] if c["S"] <= 8 else r.randint(max(1, c["S"] // 4), c["S"])
            out.append((s, r.randint(min(c["L"], max(s, c["L"] // 8)), c["L"])))
        else:
            out.append((c["S"], c["L"]))
    return out


def _table(c):
    """fp32 [max_pos, rot]: the cosines, then the sines, of position times base^(-2 i / rot)."""
    i = torch.arange(0, c["rot"], 2, dtype=torch.float64, device=DEV)
    angle = torch.arange(c["max_pos"], dtype=torch.float64, device=DEV)[:, None] * (10000.0 ** (-i / c["rot"]))[None]
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _keys_like(gen, shape):
    """Keys: a few channels much larger than the rest, some with an offset."""
    D = shape[-1]
    chan = torch.exp(0.4 * torch.randn(D, generator=gen, device=DEV))
    chan = torch.where(torch.rand(D, generator=gen, device=DEV) < 0.03, chan * 5, chan)
    off = torch.where(torch.rand(D, generator=gen, device=DEV) < 0.1, chan, torch.zeros_like(chan))
    return torch.randn(shape, generator=gen, device=DEV) * chan + off


def _regions(c, data):
    """Views of the pages' three parts: keys [pages, heads, page, D/2], values [pages, heads, page/8, D/4, 8, 2] bytes, words
    [pages, heads, page/8, 2, 8] int32."""
    P, D = c["page"], c["D"]
    n, h = data.shape[:2]
    k = data[:, :, :P * D // 2].view(n, h, P, D // 2)
    v = data[:, :, P * D // 2:P * D].view(n, h, P // 8, D // 4, 8, 2)
    w = data[:, :, P * D:].view(torch.int32).view(n, h, P // 8, 2, 8)
    return k, v, w


def _quantize(x):
    """fp32 [..., D] to codes and words, one scale and zero point for a row."""
    lo, hi = x.amin(-1, keepdim=True).clamp(max=0), x.amax(-1, keepdim=True).clamp(min=0)
    alpha = (((hi - lo) * torch.tensor(1 / 15, dtype=torch.float32, device=x.device)).view(torch.int32) & ~15).view(torch.float32)
    inv = torch.where(alpha > 0, 1.0 / alpha, torch.zeros_like(alpha))
    theta = torch.round(-lo * inv).clamp(max=15)
    code = torch.minimum(torch.maximum(torch.round(x * inv), -theta), 15 - theta) + theta
    return code.to(torch.uint8), (alpha.view(torch.int32) | theta.to(torch.int32)).squeeze(-1)


def _store(c, data, slots, k, v):
    """Quantizes fp32 k, v [T, heads, D] into the slots (page * tokens of a page + token) of the cache."""
    keys, values, words = _regions(c, data)
    page, at = slots // c["page"], slots % c["page"]
    kc, kw = _quantize(k)
    vc, vw = _quantize(v)
    keys[page, :, at] = kc[..., 0::2] | (kc[..., 1::2] << 4)
    v2 = vc[..., 0::2] | (vc[..., 1::2] << 4)
    values[page, :, at // 8, :, at % 8] = v2.view(*v2.shape[:-1], c["D"] // 4, 2)
    words[page, :, at // 8, 0, at % 8] = kw
    words[page, :, at // 8, 1, at % 8] = vw


def _load(c, data, page, at):
    """The fp32 keys and values [..., heads, D] of the tokens `at` of the pages `page`."""
    keys, values, words = _regions(c, data)

    def worth(b, w):
        code = torch.stack([b & 15, b >> 4], -1).flatten(-2).float()
        return (code - (w & 15).float()[..., None]) * (w & ~15).view(torch.float32)[..., None]

    v = values[page, :, at // 8, :, at % 8]
    return (worth(keys[page, :, at], words[page, :, at // 8, 0, at % 8]),
            worth(v.flatten(-2), words[page, :, at // 8, 1, at % 8]))


def _cache(c, n_pages):
    return torch.zeros(n_pages, c["Hkv"], c["page"] * (c["D"] + 8), dtype=torch.uint8, device=DEV)


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dt = DTYPES[c["dtype"]]
    s = {"case": c}
    if c["kind"] == "rope":
        T, H, D = c["T"], c["H"], c["D"]
        if c["packed"]:   # the heads of a row of the projection, values behind them
            x = torch.randn(T, (H + 8) * D, generator=gen, device=DEV).to(dt)[:, :H * D].view(T, H, D)
        else:
            x = torch.randn(T, H, D, generator=gen, device=DEV).to(dt)
        s["x"] = x
        if T <= 64:
            s["positions"] = torch.randint(0, c["max_pos"], (T,), generator=gen, device=DEV, dtype=torch.int32)
        else:   # a run of positions
            first = int(torch.randint(0, c["max_pos"] - T + 1, (1,), generator=gen, device=DEV))
            s["positions"] = torch.arange(first, first + T, dtype=torch.int32, device=DEV)
        s["table"] = _table(c)
        return s
    P = c["page"]
    if c["kind"] == "append":
        T, Hq, Hkv, D, runs = c["T"], c["Hq"], c["Hkv"], c["D"], c["runs"]
        # `runs` sequences of about T / runs new tokens, each behind what its last page holds already
        per = [T // runs + (i < T % runs) for i in range(runs)]
        start = torch.randint(0, c["max_pos"] - max(per), (runs,), generator=gen, device=DEV).tolist()
        need = [(a % P + n + P - 1) // P for a, n in zip(start, per)]
        pages = torch.randperm(sum(need) + 3, generator=gen, device=DEV)
        slots, positions, at = [], [], 0
        for a, n, m in zip(start, per, need):
            t = torch.arange(a % P, a % P + n, device=DEV)
            slots.append(pages[at:at + m][t // P] * P + t % P)
            positions.append(torch.arange(a, a + n, dtype=torch.int32, device=DEV))
            at += m
        s["slots"], s["positions"] = torch.cat(slots), torch.cat(positions)
        s["table"] = _table(c)
        row = torch.empty(T, (Hq + 2 * Hkv) * D, dtype=dt, device=DEV)   # rows of the fused projection
        s["q"] = row[:, :Hq * D].view(T, Hq, D) if Hq else None
        s["k"] = row[:, Hq * D:(Hq + Hkv) * D].view(T, Hkv, D)
        s["v"] = row[:, (Hq + Hkv) * D:].view(T, Hkv, D)
        if Hq:
            s["q"].copy_(torch.randn(T, Hq, D, generator=gen, device=DEV))
        s["k"].copy_(_keys_like(gen, (T, Hkv, D)))
        s["v"].copy_(0.5 * torch.randn(T, Hkv, D, generator=gen, device=DEV))
        s["data"] = _cache(c, pages.numel())
    else:
        lens = _lens(c)
        B, Hq, Hkv, D = c["B"], c["Hq"], c["Hkv"], c["D"]
        need = [(n + P - 1) // P for _, n in lens]
        pages = torch.randperm(sum(need) + 3, generator=gen, device=DEV)
        table = torch.zeros(B, max(need), dtype=torch.int32, device=DEV)
        s["data"] = _cache(c, pages.numel())
        at = 0
        for b, (_, n) in enumerate(lens):
            mine = pages[at:at + need[b]]
            at += need[b]
            table[b, :need[b]] = mine
            t = torch.arange(n, device=DEV)
            _store(c, s["data"], mine[t // P] * P + t % P, _keys_like(gen, (n, Hkv, D)),
                   0.5 * torch.randn(n, Hkv, D, generator=gen, device=DEV))
        s["pages"] = table
        s["lens"] = torch.tensor([n for _, n in lens], dtype=torch.int32, device=DEV)
        starts = [0]
        for n, _ in lens:
            starts.append(starts[-1] + n)
        s["q_starts"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
        s["q"] = torch.randn(starts[-1], Hq, D, generator=gen, device=DEV).to(dt)
    if own:   # what a program keeps beside the buffers: the cache's handle, the split's workspace
        from paper_2101_05615_amd import kv4
        s["cache"] = kv4.Cache(s["data"], Hkv, D, P)
        if c["kind"] == "attention":
            s["workspace"] = kv4.attention_workspace(s["cache"], Hq, B, max_q_len=c["S"], max_kv_len=c["L"])
    return s


# ---- the operators ------------------------------------------------------------------------------------------------------


def _rotate(c, x, positions, table, inverse=False):
    """fp32 x [T, heads, D] with its first `rot` channels rotated."""
    r = c["rot"]
    cs = table[positions.long()][:, None]
    cos, sin = cs[..., :r // 2], cs[..., r // 2:]
    if inverse:
        sin = -sin
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, x[..., r:]], -1)


def _attention(c, s):
    q, P, D = s["q"], c["page"], c["D"]
    B, S, L, Hq, Hkv = c["B"], c["S"], c["L"], c["Hq"], c["Hkv"]
    token = torch.arange(L, device=DEV)
    k, v = _load(c, s["data"], s["pages"][:, token // P].long(), (token % P).expand(B, L))      # [B, L, Hkv, D]
    starts, lens = s["q_starts"].long(), s["lens"].long()
    n = starts[1:] - starts[:-1]
    i = torch.arange(S, device=DEV)
    rows = (starts[:-1, None] + i).clamp(max=q.shape[0] - 1)
    x = q[rows].float().view(B, S, Hkv, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D)
    score = torch.matmul(x, k.permute(0, 2, 3, 1).contiguous()) * (1 / math.sqrt(D))
    score = score.view(B, Hkv, S, Hq // Hkv, L)
    last = (lens - n)[:, None] + i            # the newest key that query i may see
    seen = (token <= last[..., None]) & (token < lens[:, None, None])
    score = score.masked_fill(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    o = torch.matmul(p.view(B, Hkv, -1, L), v.permute(0, 2, 1, 3).contiguous())
    o = o.view(B, Hkv, S, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(B, S, Hq, D)
    t = torch.arange(q.shape[0], device=DEV)
    b = torch.bucketize(t, starts[1:], right=True)
    return o[b, t - starts[b]].to(q.dtype)


def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2101_05615_amd import kv4
        if c["kind"] == "rope":
            return kv4.rope(s["x"], s["positions"], s["table"], interleaved=c["interleaved"], inverse=c["inverse"])
        if c["kind"] == "append":
            q = kv4.append(s["cache"], s["k"], s["v"], s["slots"], positions=s["positions"], table=s["table"],
                           interleaved=c["interleaved"], q=s["q"])
            k, v = kv4.read(s["cache"], s["slots"], dtype=s["k"].dtype)
            return {"q": q, "k": k, "v": v}
        return kv4.attention(s["q"], s["cache"], s["pages"], s["lens"], q_starts=s["q_starts"], max_q_len=c["S"],
                             max_kv_len=c["L"], workspace=s["workspace"])
    if c["kind"] == "rope":
        return _rotate(c, s["x"].float(), s["positions"], s["table"], c["inverse"]).to(s["x"].dtype)
    if c["kind"] == "append":
        q = None if s["q"] is None else _rotate(c, s["q"].float(), s["positions"], s["table"]).to(s["q"].dtype)
        _store(c, s["data"], s["slots"], _rotate(c, s["k"].float(), s["positions"], s["table"]), s["v"].float())
        k, v = _load(c, s["data"], s["slots"] // c["page"], s["slots"] % c["page"])   # what the cache holds now
        return {"q": q, "k": k.to(s["k"].dtype), "v": v.to(s["v"].dtype)}
    return _attention(c, s)


def work(case):
    c, e = case, BYTES[case["dtype"]]
    if c["kind"] == "rope":
        n = c["T"] * c["H"] * c["D"]
        return {"bytes": 2 * n * e + c["T"] * c["rot"] * 4 + 4 * c["T"], "flops": 3 * c["T"] * c["H"] * c["rot"]}
    if c["kind"] == "append":
        T, kv, q = c["T"], c["T"] * c["Hkv"] * c["D"], c["T"] * c["Hq"] * c["D"]
        held = 2 * T * c["Hkv"] * (c["D"] // 2 + 4)   # written, and read back
        return {"bytes": 2 * q * e + 2 * kv * e + 2 * held + 2 * kv * e + T * (c["rot"] * 4 + 20),
                "flops": 3 * T * (c["Hq"] + c["Hkv"]) * c["rot"] + 2 * kv * 8}
    keys = sum(n for _, n in _lens(c))
    q = sum(n for n, _ in _lens(c)) * c["Hq"] * c["D"]
    pairs = sum(n * m - n * (n - 1) // 2 for n, m in _lens(c))
    return {"bytes": keys * c["Hkv"] * (c["D"] + 8) + 2 * q * e + 4 * (keys // c["page"] + 2 * c["B"]),
            "flops": 4 * pairs * c["Hq"] * c["D"]}


# ---- the same in 64 bits, from the definitions --------------------------------------------------------------------------


def _turn64(c, x, positions, table, sign):
    """Each pair of channels as a complex number times cos + i sin."""
    x = x.double()
    r, h = c["rot"], c["rot"] // 2
    first = torch.arange(h, device=DEV) * (2 if c["interleaved"] else 1)
    second = first + (1 if c["interleaved"] else h)
    cs = table.double()[positions.long()]
    turn = torch.complex(cs[:, :h], sign * cs[:, h:])[:, None]
    z = torch.complex(x[..., first], x[..., second]) * turn
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _held64(x):
    """What 4 bits keep of x [..., D]: the nearest of 16 evenly spaced values, zero among them, from its least to its largest."""
    x = x.double()
    lo = torch.minimum(x.min(-1, keepdim=True)[0], torch.zeros((), dtype=torch.float64, device=DEV))
    hi = torch.maximum(x.max(-1, keepdim=True)[0], torch.zeros((), dtype=torch.float64, device=DEV))
    step = (hi - lo) / 15
    bits = 2.0 ** (19 - torch.floor(torch.log2(step)))           # a scale has 20 significant bits
    step = torch.floor(step * bits) / bits
    zero = torch.clamp(torch.round(-lo / step), 0, 15)
    return (torch.clamp(torch.round(x / step) + zero, 0, 15) - zero) * step


def _token64(c, data, page, at):
    """The keys and values of one sequence's tokens: [heads, tokens, D] in 64 bits, from the bytes of the pages."""
    P, D = c["page"], c["D"]
    blk = data[page].long()                                       # [tokens, heads, bytes]
    n, h = blk.shape[:2]
    ch = torch.arange(D, device=DEV)
    at = at[:, None]

    def pick(idx):
        return torch.gather(blk, 2, idx[:, None].expand(n, h, idx.shape[1]))

    def word(which):
        b = pick(P * D + (at // 8) * 64 + which * 32 + (at % 8) * 4 + torch.arange(4, device=DEV))
        w = (b * (256 ** torch.arange(4, device=DEV))).sum(-1)
        theta = w % 16
        mant = (w % (1 << 23)) - theta
        expo = w // (1 << 23)                                     # (scales are positive and normal)
        return theta.double()[..., None], ((1 + mant.double() / (1 << 23)) * 2.0 ** (expo.double() - 127))[..., None]

    kb = pick(at * (D // 2) + ch // 2)
    vb = pick(P * D // 2 + (at // 8) * (4 * D) + (ch // 4) * 16 + (at % 8) * 2 + (ch % 4) // 2)
    out = []
    for b, (theta, alpha) in ((kb, word(0)), (vb, word(1))):
        code = torch.where(ch % 2 == 0, b % 16, b // 16).double()
        out.append((alpha * (code - theta)).transpose(0, 1))
    return out


def exact(case, seed):
    c = dict(case)
    s = prepare(c, seed)
    if c["kind"] == "rope":
        return _turn64(c, s["x"], s["positions"], s["table"], -1.0 if c["inverse"] else 1.0)
    if c["kind"] == "append":
        q = None if s["q"] is None else _turn64(c, s["q"], s["positions"], s["table"], 1.0)
        return {"q": q, "k": _held64(_turn64(c, s["k"], s["positions"], s["table"], 1.0)), "v": _held64(s["v"])}
    P, D, g = c["page"], c["D"], c["Hq"] // c["Hkv"]
    out, at = [], 0
    for b, (n, m) in enumerate(_lens(c)):
        x = s["q"][at:at + n].double().view(n, c["Hkv"], g, D)
        at += n
        best = torch.full((n, c["Hkv"], g), -math.inf, dtype=torch.float64, device=DEV)
        total, acc = torch.zeros_like(best), torch.zeros_like(x)
        limit = m - n + torch.arange(n, device=DEV)
        for first in range(0, m, 8192):                           # a piece of the keys at a time
            t = torch.arange(first, min(m, first + 8192), device=DEV)
            k, v = _token64(c, s["data"], s["pages"][b].long()[t // P], t % P)
            sc = torch.matmul(x.permute(1, 0, 2, 3).reshape(c["Hkv"], n * g, D), k.transpose(1, 2).contiguous()) / math.sqrt(D)
            sc = sc.view(c["Hkv"], n, g, -1).permute(1, 0, 2, 3)
            sc = torch.where((t[None] <= limit[:, None])[:, None, None], sc, torch.full((), -math.inf, dtype=torch.float64, device=DEV))
            new = torch.maximum(best, sc.max(-1)[0])
            keep = torch.where(best == new, torch.ones_like(best), torch.exp(best - new))
            e = torch.exp(sc - torch.where(new == -math.inf, torch.zeros_like(new), new)[..., None])
            total = total * keep + e.sum(-1)
            pv = torch.matmul(e.permute(1, 0, 2, 3).reshape(c["Hkv"], n * g, -1), v)
            acc = acc * keep[..., None] + pv.view(c["Hkv"], n, g, D).permute(1, 0, 2, 3)
            best = new
        out.append((acc / torch.where(total == 0, torch.ones_like(total), total)[..., None]).reshape(n, c["Hq"], D))
    return torch.cat(out)
