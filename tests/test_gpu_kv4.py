"""Rotary positions, the 4-bit cache and its attention on the GPU.

Rotation, quantization and read-back are fixed sequences of fp32 operations: compared with ==.  The attention is compared with
64 bits over the values that the cache holds.  Its bound per output element, with P = sum_j p_j |v_j| of that element:
    u_out |o|                       the output's type rounds once
  + u_p P                           probabilities times value scale in fp16 (2^-11), or two fp16 (2^-21) for fp32 results
  + 2 (D + 16) 2^-24 S P            scores: D fp32 additions and a few products on sum |q||k| scale <= S (fp32 queries: 2^-22 S more)
  + (L + 64) 2^-24 P                sums over L keys, exponentials, the joining of partial results
  + L 2^-28 max |v|                 fp16's smallest step, 2^-25 of numbers held times 2^4 under the largest, value scales that differ
"""
import math

import numpy as np
import pytest

import kv4_reference as ref
from gpu_util import assert_same, say

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]
U = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2101_05615_amd import kv4
    return kv4, torch, torch.device("cuda:0")


def f32(t):
    return t.float().cpu().numpy()


def strided(torch, dev, shape, dtype, gap, offset=0):
    """A [tokens, heads, D] view whose rows lie `gap` elements further apart than they need to, garbage between."""
    T, H, D = shape
    store = torch.full((T * (H * D + gap) + offset + 8,), 77.0, dtype=dtype, device=dev)
    return store[offset:offset + T * (H * D + gap)].view(T, H * D + gap)[:, :H * D].view(T, H, D), store


# ---- positions -----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("kw", [dict(), dict(base=500000.0), dict(scaling="linear", factor=4.0),
                                dict(scaling="by_index", factor=16.0, low=1.0, high=32.0, context=4096.0, magnitude=1.2772588722239782),
                                dict(scaling="by_turns", base=500000.0, factor=8.0, low=1.0, high=4.0, context=8192.0)])
@pytest.mark.parametrize("rot", [2, 32, 128, 256])
def test_table(env, kw, rot):
    kv4, torch, dev = env
    n = 40000
    got = kv4.rope_table(n, rot, device=dev, **kw).cpu().numpy()
    mag = kw.get("magnitude", 1.0)
    f = ref.frequencies(rot, kw.get("base", 10000.0), **{k: v for k, v in kw.items() if k not in ("base", "magnitude")})
    angle = np.arange(n)[:, None] * f[None]
    want = np.concatenate([np.cos(angle), np.sin(angle)], 1) * mag
    assert got.shape == (n, rot)
    # one rounding to fp32 below 2 (2^-24 at most below 1), and an angle below 4e4 whose frequency is 2^-51 off at most
    assert np.max(np.abs(got - want)) <= 2.0 ** -24 * max(1.0, 2.0 * (mag > 1)) + 4e4 * 2.0 ** -51


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,D,rot", [(1, 1, 64, 64), (7, 3, 128, 128), (33, 5, 128, 32), (300, 2, 256, 256), (5, 4, 80, 20),
                                       (9, 3, 96, 96), (2, 2, 2, 2), (13, 2, 35, 6), (70000, 1, 16, 16), (11, 40, 1024, 256)])
def test_rope(env, dtype, interleaved, T, H, D, rot):
    kv4, torch, dev = env
    dt = getattr(torch, dtype)
    rng = np.random.default_rng(T * 1000 + D + rot)
    table = kv4.rope_table(5000, rot, device=dev)
    pos = rng.integers(0, 5000, T).astype(np.int32)
    x, _ = strided(torch, dev, (T, H, D), dt, gap=5, offset=3)
    x.copy_(torch.from_numpy(rng.standard_normal((T, H, D)).astype(np.float32)).to(dev))
    before = f32(x)
    tab = table.cpu().numpy()[pos][:, None]
    p = torch.from_numpy(pos).to(dev)
    for inverse in (False, True):
        want = ref.turn(before, tab[..., :rot // 2], tab[..., rot // 2:], rot, interleaved, inverse)
        want = torch.from_numpy(want).to(dt).float().numpy()
        got = kv4.rope(x, p, table, interleaved=interleaved, inverse=inverse)
        assert_same(f32(got), want, "new output")
        out, store = strided(torch, dev, (T, H, D), dt, gap=9, offset=1)
        kv4.rope(x, p, table, interleaved=interleaved, inverse=inverse, out=out)
        assert_same(f32(out), want, "strided output")
        rest = torch.cat([store[:1], store[1:1 + T * (H * D + 9)].view(T, -1)[:, H * D:].flatten(), store[1 + T * (H * D + 9):]])
        assert (rest == 77.0).all(), "elements between the rows were written"
    y, _ = strided(torch, dev, (T, H, D), dt, gap=5, offset=3)
    y.copy_(x)
    assert kv4.rope(y, p, table, interleaved=interleaved, out=y) is y
    assert_same(f32(y), f32(kv4.rope(x, p, table, interleaved=interleaved)), "in place")


def test_rope_heads_in_any_order(env):
    kv4, torch, dev = env
    table = kv4.rope_table(100, 32, device=dev)
    x = torch.randn(6, 9, 64, device=dev)       # [heads, tokens, D]
    pos = torch.arange(9, dtype=torch.int32, device=dev)
    got = kv4.rope(x.transpose(0, 1), pos, table)
    want = kv4.rope(x.transpose(0, 1).contiguous(), pos, table)
    assert torch.equal(got, want)
    flipped = torch.empty(9, 6, 64, device=dev).transpose(0, 1).contiguous().transpose(0, 1)
    kv4.rope(x.transpose(0, 1), pos, table, out=flipped)
    assert torch.equal(flipped, want)


def test_rope_positions_outside_the_table_and_no_tokens(env):
    kv4, torch, dev = env
    for D, rot in ((64, 32), (20, 10)):
        table = kv4.rope_table(50, rot, device=dev)
        x = torch.randn(4, 2, D, device=dev)
        y = kv4.rope(x, torch.tensor([0, -1, 50, 49], dtype=torch.int32, device=dev), table)
        assert torch.isnan(y[1:3, :, :rot]).all() and torch.equal(y[:, :, rot:], x[:, :, rot:])
        assert torch.isfinite(y[[0, 3]]).all() and torch.equal(y[0], x[0])
        assert kv4.rope(x[:0], torch.empty(0, dtype=torch.int32, device=dev), table).shape == (0, 2, D)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(64, 32), (20, 12)])
def test_rope_gradient(env, interleaved, D, rot):
    """inverse=True is the gradient: against the rotation's matrix in 64 bits, and against differences of the forward pass."""
    kv4, torch, dev = env
    rng = np.random.default_rng(5)
    table = kv4.rope_table(900, rot, device=dev)
    pos = torch.tensor([777, 3], dtype=torch.int32, device=dev)
    g = torch.from_numpy(rng.standard_normal((2, 1, D)).astype(np.float32)).to(dev)
    grad = kv4.rope(g, pos, table, interleaved=interleaved, inverse=True).double().cpu().numpy()
    eye = torch.eye(D, device=dev)[:, None]                                  # one token per channel
    for t in range(2):
        at = pos[t].expand(D).contiguous()
        m = kv4.rope(eye, at, table, interleaved=interleaved)[:, 0].double().cpu().numpy()      # row i: the image of e_i
        want = m @ g[t, 0].double().cpu().numpy()
        # two products and a sum in fp32, on both sides
        assert np.max(np.abs(grad[t, 0] - want)) <= 4 * 2.0 ** -24 * float(g.abs().max()) * 2
        x = torch.from_numpy(rng.standard_normal((1, 1, D)).astype(np.float32)).to(dev).expand(D, 1, D)
        h = 2.0 ** -3
        hi = kv4.rope((x + h * eye).contiguous(), at, table, interleaved=interleaved).double()
        lo = kv4.rope((x - h * eye).contiguous(), at, table, interleaved=interleaved).double()
        diff = ((hi - lo) / (2 * h) * g[t].double()).sum((1, 2)).cpu().numpy()
        # x + h loses 2^-24 |x|, the rotation as much again; / 2 h, times |g|, two channels that move and D - 2 that do not
        assert np.max(np.abs(diff - want)) <= 16 * 2.0 ** -24 * 6 / (2 * h) * float(g.abs().max())


# ---- the cache -----------------------------------------------------------------------------------------------------------


def rows(rng, shape):
    """Channels of several sizes, with rows of zeros, of one sign, of one value, tiny, huge and nearly constant."""
    x = (rng.standard_normal(shape) * np.exp(rng.standard_normal(shape[-1]))).astype(np.float32)
    flat = x.reshape(-1, shape[-1])
    special = [lambda r: r * 0, np.abs, lambda r: -np.abs(r), lambda r: r * 0 + 3.7, lambda r: r * 1e-37, lambda r: r * np.float32(1e-42),
               lambda r: r * 1e30, lambda r: np.abs(r) * 1e-4 + 100, lambda r: np.where(np.arange(r.size) == 5, -9.0, 0.0)]
    for i, f in enumerate(special):
        if i + 1 < len(flat):
            flat[i + 1] = f(flat[i + 1])
    return x


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("P,Hkv,D,T,rot,interleaved", [(16, 1, 64, 1, 64, False), (16, 2, 64, 37, 32, True), (32, 8, 128, 5, 128, False),
                                                       (64, 3, 128, 700, 32, False), (256, 1, 256, 301, 256, True),
                                                       (128, 2, 256, 40, 16, False), (64, 4, 128, 2500, 128, True)])
def test_append_and_read(env, dtype, P, Hkv, D, T, rot, interleaved):
    kv4, torch, dev = env
    dt = getattr(torch, dtype)
    rng = np.random.default_rng(T + D + P)
    n_pages = (T + P - 1) // P + 3
    cache = kv4.new_cache(n_pages, Hkv, D, P, device=dev)
    cache.data.random_(0, 256)
    model = ref.Cache(cache.data.cpu().numpy().copy(), n_pages, Hkv, D, P)
    table = kv4.rope_table(3000, rot, device=dev)
    slots = rng.permutation(n_pages * P)[:T] if T > 64 else np.arange(11, 11 + T)
    slots = slots.astype(np.int64)
    if T > 20:
        slots[3], slots[17] = -1, n_pages * P        # padding, and a slot behind the cache
    pos = rng.integers(0, 3000, T).astype(np.int32)
    k, _ = strided(torch, dev, (T, Hkv, D), dt, gap=3, offset=1)
    v, _ = strided(torch, dev, (T, Hkv, D), dt, gap=11)
    k.copy_(torch.from_numpy(rows(rng, (T, Hkv, D))))
    v.copy_(torch.from_numpy(rows(rng, (T, Hkv, D))))
    q = torch.randn(T, 5, D, device=dev).to(dt)
    tab = table.cpu().numpy()[pos][:, None]
    cos, sin = tab[..., :rot // 2], tab[..., rot // 2:]
    p, s = torch.from_numpy(pos).to(dev), torch.from_numpy(slots).to(dev)
    got_q = kv4.append(cache, k, v, s, positions=p, table=table, interleaved=interleaved, q=q)
    assert_same(f32(got_q), torch.from_numpy(ref.turn(f32(q), cos, sin, rot, interleaved)).to(dt).float().numpy(), "queries")
    kc, kw = ref.quantize(ref.turn(f32(k), cos, sin, rot, interleaved))
    vc, vw = ref.quantize(f32(v))
    held = (slots >= 0) & (slots < n_pages * P)
    for t in np.nonzero(held)[0]:
        model.put(slots[t], kc[t], kw[t], vc[t], vw[t])
    assert_same(cache.data.cpu().numpy(), model.data.reshape(-1), "the cache's bytes")
    for out in TYPES:
        ok, ov = kv4.read(cache, s, dtype=getattr(torch, out))
        for o, c, w in ((ok, kc, kw), (ov, vc, vw)):
            want = np.where(held[:, None, None], ref.worth(c, w), np.float32(0))
            got, want = f32(o), torch.from_numpy(want).to(getattr(torch, out)).float().numpy()
            assert np.array_equal(np.isnan(got), np.isnan(want))          # (an infinity among fp16 inputs: a poisoned head)
            assert_same(np.where(np.isnan(got), 0, got), np.where(np.isnan(want), 0, want), f"read back as {out}")
    # queries in place, and keys that are rotated already
    q2 = q.clone()
    assert kv4.append(cache, k, v, s, positions=p, table=table, interleaved=interleaved, q=q2, q_out=q2) is q2
    assert torch.equal(q2, got_q)
    assert kv4.append(cache, k, v, s) is None
    kc, kw = ref.quantize(f32(k))
    for t in np.nonzero(held)[0]:
        model.put(slots[t], kc[t], kw[t], vc[t], vw[t])
    assert_same(cache.data.cpu().numpy(), model.data.reshape(-1), "unrotated keys")


def test_append_poison(env):
    """Infinities, NaN, ranges beyond fp32 and positions outside the table: the scale is NaN, the neighbours are as they were."""
    kv4, torch, dev = env
    cache = kv4.new_cache(2, 2, 64, 16, device=dev)
    cache.data.zero_()
    table = kv4.rope_table(10, 64, device=dev)
    k, v = torch.randn(8, 2, 64, device=dev), torch.randn(8, 2, 64, device=dev)
    k[1, 0, 5], k[2, 1, 63], v[3, 0, 0], v[4, 1, 17] = math.inf, math.nan, -math.inf, math.nan
    v[5, 0, 3], v[5, 0, 4] = 3e38, -3e38
    pos = torch.tensor([0, 0, 0, 0, 0, 0, 10, -1], dtype=torch.int32, device=dev)
    slots = torch.arange(9, 17, device=dev)
    kv4.append(cache, k, v, slots, positions=pos, table=table)
    rk, rv = kv4.read(cache, slots)
    nk, nv = torch.isnan(rk).all(-1).cpu(), torch.isnan(rv).all(-1).cpu()
    assert nk.nonzero().tolist() == [[1, 0], [2, 1], [6, 0], [6, 1], [7, 0], [7, 1]]
    assert nv.nonzero().tolist() == [[3, 0], [4, 1], [5, 0]]
    assert torch.isfinite(rk[~nk.to(dev)]).all() and torch.isfinite(rv[~nv.to(dev)]).all()
    model = ref.Cache(cache.data.cpu().numpy(), 2, 2, 64, 16)
    assert model.token(10)[1][0] == 0x7FC00000 and not model.token(10)[0][0].any()


def test_append_nothing(env):
    kv4, torch, dev = env
    cache = kv4.new_cache(1, 2, 64, 16, device=dev)
    cache.data.fill_(0x5A)
    e = torch.empty(0, 2, 64, device=dev)
    slots = torch.empty(0, dtype=torch.int64, device=dev)
    kv4.append(cache, e, e, slots)
    assert kv4.read(cache, slots)[0].shape == (0, 2, 64)
    x = torch.randn(5, 2, 64, device=dev)
    kv4.append(cache, x, x, torch.full((5,), -1, dtype=torch.int64, device=dev))
    assert (cache.data == 0x5A).all()


# ---- attention -----------------------------------------------------------------------------------------------------------


class Batch:
    """Sequences in a cache of garbage: pages in a random order, page-table entries behind a sequence's end invalid."""

    def __init__(self, env, lens, Hq, Hkv, D, P, dtype, seed=0, q_lens=None, spread=1.0):
        kv4, torch, dev = env
        rng = np.random.default_rng(seed)
        self.env, self.lens, self.D, self.dtype = env, lens, D, dtype
        self.q_lens = [1] * len(lens) if q_lens is None else q_lens
        need = [(m + P - 1) // P for m in lens]
        self.n_pages = sum(need) + 2
        self.cache = kv4.new_cache(self.n_pages, Hkv, D, P, device=dev)
        self.cache.data.random_(0, 256)          # unused tokens: any bits, NaN scales among them
        order, W = rng.permutation(self.n_pages), max(max(need), 1)
        table = np.full((len(lens), W + 1), -7, np.int32)
        self.slots, at = [], 0
        for b, m in enumerate(lens):
            mine = order[at:at + need[b]]
            at += need[b]
            table[b, :need[b]] = mine
            t = np.arange(m)
            self.slots.append((mine[t // P] * P + t % P).astype(np.int64) if m else np.zeros(0, np.int64))
            if m:
                k = rng.standard_normal((m, Hkv, D)) * np.exp(0.5 * rng.standard_normal((m, Hkv, 1))) * spread
                v = rng.standard_normal((m, Hkv, D)) * np.exp(1.5 * rng.standard_normal((m, Hkv, 1)))
                kv4.append(self.cache, torch.from_numpy(k.astype(np.float32)).to(dev), torch.from_numpy(v.astype(np.float32)).to(dev),
                           torch.from_numpy(self.slots[-1]).to(dev))
        self.pages = torch.from_numpy(table).to(dev)
        self.kv_lens = torch.tensor(lens, dtype=torch.int32, device=dev)
        starts = np.concatenate([[0], np.cumsum(self.q_lens)]).astype(np.int32)
        self.starts = starts
        self.q_starts = torch.from_numpy(starts).to(dev) if q_lens is not None else None
        dt = getattr(torch, dtype)
        self.q, _ = strided(torch, dev, (int(starts[-1]), Hq, D), dt, gap=7, offset=1)
        self.q.copy_(torch.from_numpy(rng.standard_normal((int(starts[-1]), Hq, D)).astype(np.float32)))

    def run(self, workspace=True, out=None, **kw):
        kv4, torch, dev = self.env
        mq = max(max(self.q_lens), 1)
        mk = kw.pop("max_kv_len", max(self.lens))
        ws = kv4.attention_workspace(self.cache, self.q.shape[1], len(self.lens), max_q_len=mq, max_kv_len=mk) if workspace is True else workspace
        return kv4.attention(self.q, self.cache, self.pages, self.kv_lens, q_starts=self.q_starts, max_q_len=mq, max_kv_len=mk,
                             workspace=ws, out=out, **kw)

    def check(self, got, causal=True, scale=None):
        q, got = f32(self.q).astype(np.float64), f32(got).astype(np.float64)
        scale = 1 / math.sqrt(self.D) if scale is None else scale
        model = ref.Cache(self.cache.data.cpu().numpy(), self.n_pages, self.cache.kv_heads, self.D, self.cache.page_tokens)
        u_p = 2.0 ** -21 if self.dtype == "float32" else 2.0 ** -11
        worst = 0.0
        for b, m in enumerate(self.lens):
            rows_ = slice(int(self.starts[b]), int(self.starts[b + 1]))
            k, v = model.load(self.slots[b])
            want, mass, size = ref.attention(q[rows_], k, v, scale, causal)
            if not want.size:
                continue
            big = float(np.abs(v).max()) if m else 0.0
            e = u_p + 2 * (self.D + 16) * 2.0 ** -24 * size + (2.0 ** -21 * size if self.dtype == "float32" else 0) + (m + 64) * 2.0 ** -24
            bound = U[self.dtype] * np.abs(want) + e * mass * (1 + U[self.dtype]) + m * 2.0 ** -28 * big + 2.0 ** -25 * (self.dtype == "float16")
            off = np.abs(got[rows_] - want)
            assert np.isfinite(got[rows_]).all(), f"sequence {b}"
            ratio = float(np.max(off / np.maximum(bound, 1e-300))) if (bound > 0).any() else float(np.max(off))
            worst = max(worst, ratio)
            assert (off <= bound).all(), f"sequence {b} of {m} keys: {ratio:.2f} times the bound at {np.argwhere(off > bound)[0]}"
        say(f"largest error: {worst:.2f} of the bound")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,Hq,Hkv,P", [(64, 2, 2, 16), (64, 16, 1, 64), (128, 8, 2, 16), (128, 32, 8, 32), (128, 5, 1, 256),
                                        (256, 4, 4, 16), (256, 14, 2, 128)])
def test_one_token(env, dtype, D, Hq, Hkv, P):
    b = Batch(env, [1, 2, 15, 16, 17, 0, 31, 32, 33, 64, 127, 130, 300], Hq, Hkv, D, P, dtype, seed=D + Hq)
    b.check(b.run())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,Hq,Hkv,P", [(64, 4, 1, 32), (128, 8, 1, 16), (128, 16, 2, 128), (256, 2, 1, 64)])
def test_keys_split_over_workgroups(env, dtype, D, Hq, Hkv, P):
    kv4, torch, dev = env
    b = Batch(env, [5000, 1, 257, 4097, 0, 2049], Hq, Hkv, D, P, dtype, seed=D)
    ws = kv4.attention_workspace(b.cache, Hq, 6, max_kv_len=5000)
    assert ws is not None
    got = b.run(ws)
    b.check(got)
    again = b.run(ws)
    assert torch.equal(got, again), "the result depends on the order in which workgroups arrive"
    assert (ws[:65536] == 0).all(), "the counters are not as a next call needs them"
    b.check(b.run(None))                               # no workspace: not split


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D,Hq,Hkv,P", [(64, 4, 2, 16), (128, 8, 2, 64), (128, 7, 1, 32), (256, 4, 2, 16)])
def test_several_queries(env, dtype, causal, D, Hq, Hkv, P):
    b = Batch(env, [5, 40, 3, 100, 0, 77, 256, 31], Hq, Hkv, D, P, dtype, seed=D + Hq, q_lens=[5, 3, 9, 1, 2, 0, 70, 31])
    b.check(b.run(causal=causal), causal=causal)       # (sequences 2 and 4 have queries before the first key: rows of 0)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_many_queries_split(env, dtype):
    b = Batch(env, [1500, 900, 130], 4, 1, 128, 32, dtype, seed=9, q_lens=[40, 33, 130])
    b.check(b.run())
    b.check(b.run(None))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,Hq,Hkv", [(64, 10, 5), (128, 6, 3), (256, 2, 1)])
def test_keys_dealt_over_a_batch(env, dtype, D, Hq, Hkv):
    """More sequences than a wave has lanes, of all lengths, some without queries or keys: keys are dealt by what is there."""
    kv4, torch, dev = env
    rng = np.random.default_rng(D)
    lens = [int(x) for x in np.exp(rng.uniform(0, math.log(1500), 70))] + [0, 1500, 1281, 1]
    q_lens = [int(x) for x in rng.integers(0, 6, 70)] + [3, 140, 33, 2]
    b = Batch(env, lens, Hq, Hkv, D, 32, dtype, seed=D, q_lens=q_lens)
    ws = kv4.attention_workspace(b.cache, Hq, len(lens), max_q_len=140, max_kv_len=1500)
    assert ws is not None
    got = b.run(ws)
    b.check(got)
    assert torch.equal(got, b.run(ws)) and (ws[:65536] == 0).all()
    b.check(b.run(ws, causal=False), causal=False)
    short = [min(m, 700) for m in lens]                # other lengths in the same workspace
    b.lens, b.slots = short, [s[:m] for s, m in zip(b.slots, short)]
    b.kv_lens.copy_(torch.tensor(short, dtype=torch.int32))
    b.check(b.run(ws, max_kv_len=1500))


def test_rows_without_keys_are_zero(env):
    kv4, torch, dev = env
    b = Batch(env, [0, 2], 4, 2, 64, 16, "float32", q_lens=[3, 4])
    got = b.run()
    assert (got[:3] == 0).all() and (got[3:5] == 0).all() and (got[5:] != 0).any(-1).all()


def test_strides_bounds_and_rows_of_nobody(env):
    """Output rows apart from each other and out of order; queries that no sequence has, and lengths above the bound."""
    kv4, torch, dev = env
    b = Batch(env, [50, 70], 8, 2, 128, 16, "bfloat16", seed=3, q_lens=[2, 3])
    want = b.run()
    store = torch.full((8, 5, 200), 5.0, dtype=torch.bfloat16, device=dev)
    out = store[:, :, 3:131].transpose(0, 1)
    b.run(out=out)
    assert torch.equal(out, want) and (store[:, :, :3] == 5).all() and (store[:, :, 131:] == 5).all()
    # queries 0 and 4 belong to nobody
    b.q_starts = torch.tensor([1, 3, 4], dtype=torch.int32, device=dev)
    out = torch.full((5, 8, 128), 5.0, dtype=torch.bfloat16, device=dev)
    b.run(out=out)
    assert (out[0] == 5).all() and (out[4] == 5).all() and (out[1:4] != 5).any()
    # a length above max_kv_len counts as max_kv_len, one below zero as zero
    b = Batch(env, [60, 60], 8, 2, 128, 16, "bfloat16", seed=4)
    b.kv_lens = torch.tensor([1 << 30, -5], dtype=torch.int32, device=dev)
    got = b.run(max_kv_len=40)
    b.kv_lens = torch.tensor([40, 0], dtype=torch.int32, device=dev)
    assert torch.equal(got, b.run(max_kv_len=40)) and (got[1] == 0).all()
    # pages that are none of the cache's read as page 0
    wild = b.pages.clone()
    wild[0, 1] = 1 << 30
    b.pages = wild
    got = b.run(max_kv_len=40)
    wild[0, 1] = 0
    assert torch.equal(got, b.run(max_kv_len=40))


@pytest.mark.parametrize("dtype", TYPES)
def test_scores_of_all_sizes(env, dtype):
    """Scores that dwarf each other (one key takes all), equal scores, queries of zero, scales of both signs and extreme queries."""
    kv4, torch, dev = env
    b = Batch(env, [700, 90], 4, 2, 128, 32, dtype, seed=12, spread=30.0)
    b.check(b.run())
    b.check(b.run(scale=-0.02), scale=-0.02)
    b.check(b.run(scale=0.0), scale=0.0)
    big = 2.0 ** (100 if dtype != "float16" else 10)
    b.q.mul_(big)
    b.check(b.run(scale=0.05 / big), scale=0.05 / big)
    b.q.mul_(2.0 ** (-180 if dtype != "float16" else -20))
    b.check(b.run())
    b.q.zero_()
    b.check(b.run())


@pytest.mark.parametrize("q_lens", [[1], [3], [20]])
def test_scores_far_below_zero(env, q_lens):
    """All scores between -4e6 and -4e8: the least negative one takes all."""
    kv4, torch, dev = env
    b = Batch(env, [100], 4, 2, 64, 16, "float32", seed=2, q_lens=q_lens)
    slots = torch.from_numpy(b.slots[0]).to(dev)
    k = (torch.arange(100, device=dev).flip(0) + 1.0)[:, None, None].repeat(1, 2, 64)
    v = torch.randn(100, 2, 64, device=dev)
    kv4.append(b.cache, k, v, slots)
    b.q.fill_(-(2.0 ** 16))
    got, held = b.run(scale=1.0), kv4.read(b.cache, slots)[1]
    for i in range(q_lens[0]):
        want = held[99 - (q_lens[0] - 1 - i)].repeat_interleave(2, 0)
        assert ((got[i] - want).abs() <= 2.0 ** -20 * want.abs()).all()


@pytest.mark.parametrize("D,n_q", [(64, 1), (64, 20), (128, 1), (128, 40), (256, 1), (256, 40)])
@pytest.mark.parametrize("n", [1, 64])
def test_keys_all_alike_give_their_value(env, D, n_q, n):
    """n tokens alike: each has a probability of 1 / n whatever the score, and an fp32 result is the value they hold.  Over 2^16 rows
    of scores of all fractions: 2^-22 of the two fp16 numbers for a probability and 2^-24 n each for its two sums."""
    kv4, torch, dev = env
    Hq, Hkv, P, B = 16, 2, 64, 4096 // n_q
    g = torch.Generator(device=dev).manual_seed(D + n_q)
    cache = kv4.new_cache(B, Hkv, D, P, device=dev)
    k, v = (torch.randn(B, Hkv, D, device=dev, generator=g).repeat_interleave(n, 0) for _ in range(2))
    kv4.append(cache, k, v, (torch.arange(B, device=dev)[:, None] * P + torch.arange(n, device=dev)).flatten())
    held = kv4.read(cache, torch.arange(B, device=dev) * P)[1].repeat_interleave(n_q, 0).repeat_interleave(Hq // Hkv, 1)
    q = torch.randn(B * n_q, Hq, D, device=dev, generator=g)
    got = kv4.attention(q, cache, torch.arange(B, device=dev, dtype=torch.int32)[:, None], torch.full((B,), n, dtype=torch.int32, device=dev),
                        q_starts=torch.arange(B + 1, dtype=torch.int32, device=dev) * n_q, max_q_len=n_q, max_kv_len=n, causal=False)
    off = ((got - held).abs() / held.abs().clamp(min=1e-30)).max()
    assert off <= 2.0 ** -21 + 2 * (n + 4) * 2.0 ** -24, f"{float(off):.1e}"


def test_value_scales_of_all_sizes(env):
    """Values 2^60 apart between tokens: the small ones count where the large ones have no weight."""
    kv4, torch, dev = env
    b = Batch(env, [200], 2, 1, 64, 16, "float32", seed=2)
    s = torch.from_numpy(b.slots[0]).to(dev)
    k, v = kv4.read(b.cache, s)
    v *= torch.exp2(torch.arange(200, device=dev) * 0.3)[:, None, None]
    kv4.append(b.cache, k, v, s)
    b.check(b.run())
    kv4.append(b.cache, k, v.flip(0).contiguous(), s)
    b.check(b.run())
    kv4.append(b.cache, k, v * 2.0 ** -120, s)
    b.check(b.run())


def test_poisoned_tokens(env):
    """A NaN key or value reaches the rows that see it, and no others."""
    kv4, torch, dev = env
    for at, which in ((30, "k"), (30, "v"), (63, "k"), (63, "v")):
        b = Batch(env, [64, 64], 4, 2, 64, 16, "float32", seed=6, q_lens=[40, 1])
        k, v = kv4.read(b.cache, torch.from_numpy(b.slots[0][at:at + 1]).to(dev))
        (k if which == "k" else v)[0, 1, 3] = float("nan")
        kv4.append(b.cache, k, v, torch.from_numpy(b.slots[0][at:at + 1]).to(dev))
        got = b.run()
        nan = torch.isnan(got).all(-1).cpu().numpy()
        want = np.zeros((41, 4), bool)
        want[max(0, at - 24):40, 2:] = True            # query i sees keys up to 24 + i
        assert (nan == want).all() and np.isfinite(f32(got)[~want]).all(), (at, which)
    b.q[5, 1, 0], b.q[6, 0, 1] = float("inf"), float("nan")
    nan = torch.isnan(b.run()).all(-1).cpu()
    assert nan[5, 1] and nan[6, 0] and not nan[5, 0] and not nan[6, 1]


def test_offsets_beyond_32_bits(env):
    """A cache of more than 4 GiB, attended to and read at its far end."""
    kv4, torch, dev = env
    P, Hkv, D = 256, 8, 256
    n = (9 << 30) // 2 // kv4.cache_bytes(1, Hkv, D, P) + 5
    cache = kv4.new_cache(n, Hkv, D, P, device=dev)
    assert cache.data.numel() > 1 << 32
    k, v = torch.randn(300, Hkv, D, device=dev), torch.randn(300, Hkv, D, device=dev)
    far, near = torch.tensor([[n - 1, n - 3]], dtype=torch.int32, device=dev), torch.tensor([[1, 0]], dtype=torch.int32, device=dev)
    t = torch.arange(300, device=dev)
    q = torch.randn(1, 16, D, device=dev)
    lens = torch.tensor([300], dtype=torch.int32, device=dev)
    got = []
    for pages in (far, near):
        kv4.append(cache, k, v, pages[0].long()[t // P] * P + t % P)
        got.append((kv4.attention(q, cache, pages, lens),) + kv4.read(cache, pages[0].long()[t // P] * P + t % P))
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_other_streams_and_graphs(env):
    """A step recorded into a graph, replayed with new inputs and other work between the replays, against the eager calls."""
    kv4, torch, dev = env
    b = Batch(env, [900, 40, 333], 8, 2, 128, 16, "bfloat16", seed=1)
    table = kv4.rope_table(2000, 128, device=dev)
    ws = kv4.attention_workspace(b.cache, 8, 3, max_kv_len=900)
    assert ws is not None
    k, v = (torch.randn(3, 2, 128, device=dev).bfloat16() for _ in range(2))
    q = torch.randn(3, 8, 128, device=dev).bfloat16()
    slots = torch.tensor([int(s[-1]) for s in b.slots], device=dev)
    pos = (b.kv_lens - 1).contiguous()
    out, turned = torch.empty_like(q), torch.empty_like(q)

    def step():
        kv4.append(b.cache, k, v, slots, positions=pos, table=table, q=q, q_out=turned)
        kv4.attention(turned, b.cache, b.pages, b.kv_lens, max_kv_len=900, workspace=ws, out=out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(3):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, device=dev))
        out.fill_(9)
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        torch.randn(1000, 1000, device=dev).sum()
        out.fill_(9)
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out)
