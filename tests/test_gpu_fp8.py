"""8-bit floats with a scale per block of 128 on the GPU: codes and scales bit for bit, products, the gated block, its backward pass and the
weights' gradient against 64 bits, at the sizes and values where they can go wrong.  Bounds: fp8_reference.py."""
import numpy as np
import pytest

import fp8_reference as ref
from gpu_util import assert_same, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2101_05615_amd import fp8
    return fp8, torch, torch.device("cuda:0")


DTYPES = ["float32", "bfloat16", "float16"]


def tensor(torch, dev, x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dev).to(getattr(torch, dtype))


def f64(t):
    return t.detach().double().cpu().numpy()


def inputs(rng, T, K, scale=1.0):
    chan = np.exp(0.4 * rng.standard_normal(K)) * np.where(rng.random(K) < 0.02, 8.0, 1.0)
    return scale * rng.standard_normal((T, K)) * chan


def weights(rng, K, N):
    return rng.standard_normal((K, N)) / np.sqrt(K)


def wide_rows(torch, x, pad=3, lead=1):
    """x as a view of wider rows that starts off any alignment but its type's."""
    store = torch.full((x.shape[0], x.shape[1] + pad + lead), 7.0, dtype=x.dtype, device=x.device)
    view = store[:, lead:lead + x.shape[1]]
    view.copy_(x)
    return view


def check_blocks(got, x, what):
    codes, byte = ref.quantize(x)
    g_codes, g_byte = got.codes.cpu().numpy(), got.scales.cpu().numpy()
    assert_same(g_byte[:, :byte.shape[1]], byte, f"{what}: scales")
    fine = np.repeat(byte != 255, 128, 1)
    zero = (codes & 127) == 0                                # (the sign of a zero is not fixed)
    assert_same(np.where(fine & ~(zero & ((g_codes & 127) == 0)), g_codes, 0), np.where(fine & ~zero, codes, 0), f"{what}: codes")


# ---- quantize, dequantize ---------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,K", [(1, 1), (3, 127), (5, 128), (7, 129), (2, 512), (9, 1000), (4, 4097), (300, 640)])
def test_quantize(env, dtype, T, K):
    fp8, torch, dev = env
    rng = np.random.default_rng(T * 1000 + K)
    x = tensor(torch, dev, inputs(rng, T, K), dtype)
    say(f"quantize {T} x {K} {dtype}")
    for view in (x, wide_rows(torch, x)):
        q = fp8.quantize(view)
        torch.cuda.synchronize()
        check_blocks(q, f64(x), f"{T}x{K} {dtype}")
        back = fp8.dequantize(q, dtype=torch.float32)
        assert_same(f64(back), ref.held(f64(x)), "values")
        out = wide_rows(torch, torch.zeros_like(x))
        fp8.dequantize(q, dtype=x.dtype, out=out)
        assert_same(f64(out), f64(back.to(x.dtype)), "values in a view")


def test_quantize_every_bfloat16(env):
    """Every finite bfloat16 in a block of its own size class: ties, subnormals, the ends of the range."""
    fp8, torch, dev = env
    bits = torch.arange(0, 0x7f80, dtype=torch.int32, device=dev)
    x = (bits << 16).view(torch.float32).to(torch.bfloat16)
    x = torch.cat([x, -x])                                   # neighbours in size share a block
    x = torch.nn.functional.pad(x, (0, -x.numel() % 1024)).view(-1, 1024)
    check_blocks(fp8.quantize(x), f64(x), "all")
    with np.errstate(over="ignore"):                         # (sizes from 2^128 - 2^123 on round to 2^128, which fp32 has not)
        assert_same(f64(fp8.dequantize(fp8.quantize(x))), ref.held(f64(x)).astype(np.float32), "values")


@pytest.mark.parametrize("top", [2.0 ** -149, 2.0 ** -130, 2.0 ** -126, 2.0 ** -119, 2.0 ** -118, 2.0 ** -9, 1.0, 448.0, 1.75, 1.7500001, 3.5,
                                 3.0e38, 3.4028234663852886e38])
def test_quantize_ends(env, top):
    fp8, torch, dev = env
    rng = np.random.default_rng(5)
    x = (rng.uniform(-1, 1, (4, 300)) * top).astype(np.float32)
    x[:, [3, 200, 299]] = np.float32(top)
    x[2, 128:256] = 0.0
    x[3, 128:256] = -0.0
    t = torch.from_numpy(x).to(dev)
    check_blocks(fp8.quantize(t), x.astype(np.float64), f"largest {top}")
    with np.errstate(over="ignore"):
        assert_same(f64(fp8.dequantize(fp8.quantize(t))), ref.held(x.astype(np.float64)).astype(np.float32), "values")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_not_finite(env, dtype, bad):
    """One such number makes its block NaN, and nothing else."""
    fp8, torch, dev = env
    rng = np.random.default_rng(6)
    x = inputs(rng, 5, 400)
    x[1, 200] = bad
    x[4, 399] = bad
    t = tensor(torch, dev, x, dtype)
    want = f64(t)
    want[1, 128:256] = want[4, 384:] = np.nan
    got = f64(fp8.dequantize(fp8.quantize(t)))
    assert np.array_equal(np.isnan(got), np.isnan(want))
    check_blocks(fp8.quantize(t), f64(t), "not finite")
    b = weights(rng, 400, 96)
    b[130, 70] = bad
    w = fp8.pack(tensor(torch, dev, b, dtype))
    y = f64(fp8.matmul(t, w))                                # every product takes the block of B in
    assert np.isnan(y).all()
    w = fp8.pack(tensor(torch, dev, weights(rng, 400, 300), dtype))
    for T in (5, 40, 200):                                   # each kernel
        big = torch.cat([t, t[:1].expand(T - 5, -1)]) if T > 5 else t
        y = np.isnan(f64(fp8.matmul(big.contiguous(), w)))
        assert y[[1, 4]].all() and not np.delete(y, [1, 4], 0).any()


# ---- weights ----------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K,N,order", [(1, 1, "rows"), (128, 256, "rows"), (130, 300, "rows"), (129, 127, "columns"), (515, 70, "columns"),
                                       (257, 520, "strided")])
@pytest.mark.parametrize("gated", [False, True])
def test_pack(env, dtype, K, N, order, gated):
    fp8, torch, dev = env
    rng = np.random.default_rng(K + N)
    say(f"pack {K} x {N} {order} {dtype} gated {gated}")

    def make():
        b = tensor(torch, dev, inputs(rng, K, N), dtype)
        if order == "columns":
            return b.t().contiguous().t()
        if order == "strided":
            store = torch.zeros(K, 2 * N + 1, dtype=b.dtype, device=dev)
            store[:, 1::2] = b
            return store[:, 1::2]
        return b

    mats = [make(), make()] if gated else [make()]
    w = (fp8.pack_gated if gated else fp8.pack)(*mats, transposed=True)
    torch.cuda.synchronize()
    for which, (b, (codes, byte)) in enumerate(zip(mats, ref.unpack(w.data.cpu().numpy(), K, N, gated))):
        want, scale = ref.quantize_weight(f64(b))
        got = codes[:K, :N]
        zero = ((want | got) & 127) == 0
        assert_same(np.where(zero, 0, got), np.where(zero, 0, want), f"codes {which}")
        assert not (codes[K:] & 127).any() and not (codes[:, N:] & 127).any()
        assert_same(byte[:, :N], np.repeat(scale, 128, 1)[:, :N], f"scales {which}")
    t = w.transposed
    assert t.n == K and t.k == (2 * ref.up(N, 128) if gated else N) and not t.gated
    (t_codes, t_byte), = ref.unpack(t.data.cpu().numpy(), t.k, t.n, False)
    for which, b in enumerate(mats):
        want, scale = ref.quantize_weight(f64(b))
        at = which * ref.up(N, 128)
        got = t_codes[at:at + N, :K].T
        zero = ((want | got) & 127) == 0
        assert_same(np.where(zero, 0, got), np.where(zero, 0, want), f"transposed codes {which}")
        assert_same(t_byte[at // 128:at // 128 + scale.shape[1], :K], np.repeat(scale, 128, 0)[:K].T, f"transposed scales {which}")
        assert not (t_codes[at + N:at + ref.up(N, 128)] & 127).any()
    assert not (t_codes[:, K:] & 127).any()


# ---- products ---------------------------------------------------------------------------------------------------------------


def compare(got, want, bound, what):
    off = np.abs(got - want)
    assert off.shape == bound.shape
    bad = ~(off <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off, worst {np.nanmax(off / bound):.2f} of the bound, at {np.argwhere(bad)[0]}"


PRODUCTS = [(1, 128, 256), (1, 1, 1), (2, 300, 70), (16, 2000, 520), (17, 640, 300), (33, 1100, 130), (64, 257, 65), (65, 128, 256), (100, 1000, 100),
            (203, 2740, 410), (300, 513, 700), (1, 8192, 64), (40, 9000, 100)]


@pytest.mark.parametrize("T,K,N", PRODUCTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_matmul(env, T, K, N, dtype):
    fp8, torch, dev = env
    rng = np.random.default_rng(T * 7 + K)
    say(f"matmul {T} x {K} x {N} {dtype}")
    x, b = tensor(torch, dev, inputs(rng, T, K), dtype), tensor(torch, dev, weights(rng, K, N), dtype)
    bias = torch.randn(N, device=dev)
    w, ws = fp8.pack(b), fp8.workspace(dev)
    x8, b8 = ref.held(f64(x)), ref.held_weight(f64(b))
    want, mass = x8 @ b8 + f64(bias), np.abs(x8) @ np.abs(b8) + np.abs(f64(bias))
    results = {}
    for out_dtype in DTYPES:
        o = getattr(torch, out_dtype)
        for wide in (None, False):
            bound = ref.sum_bound(mass, K, wide is None and out_dtype == "float32" or T <= 64)
            bound = bound + ref.rounding(np.abs(want) + bound, out_dtype)
            y = fp8.matmul(x, w, bias=bias, dtype=o, workspace=ws, wide_sums=wide)
            compare(f64(y), want, bound, f"{out_dtype} wide {wide}")
            compare(f64(fp8.matmul(x, w, bias=bias, dtype=o, wide_sums=wide)), want, bound, "without a workspace")
            assert torch.equal(y, fp8.matmul(fp8.quantize(x), w, bias=bias, dtype=o, workspace=ws, wide_sums=wide)), "from 8 bits"
            results[out_dtype, wide] = y
    # views of wider rows, in and out, which is left as it was outside
    store = torch.full((T, N + 5), 3.0, dtype=x.dtype, device=dev)
    y = fp8.matmul(wide_rows(torch, x), w, bias=bias, out=store[:, 2:2 + N], workspace=ws)
    assert torch.equal(y, results[dtype, None]) and (store[:, :2] == 3).all() and (store[:, 2 + N:] == 3).all()
    assert (ws[:fp8.COUNTER_BYTES] == 0).all()


GATED = [(1, 128, 128), (3, 300, 70), (16, 1500, 300), (33, 700, 129), (64, 128, 640), (70, 1000, 200), (150, 513, 260)]


@pytest.mark.parametrize("T,K,F", GATED)
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
def test_gated(env, T, K, F, act):
    fp8, torch, dev = env
    rng = np.random.default_rng(T * 3 + K)
    say(f"gated {T} x {K} x {F} {act}")
    dtype = DTYPES[T % 3]
    x = tensor(torch, dev, inputs(rng, T, K), dtype)
    gate, up = (tensor(torch, dev, weights(rng, K, F) * s, dtype) for s in (2.0, 1.0))
    w, ws = fp8.pack_gated(gate, up), fp8.workspace(dev)
    x8, g8, u8 = ref.held(f64(x)), ref.held_weight(f64(gate)), ref.held_weight(f64(up))
    g, u = x8 @ g8, x8 @ u8
    h, h_err = gated_reference(act, g, u, *(ref.sum_bound(np.abs(x8) @ np.abs(b), K, True) for b in (g8, u8)))
    _, h_err8 = gated_reference(act, g, u, *(ref.sum_bound(np.abs(x8) @ np.abs(b), K, False) for b in (g8, u8)))
    for out_dtype in DTYPES:
        y = fp8.gated(x, w, act, dtype=getattr(torch, out_dtype), workspace=ws)
        err = h_err if T <= 64 or out_dtype == "float32" else h_err8
        compare(f64(y), h, err + ref.rounding(np.abs(h) + err, out_dtype), out_dtype)
        compare(f64(fp8.gated(fp8.quantize(x), w, act, dtype=getattr(torch, out_dtype))), h, err + ref.rounding(np.abs(h) + err, out_dtype), "alone")
    # in 8 bits
    for wide in (False, True):
        q = fp8.gated(x, w, act, out=fp8.new_blocks(T, F, dev), workspace=ws, wide_sums=wide)
        compare(f64(fp8.dequantize(q)), ref.held(h), ref.held_bound(h, h_err if wide else h_err8) + 1e-300, f"8 bits, wide {wide}")
        codes = q.codes.cpu().numpy()
        assert not (codes[:, F:] & 127).any(), "behind the last column"
    assert (ws[:fp8.COUNTER_BYTES] == 0).all()


def gated_reference(act, g, u, g_err, u_err):
    """h and how far it may be off: errors of g and u through the slope (at most 1.2 for these activations), and fp32 arithmetic on top:
    some ten roundings, and an exponential whose argument z carries 2^-23 |z|, so a weight e^-z (1 + |z| 2^-23)."""
    a, _ = ref.activate(act, g)
    a_err = 1.2 * g_err + 2.0 ** -20 * np.abs(a) * (1 + np.abs(g)) + 2.0 ** -22 * np.abs(g)
    return a * u, a_err * (np.abs(u) + u_err) + np.abs(a) * u_err + 2.0 ** -23 * np.abs(a * u)


@pytest.mark.parametrize("T,K,F", [(1, 128, 128), (5, 300, 70), (33, 500, 129), (70, 260, 300), (260, 384, 200)])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
def test_gated_backward(env, T, K, F, act):
    fp8, torch, dev = env
    rng = np.random.default_rng(T * 3 + K)
    say(f"gated backward {T} x {K} x {F} {act}")
    dtype = DTYPES[T % 3]
    x, dh = tensor(torch, dev, inputs(rng, T, K), dtype), tensor(torch, dev, inputs(rng, T, F, 0.01), dtype)
    gate, up = (tensor(torch, dev, weights(rng, K, F) * s, dtype) for s in (2.0, 1.0))
    w, ws = fp8.pack_gated(gate, up), fp8.workspace(dev)
    xq = fp8.quantize(x)
    dgu, dgu8, h8 = fp8.gated_backward(xq, w, wide_rows(torch, dh), act, workspace=ws)
    again = fp8.gated_backward(xq, w, dh, act, workspace=ws)
    assert torch.equal(dgu, again[0]) and torch.equal(dgu8.codes, again[1].codes) and torch.equal(h8.codes, again[2].codes)
    x8, g8, u8, d = ref.held(f64(x)), ref.held_weight(f64(gate)), ref.held_weight(f64(up)), f64(dh)
    g, u = x8 @ g8, x8 @ u8
    g_err, u_err = (ref.sum_bound(np.abs(x8) @ np.abs(b), K, False) for b in (g8, u8))
    a, slope = ref.activate(act, g)
    h, h_err = gated_reference(act, g, u, g_err, u_err)
    a_err = 1.2 * g_err + 2.0 ** -20 * np.abs(a) * (1 + np.abs(g)) + 2.0 ** -22 * np.abs(g)
    # the slope's own slope is at most 1.2 for these activations (the jump of relu at 0: none of g is that near, or the slope is free there)
    s_err = 1.2 * g_err + 2.0 ** -19 * (1 + np.abs(g))
    if act == "relu":
        s_err = np.where(np.abs(g) <= g_err, 1.0, 0.0)
    dg, dg_err = d * u * slope, np.abs(d) * (u_err * (np.abs(slope) + s_err) + np.abs(u) * s_err) + 2.0 ** -22 * np.abs(d * u * slope)
    du, du_err = d * a, np.abs(d) * a_err + 2.0 ** -23 * np.abs(d * a)
    Fp = ref.up(F, 128)
    got = f64(dgu)
    for i, (want, err) in enumerate(((dg, dg_err), (du, du_err))):
        compare(got[:, i, :F], want, err + ref.rounding(np.abs(want) + err, "bfloat16"), f"dgu {i}")
        assert not got[:, i, F:].any()
        part = f64(fp8.dequantize(dgu8))[:, i * Fp:(i + 1) * Fp]
        compare(part[:, :F], ref.held(want), ref.held_bound(want, err) + 1e-300, f"dgu8 {i}")
        assert not part[:, F:].any()
    compare(f64(fp8.dequantize(h8)), ref.held(h), ref.held_bound(h, h_err) + 1e-300, "h8")
    # what the forward kernel writes, bit for bit
    q = fp8.gated(xq, w, act, out=fp8.new_blocks(T, F, dev), workspace=ws)
    assert torch.equal(q.codes, h8.codes) and torch.equal(q.scales[:, :Fp // 128], h8.scales[:, :Fp // 128])


@pytest.mark.parametrize("T,K,N", [(1, 1, 1), (3, 200, 70), (64, 128, 128), (65, 129, 131), (300, 260, 300), (1000, 100, 515), (2100, 300, 64)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_weight_gradient(env, T, K, N, dtype):
    fp8, torch, dev = env
    rng = np.random.default_rng(T + K)
    say(f"weight gradient {T} x {K} x {N} {dtype}")
    x, dy = tensor(torch, dev, inputs(rng, T, K), dtype), tensor(torch, dev, inputs(rng, T, N, 0.01), dtype)
    x8, d, ws = ref.held(f64(x)), f64(dy), fp8.workspace(dev)
    want, mass = x8.T @ d, np.abs(x8).T @ np.abs(d)
    xq = fp8.quantize(x)
    # every bit of dy: parts of 8 bits, the last one's rounding at most 2^-24 of dy (fp32; subnormal parts: 2^-133)
    bound = mass * ((64 + 32 + T / 16 * 3) * 2.0 ** -23) + np.abs(x8).sum(0)[:, None] * 2.0 ** -130
    for out_dtype in DTYPES:
        o = getattr(torch, out_dtype)
        y = fp8.weight_gradient(xq, dy, dtype=o, workspace=ws)
        compare(f64(y), want, bound + ref.rounding(np.abs(want) + bound, out_dtype), out_dtype)
        compare(f64(fp8.weight_gradient(xq, wide_rows(torch, dy), dtype=o)), want, bound + ref.rounding(np.abs(want) + bound, out_dtype), "view")
        store = torch.full((K, N + 5), 3.0, dtype=o, device=dev)
        assert torch.equal(fp8.weight_gradient(xq, dy, out=store[:, 2:2 + N], workspace=ws), y)
        assert (store[:, :2] == 3).all() and (store[:, 2 + N:] == 3).all()
    assert (ws[:fp8.COUNTER_BYTES] == 0).all()


@pytest.mark.parametrize("T,K,N", [(70, 200, 130), (2100, 140, 200), (65, 2600, 2700)])
def test_weight_gradients_of_a_pair(env, T, K, N):
    """Two in one launch: the same bits as one by one where the tiles are the same, and always within the bound."""
    fp8, torch, dev = env
    rng = np.random.default_rng(T)
    x = tensor(torch, dev, inputs(rng, T, K), "bfloat16")
    both = torch.from_numpy(inputs(rng, T, 2 * N, 0.01)).to(dev).to(torch.bfloat16)
    dys, xq, ws = (both[:, :N], both[:, N:]), fp8.quantize(x), fp8.workspace(dev)
    got = fp8.weight_gradient(xq, dys, dtype=torch.float32, workspace=ws)
    x8 = ref.held(f64(x))
    for y, dy in zip(got, dys):
        want, mass = x8.T @ f64(dy), np.abs(x8).T @ np.abs(f64(dy))
        bound = mass * ((64 + 32 + T / 16 * 3) * 2.0 ** -23)
        compare(f64(y), want, bound + ref.rounding(np.abs(want) + bound, "float32"), "pair")
    if T == 70:
        assert all(torch.equal(y, fp8.weight_gradient(xq, dy, dtype=torch.float32)) for y, dy in zip(got, dys))


def test_weight_gradient_infinite(env):
    """An infinity in dy stays one (the parts of a number are finite but the first)."""
    fp8, torch, dev = env
    for dtype in DTYPES:
        x = torch.ones(20, 130, device=dev)
        dy = torch.ones(20, 40, device=dev, dtype=getattr(torch, dtype))
        dy[3, 5], dy[4, 6], dy[5, 7] = np.inf, -np.inf, np.nan
        y = fp8.weight_gradient(fp8.quantize(x), dy, dtype=torch.float32)
        assert (y[:, 5] == np.inf).all() and (y[:, 6] == -np.inf).all() and torch.isnan(y[:, 7]).all()
        rest = [i for i in range(40) if i not in (5, 6, 7)]
        assert (y[:, rest] == 20).all()


# ---- together ---------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("T", [1, 16, 17, 64, 65, 200])
@pytest.mark.parametrize("dtype", DTYPES)
def test_feed_forward(env, T, dtype):
    fp8, torch, dev = env
    rng = np.random.default_rng(T)
    K, F = 384, 650
    say(f"feed forward {T} {dtype}")
    x = tensor(torch, dev, inputs(rng, T, K), dtype)
    gate, up, down = (tensor(torch, dev, weights(rng, *s), dtype) for s in ((K, F), (K, F), (F, K)))
    ws = fp8.workspace(dev)
    y = fp8.feed_forward(x, fp8.pack_gated(gate, up), fp8.pack(down), workspace=ws)
    x8, g8, u8, d8 = ref.held(f64(x)), *(ref.held_weight(f64(b)) for b in (gate, up, down))
    wide = T <= 64 or dtype == "float32"
    h, h_err = gated_reference("silu", x8 @ g8, x8 @ u8, *(ref.sum_bound(np.abs(x8) @ np.abs(b), K, wide) for b in (g8, u8)))
    h8, h8_err = ref.held(h), ref.held_bound(h, h_err)
    want = h8 @ d8
    bound = h8_err @ np.abs(d8) + ref.sum_bound((np.abs(h8) + h8_err) @ np.abs(d8), F, wide or dtype == "float32")
    compare(f64(y), want, bound + ref.rounding(np.abs(want) + bound, dtype), "feed forward")
    h, h_err = gated_reference("silu", x8 @ g8, x8 @ u8, *(ref.sum_bound(np.abs(x8) @ np.abs(b), K, True) for b in (g8, u8)))
    h8, h8_err = ref.held(h), ref.held_bound(h, h_err)
    bound = h8_err @ np.abs(d8) + ref.sum_bound((np.abs(h8) + h8_err) @ np.abs(d8), F, True)
    y = fp8.feed_forward(x, fp8.pack_gated(gate, up), fp8.pack(down), workspace=ws, wide_sums=True)
    compare(f64(y), h8 @ d8, bound + ref.rounding(np.abs(h8 @ d8) + bound, dtype), "wide sums")


@pytest.mark.parametrize("T", [1, 5, 70, 300])
@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_gradients(env, T, dtype):
    fp8, torch, dev = env
    rng = np.random.default_rng(T)
    K, N = 300, 200
    say(f"linear {T} {dtype}")
    x, b = (tensor(torch, dev, v, dtype).requires_grad_() for v in (inputs(rng, T, K), weights(rng, K, N)))
    ws = fp8.workspace(dev)
    y = fp8.linear(x, b, workspace=ws)
    dy = tensor(torch, dev, inputs(rng, T, N, 0.01), dtype)
    dx, db = torch.autograd.grad(y, (x, b), dy)
    x8, b8, d8 = ref.held(f64(x)), ref.held_weight(f64(b)), ref.held(f64(dy))
    wide = T <= 64 or dtype == "float32"
    for got, p, q, n, w in ((y, x8, b8, K, wide), (dx, d8, b8.T, N, wide), (db, x8.T, f64(dy), T, True)):
        want, bound = p @ q, ref.sum_bound(np.abs(p) @ np.abs(q), max(n, 3 * 128 * T // 16 if got is db else 0), w)
        compare(f64(got), want, bound + ref.rounding(np.abs(want) + bound, dtype), "linear")


def test_linear_against_differences(env):
    """On numbers that 8 bits hold, the product is linear: differences are exact."""
    fp8, torch, dev = env
    rng = np.random.default_rng(1)
    T, K, N = 6, 260, 140
    x = rng.integers(-8, 9, (T, K)).astype(np.float32)
    b = rng.integers(-8, 9, (K, N)).astype(np.float32)
    dy = rng.integers(-8, 9, (T, N)).astype(np.float32)
    x[:, ::128] = 15
    b[::128, ::128] = 15
    dy[:, ::128] = 15
    t = lambda v: torch.from_numpy(v).to(dev)  # noqa: E731
    xt, bt = t(x).requires_grad_(), t(b).requires_grad_()
    dx, db = torch.autograd.grad(fp8.linear(xt, bt), (xt, bt), t(dy))
    for _ in range(10):
        i, j = rng.integers(T), rng.integers(1, 128)
        step = np.zeros_like(x)
        step[i, j] = 1.0
        up, down = (f64(fp8.linear(t(x + s * step), t(b))) for s in (1, -1))
        assert ((up - down) / 2 * dy).sum() == f64(dx)[i, j]
        i, j = rng.integers(1, 128), rng.integers(1, 128)
        step = np.zeros_like(b)
        step[i, j] = 1.0
        up, down = (f64(fp8.linear(t(x), t(b + s * step))) for s in (1, -1))
        assert ((up - down) / 2 * dy).sum() == f64(db)[i, j]


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
def test_gated_against_differences(env, act):
    """Central differences of the gated kernel's fp32 result, one channel of x moved between numbers that 8 bits hold.  The error of a
    difference is (step of g or u)^3 / 6 of the third derivative (at most 3 for a(g) u with |u| up to 3), fp32 results 2^-22 of their
    size; relu where no g changes sign."""
    fp8, torch, dev = env
    rng = np.random.default_rng(2)
    T, K, F = 4, 128, 96
    x = np.where(rng.random((T, K)) < 0.5, 1.25, -1.25).astype(np.float32)
    x[:, 0] = 1.75
    gate, up = ((rng.standard_normal((K, F)) * 2.0 ** -4).astype(np.float32) for _ in range(2))
    t = lambda v: torch.from_numpy(v).to(dev)  # noqa: E731
    w = fp8.pack_gated(t(gate), t(up), transposed=True)
    g8, u8 = ref.held_weight(gate.astype(np.float64)), ref.held_weight(up.astype(np.float64))
    dh = np.zeros((T, F), np.float32)
    for c in range(1, 12):
        step = np.zeros_like(x)
        step[:, c] = 0.125
        high, low = (f64(fp8.gated(t(x + s * step), w, act, dtype=torch.float32)) for s in (1, -1))
        slope = (high - low) / 0.25                           # of every h in channel c
        dh[:] = 1.0
        dgu = f64(fp8.gated_backward(fp8.quantize(t(x)), w, t(dh), act)[0])[:, :, :F]
        want = dgu[:, 0] * g8[c] + dgu[:, 1] * u8[c]
        d = 0.125 * (np.abs(g8[c]) + np.abs(u8[c]))
        u = np.abs(x.astype(np.float64) @ u8) + d
        bound = d ** 3 / 0.125 * (1 + u) + 2.0 ** -8 * (np.abs(dgu[:, 0] * g8[c]) + np.abs(dgu[:, 1] * u8[c])) + (1 + np.abs(high)) * 2.0 ** -20 / 0.25
        # sums on the 8-bit cores in the backward pass
        bound = bound + 2.0 ** -9 * (1 + u) * (np.abs(x).astype(np.float64) @ (np.abs(g8) + np.abs(u8))) * (np.abs(g8[c]) + np.abs(u8[c]))
        calm = np.abs(x.astype(np.float64) @ g8) > 2 * d if act == "relu" else np.ones_like(bound, bool)
        assert calm.mean() > 0.5
        compare(np.where(calm, slope, 0), np.where(calm, want, 0), bound, act)


@pytest.mark.parametrize("T,act,dtype", [(1, "silu", "bfloat16"), (70, "gelu", "float16"), (130, "gelu_tanh", "float32"), (300, "relu", "bfloat16")])
def test_gated_mlp_gradients(env, T, act, dtype):
    """The whole block against the composition of its parts, which are compared with 64 bits above: every gradient bit for bit."""
    fp8, torch, dev = env
    rng = np.random.default_rng(T)
    K, F = 260, 390
    say(f"gated mlp {T} {act} {dtype}")
    x = tensor(torch, dev, inputs(rng, T, K), dtype).requires_grad_()
    gate, up, down = (tensor(torch, dev, weights(rng, *s), dtype).requires_grad_() for s in ((K, F), (K, F), (F, K)))
    dy = tensor(torch, dev, inputs(rng, T, K, 0.01), dtype)
    y = fp8.gated_mlp(x, gate, up, down, act)
    grads = torch.autograd.grad(y, (x, gate, up, down), dy)
    with torch.no_grad():
        w_in, w_out, xq = fp8.pack_gated(gate, up, transposed=True), fp8.pack(down, transposed=True), fp8.quantize(x)
        h8 = fp8.gated(xq, w_in, act, out=fp8.new_blocks(T, F, dev))
        assert torch.equal(y, fp8.matmul(h8, w_out, dtype=x.dtype))
        dh = fp8.matmul(fp8.quantize(dy), w_out.transposed, dtype=torch.float32, wide_sums=False)
        dgu, dgu8, _ = fp8.gated_backward(xq, w_in, dh, act)
        want = (fp8.matmul(dgu8, w_in.transposed, dtype=x.dtype), fp8.weight_gradient(xq, dgu[:, 0, :F], dtype=x.dtype),
                fp8.weight_gradient(xq, dgu[:, 1, :F], dtype=x.dtype), fp8.weight_gradient(h8, dy, dtype=x.dtype))
    for got, expect in zip(grads, want):
        assert got.dtype == expect.dtype and torch.equal(got, expect)
    # and the gradient of x against the formula: dgu in 8 bits times the weights
    d8 = f64(fp8.dequantize(dgu8))
    g8, u8 = ref.held_weight(f64(gate)), ref.held_weight(f64(up))
    Fp = ref.up(F, 128)
    formula = d8[:, :F] @ g8.T + d8[:, Fp:Fp + F] @ u8.T
    mass = np.abs(d8[:, :F]) @ np.abs(g8.T) + np.abs(d8[:, Fp:Fp + F]) @ np.abs(u8.T)
    bound = ref.sum_bound(mass, 2 * Fp, T <= 64 or dtype == "float32")
    compare(f64(grads[0]), formula, bound + ref.rounding(np.abs(formula) + bound, dtype), "dx")


def test_some_gradients_only(env):
    fp8, torch, dev = env
    x, gate, up, down = (torch.randn(s, device=dev) for s in ((20, 130), (130, 70), (130, 70), (70, 130)))
    full = [t.clone().requires_grad_() for t in (x, gate, up, down)]
    want = torch.autograd.grad(fp8.gated_mlp(*full).sum(), full)
    for i in range(4):
        some = [t.clone().requires_grad_(j == i) for j, t in enumerate((x, gate, up, down))]
        got, = torch.autograd.grad(fp8.gated_mlp(*some).sum(), some[i])
        assert torch.equal(got, want[i])
    assert not fp8.gated_mlp(x, gate, up, down).requires_grad
    b = torch.randn(130, 50, device=dev)
    for flags in ((True, False), (False, True)):
        xs, bs = x.clone().requires_grad_(flags[0]), b.clone().requires_grad_(flags[1])
        torch.autograd.grad(fp8.linear(xs, bs).sum(), [t for t in (xs, bs) if t.requires_grad])


def test_no_tokens(env):
    fp8, torch, dev = env
    gate, up, down = (torch.randn(s, device=dev).requires_grad_() for s in ((130, 70), (130, 70), (70, 130)))
    x = torch.randn(0, 130, device=dev).requires_grad_()
    y = fp8.gated_mlp(x, gate, up, down)
    assert y.shape == (0, 130)
    grads = torch.autograd.grad(y.sum(), (x, gate, up, down))
    assert grads[0].shape == (0, 130) and all((g == 0).all() and g.shape == p.shape for g, p in zip(grads[1:], (gate, up, down)))
    with torch.no_grad():
        assert fp8.feed_forward(x, fp8.pack_gated(gate, up), fp8.pack(down)).shape == (0, 130)
        assert fp8.dequantize(fp8.quantize(x)).shape == (0, 130)


def test_captured(env):
    """A training step and a generation step recorded into graphs, replayed several times on new inputs with eager work between; a workspace of
    their own."""
    fp8, torch, dev = env
    T, K, F = 70, 300, 260
    data = [torch.randn(s, device=dev) for s in ((T, K), (K, F), (K, F), (F, K), (T, K))]
    w_in, w_out = fp8.pack_gated(data[1], data[2]), fp8.pack(data[3])
    few = torch.randn(3, K, device=dev)

    def step(x, gate, up, down, dy, ws):
        x, gate, up, down = (t.detach().requires_grad_() for t in (x, gate, up, down))
        y = fp8.gated_mlp(x, gate, up, down, workspace=ws)
        return (y.detach(),) + torch.autograd.grad(y, (x, gate, up, down), dy)

    own, other = fp8.workspace(dev), fp8.workspace(dev)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*data, own)
        fp8.feed_forward(few, w_in, w_out, workspace=own)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(*data, own)
        y = fp8.feed_forward(few, w_in, w_out, workspace=own)
    for turn in range(4):
        for t in data:
            t.copy_(torch.randn(t.shape, device=dev))
        few.copy_(torch.randn(few.shape, device=dev))
        graph.replay()
        want = step(*data, other)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), turn
        assert torch.equal(y, fp8.feed_forward(few, w_in, w_out, workspace=other)), turn


def test_another_stream(env):
    fp8, torch, dev = env
    side = torch.cuda.Stream()
    x, b = torch.randn(40, 700, device=dev), torch.randn(700, 300, device=dev)
    want = fp8.matmul(x, fp8.pack(b))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ws = fp8.workspace(dev)
        got = fp8.matmul(x, fp8.pack(b), workspace=ws)
        again = fp8.matmul(x, fp8.pack(b), workspace=ws)
    side.synchronize()
    bound = 1e-5 * float(want.abs().max())
    assert (got - want).abs().max() < bound and torch.equal(got, again)


def test_beyond_32_bits(env):
    """Codes, and rows of the result, whose offsets pass 2^31 and 2^32."""
    fp8, torch, dev = env
    K, T = 16384, 270000
    codes = torch.zeros((T, K), dtype=torch.uint8, device=dev)
    scales = torch.full((T, K // 128), 127, dtype=torch.uint8, device=dev)
    rng = np.random.default_rng(0)
    rows = [0, 131071, 131072, 262143, 262144, T - 1]
    x = rng.standard_normal((len(rows), K))
    c, s = ref.quantize(x)
    codes[rows], scales[rows] = torch.from_numpy(c).to(dev), torch.from_numpy(s).to(dev)
    big = fp8.Blocks(codes, scales, K)
    b = weights(rng, K, 40)
    y = fp8.matmul(big, fp8.pack(tensor(torch, dev, b, "float32")), dtype=torch.float32)
    x8, b8 = ref.held(x), ref.held_weight(f64(tensor(torch, dev, b, "float32")))
    want = x8 @ b8
    compare(f64(y[rows]), want, ref.sum_bound(np.abs(x8) @ np.abs(b8), K, True) + 2.0 ** -24 * np.abs(want), "rows")
    others = torch.ones(T, dtype=torch.bool, device=dev)
    others[rows] = False
    assert not y[others].any()
    back = fp8.dequantize(fp8.Blocks(codes[131072:], scales[131072:], K), dtype=torch.bfloat16)
    assert_same(f64(back[262144 - 131072]), ref.held(x)[4], "values")
    del back, y
    dy = torch.zeros(T, 8, device=dev)
    dy[rows] = 1.0
    g = fp8.weight_gradient(big, dy, workspace=fp8.workspace(dev))
    want = x8.sum(0)
    compare(f64(g), np.repeat(want[:, None], 8, 1), np.repeat((np.abs(x8).sum(0) * 2.0 ** -20)[:, None], 8, 1), "gradient")


# ---- enough rows and columns for the kernel of 256 x 256 tiles ------------------------------------------------------------------


def big64(torch, dev, a, b):
    return (torch.from_numpy(a).to(dev) @ torch.from_numpy(b).to(dev)).cpu().numpy()


@pytest.mark.parametrize("T,K,N", [(2500, 300, 5200), (2561, 128, 5121), (300, 1100, 25600)])
def test_matmul_large_tiles(env, T, K, N):
    fp8, torch, dev = env
    rng = np.random.default_rng(T)
    say(f"large tiles {T} x {K} x {N}")
    x, b = tensor(torch, dev, inputs(rng, T, K), "bfloat16"), tensor(torch, dev, weights(rng, K, N), "bfloat16")
    bias = torch.randn(N, device=dev)
    w, x8, b8 = fp8.pack(b), ref.held(f64(x)), ref.held_weight(f64(b))
    want = big64(torch, dev, x8, b8) + f64(bias)
    bound = ref.sum_bound(big64(torch, dev, np.abs(x8), np.abs(b8)) + np.abs(f64(bias)), K, False)
    for dtype in DTYPES:
        store = torch.full((T, N + 5), 3.0, dtype=getattr(torch, dtype), device=dev)
        fp8.matmul(x, w, bias=bias, out=store[:, 2:2 + N], wide_sums=False)
        compare(f64(store[:, 2:2 + N]), want, bound + ref.rounding(np.abs(want) + bound, dtype), dtype)
        assert (store[:, :2] == 3).all() and (store[:, 2 + N:] == 3).all()
    # a product whose sums stay exact on the 8-bit cores too: every row against the kernel of smaller tiles
    x = torch.randint(-2, 3, (T, K), device=dev).to(torch.bfloat16)
    b = torch.randint(-2, 3, (K, N), device=dev).to(torch.bfloat16)
    w = fp8.pack(b)
    y = fp8.matmul(x, w, dtype=torch.float32, wide_sums=False)
    assert torch.equal(y, torch.cat([fp8.matmul(part.contiguous(), w, dtype=torch.float32) for part in x.split(100)]))
    assert torch.equal(y.double(), x.double() @ b.double())


@pytest.mark.parametrize("T,N", [(1025, 300), (2100, 1900)])                  # tiles of 64 rows; with sums in fp32 of 128 too
@pytest.mark.parametrize("K", [128, 250, 384, 500, 640, 2300])                # one block to five, and enough to be dealt over workgroups
def test_matmul_small_tiles(env, T, K, N):
    fp8, torch, dev = env
    rng = np.random.default_rng(T + K)
    say(f"small tiles {T} x {K} x {N}")
    x, b = tensor(torch, dev, inputs(rng, T, K), "bfloat16"), tensor(torch, dev, weights(rng, K, N), "bfloat16")
    bias = torch.randn(N, device=dev)
    w, ws, x8, b8 = fp8.pack(b), fp8.workspace(dev), ref.held(f64(x)), ref.held_weight(f64(b))
    want, mass = big64(torch, dev, x8, b8) + f64(bias), big64(torch, dev, np.abs(x8), np.abs(b8)) + np.abs(f64(bias))
    whole = torch.randint(-2, 3, (T, K), device=dev).to(torch.bfloat16)         # sums that stay exact either way
    whole_b = torch.randint(-2, 3, (K, N), device=dev).to(torch.bfloat16)
    whole_w = fp8.pack(whole_b)
    for wide in (False, True):
        for workspace in (None, ws):
            for dtype in DTYPES:
                bound = ref.sum_bound(mass, K, wide)
                y = fp8.matmul(x, w, bias=bias, dtype=getattr(torch, dtype), workspace=workspace, wide_sums=wide)
                compare(f64(y), want, bound + ref.rounding(np.abs(want) + bound, dtype), f"{dtype} wide {wide} workspace {workspace is not None}")
            y = fp8.matmul(whole, whole_w, dtype=torch.float32, workspace=workspace, wide_sums=wide)
            assert torch.equal(y.double(), whole.double() @ whole_b.double()), f"wide {wide} workspace {workspace is not None}"
    assert (ws[:fp8.COUNTER_BYTES] == 0).all()


@pytest.mark.parametrize("T,K,F", [(2500, 300, 2700), (2561, 140, 2561)])
@pytest.mark.parametrize("act", ["silu", "relu"])
def test_gated_large_tiles(env, T, K, F, act):
    fp8, torch, dev = env
    rng = np.random.default_rng(T)
    say(f"gated, large tiles {T} x {K} x {F} {act}")
    x, dh = tensor(torch, dev, inputs(rng, T, K), "bfloat16"), tensor(torch, dev, inputs(rng, T, F, 0.01), "float32")
    gate, up = (tensor(torch, dev, weights(rng, K, F) * s, "bfloat16") for s in (2.0, 1.0))
    w, xq = fp8.pack_gated(gate, up), fp8.quantize(x)
    x8, g8, u8, d = ref.held(f64(x)), ref.held_weight(f64(gate)), ref.held_weight(f64(up)), f64(dh)
    g, u = big64(torch, dev, x8, g8), big64(torch, dev, x8, u8)
    g_err, u_err = (ref.sum_bound(big64(torch, dev, np.abs(x8), np.abs(b)), K, False) for b in (g8, u8))
    a, slope = ref.activate(act, g)
    h, h_err = gated_reference(act, g, u, g_err, u_err)
    for dtype in DTYPES:
        y = fp8.gated(xq, w, act, dtype=getattr(torch, dtype), wide_sums=False)
        compare(f64(y), h, h_err + ref.rounding(np.abs(h) + h_err, dtype), dtype)
    q = fp8.gated(xq, w, act, out=fp8.new_blocks(T, F, dev))
    got, held_f32 = f64(fp8.dequantize(q)), fp8.gated(xq, w, act, dtype=torch.float32, wide_sums=False)
    check_blocks(q, f64(held_f32), "the 8-bit form of the same kernel's fp32 result")
    assert not (q.codes[:, F:] & 127).any()
    dgu, dgu8, h8 = fp8.gated_backward(xq, w, dh, act)
    Fp = ref.up(F, 128)
    assert torch.equal(h8.codes, q.codes) and torch.equal(h8.scales[:, :Fp // 128], q.scales[:, :Fp // 128])
    s_err = np.where(np.abs(g) <= g_err, 1.0, 0.0) if act == "relu" else 1.2 * g_err + 2.0 ** -19 * (1 + np.abs(g))
    a_err = 1.2 * g_err + 2.0 ** -20 * np.abs(a) * (1 + np.abs(g)) + 2.0 ** -22 * np.abs(g)
    for i, (want, err) in enumerate(((d * u * slope, np.abs(d) * (u_err * (np.abs(slope) + s_err) + np.abs(u) * s_err) + 2.0 ** -22 * np.abs(d * u * slope)),
                                     (d * a, np.abs(d) * a_err + 2.0 ** -23 * np.abs(d * a)))):
        compare(f64(dgu[:, i, :F]), want, err + ref.rounding(np.abs(want) + err, "bfloat16"), f"dgu {i}")
        assert not dgu[:, i, F:].any()
        # the 8-bit form is of the fp32 value, which dgu has to half a step: no further than that from the 8-bit form of dgu
        part, near = f64(fp8.dequantize(dgu8))[:, i * Fp:i * Fp + F], f64(dgu[:, i, :F])
        compare(part, ref.held(near), ref.held_bound(near, ref.rounding(np.abs(near), "bfloat16") * 1.01) + 1e-300, f"dgu8 {i}")


@pytest.mark.parametrize("T,K,N", [(130, 3601, 3700), (1, 3800, 3841), (257, 130, 51400)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_weight_gradient_large_tiles(env, T, K, N, dtype):
    fp8, torch, dev = env
    rng = np.random.default_rng(T + K)
    say(f"weight gradient, large tiles {T} x {K} x {N} {dtype}")
    x, dy = tensor(torch, dev, inputs(rng, T, K), dtype), tensor(torch, dev, inputs(rng, T, N, 0.01), dtype)
    x8, d = ref.held(f64(x)), f64(dy)
    want, mass = big64(torch, dev, x8.T.copy(), d), big64(torch, dev, np.abs(x8).T.copy(), np.abs(d))
    bound = mass * ((64 + 32 + T / 16 * 3) * 2.0 ** -23) + np.abs(x8).sum(0)[:, None] * 2.0 ** -130
    store = torch.full((K, N + 5), 3.0, dtype=torch.float32, device=dev)
    y = fp8.weight_gradient(fp8.quantize(x), wide_rows(torch, dy), dtype=torch.float32, out=store[:, 2:2 + N])
    compare(f64(y), want, bound + ref.rounding(np.abs(want) + bound, "float32"), "fp32")
    assert (store[:, :2] == 3).all() and (store[:, 2 + N:] == 3).all()
    y = fp8.weight_gradient(fp8.quantize(x), dy, dtype=torch.bfloat16)
    compare(f64(y), want, bound + ref.rounding(np.abs(want) + bound, "bfloat16"), "bf16")
