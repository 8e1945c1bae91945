"""Attention over values of very different sizes: what a row does not see, or gives no weight, takes nothing from its result.

Compared with 64 bits over the values that the cache holds.  The bound per output element is that of test_gpu_kv4.py but for its last
term, which goes by the tokens that carry weight for the row: with P = sum_j p_j |v_j| of the element,
    u_out |o|  +  u_p P  +  2 (D + 16) 2^-24 S P  +  (m + 64) 2^-24 P        as there
  + 2^-21 S P + (K + 64) 2^-24 P     fp32 results: queries in two fp16; the exponent, at most K + 64 in size for a token that counts
                                     where value scales are up to 2^K apart, is rounded once
  + m 2^-28 max_j p_j span_j         fp16's smallest step, 2^-25 of numbers of which the row's largest is at least 2^3.5, times the
                                     span of 15 codes of that token
"""
import math

import numpy as np
import pytest

import kv4_reference as ref

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]
U = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
HQ, HKV = 4, 2


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2101_05615_amd import kv4
    return kv4, torch, torch.device("cuda:0")


def run(env, k, v, q, P=32, causal=True, split=False):
    """One sequence of keys k and values v [m, HKV, D] fp32, queries q [n, HQ, D] of its last tokens: (output, held keys, values, spans)."""
    kv4, torch, dev = env
    m, n, D = k.shape[0], q.shape[0], k.shape[2]
    n_pages = (m + P - 1) // P
    cache = kv4.new_cache(n_pages, HKV, D, P, device=dev)
    slots = torch.arange(m, device=dev)
    kv4.append(cache, torch.from_numpy(k.astype(np.float32)).to(dev), torch.from_numpy(v.astype(np.float32)).to(dev), slots)
    ws = kv4.attention_workspace(cache, HQ, 1, max_q_len=n, max_kv_len=m) if split else None
    assert not split or ws is not None
    got = kv4.attention(q.to(dev), cache, torch.arange(n_pages, dtype=torch.int32, device=dev)[None], torch.tensor([m], dtype=torch.int32, device=dev),
                        q_starts=torch.tensor([0, n], dtype=torch.int32, device=dev), max_q_len=n, max_kv_len=m, causal=causal, workspace=ws)
    model = ref.Cache(cache.data.cpu().numpy(), n_pages, HKV, D, P)
    tokens = [model.token(t) for t in range(m)]
    hk, hv = (np.stack([ref.worth(t[i], t[i + 1]) for t in tokens]).astype(np.float64) for i in (0, 2))
    span = 15 * (np.stack([t[3] for t in tokens]) & np.uint32(0xFFFFFFF0)).view(np.float32).astype(np.float64)
    return got.double().cpu().numpy(), hk, hv, span


def check(got, q, k, v, span, dtype, K, causal=True, rows=None):
    """K: log2 of how far apart value scales are."""
    n, m, D = q.shape[0], k.shape[0], k.shape[2]
    q = q.double().cpu().numpy()
    worst = 0.0
    for i in range(n) if rows is None else rows:
        seen = m - n + i + 1 if causal else m
        for h in range(HQ):
            kk, vv = k[:seen, h // (HQ // HKV)], v[:seen, h // (HQ // HKV)]
            s = kk @ q[i, h] / math.sqrt(D)
            size = float(np.max(np.abs(kk) @ np.abs(q[i, h]))) / math.sqrt(D)
            p = np.exp(s - s.max())
            p /= p.sum()
            want, mass = p @ vv, p @ np.abs(vv)
            e = (2.0 ** -21 if dtype == "float32" else 2.0 ** -11) + 2 * (D + 16) * 2.0 ** -24 * size + (m + 64) * 2.0 ** -24
            if dtype == "float32":
                e += 2.0 ** -21 * size + (K + 64) * 2.0 ** -24
            bound = U[dtype] * np.abs(want) + e * mass * (1 + U[dtype]) + m * 2.0 ** -28 * np.max(p * span[:seen, h // (HQ // HKV)])
            bound = bound + 2.0 ** -25 * (dtype == "float16")
            off = np.abs(got[i, h] - want)
            assert np.isfinite(got[i, h]).all(), (i, h)
            worst = max(worst, float(np.max(off / bound)))
            assert (off <= bound).all(), f"row {i}, head {h}: {np.max(off / bound):.2f} times the bound"
    return worst


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,n", [(64, 4), (128, 4), (128, 16), (256, 4), (64, 40), (128, 70), (256, 40)])
@pytest.mark.parametrize("k", [0, 8, 16, 24, 64])
def test_a_later_token_with_large_values(env, dtype, D, n, k):
    """The last token's values are 2^k larger: rows before the last do not see it, in the same tile or not."""
    kv4, torch, dev = env
    rng = np.random.default_rng(D + n)
    m = 600
    keys, values = 0.3 * rng.standard_normal((m, HKV, D)), rng.standard_normal((m, HKV, D))
    values[-1] *= 2.0 ** k
    q = torch.from_numpy(rng.standard_normal((n, HQ, D)).astype(np.float32)).to(getattr(torch, dtype))
    got, hk, hv, span = run(env, keys, values, q)
    check(got, q, hk, hv, span, dtype, k, rows=sorted({0, 1, n // 2, n - 2}))
    if dtype != "float16" or k < 16:
        check(got, q, hk, hv, span, dtype, k, rows=[n - 1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 8, 40])
@pytest.mark.parametrize("at", [0, 37, 399])
@pytest.mark.parametrize("k", [20, 60])
def test_large_values_without_weight(env, dtype, n, at, k):
    """One token has values 2^k larger and a score about 200 below the others': e^-200 of 2^k is nothing, and the others keep their digits."""
    kv4, torch, dev = env
    rng = np.random.default_rng(at + n)
    m, D = 400, 64
    keys, values = 0.2 * rng.standard_normal((m, HKV, D)), rng.standard_normal((m, HKV, D))
    keys[at], values[at] = -25.0, values[at] * 2.0 ** k
    q = torch.from_numpy((1 + 0.1 * rng.standard_normal((n, HQ, D))).astype(np.float32)).to(getattr(torch, dtype))
    got, hk, hv, span = run(env, keys, values, q, causal=False)
    check(got, q, hk, hv, span, dtype, k, causal=False, rows=sorted({0, n // 2, n - 1}))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("first", [True, False])
def test_shares_whose_values_differ(env, dtype, n, first):
    """Keys split over workgroups: half of the keys have all the weight and values of ordinary size, the others values 2^60 larger and none."""
    kv4, torch, dev = env
    rng = np.random.default_rng(n)
    m, D = 3000, 64
    keys, values = 0.2 * rng.standard_normal((m, HKV, D)), rng.standard_normal((m, HKV, D))
    half = slice(0, m // 2) if first else slice(m // 2, m)
    keys[half], values[half] = -25.0, values[half] * 2.0 ** 60
    q = torch.from_numpy((1 + 0.1 * rng.standard_normal((n, HQ, D))).astype(np.float32)).to(getattr(torch, dtype))
    got, hk, hv, span = run(env, keys, values, q, causal=False, split=True)
    check(got, q, hk, hv, span, dtype, 60, causal=False, rows=sorted({0, n - 1}))


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("size", [2.0 ** -100, 1.0, 2.0 ** 100])
def test_tokens_of_zeros(env, n, size):
    """Tokens whose values are all zero, first and between: they have probability and nothing else.  All of them zero: the result is 0."""
    kv4, torch, dev = env
    rng = np.random.default_rng(n)
    m, D = 300, 64
    keys, values = 0.3 * rng.standard_normal((m, HKV, D)), size * rng.standard_normal((m, HKV, D))
    values[:100], values[150:180] = 0.0, 0.0
    q = torch.from_numpy(rng.standard_normal((n, HQ, D)).astype(np.float32))
    got, hk, hv, span = run(env, keys, values, q)
    check(got, q, hk, hv, span, "float32", 0, rows=[0, n - 1])
    assert (run(env, keys, values * 0, q)[0] == 0).all()


@pytest.mark.parametrize("n", [2, 40])
@pytest.mark.parametrize("k", [40, 64])
def test_many_keys_before_a_token_with_large_values(env, n, k):
    """20000 keys of about equal weight, so that their sum is large where the last token's values change the common reference."""
    kv4, torch, dev = env
    rng = np.random.default_rng(n)
    m, D = 20000, 64
    keys, values = 0.1 * rng.standard_normal((m, HKV, D)), rng.standard_normal((m, HKV, D))
    values[-1] *= 2.0 ** k
    q = torch.from_numpy(rng.standard_normal((n, HQ, D)).astype(np.float32))
    got, hk, hv, span = run(env, keys, values, q)
    check(got, q, hk, hv, span, "float32", k, rows=[0, n - 1])
