"""fp16 results of the attention: as precise over many query rows as over few.

Bound per element, with P = sum_j p_j |v_j| and S the largest sum |q||k| scale:
    2^-11 |o|                            the result's own rounding
  + 2^-21 P                              probabilities times value scale in two fp16 numbers
  + 2 (D + 16) 2^-24 S P                 scores: D fp32 additions and a few products
  + (m + 64) 2^-24 P                     sums over m keys, exponentials, the joining of partial results
  + m 2^-28 max_j p_j span_j + 2^-25     fp16's smallest step: of the weights, of the result
One fp16 number for a probability would be up to 2^-11 P off where one key has most of the weight.
"""
import math

import numpy as np
import pytest

import kv4_reference as ref
from gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,P,split", [(64, 16, False), (64, 64, True), (128, 16, False), (128, 64, True), (256, 32, False), (256, 16, True)])
@pytest.mark.parametrize("n", [4, 16, 17, 40, 130])
def test_fp16_results(D, P, split, n):
    import torch
    from paper_2101_05615_amd import kv4
    assert torch.cuda.is_available(), "this test needs the MI355X"
    dev, rng = torch.device("cuda:0"), np.random.default_rng(D + n)
    m, Hq, Hkv = 1500 if split else 300, 4, 2
    n_pages = (m + P - 1) // P
    cache = kv4.new_cache(n_pages, Hkv, D, P, device=dev)
    k, v = rng.standard_normal((m, Hkv, D)), rng.standard_normal((m, Hkv, D))
    v *= np.exp(0.7 * rng.standard_normal((m, Hkv, 1)))
    kv4.append(cache, *(torch.from_numpy(x.astype(np.float32)).to(dev) for x in (k, v)), torch.arange(m, device=dev))
    # a query is one of the keys it sees, so that this one has most of the weight, and a little of everything
    mine = rng.integers(0, m - n, (n, Hq))
    q = 3 / math.sqrt(D) * np.stack([np.stack([k[mine[i, h], h // 2] for h in range(Hq)]) for i in range(n)]) + 0.3 * rng.standard_normal((n, Hq, D))
    q = torch.from_numpy(q).half()
    ws = kv4.attention_workspace(cache, Hq, 1, max_q_len=n, max_kv_len=m) if split else None
    got = kv4.attention(q.to(dev), cache, torch.arange(n_pages, dtype=torch.int32, device=dev)[None], torch.tensor([m], dtype=torch.int32, device=dev),
                        q_starts=torch.tensor([0, n], dtype=torch.int32, device=dev), max_q_len=n, max_kv_len=m, scale=1 / 3, workspace=ws)
    got, q = got.double().cpu().numpy(), q.double().numpy()
    model = ref.Cache(cache.data.cpu().numpy(), n_pages, Hkv, D, P)
    tokens = [model.token(t) for t in range(m)]
    hk, hv = (np.stack([ref.worth(t[i], t[i + 1]) for t in tokens]).astype(np.float64) for i in (0, 2))
    span = 15 * (np.stack([t[3] for t in tokens]) & np.uint32(0xFFFFFFF0)).view(np.float32).astype(np.float64)
    worst = 0.0
    for i in sorted({0, 1, 15, 16, 33, n // 2, n - 1} & set(range(n))):
        seen = m - n + i + 1
        for h in range(Hq):
            kk, vv = hk[:seen, h // 2], hv[:seen, h // 2]
            s, size = kk @ q[i, h] / 3, float(np.max(np.abs(kk) @ np.abs(q[i, h]))) / 3
            p = np.exp(s - s.max())
            p /= p.sum()
            want, mass = p @ vv, p @ np.abs(vv)
            e = 2.0 ** -21 + 2 * (D + 16) * 2.0 ** -24 * size + (m + 64) * 2.0 ** -24
            bound = 2.0 ** -11 * np.abs(want) + e * mass * (1 + 2.0 ** -11) + m * 2.0 ** -28 * np.max(p * span[:seen, h // 2]) + 2.0 ** -25
            off = np.abs(got[i, h] - want)
            worst = max(worst, float(np.max(off / bound)))
            assert (off <= bound).all(), f"row {i}, head {h}: {np.max(off / bound):.2f} times the bound"
    say(f"largest error: {worst:.2f} of the bound")
