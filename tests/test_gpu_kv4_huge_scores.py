"""Attention with scores of up to 2^28, where neighbouring fp32 numbers are 32 apart: the key with the largest score takes all, and the
result is its value.

Bound: one rounding to the output's type, 2^-11 for a 16-bit type's weight in one fp16 number, 2^-21 for an fp32 result's in two, and
2^-22 for the sums of up to 65 numbers of which all but one are 0 and the division.  The value scales of one sequence are within 2^8, so that
the weight of a key whose scale is not the largest is at least 2^-8 2^4 and its second fp16 number, in steps of 2^-24, is right to 2^-21.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = {"float32": 2.0 ** -24 + 2.0 ** -20, "bfloat16": 2.0 ** -8 + 2.0 ** -10, "float16": 2.0 ** -11 + 2.0 ** -10}


@pytest.mark.parametrize("dtype", sorted(U))
@pytest.mark.parametrize("n", [1, 12, 20, 50])
@pytest.mark.parametrize("m", [1, 3, 65])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_largest_score_takes_all(dtype, n, m, sign):
    import torch
    from paper_2101_05615_amd import kv4
    assert torch.cuda.is_available(), "this test needs the MI355X"
    dev, rng = torch.device("cuda:0"), np.random.default_rng(n * 100 + m)
    B, P, D, Hq, Hkv = 64, 128, 64, 4, 2
    cache = kv4.new_cache(B, Hkv, D, P, device=dev)
    # keys of one sign and scores in steps of 1/128 of the largest, in any order: 2^17 apart at least
    size = np.stack([rng.permutation(128)[:m] + 1.0 for _ in range(B)])[:, :, None, None] / 128
    k = (size * np.ones((B, m, Hkv, D))).astype(np.float32)
    v = (rng.standard_normal((B, m, Hkv, D)) * np.exp2(rng.uniform(-4, 4, (B, m, Hkv, 1)))).astype(np.float32)
    slots = (torch.arange(B, device=dev)[:, None] * P + torch.arange(m, device=dev)).flatten()
    kv4.append(cache, torch.from_numpy(k.reshape(-1, Hkv, D)).to(dev), torch.from_numpy(v.reshape(-1, Hkv, D)).to(dev), slots)
    hk, hv = (x.view(B, m, Hkv, D).double().cpu().numpy() for x in kv4.read(cache, slots))
    q = torch.from_numpy((sign * rng.uniform(0.5, 1.0, (B * n, Hq, D))).astype(np.float32)).to(getattr(torch, dtype))
    scale = 2.0 ** 28 / D                                    # scores from 2^20 to 2^28
    got = kv4.attention(q.to(dev), cache, torch.arange(B, dtype=torch.int32, device=dev)[:, None],
                        torch.full((B,), m, dtype=torch.int32, device=dev), q_starts=torch.arange(B + 1, dtype=torch.int32, device=dev) * n,
                        max_q_len=n, max_kv_len=m, scale=scale, causal=False).double().cpu().numpy().reshape(B, n, Hq, D)
    q = q.double().numpy().reshape(B, n, Hq, D)
    for h in range(Hq):
        score = np.matmul(q[:, :, h], hk[:, :, h // 2].transpose(0, 2, 1)) * scale
        top = np.sort(score, -1)
        assert np.abs(score).max() <= 2.0 ** 28 * 1.01 and (m == 1 or (top[..., -1] - top[..., -2]).min() > 2.0 ** 16)
        want = np.take_along_axis(hv[:, :, h // 2], score.argmax(-1)[:, :, None], 1)
        assert np.isfinite(got[:, :, h]).all()
        assert (np.abs(got[:, :, h] - want) <= U[dtype] * np.abs(want)).all(), f"head {h}: {np.max(np.abs(got[:, :, h] - want) / np.abs(want)):.1e}"
