"""Rotation angles scaled by the index of the pair: contexts and bases for which the far end of the ramp lies behind the last pair."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def by_index(rot, base, factor, low, high, context):
    """w rises from the pair that makes `high` turns (rounded down) to the one that makes `low` (rounded up), both within 0 .. rot - 1."""
    pair = lambda turns: rot * math.log(context / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
    first, last = max(math.floor(pair(high)), 0), min(max(math.ceil(pair(low)), 0), rot - 1)
    i = np.arange(rot // 2, dtype=np.float64)
    w = np.clip((i - first) / max(last - first, 0.001), 0, 1)
    f = base ** (-2 * i / rot)
    return f * (1 - w) + f / factor * w, w, last


@pytest.mark.parametrize("rot", [32, 64, 128, 256])
@pytest.mark.parametrize("base,context", [(10000.0, 4096.0), (10000.0, 65536.0), (10000.0, 131072.0), (500.0, 8192.0), (10000.0, 4.0), (2.0, 1e9)])
def test_by_index(rot, base, context):
    import torch
    from paper_2101_05615_amd import kv4
    n, kw = 40000, dict(factor=4.0, low=1.0, high=32.0, context=context)
    f, w, last = by_index(rot, base, **kw)
    if (base, context) in ((10000.0, 65536.0), (10000.0, 131072.0), (500.0, 8192.0)):
        assert last > rot // 2 - 1 and w[-1] < 1          # (what this test is for: the last pair is not interpolated in full)
    got = kv4.rope_table(n, rot, base=base, scaling="by_index", device="cuda:0", **kw).cpu().numpy()
    angle = np.arange(n)[:, None] * f[None]
    want = np.concatenate([np.cos(angle), np.sin(angle)], 1)
    # one rounding to fp32, and an angle below 4e4 whose frequency is a power and three roundings off on either side
    assert np.max(np.abs(got - want)) <= 2.0 ** -25 + 4e4 * 2.0 ** -49
