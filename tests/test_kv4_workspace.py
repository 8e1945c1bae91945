"""Sizes of the attention's workspace without a GPU: one for the largest extents serves every smaller call."""
import ctypes
import os
import random

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def kv4():
    if not os.path.exists(os.path.join(ROOT, "paper_2101_05615_amd", "libqgemm.so")):
        import __graft_entry__ as g
        g.build()
    from paper_2101_05615_amd import kv4
    return kv4


def size(kv4, D, Hkv, group, batch, max_q, max_kv):
    c = kv4.CacheDesc(data=4096, n_pages=1 << 16, kv_heads=Hkv, head_dim=D, page_tokens=64)      # (never dereferenced)
    return kv4.lib.qg_kv4_attention_workspace_bytes(ctypes.byref(c), Hkv * group, batch, max_q, max_kv)


def test_a_shorter_call_wants_no_more(kv4):
    # 8 KV heads of 128 channels, 32 query heads: a few keys less may make more shares, and a smaller batch as well
    lens = [1, 256, 512, 513, 777, 1024, 1025, 8192, 8193, 8300, 10000, 131072]
    sizes = [size(kv4, 128, 8, 4, 1, 1, n) for n in lens]
    assert sizes == sorted(sizes) and sizes[2] == 0 and sizes[3] > 0
    sizes = [size(kv4, 128, 8, 4, b, 1, 8192) for b in (1, 2, 16, 31, 32, 33, 64, 1000)]
    assert sizes == sorted(sizes) and sizes[0] > 0


@pytest.mark.parametrize("D", [64, 128, 256])
def test_sizes_grow_with_every_extent(kv4, D):
    rng = random.Random(D)
    for _ in range(3000):
        Hkv, group = rng.choice([1, 2, 3, 8]), rng.choice([1, 2, 4, 7, 16])
        large = [int(2 ** rng.uniform(0, 8)), int(2 ** rng.uniform(0, 9)), int(2 ** rng.uniform(6, 17))]
        small = [rng.randint(1, x) for x in large]
        assert size(kv4, D, Hkv, group, *small) <= size(kv4, D, Hkv, group, *large), (Hkv, group, small, large)


def test_no_more_than_a_call_can_fill(kv4):
    # one KV head, 33 rows, 1025 keys: three shares of 128 rows, each a row of results and two numbers
    assert size(kv4, 128, 1, 1, 1, 33, 1025) <= kv4.COUNTER_BYTES + 3 * 128 * (128 + 2) * 4
    assert size(kv4, 128, 1, 1, 1, 33, 1025) > kv4.COUNTER_BYTES
