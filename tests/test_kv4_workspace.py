"""Sizes of the attention's workspace without a GPU."""
import ctypes
import os

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


def test_no_more_than_a_call_can_fill(kv4):
    # one KV head, 33 rows, 1025 keys: three shares of 128 rows, each a row of results and two numbers
    assert size(kv4, 128, 1, 1, 1, 33, 1025) <= kv4.COUNTER_BYTES + 3 * 128 * (128 + 2) * 4
    assert size(kv4, 128, 1, 1, 1, 33, 1025) > kv4.COUNTER_BYTES
