"""Build-time guard for the kernels of the 4-bit cache: no private memory, no spilled vector registers, and the waves per SIMD that their
workgroups are sized for.  hipcc reports the resources while cross-compiling (no GPU needed)."""
import re
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_kernel_resources import _resources


@pytest.mark.timeout(600)
def test_kernels_stay_in_registers():
    with ThreadPoolExecutor(4) as ex:
        few, many, cache, rope = ex.map(_resources, ["kv4_attention.hip", "kv4_attention_rows.hip", "kv4_cache.hip", "rope.hip"])
    assert len(few) == 30 and len(many) == 18 and len(cache) == 18 and len(rope) == 7, "the resource report was not parsed"
    for name, r in {**few, **many, **cache, **rope}.items():
        assert r["ScratchSize [bytes/lane]"] == 0 and r["VGPRs Spill"] == 0, f"{name}: {r}"
    for name, r in few.items():       # <head_dim, query parts, type, row tiles, small pages>
        d, _, _, tiles = (int(x) for x in re.search(r"kernelILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)E", name).groups())
        assert r["Occupancy [waves/SIMD]"] >= (2 if d == 256 or tiles == 2 else 3), f"{name}: {r}"
    for name, r in many.items():
        assert r["Occupancy [waves/SIMD]"] >= 2, f"{name}: {r}"
    for name, r in {**cache, **{n: r for n, r in rope.items() if "table" not in n}}.items():
        assert r["Occupancy [waves/SIMD]"] >= 7, f"{name}: {r}"
