"""Build-time guard for the kernels of the 8-bit floats: no private memory, no spilled vector registers, and the waves per SIMD that they
are sized for.  hipcc reports the resources while cross-compiling (no GPU needed)."""
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_kernel_resources import _resources


@pytest.mark.timeout(600)
def test_kernels_stay_in_registers():
    with ThreadPoolExecutor(4) as ex:
        quantize, tile, stream, gradient = ex.map(_resources, ["fp8_quantize.hip", "fp8_tile.hip", "fp8_stream.hip", "fp8_gradient.hip"])
    assert len(quantize) == 9 and tile and stream and gradient, "the resource report was not parsed"
    for name, r in {**quantize, **tile, **stream, **gradient}.items():
        assert r["ScratchSize [bytes/lane]"] == 0 and r["VGPRs Spill"] == 0, f"{name}: {r}"
