"""8-bit floats with a scale per block of 128 without a GPU: sizes, refusals before any device work, and the plain implementation that the
GPU tests compare with."""
import ctypes
import os

import numpy as np
import pytest

import fp8_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ENULL, EINVAL, EALIGN, EWORKSPACE, EUNSUPPORTED = -1, -2, -3, -4, -7
FAKE = 1 << 16   # never dereferenced: every call below is refused before any device work


@pytest.fixture(scope="module")
def fp8():
    if not os.path.exists(os.path.join(ROOT, "paper_2101_05615_amd", "libqgemm.so")):
        import __graft_entry__ as g
        g.build()
    from paper_2101_05615_amd import fp8
    return fp8


def test_sizes(fp8):
    lib = fp8.lib
    assert lib.qg_fp8_codes_bytes(3, 1) == 3 * 128 and lib.qg_fp8_scales_bytes(3, 1) == 3 * 4
    assert lib.qg_fp8_codes_bytes(300000, 16384) == 300000 * 16384 and lib.qg_fp8_scales_bytes(7, 16384) == 7 * 128
    assert lib.qg_fp8_scales_bytes(2, 513) == 2 * 8
    for bad in [(-1, 5), (1, 0), (1, (1 << 20) + 1), ((1 << 28) + 1, 1)]:
        assert lib.qg_fp8_codes_bytes(*bad) == 0 and lib.qg_fp8_scales_bytes(*bad) == 0, bad
    assert lib.qg_fp8_weight_bytes(1, 1, 0) == 4 * 8192 + 4 * 16
    assert lib.qg_fp8_weight_bytes(130, 257, 0) == 8 * 2 * 8192 + 8 * 16
    assert lib.qg_fp8_weight_bytes(130, 129, 1) == 8 * 2 * 8192 + 8 * 16
    assert lib.qg_fp8_weight_bytes(65536, 65536, 1) == 2 * 65536 ** 2 + 2048 * 512 * 4
    for bad in [(0, 1, 0), (1, 0, 0), (1, 1, 2), (1, 1, -1), ((1 << 20) + 1, 1, 0), (1, (1 << 20) + 1, 0)]:
        assert lib.qg_fp8_weight_bytes(*bad) == 0, bad


def blocks(fp8, tokens=4, channels=300, codes=FAKE, scales=FAKE):
    return ctypes.byref(fp8._BlocksDesc(codes, scales, tokens, channels))


def rows(fp8, data=FAKE, stride=1024):
    return ctypes.byref(fp8._Rows(data, stride))


@pytest.mark.parametrize("name", ["qg_fp8_quantize", "qg_fp8_dequantize"])
def test_quantize_refusals(fp8, name):
    def call(x=None, dtype=0, to=None):
        x, to = x or rows(fp8), to or blocks(fp8)
        f = getattr(fp8.lib, name)
        return f(x, dtype, to, None) if name == "qg_fp8_quantize" else f(to, dtype, x, None)

    assert call(dtype=3) == EINVAL and call(dtype=-1) == EINVAL
    assert call(x=rows(fp8, None)) == ENULL and call(to=blocks(fp8, codes=None)) == ENULL and call(to=blocks(fp8, scales=None)) == ENULL
    assert call(x=rows(fp8, FAKE + 2)) == EALIGN and call(x=rows(fp8, FAKE + 1), dtype=1) == EALIGN
    assert call(to=blocks(fp8, codes=FAKE + 8)) == EALIGN and call(to=blocks(fp8, scales=FAKE + 2)) == EALIGN
    assert call(to=blocks(fp8, tokens=-1)) == EINVAL and call(to=blocks(fp8, channels=0)) == EINVAL
    assert call(to=blocks(fp8, channels=(1 << 20) + 1)) == EINVAL and call(to=blocks(fp8, tokens=(1 << 28) + 1)) == EINVAL
    assert call(to=blocks(fp8, tokens=1 << 28, channels=1 << 20)) == EUNSUPPORTED
    assert call(to=blocks(fp8, tokens=0, codes=None, scales=None), x=rows(fp8, None)) == 0
    f = getattr(fp8.lib, name)
    assert f(None, 0, blocks(fp8) if name == "qg_fp8_quantize" else rows(fp8), None) == ENULL


def weight(fp8, k=300, n=200, gated=0, data=FAKE):
    return ctypes.byref(fp8._WeightDesc(data, k, n, gated))


def test_pack_refusals(fp8):
    m = lambda data=FAKE: ctypes.byref(fp8._Matrix(data, 200, 1))  # noqa: E731

    def call(b=m(), up=None, k=300, n=200, dtype=1, w=weight(fp8), t=None):
        return fp8.lib.qg_fp8_pack(b, up, k, n, dtype, w, t, None)

    assert call(b=None) == ENULL and call(w=None) == ENULL and call(b=m(None)) == ENULL and call(w=weight(fp8, data=None)) == ENULL
    assert call(up=m(None), w=weight(fp8, gated=1)) == ENULL
    assert call(dtype=7) == EINVAL and call(k=0) == EINVAL and call(n=-5) == EINVAL
    assert call(w=weight(fp8, k=301)) == EINVAL and call(w=weight(fp8, n=201)) == EINVAL and call(w=weight(fp8, gated=1)) == EINVAL
    assert call(up=m()) == EINVAL                                                 # a pair into a plain buffer
    assert call(t=weight(fp8, 300, 200)) == EINVAL and call(t=weight(fp8, 200, 300, 1)) == EINVAL
    assert call(up=m(), w=weight(fp8, gated=1), t=weight(fp8, 400, 300)) == EINVAL   # (2 * 256)
    assert call(b=m(FAKE + 1)) == EALIGN and call(w=weight(fp8, data=FAKE + 8)) == EALIGN and call(b=m(FAKE + 2), dtype=0) == EALIGN


def product(fp8, **kw):
    a = dict(x=fp8._BlocksDesc(FAKE, FAKE, 40, 300), x_rows=fp8._Rows(None, 0), x_dtype=0, tokens=40, out=fp8._Rows(FAKE, 200), dtype=1,
             activation=0, wide_sums=0, bias=None, workspace=None, workspace_bytes=0)
    a.update(kw)
    return ctypes.byref(fp8._Product(*[a[n] for n, _ in fp8._Product._fields_]))


def common_refusals(fp8, call, gated):
    none = fp8._BlocksDesc(None, None, 0, 0)
    assert call(p=None) == ENULL and call(w=None) == ENULL and call(w=weight(fp8, gated=gated, data=None)) == ENULL
    assert call(w=weight(fp8, gated=1 - gated)) == EINVAL and call(w=weight(fp8, gated=gated, data=FAKE + 4)) == EALIGN
    assert call(tokens=-1) == EINVAL and call(tokens=41) == EINVAL and call(wide_sums=2) == EINVAL
    assert call(x=fp8._BlocksDesc(FAKE, FAKE, 40, 301)) == EINVAL and call(x=fp8._BlocksDesc(FAKE, None, 40, 300)) == ENULL
    assert call(x=fp8._BlocksDesc(FAKE + 8, FAKE, 40, 300)) == EALIGN
    assert call(x=none) == ENULL
    raw = dict(x=none, x_rows=fp8._Rows(FAKE, 300))
    assert call(**raw) == EUNSUPPORTED                                            # more than QG_FP8_FEW tokens
    assert call(**raw, x_dtype=9, tokens=3) == EINVAL
    assert call(x=none, x_rows=fp8._Rows(FAKE + 2, 300), tokens=3) == EALIGN
    assert call(**raw, tokens=3) == EUNSUPPORTED                                  # 300 channels are no multiple of 16
    assert call(workspace=FAKE, workspace_bytes=fp8.WORKSPACE_BYTES - 1) == EWORKSPACE
    assert call(workspace=FAKE + 4, workspace_bytes=fp8.WORKSPACE_BYTES) == EALIGN
    assert call(tokens=0, x=none, out=fp8._Rows(None, 0)) == 0


def test_matmul_refusals(fp8):
    def call(p=0, w=weight(fp8), **kw):
        return fp8.lib.qg_fp8_matmul(w, product(fp8, **kw) if p == 0 else p, None)

    common_refusals(fp8, call, 0)
    assert call(dtype=3) == EINVAL and call(out=fp8._Rows(None, 0)) == ENULL and call(out=fp8._Rows(FAKE + 1, 200)) == EALIGN
    assert call(bias=FAKE + 2) == EALIGN
    assert call(w=weight(fp8, 300, 1 << 20), x=fp8._BlocksDesc(FAKE, FAKE, 1 << 28, 300), tokens=1 << 28) == EUNSUPPORTED


def test_gated_refusals(fp8):
    def call(p=0, w=weight(fp8, gated=1), held=None, **kw):
        return fp8.lib.qg_fp8_gated(w, product(fp8, **kw) if p == 0 else p, held, None)

    common_refusals(fp8, call, 1)
    assert call(activation=4) == EINVAL and call(activation=-1) == EINVAL and call(bias=FAKE) == EINVAL and call(dtype=3) == EINVAL
    nowhere = fp8._Rows(None, 0)
    assert call(out=nowhere) == ENULL and call(held=blocks(fp8, 40, 200)) == EINVAL
    assert call(out=nowhere, held=blocks(fp8, 39, 200)) == EINVAL and call(out=nowhere, held=blocks(fp8, 40, 300)) == EINVAL
    assert call(out=nowhere, held=blocks(fp8, 3, 200), tokens=3, x=fp8._BlocksDesc(None, None, 0, 0), x_rows=fp8._Rows(FAKE, 300)) == EUNSUPPORTED


def test_gated_backward_refusals(fp8):
    def call(p=0, w=weight(fp8, gated=1), dh=rows(fp8), dh_dtype=0, dgu=FAKE, both=blocks(fp8, 40, 512), held=blocks(fp8, 40, 200), **kw):
        return fp8.lib.qg_fp8_gated_backward(w, product(fp8, **kw) if p == 0 else p, dh, dh_dtype, dgu, both, held, None)

    common_refusals(fp8, call, 1)
    assert call(dh=None) == ENULL and call(both=None) == ENULL and call(held=None) == ENULL and call(dgu=None) == ENULL
    assert call(dh=rows(fp8, None)) == ENULL and call(dh=rows(fp8, FAKE + 2)) == EALIGN and call(dgu=FAKE + 8) == EALIGN
    assert call(dh_dtype=3) == EINVAL and call(activation=9) == EINVAL
    assert call(both=blocks(fp8, 40, 400)) == EINVAL and call(held=blocks(fp8, 40, 256)) == EINVAL
    raw = dict(x=fp8._BlocksDesc(None, None, 0, 0), x_rows=fp8._Rows(FAKE, 300), tokens=3, both=blocks(fp8, 3, 512), held=blocks(fp8, 3, 200))
    assert call(**raw) == EUNSUPPORTED
    assert call(wide_sums=1) == EUNSUPPORTED
    assert call(w=weight(fp8, 300, 7, 1), held=blocks(fp8, 40, 7), both=blocks(fp8, 40, 256)) == EUNSUPPORTED   # fewer than 8 columns
    wide = (1 << 20) - 100
    assert call(w=weight(fp8, 300, wide, 1)) == EINVAL                            # the pair's gradient would have too many channels


def test_weight_gradient_refusals(fp8):
    def call(x=blocks(fp8), dy=rows(fp8), dy_dtype=0, n=200, out=rows(fp8), dtype=0, ws=None, size=0, dy2=None, out2=None):
        return fp8.lib.qg_fp8_weight_gradient(x, dy, dy2, dy_dtype, n, out, out2, dtype, ws, size, None)

    assert call(x=None) == ENULL and call(dy=None) == ENULL and call(out=None) == ENULL
    assert call(dy=rows(fp8, None)) == ENULL and call(out=rows(fp8, None)) == ENULL and call(x=blocks(fp8, codes=None)) == ENULL
    assert call(dy_dtype=3) == EINVAL and call(dtype=3) == EINVAL and call(n=0) == EINVAL and call(n=(1 << 20) + 1) == EINVAL
    assert call(dy=rows(fp8, FAKE + 2)) == EALIGN and call(out=rows(fp8, FAKE + 2)) == EALIGN
    assert call(dy2=rows(fp8)) == ENULL and call(out2=rows(fp8)) == ENULL and call(dy2=rows(fp8, FAKE + 2), out2=rows(fp8)) == EALIGN
    assert call(dy2=rows(fp8), out2=rows(fp8, None)) == ENULL
    assert call(ws=FAKE, size=100) == EWORKSPACE and call(ws=FAKE + 4, size=fp8.WORKSPACE_BYTES) == EALIGN


def test_python_refusals(fp8):
    """Arguments that the module itself refuses, on tensors without a GPU."""
    import torch
    with pytest.raises(RuntimeError, match="cpu"):
        fp8.quantize(torch.zeros(3, 4))
    with pytest.raises(AssertionError):
        fp8.quantize(torch.zeros(3, 4, dtype=torch.float64))
    with pytest.raises(AssertionError):
        fp8.quantize(torch.zeros(3, 8)[:, ::2])
    with pytest.raises(AssertionError):
        fp8.quantize(torch.zeros(3))
    with pytest.raises(RuntimeError, match="gradient"):
        fp8.matmul(torch.zeros(3, 4, requires_grad=True), None)
    for bad in [(3, 0), (-1, 3), (3, (1 << 20) + 1)]:
        with pytest.raises(Exception):
            fp8.new_blocks(*bad, device="cpu")


# ---- the plain implementation itself --------------------------------------------------------------------------------------------


def test_numbers():
    """Against torch's own e4m3 type."""
    import torch
    every = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    assert np.array_equal(ref.value(every.numpy(), np.full(256, 127)), every.view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.uniform(-448, 448, 20000), rng.uniform(-0.05, 0.05, 20000), ref.MIDDLES, -ref.MIDDLES]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ref.round_codes(x.astype(np.float64)), want)


def test_scale_bytes():
    amax = np.array([0.0, 2.0 ** -149, 2.0 ** -118, 2.0 ** -117, 1.0, 1.75, 1.7500001, 448.0, 448.0001, 3.0e38, np.inf, np.nan])
    assert ref.byte_of(amax).tolist() == [0, 0, 1, 2, 119, 119, 120, 127, 128, 247, 255, 255]
    for a in amax[1:10]:
        e = float(ref.byte_of(a)) - 127
        assert a <= 448 * 2.0 ** e and (e == -127 or a > 448 * 2.0 ** (e - 1))
