"""The positions, the 4-bit cache and its attention without a GPU: sizes, refusals before any device work, and the plain
implementation that the GPU tests compare with."""
import ctypes
import os

import numpy as np
import pytest

import kv4_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def kv4():
    if not os.path.exists(os.path.join(ROOT, "paper_2101_05615_amd", "libqgemm.so")):
        import __graft_entry__ as g
        g.build()
    from paper_2101_05615_amd import kv4
    return kv4


FAKE = 4096   # never dereferenced: every call below is refused before any device work


def test_cache_bytes(kv4):
    assert kv4.cache_bytes(1, 1, 64, 16) == 16 * 72
    assert kv4.cache_bytes(3, 8, 128, 64) == 3 * 8 * 64 * 136
    assert kv4.cache_bytes(1 << 20, 8, 256, 256) == (1 << 20) * 8 * 256 * 264      # beyond 32 bits
    for bad in [(0, 1, 64, 16), (1, 0, 64, 16), (1, 1, 96, 16), (1, 1, 64, 8), (1, 1, 64, 48), (1, 1, 64, 512), (-1, 1, 64, 16), (1, 40000, 64, 16)]:
        assert kv4.cache_bytes(*bad) == 0, bad


def test_table_refusals(kv4):
    lib = kv4.lib
    good = dict(base=10000.0, factor=2.0, low=1.0, high=4.0, context=100.0, magnitude=1.0, scaling=kv4.ROPE_BY_TURNS, rot=64, max_pos=10)
    inf, nan = float("inf"), float("nan")

    def call(table=FAKE, **kw):
        return lib.qg_rope_table(ctypes.byref(kv4.RopeParams(**{**good, **kw})), table, None)

    for bad in [dict(base=1.0), dict(base=inf), dict(base=nan), dict(factor=0.5), dict(factor=nan), dict(low=0.0), dict(low=4.0), dict(high=inf),
                dict(context=0.0), dict(context=nan), dict(magnitude=0.0), dict(magnitude=inf), dict(scaling=4), dict(scaling=-1), dict(rot=0),
                dict(rot=63), dict(rot=258), dict(max_pos=0)]:
        assert call(**bad) == -2, bad
    assert call(table=None) == -1 and lib.qg_rope_table(None, FAKE, None) == -1
    assert call(table=FAKE + 4) == -3


def rope_args(kv4, **kw):
    a = dict(x=kv4.Heads(FAKE, 128, 64), dtype=1, tokens=3, heads=2, head_dim=64, positions=FAKE, table=FAKE, max_pos=10, rot=64,
             interleaved=0, inverse=0, y=kv4.Heads(2 * FAKE, 128, 64))
    a.update(kw)
    x, y = a["x"], a["y"]
    return [ctypes.byref(x) if x else None, a["dtype"], a["tokens"], a["heads"], a["head_dim"], a["positions"], a["table"], a["max_pos"],
            a["rot"], a["interleaved"], a["inverse"], ctypes.byref(y) if y else None, None]


def test_rope_refusals(kv4):
    H = kv4.Heads
    for code, bad in [(-1, dict(x=None)), (-1, dict(y=None)), (-1, dict(x=H(None, 1, 1))), (-1, dict(positions=None)), (-1, dict(table=None)),
                      (-2, dict(dtype=3)), (-2, dict(dtype=-1)), (-2, dict(tokens=-1)), (-2, dict(heads=0)), (-2, dict(head_dim=1)),
                      (-2, dict(head_dim=1025)), (-2, dict(rot=66)), (-2, dict(rot=0)), (-2, dict(rot=7)), (-2, dict(max_pos=0)),
                      (-2, dict(interleaved=2)), (-2, dict(inverse=-1)), (-2, dict(y=H(FAKE, 64, 128))), (-3, dict(x=H(FAKE + 1, 128, 64))),
                      (-3, dict(dtype=0, y=H(2 * FAKE + 2, 128, 64))), (-3, dict(table=FAKE + 8)), (-3, dict(positions=FAKE + 2))]:
        assert kv4.lib.qg_rope(*rope_args(kv4, **bad)) == code, (code, bad)
    assert kv4.lib.qg_rope(*rope_args(kv4, tokens=0, positions=None, x=H(None, 1, 1), y=H(None, 1, 1))) == 0    # nothing to do


def desc(kv4, **kw):
    return kv4.CacheDesc(**{**dict(data=FAKE, n_pages=4, kv_heads=2, head_dim=64, page_tokens=16), **kw})


def test_append_and_read_refusals(kv4):
    H, lib = kv4.Heads, kv4.lib

    def append(cache=None, none=False, **kw):
        p = kv4.AppendParams(k=H(FAKE, 128, 64), v=H(FAKE, 128, 64), slots=FAKE, positions=FAKE, table=FAKE, q=H(FAKE, 256, 64),
                             q_out=H(2 * FAKE, 256, 64), dtype=1, tokens=3, q_heads=4, max_pos=10, rot=32, interleaved=0)
        for k, v in kw.items():
            setattr(p, k, v)
        return lib.qg_kv4_append(ctypes.byref(cache or desc(kv4)), None if none else ctypes.byref(p), None)

    for code, bad in [(-1, dict(none=True)), (-1, dict(cache=desc(kv4, data=None))), (-3, dict(cache=desc(kv4, data=FAKE + 16))),
                      (-2, dict(cache=desc(kv4, head_dim=80))), (-2, dict(cache=desc(kv4, page_tokens=20))), (-2, dict(cache=desc(kv4, n_pages=0))),
                      (-2, dict(dtype=9)), (-2, dict(tokens=-1)), (-2, dict(tokens=1000001)), (-2, dict(q_heads=-1)), (-2, dict(q_heads=65535)),
                      (-1, dict(slots=None)), (-3, dict(slots=FAKE + 4)), (-1, dict(k=H(None, 1, 1))), (-1, dict(v=H(None, 1, 1))),
                      (-1, dict(q=H(None, 1, 1))), (-1, dict(q_out=H(None, 1, 1))), (-3, dict(k=H(FAKE + 1, 128, 64))),
                      (-2, dict(q_out=H(FAKE, 64, 64))), (-1, dict(table=None)), (-7, dict(rot=24)), (-2, dict(rot=128)), (-2, dict(max_pos=0)),
                      (-2, dict(interleaved=5))]:
        assert append(**bad) == code, (code, bad)
    assert append(tokens=0, slots=None, k=H(None, 1, 1)) == 0
    assert lib.qg_kv4_append(None, ctypes.byref(kv4.AppendParams()), None) == -1

    def read(cache=None, slots=FAKE, tokens=2, dtype=0, k=H(FAKE, 128, 64), v=H(FAKE, 128, 64)):
        return lib.qg_kv4_read(ctypes.byref(cache or desc(kv4)), slots, tokens, dtype, ctypes.byref(k) if k else None,
                               ctypes.byref(v) if v else None, None)

    for code, bad in [(-1, dict(k=None)), (-1, dict(v=None)), (-1, dict(slots=None)), (-3, dict(slots=FAKE + 4)), (-2, dict(dtype=3)),
                      (-2, dict(tokens=-2)), (-2, dict(cache=desc(kv4, kv_heads=0))), (-3, dict(k=H(FAKE + 2, 128, 64)))]:
        assert read(**bad) == code, (code, bad)
    assert read(tokens=0, slots=None) == 0


def attention_params(kv4, **kw):
    H = kv4.Heads
    p = kv4.AttentionParams(q=H(FAKE, 256, 64), out=H(FAKE, 256, 64), pages=FAKE, kv_lens=FAKE, q_starts=FAKE, workspace=FAKE,
                            workspace_bytes=1 << 30, scale=0.1, dtype=1, tokens=3, q_heads=4, batch=2, pages_stride=4, max_q_len=2,
                            max_kv_len=64, causal=1)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def test_attention_refusals(kv4):
    H, lib = kv4.Heads, kv4.lib

    def call(cache=None, **kw):
        return lib.qg_kv4_attention(ctypes.byref(cache or desc(kv4)), ctypes.byref(attention_params(kv4, **kw)), None)

    long = dict(pages_stride=1 << 16, max_kv_len=1 << 20)
    for code, bad in [(-2, dict(cache=desc(kv4, head_dim=32))), (-2, dict(dtype=5)), (-2, dict(tokens=-1)), (-2, dict(q_heads=3)), (-2, dict(q_heads=0)),
                      (-2, dict(batch=-1)), (-2, dict(max_q_len=-1)), (-2, dict(max_kv_len=65)), (-2, dict(max_kv_len=-1)), (-2, dict(scale=float("nan"))),
                      (-2, dict(scale=float("inf"))), (-2, dict(causal=2)), (-2, dict(pages_stride=-1, max_kv_len=0)), (-2, dict(q_starts=None)),
                      (-1, dict(kv_lens=None)), (-1, dict(pages=None)), (-1, dict(q=H(None, 1, 1))), (-1, dict(out=H(None, 1, 1))),
                      (-3, dict(kv_lens=FAKE + 2)), (-3, dict(pages=FAKE + 1)), (-3, dict(q_starts=FAKE + 2)), (-3, dict(out=H(FAKE + 1, 256, 64))),
                      (-4, dict(workspace_bytes=100, **long)), (-3, dict(workspace=FAKE + 8, **long)), (-2, dict(max_q_len=1 << 28))]:
        assert call(**bad) == code, (code, bad)
    for nothing in [dict(tokens=0), dict(batch=0), dict(max_q_len=0)]:
        assert call(kv_lens=None, pages=None, q=H(None, 1, 1), **nothing) == 0, nothing
    assert lib.qg_kv4_attention(ctypes.byref(desc(kv4)), None, None) == -1


def test_workspace_bytes(kv4):
    lib, c = kv4.lib, desc(kv4, n_pages=1 << 16)

    def size(q_heads, batch, max_q, max_kv):
        return lib.qg_kv4_attention_workspace_bytes(ctypes.byref(c), q_heads, batch, max_q, max_kv)

    assert size(8, 1, 1, 100) == 0                       # short: one workgroup has it all
    assert size(8, 1, 1, 100000) > 0
    assert size(7, 1, 1, 100000) == 0 and size(8, 0, 1, 1000) == 0 and size(8, 1, 0, 1000) == 0 and size(8, 1, 1, 0) == 0
    assert lib.qg_kv4_attention_workspace_bytes(None, 8, 1, 1, 1000) == 0


# ---- the plain implementation itself --------------------------------------------------------------------------------------


def test_reference_quantization_by_hand():
    x = np.zeros((4, 64), np.float32)
    x[0, :3] = [15.0, 7.49, -0.1]           # span 15.1: alpha a little above 1, theta 0: the negative one becomes 0
    x[1, 0], x[1, 1] = -5.0, 10.0           # alpha 1, theta 5
    x[3, 7] = 4.0
    code, word = ref.quantize(x)
    v = ref.worth(code, word)
    assert word[1] & 15 == 5 and code[1, 0] == 0 and code[1, 1] == 15 and v[1, 0] == -5 and v[1, 1] == 10 and (v[1, 2:] == 0).all()
    assert word[2] == 0 and (v[2] == 0).all()
    assert word[3] & 15 == 0 and code[3, 7] == 15 and abs(v[3, 7] - 4) < 1e-4 and (np.delete(v[3], 7) == 0).all()
    assert abs(v[0, 0] - 15.1) < 0.2 and word[0] & 15 == 0 and v[0, 2] == 0


def test_reference_quantization_is_within_half_a_step():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((500, 128)) * np.exp(rng.standard_normal((500, 1)) * 5)).astype(np.float32)
    code, word = ref.quantize(x)
    alpha = (word & np.uint32(0xFFFFFFF0)).view(np.float32)
    # rounding to a step, one end of the range cut by up to half a step more because theta is a whole number
    assert (np.abs(ref.worth(code, word) - x) <= 1.0001 * alpha[:, None]).all() and code.max() == 15 and code.min() == 0
    assert (np.abs(ref.worth(code, word) - x) <= 0.5001 * alpha[:, None]).mean() > 0.98


def test_reference_cache_round_trip():
    rng = np.random.default_rng(1)
    c = ref.Cache(np.zeros(3 * 2 * 32 * 72, np.uint8), 3, 2, 64, 32)
    code, word = ref.quantize(rng.standard_normal((2, 2, 2, 64)).astype(np.float32))
    for i, slot in enumerate((5, 95)):
        c.put(slot, code[i, 0], word[i, 0], code[i, 1], word[i, 1])
    for i, slot in enumerate((5, 95)):
        kc, kw, vc, vw = c.token(slot)
        assert (kc == code[i, 0]).all() and (kw == word[i, 0]).all() and (vc == code[i, 1]).all() and (vw == word[i, 1]).all()


def test_reference_attention_against_torch():
    import torch
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((3, 4, 64)), rng.standard_normal((9, 2, 64)), rng.standard_normal((9, 2, 64))
    got, _, _ = ref.attention(q, k, v, 0.3, True)
    t = [torch.from_numpy(x).transpose(0, 1) for x in (q, np.repeat(k, 2, 1), np.repeat(v, 2, 1))]
    mask = torch.arange(9)[None] <= 6 + torch.arange(3)[:, None]
    want = torch.nn.functional.scaled_dot_product_attention(*t, attn_mask=mask, scale=0.3).transpose(0, 1).numpy()
    assert np.allclose(got, want, atol=1e-12)
    assert (ref.attention(q, k[:2], v[:2], 0.3, True)[0][0] == 0).all()


def test_reference_frequencies():
    f = ref.frequencies(64, 10000.0)
    assert f[0] == 1 and abs(f[-1] - 10000.0 ** (-62 / 64)) < 1e-18
    for kind in ("by_index", "by_turns"):
        g = ref.frequencies(64, 10000.0, kind, factor=8.0, low=1.0, high=32.0, context=4096.0)
        turns = 4096 * f / (2 * np.pi)
        assert np.array_equal(g[turns > 64], f[turns > 64]) and np.allclose(g[turns < 0.5], f[turns < 0.5] / 8)
        assert (g <= f).all() and (g >= f / 8 * (1 - 1e-12)).all()
