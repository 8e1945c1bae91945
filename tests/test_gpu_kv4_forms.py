"""Forms of the kernels that take over at certain sizes: two tiles of query rows a wave, two workgroups over the rows of 256 channels, keys
split among those, and the launches of large calls.  Bounds and oracles as in test_gpu_kv4.py."""
import numpy as np
import pytest

import kv4_reference as ref
from gpu_util import assert_same
from test_gpu_kv4 import TYPES, Batch, f32, rows, strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2101_05615_amd import kv4
    return kv4, torch, torch.device("cuda:0")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,P", [(64, 16), (64, 64), (128, 16), (128, 32), (256, 16), (256, 128)])
@pytest.mark.parametrize("q_lens", [[5, 1, 5, 4, 0, 5], [8, 8, 3, 8, 1, 7]])
def test_up_to_32_rows(env, dtype, D, P, q_lens):
    """Four query heads to a KV head: 20 and 32 rows, some sequences with fewer (a wave's second tile of rows, or workgroup, has none)."""
    b = Batch(env, [33, 64, 5, 131, 0, 200], 8, 2, D, P, dtype, seed=D + P, q_lens=q_lens)
    b.check(b.run())
    b.check(b.run(causal=False), causal=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,P,q_len", [(64, 32, 5), (64, 16, 8), (128, 16, 5), (128, 64, 8), (256, 64, 3), (256, 16, 4), (256, 32, 5), (256, 64, 8)])
def test_up_to_32_rows_split(env, dtype, D, P, q_len):
    """The same with keys split over workgroups: 12 to 32 rows, up to 32 rows of 256 channels in the join."""
    kv4, torch, dev = env
    b = Batch(env, [3000, 700, 2049, 1], 4, 1, D, P, dtype, seed=D + q_len, q_lens=[q_len, q_len, 2, 1])
    ws = kv4.attention_workspace(b.cache, 4, 4, max_q_len=q_len, max_kv_len=3000)
    ws[kv4.COUNTER_BYTES:] = 0xFF
    got = b.run(ws)
    b.check(got)
    assert (ws[kv4.COUNTER_BYTES:] != 0xFF).any() and (ws[:kv4.COUNTER_BYTES] == 0).all()
    assert torch.equal(got, b.run(ws))
    b.check(b.run(ws, causal=False), causal=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H,D,rot,interleaved", [(4099, 16, 64, 64, False), (2049, 20, 128, 64, True), (1201, 16, 256, 256, False)])
def test_rope_of_many_heads(env, dtype, T, H, D, rot, interleaved):
    """Launches of workgroups of 256 threads, an odd number of tokens, rows of a wider tensor."""
    kv4, torch, dev = env
    assert T * H * (D // 16) >= 256 * 1024
    rng = np.random.default_rng(T)
    dt = getattr(torch, dtype)
    table = kv4.rope_table(5000, rot, device=dev)
    pos = rng.integers(0, 5000, T).astype(np.int32)
    x, _ = strided(torch, dev, (T, H, D), dt, gap=D + 1, offset=1)
    x.copy_(torch.from_numpy(rng.standard_normal((T, H, D)).astype(np.float32)))
    tab = table.cpu().numpy()[pos][:, None]
    want = torch.from_numpy(ref.turn(f32(x), tab[..., :rot // 2], tab[..., rot // 2:], rot, interleaved)).to(dt).float().numpy()
    assert_same(f32(kv4.rope(x, torch.from_numpy(pos).to(dev), table, interleaved=interleaved)), want, "rotated")


@pytest.mark.parametrize("T,H,D,rot", [(70001, 64, 16, 16), (524291, 1, 6, 4)])
def test_rope_of_more_heads_than_a_launch_numbers(env, T, H, D, rot):
    """Beyond 2^22 heads of tokens a second span of workgroups; beyond 65535 times eight tokens, extents off 16, a second round."""
    kv4, torch, dev = env
    rng = np.random.default_rng(T)
    table = kv4.rope_table(5000, rot, device=dev)
    pos = rng.integers(0, 5000, T).astype(np.int32)
    x = torch.from_numpy(rng.standard_normal((T, H, D), dtype=np.float32)).to(dev).bfloat16()
    tab = table.cpu().numpy()[pos][:, None]
    want = torch.from_numpy(ref.turn(f32(x), tab[..., :rot // 2], tab[..., rot // 2:], rot, False)).bfloat16()
    assert torch.equal(kv4.rope(x, torch.from_numpy(pos).to(dev), table).cpu(), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("P,Hkv,Hq,D,T,rot,interleaved", [(64, 8, 3, 128, 2101, 128, False), (16, 4, 4, 64, 8209, 32, True), (256, 8, 1, 256, 1031, 128, False)])
def test_long_prompts(env, dtype, P, Hkv, Hq, D, T, rot, interleaved):
    """Appends and reads of workgroups of 256 threads, spread over the XCDs, an odd number of tokens; the cache's bytes."""
    kv4, torch, dev = env
    assert T * (D // 16) * 2 * Hkv >= 256 * 1024
    dt, rng = getattr(torch, dtype), np.random.default_rng(T)
    n_pages = (T + P - 1) // P + 2
    cache = kv4.new_cache(n_pages, Hkv, D, P, device=dev)
    cache.data.random_(0, 256)
    model = ref.Cache(cache.data.cpu().numpy().copy(), n_pages, Hkv, D, P)
    table = kv4.rope_table(9000, rot, device=dev)
    slots = (rng.permutation(n_pages)[np.arange(T) // P] * P + np.arange(T) % P).astype(np.int64)
    slots[[3, T - 2]] = -1
    pos = np.arange(7, 7 + T, dtype=np.int32)
    row = torch.from_numpy(rng.standard_normal((T, (Hq + 2 * Hkv) * D)).astype(np.float32)).to(dev).to(dt)      # a fused projection's rows
    q, k, v = (row[:, a * D:b * D].view(T, b - a, D) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
    k.copy_(torch.from_numpy(rows(rng, (T, Hkv, D))))
    tab = table.cpu().numpy()[pos][:, None]
    cos, sin = tab[..., :rot // 2], tab[..., rot // 2:]
    s = torch.from_numpy(slots).to(dev)
    got = kv4.append(cache, k, v, s, positions=torch.from_numpy(pos).to(dev), table=table, interleaved=interleaved, q=q)
    assert_same(f32(got), torch.from_numpy(ref.turn(f32(q), cos, sin, rot, interleaved)).to(dt).float().numpy(), "queries")
    (kc, kw), (vc, vw) = ref.quantize(ref.turn(f32(k), cos, sin, rot, interleaved)), ref.quantize(f32(v))
    for t in np.nonzero(slots >= 0)[0]:
        model.put(slots[t], kc[t], kw[t], vc[t], vw[t])
    assert_same(cache.data.cpu().numpy(), model.data.reshape(-1), "the cache's bytes")
    held = (slots >= 0)[:, None, None]
    for o, c, w in zip(kv4.read(cache, s, dtype=dt), (kc, vc), (kw, vw)):
        got, want = f32(o), torch.from_numpy(np.where(held, ref.worth(c, w), np.float32(0))).to(dt).float().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want))          # (an infinity among fp16 inputs: a poisoned head)
        assert_same(np.where(np.isnan(got), 0, got), np.where(np.isnan(want), 0, want), "read back")
