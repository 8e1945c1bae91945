"""The example block: quantized products, rotation, 4-bit cache and attention together, piece by piece and token by token.  The products
have one right result (the oracle's); the attention between them is compared with 64 bits over the values that the cache holds."""
import math

import numpy as np
import pytest

import kv4_reference as ref
from gpu_util import assert_same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2101_05615_amd import attention_block
    import oracle
    oracle.build()
    return attention_block, torch, torch.device("cuda:0"), oracle


def product(oracle, x, side):
    codes, alpha, x_alpha = side[4]
    a = oracle.quantize_f32(np.ascontiguousarray(x), side[2], side[3])
    return oracle.gemm_u8s8_dequant_f32(a, side[3], codes, [0], None, x_alpha * alpha, False)


@pytest.mark.parametrize("heads,kv_heads,D,page", [(4, 2, 64, 16), (8, 1, 128, 32)])
def test_block(env, heads, kv_heads, D, page):
    ab, torch, dev, oracle = env
    rng = np.random.default_rng(3)
    hidden, batch = 96, 3
    w = lambda i, o: (rng.standard_normal((i, o)) / np.sqrt(i)).astype(np.float32)  # noqa: E731
    block = ab.AttentionBlock(w(hidden, (heads + 2 * kv_heads) * D), w(heads * D, hidden), heads, kv_heads, D, n_pages=40, page_tokens=page,
                              max_pos=200, x_range=(-4.0, 4.0), o_range=(-2.0, 2.0), rot=D // 2)
    seqs = ab.Batch(block, batch, 100)
    ws = block.workspace(batch, 40, 100)
    table = block.table.cpu().numpy()
    for new in ([40, 33, 7], [1, 1, 1], [5, 0, 20], [1, 1, 1]):
        pos, slots, lens, starts = seqs.grow(new)
        x = torch.from_numpy(rng.standard_normal((sum(new), hidden)).astype(np.float32)).to(dev)
        y = block(x, pos, slots, seqs.pages, lens, starts, max_q_len=40, max_kv_len=100, workspace=ws)
        torch.cuda.synchronize()
        row = product(oracle, x.cpu().numpy(), block.qkv)
        T, r = sum(new), table.shape[1]
        qh, kh, vh = (row[:, a * D:b * D].reshape(T, -1, D) for a, b in ((0, heads), (heads, heads + kv_heads), (heads + kv_heads, heads + 2 * kv_heads)))
        cs = table[pos.cpu().numpy()][:, None]
        qh, kh = (ref.turn(v, cs[..., :r // 2], cs[..., r // 2:], r, False) for v in (qh, kh))
        model = ref.Cache(block.cache.data.cpu().numpy(), 40, kv_heads, D, page)
        for t, s in enumerate(slots.cpu().numpy()):
            kc, kw, vc, vw = model.token(s)
            for got, want in zip((kc, kw, vc, vw), ref.quantize(kh[t]) + ref.quantize(vh[t])):
                assert_same(got, want, f"token {t} in the cache")
        # the output product of the attention's own result, and that result against 64 bits
        o = ab.kv4.attention(torch.from_numpy(qh).to(dev), block.cache, seqs.pages, lens, q_starts=starts, max_q_len=40, max_kv_len=100, workspace=ws)
        o = o.cpu().numpy()
        assert_same(y.cpu().numpy(), product(oracle, o.reshape(T, -1), block.out), "output product")
        for b in range(batch):
            t = np.arange(seqs.lens[b])
            k, v = model.load(seqs.pages[b].cpu().numpy()[t // page].astype(np.int64) * page + t % page)
            mine = slice(int(starts[b]), int(starts[b + 1]))
            want, mass, size = ref.attention(qh[mine].astype(np.float64), k, v, 1 / math.sqrt(D), True)
            # (the bound of test_gpu_kv4.py for fp32)
            bound = 2.0 ** -24 * np.abs(want) + (2.0 ** -21 * (1 + size) + 2 * (D + 16) * 2.0 ** -24 * size + 200 * 2.0 ** -24) * mass + 1e-6 * np.abs(v).max(initial=0)
            assert (np.abs(o[mine] - want) <= bound).all()


def test_example_runs(env, capsys):
    ab = env[0]
    ab.main(steps=3)
    lines = capsys.readouterr().out.splitlines()
    off = [float(line.split(" off")[0].split()[-1]) for line in lines if " off" in line]
    # 4-bit values of random weights are about 15 % off, and nothing averages that out; a wrong rotation, mask or page is of the order of 1
    assert len(off) == 6 and max(off) < 0.2, lines
