"""What the calls of kv4 take an argument to be that is not given."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2101_05615_amd import kv4
    return kv4, torch, torch.device("cuda:0")


def filled(env, lens, P=16, Hkv=2, D=64):
    """A cache with sequences of these lengths: (cache, pages, kv_lens)."""
    kv4, torch, dev = env
    W = max((m + P - 1) // P for m in lens)
    cache = kv4.new_cache(W * len(lens), Hkv, D, P, device=dev)
    pages = torch.arange(W * len(lens), dtype=torch.int32, device=dev).view(len(lens), W)
    for b, m in enumerate(lens):
        k, v = torch.randn(m, Hkv, D, device=dev), torch.randn(m, Hkv, D, device=dev)
        kv4.append(cache, k, v, b * W * P + torch.arange(m, device=dev))
    return cache, pages, torch.tensor(lens, dtype=torch.int32, device=dev)


@pytest.mark.parametrize("q_lens", [[5, 1, 3], [40, 0, 20], [1, 1, 1]])
def test_queries_of_a_sequence(env, q_lens):
    """With q_starts and no max_q_len every row of q is computed (new results reuse memory full of NaN here)."""
    kv4, torch, dev = env
    cache, pages, lens = filled(env, [50, 33, 40])
    T = sum(q_lens)
    starts = torch.tensor([0, q_lens[0], q_lens[0] + q_lens[1], T], dtype=torch.int32, device=dev)
    q = torch.randn(T, 4, 64, device=dev)
    want = kv4.attention(q, cache, pages, lens, q_starts=starts, max_q_len=T)
    junk = torch.full((T, 4, 64), float("nan"), device=dev)
    del junk
    got = kv4.attention(q, cache, pages, lens, q_starts=starts)
    assert torch.equal(got, want) and torch.isfinite(want).all()


def test_one_query_without_starts(env):
    kv4, torch, dev = env
    cache, pages, lens = filled(env, [50, 33, 40])
    q = torch.randn(3, 4, 64, device=dev)
    one = torch.arange(4, dtype=torch.int32, device=dev)
    assert torch.equal(kv4.attention(q, cache, pages, lens), kv4.attention(q, cache, pages, lens, q_starts=one, max_q_len=1))


def test_block_takes_all_queries(env):
    """The example block, prompts of several tokens and no max_q_len."""
    kv4, torch, dev = env
    import numpy as np
    from paper_2101_05615_amd.attention_block import AttentionBlock, Batch
    rng = np.random.default_rng(0)
    w = lambda i, o: (rng.standard_normal((i, o)) / np.sqrt(i)).astype(np.float32)  # noqa: E731
    out = []
    x = torch.randn(30, 96, device=dev)
    wq, wo = w(96, 8 * 64), w(4 * 64, 96)
    for kw in (dict(max_q_len=18), {}):
        block = AttentionBlock(wq, wo, 4, 2, 64, n_pages=8, page_tokens=16, max_pos=64, x_range=(-4.0, 4.0), o_range=(-2.0, 2.0))
        pos, slots, lens, starts = (seqs := Batch(block, 2, 32)).grow([18, 12])
        junk = torch.full((30, 4, 64), float("nan"), device=dev)
        del junk
        out.append(block(x, pos, slots, seqs.pages, lens, starts, **kw))
    assert torch.isfinite(out[0]).all()
    # (the same sums in another order where the bound chooses another kernel: one step of the 8-bit activations of the output product)
    assert (out[0] - out[1]).abs().max() <= 2 * (4.0 / 255) * np.abs(wo).max()


def test_workspace_for_any_length(env):
    """attention() without max_kv_len takes what the page table holds; attention_workspace() without it serves that, and keys are split."""
    kv4, torch, dev = env
    cache, pages, lens = filled(env, [3000])
    ws = kv4.attention_workspace(cache, 4, 1)
    assert ws is not None and ws.numel() == kv4.attention_workspace_bytes(cache, 4, 1) >= kv4.attention_workspace_bytes(cache, 4, 1, max_kv_len=3000)
    q = torch.randn(1, 4, 64, device=dev)
    ws[kv4.COUNTER_BYTES:] = 0xFF
    got = kv4.attention(q, cache, pages, lens, workspace=ws)
    assert (ws[kv4.COUNTER_BYTES:] != 0xFF).any()                       # (partial results went through it)
    assert torch.equal(got, kv4.attention(q, cache, pages, lens, max_kv_len=pages.shape[1] * 16,
                                          workspace=kv4.attention_workspace(cache, 4, 1, max_kv_len=pages.shape[1] * 16)))
