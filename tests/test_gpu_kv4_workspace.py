"""One workspace of the attention for calls of all extents up to those that it was made for."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("D,Hq,Hkv", [(64, 4, 2), (128, 8, 1), (256, 4, 2)])
def test_workspace_of_the_largest_call(dtype, D, Hq, Hkv):
    import torch
    from paper_2101_05615_amd import kv4
    assert torch.cuda.is_available(), "this test needs the MI355X"
    dev, P, B, Q, L = torch.device("cuda:0"), 64, 40, 60, 4000
    W = (L + P - 1) // P
    cache = kv4.new_cache(W, Hkv, D, P, device=dev)             # one history, which all sequences share
    g = torch.Generator(device=dev).manual_seed(D)
    k, v = (torch.randn(L, Hkv, D, device=dev, generator=g) for _ in range(2))
    kv4.append(cache, k, v, torch.arange(L, device=dev))
    pages = torch.arange(W, dtype=torch.int32, device=dev).repeat(B, 1)
    all_q = torch.randn(B * Q, Hq, D, device=dev, generator=g).to(getattr(torch, dtype))
    ws = kv4.attention_workspace(cache, Hq, B, max_q_len=Q, max_kv_len=L)
    ws[kv4.COUNTER_BYTES:] = 0xFF                              # (only the counters need to be zero)
    split = 0
    for b, n, m in [(B, Q, L), (1, 1, L), (1, 1, L - 1), (1, 1, 1025), (1, 1, 2500), (3, 1, 3333), (16, 1, L), (B, 1, L), (1, Q, L), (1, 40, 1100),
                    (2, 33, L), (5, 7, 2000), (1, 9, 513), (B, 20, 1500), (1, 1, 100)]:
        q, t = all_q[:b * n], torch.arange(b + 1, dtype=torch.int32, device=dev) * n
        lens = (m - torch.arange(b, dtype=torch.int32, device=dev) * 37 % m).int().contiguous()
        own = kv4.attention_workspace(cache, Hq, b, max_q_len=n, max_kv_len=m)
        split += own is not None
        want = kv4.attention(q, cache, pages[:b], lens, q_starts=t, max_q_len=n, max_kv_len=m, workspace=own)
        got = kv4.attention(q, cache, pages[:b], lens, q_starts=t, max_q_len=n, max_kv_len=m, workspace=ws)
        assert torch.equal(got, want), (b, n, m)
        assert (ws[:kv4.COUNTER_BYTES] == 0).all(), (b, n, m)
    assert split > 10
