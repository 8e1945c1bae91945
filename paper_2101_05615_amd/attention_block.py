"""The attention of one decoder layer with quantized weights and a quantized cache, as a serving program would run it:

    fp32 activations -> int8 weights, one product for queries, keys and values (gemm_f32s8_dequant_f32)
    -> rotary positions, keys and values into the paged 4-bit cache (kv4.append)
    -> attention over the cache (kv4.attention)
    -> int8 weights, the output product (gemm_f32s8_dequant_f32)

`python -m paper_2101_05615_amd.attention_block` reads a batch of prompts in pieces, generates some tokens with the generation step
recorded into a HIP graph, compares everything with plain 64-bit arithmetic over the same weights and prints both errors and times.
"""
import numpy as np
import torch

from . import kv4
from . import qgemm as q


class AttentionBlock:
    """Weights are [in, out] fp32 (host), quantized per output channel to int8; activations by one scale and zero point."""

    def __init__(self, w_qkv, w_out, heads, kv_heads, head_dim, n_pages, page_tokens, max_pos, x_range, o_range, rot=None, device="cuda"):
        self.heads, self.kv_heads, self.head_dim, self.device = heads, kv_heads, head_dim, torch.device(device)
        self.qkv, self.out = self._pack(w_qkv, x_range), self._pack(w_out, o_range)
        self.table = kv4.rope_table(max_pos, rot or head_dim, device=device)
        self.cache = kv4.new_cache(n_pages, kv_heads, head_dim, page_tokens, device=device)

    def _pack(self, w, x_range):
        alpha = np.maximum(np.abs(w).max(0) / 127, 1e-12).astype(np.float32)         # per output channel, theta_B = 0
        codes = np.clip(np.rint(w / alpha), -127, 127).astype(np.int8)
        lo, hi = min(x_range[0], 0.0), max(x_range[1], 0.0)
        x_alpha = np.float32((hi - lo) / 255)
        zp = int(np.clip(round(-lo / float(x_alpha)), 0, 255))
        packed = q.pack_b(torch.from_numpy(codes).to(self.device), [0])
        scales = torch.from_numpy(x_alpha * alpha).to(self.device)
        return packed, scales, np.float32(1) / x_alpha, zp, (codes, alpha, x_alpha)

    def _product(self, x, side):
        packed, scales, inv, zp, _ = side
        return q.gemm_f32s8_dequant_f32(x, inv, zp, packed, None, scales, False)

    def project_in(self, x):
        """x fp32 [tokens, hidden] -> queries, keys, values: views of the product's rows."""
        T, H, G, D = x.shape[0], self.heads, self.kv_heads, self.head_dim
        row = self._product(x, self.qkv)
        return (row[:, :H * D].view(T, H, D), row[:, H * D:(H + G) * D].view(T, G, D), row[:, (H + G) * D:].view(T, G, D))

    def project_out(self, o):
        return self._product(o.view(o.shape[0], -1), self.out)

    def workspace(self, batch, max_q_len, max_kv_len):
        return kv4.attention_workspace(self.cache, self.heads, batch, max_q_len=max_q_len, max_kv_len=max_kv_len)

    def __call__(self, x, positions, slots, pages, kv_lens, q_starts=None, max_q_len=None, max_kv_len=None, workspace=None):
        """x [tokens, hidden] of new tokens, their positions and cache slots; the rest as kv4.attention (kv_lens counts the new ones)."""
        qh, kh, vh = self.project_in(x)
        kv4.append(self.cache, kh, vh, slots, positions=positions, table=self.table, q=qh, q_out=qh)
        o = kv4.attention(qh, self.cache, pages, kv_lens, q_starts=q_starts, max_q_len=max_q_len, max_kv_len=max_kv_len, workspace=workspace)
        return self.project_out(o)


class Batch:
    """Page bookkeeping of some sequences that grow: which pages they own, how long they are."""

    def __init__(self, block, batch, max_len, seed=0):
        self.P, self.dev = block.cache.page_tokens, block.device
        per = (max_len + self.P - 1) // self.P
        assert batch * per <= block.cache.n_pages
        order = torch.from_numpy(np.random.default_rng(seed).permutation(block.cache.n_pages)[:batch * per]).to(self.dev)
        self.pages = order.view(batch, per).to(torch.int32).contiguous()
        self.lens = [0] * batch

    def grow(self, new):
        """`new` tokens for each sequence: (positions, slots, kv_lens, q_starts), the lengths updated."""
        pos, slots, starts = [], [], [0]
        for b, n in enumerate(new):
            t = torch.arange(self.lens[b], self.lens[b] + n, device=self.dev)
            pos.append(t.to(torch.int32))
            slots.append(self.pages[b, t // self.P].long() * self.P + t % self.P)
            self.lens[b] += n
            starts.append(starts[-1] + n)
        as_int = lambda v: torch.tensor(v, dtype=torch.int32, device=self.dev)  # noqa: E731
        return torch.cat(pos), torch.cat(slots), as_int(self.lens), as_int(starts)


def _plain(block, history, new):
    """The new tokens' outputs in 64 bits over unquantized activations and cache: what quantization as a whole costs."""
    codes, alpha, _ = block.qkv[4]
    w_in = torch.from_numpy(codes.astype(np.float64) * alpha).to(block.device)
    codes, alpha, _ = block.out[4]
    w_out = torch.from_numpy(codes.astype(np.float64) * alpha).to(block.device)
    H, G, D = block.heads, block.kv_heads, block.head_dim
    out = []
    for x, n in zip(history, new):
        row = x.double() @ w_in
        T, r = x.shape[0], block.table.shape[1]
        cs = block.table[:T].double()[:, None]
        c, s = cs[..., :r // 2], cs[..., r // 2:]

        def turn(y):
            a, b = y[..., :r // 2], y[..., r // 2:r]
            return torch.cat([a * c - b * s, b * c + a * s, y[..., r:]], -1)

        qh, kh, vh = turn(row[:, :H * D].view(T, H, D)), turn(row[:, H * D:(H + G) * D].view(T, G, D)), row[:, (H + G) * D:].view(T, G, D)
        kh, vh = kh.repeat_interleave(H // G, 1), vh.repeat_interleave(H // G, 1)
        score = torch.matmul(qh[T - n:].transpose(0, 1), kh.permute(1, 2, 0).contiguous()) / D ** 0.5
        seen = torch.arange(T, device=x.device)[None] <= torch.arange(T - n, T, device=x.device)[:, None]
        p = score.masked_fill(~seen, float("-inf")).softmax(-1)
        out.append(torch.matmul(p, vh.transpose(0, 1).contiguous()).transpose(0, 1).reshape(n, H * D) @ w_out)
    return torch.cat(out)


def main(batch=4, hidden=1024, heads=8, kv_heads=2, head_dim=128, prompt=300, pieces=3, steps=8):
    rng = np.random.default_rng(0)
    dev = torch.device("cuda:0")
    w = lambda i, o: (rng.standard_normal((i, o)) / np.sqrt(i)).astype(np.float32)  # noqa: E731
    block = AttentionBlock(w(hidden, (heads + 2 * kv_heads) * head_dim), w(heads * head_dim, hidden), heads, kv_heads, head_dim, n_pages=64,
                           page_tokens=32, max_pos=512, x_range=(-4.0, 4.0), o_range=(-3.0, 3.0))
    seqs, max_len = Batch(block, batch, prompt + steps), prompt + steps
    ws = block.workspace(batch, prompt, max_len)
    history = [torch.zeros(0, hidden, device=dev) for _ in range(batch)]

    def error(y, new):
        want = _plain(block, history, new)
        return float((y.double() - want).norm() / want.norm())

    left = [prompt - 7 * b for b in range(batch)]              # prompts of different lengths, read in pieces
    for piece in range(pieces):
        new = [n // pieces if piece < pieces - 1 else n - n // pieces * (pieces - 1) for n in left]
        x = torch.randn(sum(new), hidden, device=dev).clamp_(-4, 4)
        for b, part in enumerate(x.split(new)):
            history[b] = torch.cat([history[b], part])
        pos, slots, lens, starts = seqs.grow(new)
        y = block(x, pos, slots, seqs.pages, lens, starts, max_q_len=max(new), max_kv_len=max_len, workspace=ws)
        print(f"piece {piece}: {sum(new)} tokens, {error(y, new):.3f} off unquantized 64 bits", flush=True)

    # one token a sequence: recorded once, replayed with new inputs
    x = torch.zeros(batch, hidden, device=dev)
    pos, slots, lens, _ = seqs.grow([1] * batch)
    call = lambda: block(x, pos, slots, seqs.pages, lens, max_kv_len=max_len, workspace=ws)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = call()
    for step in range(steps):
        x.copy_(torch.randn(batch, hidden, device=dev).clamp_(-4, 4))
        for b in range(batch):
            history[b] = torch.cat([history[b], x[b:b + 1]])
        if step:
            for a, b in zip((pos, slots, lens), seqs.grow([1] * batch)):
                a.copy_(b)
        graph.replay()
        print(f"step {step}: {error(y, [1] * batch):.3f} off", flush=True)
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    for _ in range(50):
        graph.replay()
    b.record()
    torch.cuda.synchronize()
    print(f"a step of {batch} sequences, {max(seqs.lens)} keys: {a.elapsed_time(b) / 50 * 1e3:.1f} us")


if __name__ == "__main__":
    main()
