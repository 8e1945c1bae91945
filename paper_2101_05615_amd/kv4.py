"""Rotary positions, the paged 4-bit key/value cache and the attention over it (include/qgemm.h, the qg_rope* and qg_kv4_* calls).

    table = kv4.rope_table(max_pos, rot)                                   # once per model
    cache = kv4.new_cache(n_pages, kv_heads, head_dim, page_tokens)        # once per layer
    q = kv4.append(cache, k, v, slots, positions=pos, table=table, q=q)    # rotate q and k, store k and v in 4 bits
    o = kv4.attention(q, cache, pages, kv_lens)                            # one query token per sequence

Tensors of heads are [tokens, heads, head_dim] in float32, bfloat16 or float16 with any strides but a unit stride of channels:
views of a fused projection's rows are taken as they are.  rope() is differentiable; what goes through the cache carries no gradient.
Argument marshalling only, like qgemm.py: the calls that a program repeats first go through the extension module, and only a call that
it declines is marshalled, and its error named, here.
"""
import ctypes
import math

import torch
from torch.autograd import forward_ad

from .qgemm import QGemmError, _binding, _check, _stream, lib

F32, BF16, F16 = 0, 1, 2
COUNTER_BYTES = 65536   # QG_KV4_COUNTER_BYTES
MAX_KV_LEN = 1 << 30    # of a call
_TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
ROPE_PLAIN, ROPE_LINEAR, ROPE_BY_INDEX, ROPE_BY_TURNS = 0, 1, 2, 3
_SCALINGS = {"plain": ROPE_PLAIN, "linear": ROPE_LINEAR, "by_index": ROPE_BY_INDEX, "by_turns": ROPE_BY_TURNS}


class Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class RopeParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("base", "factor", "low", "high", "context", "magnitude")] + \
               [(n, ctypes.c_int32) for n in ("scaling", "rot", "max_pos")]


class CacheDesc(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p)] + [(n, ctypes.c_int32) for n in ("n_pages", "kv_heads", "head_dim", "page_tokens")]


class AppendParams(ctypes.Structure):
    _fields_ = [("k", Heads), ("v", Heads), ("slots", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("q", Heads), ("q_out", Heads)] + \
               [(n, ctypes.c_int32) for n in ("dtype", "tokens", "q_heads", "max_pos", "rot", "interleaved")]


class AttentionParams(ctypes.Structure):
    _fields_ = [("q", Heads), ("out", Heads), ("pages", ctypes.c_void_p), ("kv_lens", ctypes.c_void_p), ("q_starts", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t), ("scale", ctypes.c_float)] + \
               [(n, ctypes.c_int32) for n in ("dtype", "tokens", "q_heads", "batch", "pages_stride", "max_q_len", "max_kv_len", "causal")]


def _declare():
    vp, i, P = ctypes.c_void_p, ctypes.c_int, ctypes.POINTER
    lib.qg_rope_table.argtypes = [P(RopeParams), vp, vp]
    lib.qg_rope.argtypes = [P(Heads), i, i, i, i, vp, vp, i, i, i, i, P(Heads), vp]
    lib.qg_kv4_bytes.argtypes = [i, i, i, i]
    lib.qg_kv4_bytes.restype = ctypes.c_size_t
    lib.qg_kv4_append.argtypes = [P(CacheDesc), P(AppendParams), vp]
    lib.qg_kv4_read.argtypes = [P(CacheDesc), vp, i, i, P(Heads), P(Heads), vp]
    lib.qg_kv4_attention_workspace_bytes.argtypes = [P(CacheDesc), i, i, i, i]
    lib.qg_kv4_attention_workspace_bytes.restype = ctypes.c_size_t
    lib.qg_kv4_attention.argtypes = [P(CacheDesc), P(AttentionParams), vp]


_declare()


def _heads(x):
    return Heads(x.data_ptr(), x.stride(0), x.stride(1))


def _check_heads(x, like=None, heads=None, head_dim=None):
    assert x.is_cuda and x.dim() == 3 and x.dtype in _TYPES and (x.stride(2) == 1 or x.shape[2] <= 1)
    assert like is None or (x.dtype == like.dtype and x.shape[0] == like.shape[0])
    assert (heads is None or x.shape[1] == heads) and (head_dim is None or x.shape[2] == head_dim)


def _check_ints(x, dtype, *shape):
    assert x.is_cuda and x.dtype == dtype and x.is_contiguous() and tuple(x.shape) == shape


def _check_table(table):
    assert table.is_cuda and table.dtype == torch.float32 and table.dim() == 2 and table.is_contiguous()


def rope_table(max_pos, rot, base=10000.0, scaling="plain", factor=1.0, low=1.0, high=32.0, context=0.0, magnitude=1.0, device="cuda"):
    """fp32 [max_pos, rot]: the cosines, then the sines, of every position.  scaling: "plain", "linear", "by_index" or "by_turns"
    (qgemm.h: qg_rope_params)."""
    table = torch.empty((max_pos, rot), dtype=torch.float32, device=device)
    p = RopeParams(base, factor, low, high, context, magnitude, _SCALINGS[scaling], rot, max_pos)
    with torch.cuda.device(table.device):
        _check(lib.qg_rope_table(ctypes.byref(p), table.data_ptr(), _stream()), "qg_rope_table")
    return table


def rope(x, positions, table, interleaved=False, inverse=False, out=None):
    """x [tokens, heads, head_dim] with the first table.shape[1] channels of every head turned by the token's position (int32
    [tokens]); inverse: turned back, the gradient.  `out` may be x.  Differentiable in x where `out` is not given."""
    if x.requires_grad or table.requires_grad or forward_ad._current_level >= 0 or (out is not None and out.requires_grad):
        if _tracked(table) or (out is not None and (_tracked(x) or _tracked(out))):
            raise RuntimeError("kv4.rope has a gradient for x alone, and none with out=")
        if _tracked(x):
            return _Rope.apply(x, positions, table, interleaved, inverse)
    return _rope(x, positions, table, interleaved, inverse, out)


def _tracked(x):
    return (x.requires_grad and torch.is_grad_enabled()) or (forward_ad._current_level >= 0 and forward_ad.unpack_dual(x).tangent is not None)


class _Rope(torch.autograd.Function):
    """A linear map: its gradient is the map turned back, its differential the map itself."""

    @staticmethod
    def forward(ctx, x, positions, table, interleaved, inverse):
        ctx.save_for_backward(positions, table)
        ctx.save_for_forward(positions, table)
        ctx.interleaved, ctx.inverse = interleaved, inverse
        return _rope(x, positions, table, interleaved, inverse)

    @staticmethod
    def backward(ctx, g):
        g = g if g.stride(2) == 1 else g.contiguous()          # (of a sum, say: one number with strides of 0)
        return (rope(g, *ctx.saved_tensors, ctx.interleaved, not ctx.inverse),) + (None,) * 4

    @staticmethod
    def jvp(ctx, t, *_):
        t = t if t.stride(2) == 1 else t.contiguous()
        return rope(t, *ctx.saved_tensors, ctx.interleaved, ctx.inverse)


def _rope(x, positions, table, interleaved=False, inverse=False, out=None):
    done = _binding.rope(x, positions, table, interleaved, inverse, out)
    if done is not None:
        return done
    _check_heads(x)
    _check_table(table)
    T, H, D = x.shape
    _check_ints(positions, torch.int32, T)
    if out is None:
        out = torch.empty((T, H, D), dtype=x.dtype, device=x.device)
    else:
        _check_heads(out, x, H, D)
    a, b = _heads(x), _heads(out)
    _check(lib.qg_rope(ctypes.byref(a), _TYPES[x.dtype], T, H, D, positions.data_ptr(), table.data_ptr(), table.shape[0], table.shape[1],
                       int(bool(interleaved)), int(bool(inverse)), ctypes.byref(b), _stream()), "qg_rope")
    return out


def cache_bytes(n_pages, kv_heads, head_dim, page_tokens):
    """Bytes of the buffer of such a cache (0: not supported)."""
    return lib.qg_kv4_bytes(n_pages, kv_heads, head_dim, page_tokens)


class Cache:
    """A caller's uint8 buffer (contiguous, 64-byte aligned) as the 4-bit cache of one layer."""

    def __init__(self, data, kv_heads, head_dim, page_tokens):
        assert data.is_cuda and data.dtype == torch.uint8 and data.is_contiguous()
        per = cache_bytes(1, kv_heads, head_dim, page_tokens)
        if per == 0 or data.numel() < per:
            raise QGemmError(-2, "qg_kv4_bytes")
        self.data, self.n_pages = data, data.numel() // per
        self.kv_heads, self.head_dim, self.page_tokens = kv_heads, head_dim, page_tokens
        self._desc = CacheDesc(data.data_ptr(), self.n_pages, kv_heads, head_dim, page_tokens)
        self._ref, self._fast = ctypes.byref(self._desc), ctypes.addressof(self._desc)


def new_cache(n_pages, kv_heads, head_dim, page_tokens, device="cuda"):
    n = cache_bytes(n_pages, kv_heads, head_dim, page_tokens)
    if n == 0:
        raise QGemmError(-2, "qg_kv4_bytes")
    return Cache(torch.empty(n, dtype=torch.uint8, device=device), kv_heads, head_dim, page_tokens)


def append(cache, k, v, slots, positions=None, table=None, interleaved=False, q=None, q_out=None):
    """Stores k and v [tokens, kv_heads, head_dim] in the slots (int64 [tokens]; -1: not stored) in 4 bits, k rotated by its
    position if `positions` (int32 [tokens]) and `table` are given.  q [tokens, heads, head_dim] is rotated in the same pass into
    q_out (new; may be q), which is returned (None without q)."""
    done = _binding.kv4_append(cache, k, v, slots, positions, table, interleaved, q, q_out)
    if done is not None:
        return None if done is True else done
    _check_heads(k, None, cache.kv_heads, cache.head_dim)
    _check_heads(v, k, cache.kv_heads, cache.head_dim)
    T = k.shape[0]
    _check_ints(slots, torch.int64, T)
    p = AppendParams()
    p.k, p.v, p.slots = _heads(k), _heads(v), slots.data_ptr()
    if positions is not None:
        _check_ints(positions, torch.int32, T)
        _check_table(table)
        p.positions, p.table, p.max_pos, p.rot = positions.data_ptr(), table.data_ptr(), table.shape[0], table.shape[1]
    if q is not None:
        _check_heads(q, k, None, cache.head_dim)
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        else:
            _check_heads(q_out, q, q.shape[1], cache.head_dim)
        p.q, p.q_out, p.q_heads = _heads(q), _heads(q_out), q.shape[1]
    else:
        assert q_out is None
    p.dtype, p.tokens, p.interleaved = _TYPES[k.dtype], T, int(bool(interleaved))
    _check(lib.qg_kv4_append(cache._ref, ctypes.byref(p), _stream()), "qg_kv4_append")
    return q_out


def read(cache, slots, dtype=torch.float32, k=None, v=None):
    """What the slots (int64 [tokens]) hold: (keys, values) [tokens, kv_heads, head_dim] of `dtype`; outside the cache: zeros."""
    done = _binding.kv4_read(cache, slots, _TYPES[dtype], k, v)
    if done is not None:
        return done
    T = slots.shape[0]
    _check_ints(slots, torch.int64, T)
    shape = (T, cache.kv_heads, cache.head_dim)
    k = torch.empty(shape, dtype=dtype, device=slots.device) if k is None else k
    v = torch.empty(shape, dtype=dtype, device=slots.device) if v is None else v
    _check_heads(k, None, *shape[1:])
    _check_heads(v, k, *shape[1:])
    assert k.dtype == dtype and k.shape[0] == T
    a, b = _heads(k), _heads(v)
    _check(lib.qg_kv4_read(cache._ref, slots.data_ptr(), T, _TYPES[dtype], ctypes.byref(a), ctypes.byref(b), _stream()), "qg_kv4_read")
    return k, v


def attention_workspace_bytes(cache, q_heads, batch, max_q_len=1, max_kv_len=None):
    """Bytes that attention() with at most these extents wants (max_kv_len by default: any length); 0: no call splits its keys."""
    max_kv_len = MAX_KV_LEN if max_kv_len is None else max_kv_len
    return lib.qg_kv4_attention_workspace_bytes(cache._ref, q_heads, batch, max_q_len, max_kv_len)


def attention_workspace(cache, q_heads, batch, max_q_len=1, max_kv_len=None):
    """A workspace for attention() with at most these extents (max_kv_len by default: any length); None where no call splits its keys.
    One per stream that calls run on."""
    n = attention_workspace_bytes(cache, q_heads, batch, max_q_len, max_kv_len)
    if n == 0:
        return None
    ws = torch.empty(n, dtype=torch.uint8, device=cache.data.device)
    _check(lib.qg_gemm_workspace_init(ws.data_ptr(), min(n, COUNTER_BYTES), _stream()), "qg_gemm_workspace_init")
    return ws


def attention(q, cache, pages, kv_lens, q_starts=None, max_q_len=None, max_kv_len=None, scale=None, causal=True, workspace=None, out=None):
    """softmax(scale q k) v over the cached tokens of every sequence: q [tokens, heads, head_dim]; pages int32 [batch, n] names the
    pages of a sequence in order; kv_lens int32 [batch] its tokens.  q_starts int32 [batch + 1]: the rows of q that belong to a
    sequence, its last tokens (causal: query i of n sees the keys up to kv_len - n + i); None: one row each.  max_q_len,
    max_kv_len: the most of any sequence (default: the rows of q, or one without q_starts; what the page table holds), near bounds are
    faster.  Rows of q that no sequence has are not written: in a new result they hold anything.  scale: 1 / sqrt(head_dim)."""
    if max_q_len is None:
        max_q_len = 1 if q_starts is None else q.shape[0]
    done = _binding.kv4_attention(cache, q, pages, kv_lens, q_starts, max_q_len, max_kv_len, scale, causal, workspace, out)
    if done is not None:
        return done
    _check_heads(q, None, None, cache.head_dim)
    T, H, D = q.shape
    B, W = pages.shape
    assert H % cache.kv_heads == 0
    assert pages.is_cuda and pages.dtype == torch.int32 and (pages.stride(1) == 1 or W <= 1)
    _check_ints(kv_lens, torch.int32, B)
    if q_starts is not None:
        _check_ints(q_starts, torch.int32, B + 1)
    if out is None:
        out = torch.empty((T, H, D), dtype=q.dtype, device=q.device)
    else:
        _check_heads(out, q, H, D)
    p = AttentionParams()
    p.q, p.out, p.pages, p.kv_lens = _heads(q), _heads(out), pages.data_ptr(), kv_lens.data_ptr()
    p.q_starts = None if q_starts is None else q_starts.data_ptr()
    if workspace is not None:
        p.workspace, p.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    p.scale = 1.0 / math.sqrt(D) if scale is None else scale
    p.dtype, p.tokens, p.q_heads, p.batch, p.pages_stride = _TYPES[q.dtype], T, H, B, pages.stride(0) if B > 1 else W
    p.max_q_len, p.max_kv_len, p.causal = max_q_len, W * cache.page_tokens if max_kv_len is None else max_kv_len, int(bool(causal))
    assert p.max_kv_len <= W * cache.page_tokens
    _check(lib.qg_kv4_attention(cache._ref, ctypes.byref(p), _stream()), "qg_kv4_attention")
    return out
