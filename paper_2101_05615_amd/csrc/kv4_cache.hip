// Writing the 4-bit key/value cache, with the rotation of keys and queries on the way, and reading it back.
//
// A head of a token is quantized by itself (Eq. 1: alpha and theta from its least and largest channel), so D / 16 neighbouring
// lanes hold it in registers, 16 channels each, find the two extremes with cross-lane operations and store codes and word:
// one pass over the inputs, nothing in between.  Bound by memory (a long prompt) or by the launch (one token per sequence).
#include "qg_kv4.h"

namespace {

// The value of a neighbour in the row of 16 lanes, whose distance is a power of two: pairs, fours, eights, sixteens are folded in turn
template <int STEP>
__device__ inline float folded(float x) {
  constexpr int ctrl = STEP == 1 ? 0xB1 : STEP == 2 ? 0x4E : STEP == 4 ? 0x141 : 0x140;  // quad_perm, row_half_mirror, row_mirror
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), ctrl, 0xf, 0xf, true));
}
template <int LANES, typename F>
__device__ inline float fold(float x, F f) {
  x = f(x, folded<1>(x));
  x = f(x, folded<2>(x));
  if (LANES >= 8) x = f(x, folded<4>(x));
  if (LANES >= 16) x = f(x, folded<8>(x));
  return x;
}

template <int D>
struct head_codes {
  unsigned a, b;  // eight codes each, the lowest channel in the low bits
  unsigned word;
};

// The definition in qgemm.h, operation for operation
template <int D>
__device__ inline head_codes<D> quantize(const float* a, const float* b) {
  float lo = 0.0f, hi = 0.0f, bad = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo = fminf(lo, fminf(a[i], b[i]));
    hi = fmaxf(hi, fmaxf(a[i], b[i]));
    bad = bad + a[i] * 0.0f + b[i] * 0.0f;  // NaN once a channel is no finite number (the extremes skip a NaN)
  }
  lo = fold<D / 16>(lo, [](float x, float y) { return fminf(x, y); });
  hi = fold<D / 16>(hi, [](float x, float y) { return fmaxf(x, y); });
  bad = fold<D / 16>(bad, [](float x, float y) { return x + y; });
  const float span = (hi - lo) * (1.0f / 15.0f) + bad;
  head_codes<D> r = {0u, 0u, 0u};
  if (!(span < __builtin_inff())) {
    r.word = 0x7fc00000u;  // NaN, theta 0
    return r;
  }
  const unsigned bits = __builtin_bit_cast(unsigned, span) & ~15u;
  if (bits < 0x00800000u) return r;
  const float inv = 1.0f / __builtin_bit_cast(float, bits);
  const float theta = fminf(rintf(-lo * inv), 15.0f);
  r.word = bits | (unsigned)theta;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    r.a |= (unsigned)(fminf(fmaxf(rintf(a[i] * inv), -theta), 15.0f - theta) + theta) << (4 * i);
    r.b |= (unsigned)(fminf(fmaxf(rintf(b[i] * inv), -theta), 15.0f - theta) + theta) << (4 * i);
  }
  return r;
}

// Keys and values: a workgroup takes one head of neighbouring tokens, so that the 16-bit words of values that neighbours put next to each
// other leave it together.  Queries, as nothing of theirs is brought together: the heads of a token side by side, so that rows are read
// and written in one piece.  (8192 tokens, 32 query and 8 KV heads of 128 channels, and the read-back: 47 us, 55 with some heads of eight tokens for
// all three.)
template <int D, int TYPE>
__global__ void qg_kv4_append_kernel(qg_kv4_append_args p, int kv_blocks, int across) {
  typedef typename qg_elem<TYPE>::t t;
  constexpr int LANES = D / 16;
  const int per = (int)blockDim.x / LANES, local = (int)threadIdx.x / LANES, lane = (int)threadIdx.x % LANES;
  const bool is_q = (int)blockIdx.x >= kv_blocks;
  int head, token;
  bool is_v = false;
  if (is_q) {
    const unsigned unit = (blockIdx.x - kv_blocks) * per + local;
    token = (int)(unit / (unsigned)p.q_heads);
    head = (int)(unit - (unsigned)token * p.q_heads);
  } else {
    const unsigned kinds = 2 * p.c.heads, span = across * kinds, group = blockIdx.x / span, in_group = blockIdx.x - group * span;
    const int block = (int)(group * across + in_group % across), kind = (int)(in_group / across);
    is_v = kind >= p.c.heads;
    head = is_v ? kind - p.c.heads : kind;
    token = block * per + local;
  }
  if (token >= p.tokens) return;  // (a head's lanes go together)
  const t* x = is_q   ? static_cast<const t*>(p.q) + token * p.q_token + head * p.q_head
               : is_v ? static_cast<const t*>(p.v) + token * p.v_token + head * p.v_head
                      : static_cast<const t*>(p.k) + token * p.k_token + head * p.k_head;
  const bool turn = !is_v && p.positions != nullptr;
  const qg_runs r = qg_runs_of(lane, turn ? p.rot : 0, p.interleaved);
  float a[8], b[8];
  qg_load<TYPE, 8>(x + r.a, a);
  qg_load<TYPE, 8>(x + r.b, b);
  if (turn) {
    const int pos = p.positions[token];
    qg_turn_runs(a, b, r, (unsigned)pos < (unsigned)p.max_pos ? p.table + (size_t)pos * p.rot : nullptr, p.rot, p.interleaved, 1.0f);
  }
  if (is_q) {
    t* y = static_cast<t*>(p.q_out) + token * p.o_token + head * p.o_head;
    qg_store<TYPE, 8>(y + r.a, a);
    qg_store<TYPE, 8>(y + r.b, b);
    return;
  }
  const int64_t slot = p.slots[token];
  if (slot < 0 || slot >= (int64_t)p.c.n_pages << p.c.lgp) return;
  const int page = (int)(slot >> p.c.lgp), P = 1 << p.c.lgp, at = (int)slot & (P - 1);
  uint8_t* block = p.c.data + qg_kv4_block<D>(p.c, page, head);
  const head_codes<D> h = quantize<D>(a, b);
  if (is_v) {
    uint16_t* v = reinterpret_cast<uint16_t*>(block + (size_t)P * (D / 2)) + (size_t)(at >> 3) * (2 * D) + (at & 7);
    v[(r.a / 4) * 8] = (uint16_t)h.a;
    v[(r.a / 4) * 8 + 8] = (uint16_t)(h.a >> 16);
    v[(r.b / 4) * 8] = (uint16_t)h.b;
    v[(r.b / 4) * 8 + 8] = (uint16_t)(h.b >> 16);
  } else {
    unsigned* k = reinterpret_cast<unsigned*>(block + (size_t)at * (D / 2));
    k[r.a / 8] = h.a;
    k[r.b / 8] = h.b;
  }
  if (lane == 0) reinterpret_cast<unsigned*>(block + (size_t)P * D)[(at >> 3) * 16 + (is_v ? 8 : 0) + (at & 7)] = h.word;
}

template <int D, int TYPE>
__global__ void qg_kv4_read_kernel(qg_kv4_read_args p, int across) {
  typedef typename qg_elem<TYPE>::t t;
  constexpr int LANES = D / 16;
  const unsigned kinds = 2 * p.c.heads, span = across * kinds, group = blockIdx.x / span, in_group = blockIdx.x - group * span;
  const int kind = (int)(in_group / across);
  const int lane = (int)threadIdx.x % LANES;
  const long long token = ((long long)(group * across + in_group % across) * blockDim.x + threadIdx.x) / LANES;
  if (token >= p.tokens) return;
  const bool is_v = kind >= p.c.heads;
  const int head = is_v ? kind - p.c.heads : kind;
  t* y = is_v ? static_cast<t*>(p.v) : static_cast<t*>(p.k);
  if (y == nullptr) return;
  y += is_v ? token * p.v_token + head * p.v_head : token * p.k_token + head * p.k_head;
  const int64_t slot = p.slots[token];
  unsigned w[2] = {0u, 0u}, word = 0u;
  if (slot >= 0 && slot < (int64_t)p.c.n_pages << p.c.lgp) {
    const int page = (int)(slot >> p.c.lgp), P = 1 << p.c.lgp, at = (int)slot & (P - 1);
    const uint8_t* block = p.c.data + qg_kv4_block<D>(p.c, page, head);
    if (is_v) {
      const uint16_t* v = reinterpret_cast<const uint16_t*>(block + (size_t)P * (D / 2)) + (size_t)(at >> 3) * (2 * D) + (at & 7);
      w[0] = v[(4 * lane) * 8] | (unsigned)v[(4 * lane + 1) * 8] << 16;
      w[1] = v[(4 * lane + 2) * 8] | (unsigned)v[(4 * lane + 3) * 8] << 16;
    } else {
      const unsigned* k = reinterpret_cast<const unsigned*>(block + (size_t)at * (D / 2));
      w[0] = k[2 * lane];
      w[1] = k[2 * lane + 1];
    }
    word = reinterpret_cast<const unsigned*>(block + (size_t)P * D)[(at >> 3) * 16 + (is_v ? 8 : 0) + (at & 7)];
  }
  const float alpha = __builtin_bit_cast(float, word & ~15u);
  const int theta = (int)(word & 15u);
  float x[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = alpha * (float)((int)(w[i / 8] >> (4 * (i % 8)) & 15u) - theta);
  qg_store<TYPE, 8>(y + 16 * lane, x);
  qg_store<TYPE, 8>(y + 16 * lane + 8, x + 8);
}


#define QG_BY_TYPE(KERNEL, D, ...)                                                                      \
  switch (dtype) {                                                                                      \
    case QG_F32: hipLaunchKernelGGL((KERNEL<D, QG_F32>), grid, dim3(block), 0, s, __VA_ARGS__); break;  \
    case QG_BF16: hipLaunchKernelGGL((KERNEL<D, QG_BF16>), grid, dim3(block), 0, s, __VA_ARGS__); break; \
    default: hipLaunchKernelGGL((KERNEL<D, QG_F16>), grid, dim3(block), 0, s, __VA_ARGS__);             \
  }
#define QG_BY_HEAD(KERNEL, ...)                             \
  switch (head_dim) {                                       \
    case 64: QG_BY_TYPE(KERNEL, 64, __VA_ARGS__); break;    \
    case 128: QG_BY_TYPE(KERNEL, 128, __VA_ARGS__); break;  \
    default: QG_BY_TYPE(KERNEL, 256, __VA_ARGS__);          \
  }

// one wave a workgroup while that leaves CUs idle otherwise
int block_of(long long threads) { return threads < 256 * 1024 ? 64 : 256; }
// Workgroups of neighbouring tokens side by side, those of a token's heads behind each other: ids that differ by eight share an L2
// (8192 tokens of 32 query and 8 KV heads: rows of the table fetched once instead of by every XCD, 40 -> 36 us; read-back 11.4 -> 11.2).
// Small calls: ids in their order, no workgroups for nothing.
int across_of(long long blocks, int kinds) { return blocks >= 64 && blocks * kinds >= 1024 ? 8 : 1; }

}  // namespace

hipError_t qg_launch_kv4_append(const qg_kv4_append_args& a, int head_dim, int dtype, hipStream_t s) {
  const int kinds = 2 * a.c.heads + a.q_heads, lanes = head_dim / 16, block = block_of((long long)a.tokens * lanes * kinds), per = block / lanes;
  const long long blocks = ((long long)a.tokens + per - 1) / per;
  const int across = across_of(blocks, 2 * a.c.heads);
  const int kv_blocks = (int)((blocks + across - 1) / across * across * (2 * a.c.heads));
  const dim3 grid((unsigned)(kv_blocks + ((long long)a.tokens * a.q_heads + per - 1) / per));
  QG_BY_HEAD(qg_kv4_append_kernel, a, kv_blocks, across)
  return hipGetLastError();
}

hipError_t qg_launch_kv4_read(const qg_kv4_read_args& a, int head_dim, int dtype, hipStream_t s) {
  const int kinds = 2 * a.c.heads, lanes = head_dim / 16, block = block_of((long long)a.tokens * lanes * kinds);
  const long long blocks = ((long long)a.tokens * lanes + block - 1) / block;
  const int across = across_of(blocks, kinds);
  const dim3 grid((unsigned)((blocks + across - 1) / across * across * kinds));
  QG_BY_HEAD(qg_kv4_read_kernel, a, across)
  return hipGetLastError();
}
