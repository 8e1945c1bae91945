// Attention over the 4-bit key/value cache.
//
// A wave owns 16 query rows (the query heads that share a KV head, times the queries of a sequence), or NR times that, and walks
// over tiles of 32 tokens.  Both products run on v_mfma_f32_16x16x32_f16, transposed:
//   S^T = K Q^T   first operand 16 tokens x 32 channels, second 32 channels x 16 rows
//   O^T = V^T P^T first operand 16 channels x 32 tokens, second 32 tokens x 16 rows
// so that a lane keeps to one query row (its column l % 16) from the scores to the output: the running maximum and sum are a
// register each, and what a lane gets of S^T, tokens 8g .. 8g+7 (g = l / 16; the rows of the two key tiles are dealt that way),
// is in place as the second operand of the other product.
//
// The codes never become dequantized numbers: the scales go to the other side, a key's onto the score, a value's onto the
// probability.  The 16 scale-and-theta words of 8 tokens lie in the 16 lanes of a DPP row, where every lane of the row reaches them
// as an operand.  The zero points:
//   values  code - theta is a whole number of at most 15 and exact in fp16.  A dword of codes becomes eight of them with one shift,
//           four and-or (the exponent of 1024 put around a nibble) and four packed additions that take away 1024 + theta.
//   keys    a nibble alone in bits 4 to 7 of an fp16 is the number code * 2^-20, which the matrix cores take as it is (four ANDs and
//           three shifts), and theta comes off the sum, sum q (code - theta) = sum q code - theta sum q, with one fused multiply-add
//           per score.  fp32 results would see the cancellation: there keys go as values do.
// (Taking theta off the second product's sums as well is 10 % fewer instructions, but where the token that has all the weight is
// worth 0, 2^-21 of its neighbours' size is left: measured, 6 % of a result that came from the other tokens.  Nibbles in bits 0
// to 3 would save two shifts, but products of numbers this small are aligned by the exponent 2^-14 that their format gives them:
// over 32 products code * 2^-24 measured 2e-6 off the sum of their sizes, code * 2^-20 5e-8.)
//
// Rounding.  Queries become fp16 after a power of two per row that puts the largest channel near 2^14: exact for fp16 and
// bf16 channels down to 2^-24 of the largest; fp32 queries take two fp16 (22 bits).  Probabilities times value scale become fp16
// (two for fp32 results) against a running reference for both, so that they lie below 2^14 and keep 11 bits down to 2^-14.
// Scores, maxima, sums and outputs are fp32.
#include "qg_kv4.h"

namespace {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

constexpr int TILE = 32;    // tokens of a wave's step
constexpr int WAVES = 4;    // of a workgroup
constexpr float START = -1e30f;  // the running maximum before the first key
constexpr float BOOST = 4.0f;    // probabilities are held times 2^BOOST ...
constexpr float SLACK = 12.0f;   // ... and the reference moves when one would pass 2^SLACK

template <int J>
__device__ inline float row_lane(float x) {  // lane J of the caller's row of 16
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x150 + J, 0xf, 0xf, true));
}
template <int J>
__device__ inline unsigned row_lane(unsigned x) {
  return (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x150 + J, 0xf, 0xf, true);
}

union frag {
  unsigned u[4];
  h2 h[4];
  h8 v;
};

__device__ inline h2 as_h2(unsigned x) { return __builtin_bit_cast(h2, x); }

// Eight codes of a dword as four pairs (nibbles 0 4, 1 5, 2 6, 3 7), times 2^-20
__device__ inline void spread(unsigned x, unsigned* out) {
  out[0] = x << 4 & 0x00f000f0u;
  out[1] = x & 0x00f000f0u;
  out[2] = x >> 4 & 0x00f000f0u;
  out[3] = x >> 8 & 0x00f000f0u;
}

// The same less theta, in units of 1: 1024 + c or 1024 + 16 c, whose bits are a nibble under the exponent of 1024, less 1024 + theta.
// low: -(1024 + theta) twice; high: -(64 + theta).  (The masks live in registers: and-or takes no constants.)
struct masks {
  unsigned even, odd, magic;
  __device__ inline masks() : even(0x000f000fu), odd(0x00f000f0u), magic(0x64006400u) { asm("" : "+s"(even), "+s"(odd), "+v"(magic)); }
};
__device__ inline void spread_less(unsigned x, const masks& m, h2 low, h2 high, unsigned* out) {
  const h2 sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f};
  const unsigned y = x >> 8;
  out[0] = __builtin_bit_cast(unsigned, as_h2((x & m.even) | m.magic) + low);
  out[1] = __builtin_bit_cast(unsigned, __builtin_elementwise_fma(as_h2((x & m.odd) | m.magic), sixteenth, high));
  out[2] = __builtin_bit_cast(unsigned, as_h2((y & m.even) | m.magic) + low);
  out[3] = __builtin_bit_cast(unsigned, __builtin_elementwise_fma(as_h2((y & m.odd) | m.magic), sixteenth, high));
}

template <int D>
struct tile_bits {
  unsigned k[2][D / 32];  // tile a of 16 tokens: D / 4 channels of one token
  u4 v[D / 64];           // four channels of 8 tokens each
  unsigned w;             // a word of the row's 8 tokens: keys 0 .. 7, then values
};

// What a wave reads of the cache.  SMALL: pages of 16 tokens, two to a tile; otherwise a tile lies in one page, whose address is
// the same for all lanes.
template <int D, bool SMALL>
struct reader {
  uint8_t* data;
  const int32_t* table;  // the sequence's pages
  int n_pages, heads, lgp, head, last_page;   // the last page that holds a key
  unsigned key_lane, value_lane, word_lane;   // this lane's bytes past the tile's
  bool key_half, value_half;                  // SMALL: the lane's run of 8 tokens lies in the tile's second page

  __device__ inline reader(const qg_kv4_attention_args& p, int seq, int kv_head, int keys, int r, int g)
      : data(p.c.data), table(p.pages + (int64_t)seq * p.pages_stride), n_pages(p.c.n_pages), heads(p.c.heads), lgp(SMALL ? 4 : p.c.lgp),
        head(kv_head), last_page(max((keys - 1) >> (SMALL ? 4 : p.c.lgp), 0)) {
    const int key_run = r >> 2, key_at = SMALL ? key_run & 1 : key_run, value_at = SMALL ? g & 1 : g;
    key_lane = (unsigned)((8 * key_at + (r & 3)) * (D / 2) + g * (D / 8));
    value_lane = (unsigned)(value_at * (4 * D) + r * (D / 4));
    word_lane = (unsigned)(value_at * 64 + r * 4);
    key_half = key_run >= 2;
    value_half = g >= 2;
  }
  __device__ inline const uint8_t* block(int index) const {
    unsigned page = (unsigned)table[min(index, last_page)];
    page = page < (unsigned)n_pages ? page : 0u;
    return data + ((size_t)page * heads + head) * ((size_t)(D + 8) << lgp);
  }
  __device__ inline void load(int t0, tile_bits<D>& b) const {
    const int P = 1 << lgp;
    const uint8_t *kb, *vb, *wb;
    if (SMALL) {
      const uint8_t *first = block(t0 >> 4), *second = block((t0 >> 4) + 1);
      kb = key_half ? second : first;
      vb = (value_half ? second : first) + 16 * (D / 2);
      wb = vb + 16 * (D / 2);
    } else {
      const uint8_t* page = block(t0 >> lgp);
      const int at = t0 & (P - 1);
      kb = page + at * (D / 2);
      vb = page + (P + at) * (D / 2);
      wb = page + P * D + at * 8;
    }
    const uint8_t* k = kb + key_lane;
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      if (D == 64) {
        const uint2 x = *reinterpret_cast<const uint2*>(k + a * 4 * (D / 2));
        b.k[a][0] = x.x;
        b.k[a][1] = x.y;
      } else {
#pragma unroll
        for (int i = 0; i < D / 128; ++i) {
          const u4 x = reinterpret_cast<const u4*>(k + a * 4 * (D / 2))[i];
#pragma unroll
          for (int j = 0; j < 4; ++j) b.k[a][4 * i + j] = x[j];
        }
      }
    }
    const uint8_t* v = vb + value_lane;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) b.v[i] = reinterpret_cast<const u4*>(v)[i];
    b.w = *reinterpret_cast<const unsigned*>(wb + word_lane);
  }
};

// The state of a wave: NR tiles of 16 rows
template <int D, int DIG, int NR>
struct state {
  frag q[NR][DIG][D / 32];
  f4 o[NR][D / 16];
  float m[NR], l[NR];              // reference of the exponents (log2), sum (this lane's tokens)
  float factor[NR], factor_lo[NR]; // log2 score of a product and a key's scale, in two parts (the second: DIG 2)
  float q_sum[NR];                 // DIG 1: less the sum of the queries, times 2^-20
  int limit[NR];                   // last token that the row sees
  int vref;                        // biased exponent of the value scales' reference, 1 .. 253
};

__device__ inline float across_max(float x) {  // over the four lanes of a row of queries
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float across_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

template <int DIG>
__device__ inline float exponent(float z, float factor, float factor_lo, float base) {
  // DIG 2: the factor's own rounding (2^-24 of every score) is more than the rest of an fp32 result's error
  return DIG == 2 ? __builtin_fmaf(z, factor, __builtin_fmaf(z, factor_lo, base)) : __builtin_fmaf(z, factor, base);
}

// One tile.  MASKED: tokens from `end` on are not there, and a row may end inside.
template <int D, int DIG, int NR, bool MASKED>
__device__ inline void step(state<D, DIG, NR>& s, const tile_bits<D>& b, int t0, int end, int r, int g) {
  unsigned word = b.w;
  if (MASKED && t0 + 8 * g + (r & 7) >= end) word = 0u;
  const unsigned theta = word & 15u;
  const float scale = __builtin_bit_cast(float, word & ~15u);
  const masks m;

  // ---- scores
  f4 z[NR][2];
#pragma unroll
  for (int a = 0; a < 2; ++a) {
    h2 low = {}, high = {};
    if (DIG == 2) {
      // theta of the token that this lane holds as first operand: row r of tile a is token 8 (r / 4) + 4 a + r % 4
      const unsigned th = (unsigned)__builtin_amdgcn_ds_bpermute((16 * (r >> 2) + 4 * a + (r & 3)) * 4, (int)theta) * 0x10001u;
      low = as_h2(th + 0xE400E400u);
      high = as_h2((th << 4) + 0xD400D400u);
    }
#pragma unroll
    for (int n = 0; n < NR; ++n) z[n][a] = (f4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      frag k;
      if (DIG == 2)
        spread_less(b.k[a][i], m, low, high, k.u);
      else
        spread(b.k[a][i], k.u);
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int d = 0; d < DIG; ++d) z[n][a] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k.v, s.q[n][d][i].v, z[n][a], 0, 0, 0);
    }
  }

  // ---- exponents; the references move rarely
  const float ks[8] = {row_lane<0>(scale), row_lane<1>(scale), row_lane<2>(scale), row_lane<3>(scale),
                       row_lane<4>(scale), row_lane<5>(scale), row_lane<6>(scale), row_lane<7>(scale)};
  if (DIG == 1) {
    const float t = (float)theta;
    const float zp[8] = {row_lane<0>(t), row_lane<1>(t), row_lane<2>(t), row_lane<3>(t),
                         row_lane<4>(t), row_lane<5>(t), row_lane<6>(t), row_lane<7>(t)};
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int j = 0; j < 8; ++j) z[n][j >> 2][j & 3] = __builtin_fmaf(zp[j], s.q_sum[n], z[n][j >> 2][j & 3]);
  }
  const int vexp = (word & 0x7f800000u) != 0x7f800000u && r >= 8 ? min((int)(word >> 23 & 255u), 253) : 0;
  bool move = vexp > s.vref;
  float y[NR][8];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const float base = BOOST - s.m[n];
    float top = -__builtin_inff();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      z[n][j >> 2][j & 3] *= ks[j];
      y[n][j] = exponent<DIG>(z[n][j >> 2][j & 3], s.factor[n], s.factor_lo[n], base);
      if (MASKED) {
        const int t = t0 + 8 * g + j;
        if (t >= end || t > s.limit[n]) y[n][j] = -__builtin_inff();
      }
      top = fmaxf(top, y[n][j]);
    }
    move |= top > SLACK;
  }
  if (__builtin_expect(__ballot(move) != 0ull, 0)) {
    int e = vexp;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) e = max(e, __shfl_xor(e, d));
    const int vref = max(s.vref, e);
    const float shrink = __builtin_amdgcn_exp2f((float)(s.vref - vref));
    s.vref = vref;
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      float high = -__builtin_inff();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int t = t0 + 8 * g + j;
        const float x = z[n][j >> 2][j & 3] * s.factor[n];
        high = fmaxf(high, MASKED && (t >= end || t > s.limit[n]) ? -__builtin_inff() : x);
      }
      const float top = fmaxf(s.m[n], across_max(high));
      const float f = __builtin_amdgcn_exp2f(s.m[n] - top);
      s.m[n] = top;
      s.l[n] *= f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) s.o[n][i] *= f * shrink;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        y[n][j] = exponent<DIG>(z[n][j >> 2][j & 3], s.factor[n], s.factor_lo[n], BOOST - top);
        if (MASKED) {
          const int t = t0 + 8 * g + j;
          if (t >= end || t > s.limit[n]) y[n][j] = -__builtin_inff();
        }
      }
    }
  }

  // ---- probabilities times value scale
  const float vscale = scale * __builtin_bit_cast(float, (unsigned)(254 - s.vref) << 23);
  const float vs[8] = {row_lane<8>(vscale),  row_lane<9>(vscale),  row_lane<10>(vscale), row_lane<11>(vscale),
                       row_lane<12>(vscale), row_lane<13>(vscale), row_lane<14>(vscale), row_lane<15>(vscale)};
  frag p[NR][DIG];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float e = __builtin_amdgcn_exp2f(y[n][j]);
      s.l[n] += e;
      float x = e * vs[j];
      if (MASKED) {
        const int t = t0 + 8 * g + j;
        if (t >= end || t > s.limit[n]) x = 0.0f;  // (a masked value may be NaN)
      }
      const _Float16 hi = (_Float16)x;
      p[n][0].v[j] = hi;
      if (DIG == 2) p[n][DIG - 1].v[j] = (_Float16)(x - (float)hi);
    }
  }

  // ---- output.  theta of tokens 2 i and 2 i + 1 in a pair, from the lanes of the row that hold their words
  const unsigned next = (unsigned)__builtin_amdgcn_mov_dpp((int)theta, 0x101, 0xf, 0xf, true);  // row_shl:1
  const unsigned pair = theta | next << 16;
  const unsigned low = pair + 0xE400E400u, high = (pair << 4) + 0xD400D400u;
  const h2 lows[4] = {as_h2(row_lane<8>(low)), as_h2(row_lane<10>(low)), as_h2(row_lane<12>(low)), as_h2(row_lane<14>(low))};
  const h2 highs[4] = {as_h2(row_lane<8>(high)), as_h2(row_lane<10>(high)), as_h2(row_lane<12>(high)), as_h2(row_lane<14>(high))};
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    frag v[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      unsigned x[4];
      spread_less(b.v[i][t], m, lows[t], highs[t], x);
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c].u[t] = x[c];
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int d = 0; d < DIG; ++d) s.o[n][4 * i + c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[c].v, p[n][d].v, s.o[n][4 * i + c], 0, 0, 0);
  }
}

// The queries of a lane: row `row` of its column, channels (D/4) g .. of it, as fp16 scaled by a power of two
template <int D, int DIG, int NR, int TYPE>
__device__ inline void load_q(state<D, DIG, NR>& s, int n, const typename qg_elem<TYPE>::t* q, bool there, float scale_log2e,
                              float scale_log2e_lo, int g) {
  float x[D / 4];
  if (there) {
    qg_load<TYPE, D / 4>(q + g * (D / 4), x);
  } else {
#pragma unroll
    for (int i = 0; i < D / 4; ++i) x[i] = 0.0f;
  }
  unsigned top = 0u;
#pragma unroll
  for (int i = 0; i < D / 4; ++i) top = max(top, __builtin_bit_cast(unsigned, x[i]) & 0x7fffffffu);
  top = max(top, (unsigned)__shfl_xor((int)top, 16));
  top = max(top, (unsigned)__shfl_xor((int)top, 32));
  const int shift = top == 0u ? 0 : 14 + 127 - max((int)(top >> 23), 1);
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = 8 * i + (j >> 1) + 4 * (j & 1);  // the order in which the codes of a dword are spread
      // (an infinity or NaN: the row's scores become NaN)
      const float y = top < 0x7f800000u ? __builtin_ldexpf(x[c], shift) : __builtin_nanf("");
      const _Float16 hi = (_Float16)y;
      s.q[n][0][i].v[j] = hi;
      if (DIG == 2) s.q[n][DIG - 1][i].v[j] = (_Float16)(y - (float)hi);
      if (DIG == 1) sum += (float)hi;
    }
  if (DIG == 1) s.q_sum[n] = across_sum(sum) * -0x1p-20f;
  s.factor[n] = __builtin_ldexpf(scale_log2e, (DIG == 1 ? 20 : 0) - shift);
  s.factor_lo[n] = __builtin_ldexpf(scale_log2e_lo, -shift);
}

// Four consecutive channels of a finished row
template <int TYPE>
__device__ inline void write_out(const qg_kv4_attention_args& p, int token, int head, int c, const float* x) {
  typedef typename qg_elem<TYPE>::t t;
  qg_store<TYPE, 4>(static_cast<t*>(p.out) + (int64_t)token * p.o_token + (int64_t)head * p.o_head + c, x);
}

__device__ inline void hand_in(float* to, float a, float b) {  // past the caches that other workgroups do not share
  __hip_atomic_store(reinterpret_cast<u64*>(to), (u64)__builtin_bit_cast(unsigned, a) | (u64)__builtin_bit_cast(unsigned, b) << 32,
                     __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// TOKENS: the workgroup's waves share the same rows and split its tokens; otherwise they split its rows.
template <int D, int DIG, int TYPE, int NR, bool TOKENS, bool SMALL>
__global__ __launch_bounds__(64 * WAVES, 2) void qg_kv4_attention_kernel(qg_kv4_attention_args p) {
  constexpr int ROWS = 16 * NR * (TOKENS ? 1 : WAVES);  // of the workgroup
  constexpr int PITCH = D + 4;
  __shared__ float part[TOKENS ? WAVES * ROWS * PITCH : 1];
  __shared__ float part_lse[TOKENS ? WAVES * ROWS : 1];
  __shared__ int ticket_s;

  // workgroups over the rows of one (sequence, KV head, share of the keys) read the same keys: ids that differ by eight share an L2
  const int units = p.batch * p.c.heads * p.split;
  const int id = (int)blockIdx.x, unit = (id / (8 * p.row_blocks)) * 8 + id % 8;
  if (unit >= units) return;
  const int rb = p.row_blocks - 1 - (id / 8) % p.row_blocks;  // (the rows that see the most keys first)
  const int slice = unit % p.split, head = (unit / p.split) % p.c.heads, seq = unit / p.split / p.c.heads;

  int q0 = seq, n = 1;
  if (p.q_starts != nullptr) {
    q0 = min(max(p.q_starts[seq], 0), p.tokens);
    n = min(max(p.q_starts[seq + 1], q0), p.tokens) - q0;
  }
  const int keys = min(max(p.kv_lens[seq], 0), p.max_kv_len);
  const int rows = min(n, p.max_q_len) * p.group, row0 = rb * ROWS;
  if (row0 >= rows) return;
  const int last_row = min(row0 + ROWS, rows) - 1;
  const int seen = p.causal ? min(max(keys - n + last_row / p.group + 1, 0), keys) : keys;  // keys that some row sees
  const int slices = max((seen + p.chunk - 1) / p.chunk, 1);
  if (slice >= slices) return;
  const int lo = slice * p.chunk, hi = min(lo + p.chunk, seen);

  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int wave_row = row0 + (TOKENS ? 0 : wave * 16 * NR);

  state<D, DIG, NR> s;
  s.vref = 1;
#pragma unroll
  for (int nr = 0; nr < NR; ++nr) {
    const int row = wave_row + nr * 16 + r, i = row / p.group;
    const bool there = row < rows;
    const typename qg_elem<TYPE>::t* q = static_cast<const typename qg_elem<TYPE>::t*>(p.q) +
                                         (there ? (int64_t)(q0 + i) * p.q_token + (int64_t)(head * p.group + row - i * p.group) * p.q_head : 0);
    load_q<D, DIG, NR, TYPE>(s, nr, q, there, p.scale_log2e, p.scale_log2e_lo, g);
    s.limit[nr] = !there ? 0x7fffffff : p.causal ? keys - n + i : keys - 1;
    s.m[nr] = START;
    s.l[nr] = 0.0f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) s.o[nr][c] = (f4){0.0f, 0.0f, 0.0f, 0.0f};
  }
  // the first token that some row of the wave does not see
  const int whole = min(hi, p.causal ? keys - n + wave_row / p.group + 1 : keys);

  if (wave_row < rows) {
    const reader<D, SMALL> in(p, seq, head, keys, r, g);
    constexpr int STRIDE = TILE * (TOKENS ? WAVES : 1);
    int t0 = lo + (TOKENS ? wave * TILE : 0);
    if (t0 < hi) {
      // two tiles in turn, each requested while the other one is worked on (past the end: the last one again)
      const int last = t0 + (hi - 1 - t0) / STRIDE * STRIDE;
      tile_bits<D> a, b;
      in.load(t0, a);
      while (t0 + STRIDE + TILE <= whole) {
        in.load(min(t0 + STRIDE, last), b);
        step<D, DIG, NR, false>(s, a, t0, hi, r, g);
        t0 += STRIDE;
        in.load(min(t0 + STRIDE, last), a);
        step<D, DIG, NR, false>(s, b, t0, hi, r, g);
        t0 += STRIDE;
      }
      for (; t0 < hi; t0 += STRIDE) {
        in.load(min(t0 + STRIDE, last), b);
        step<D, DIG, NR, true>(s, a, t0, hi, r, g);
        a = b;
      }
    }
  }

  // ---- the wave's result: rows divided by their sum, and the sum's log2
  float lse[NR];
#pragma unroll
  for (int nr = 0; nr < NR; ++nr) {
    const float l = across_sum(s.l[nr]);
    lse[nr] = s.m[nr] + __builtin_amdgcn_logf(l);  // -infinity: no key
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) s.o[nr][c][e] = __builtin_ldexpf(s.o[nr][c][e] * inv, s.vref - 127);
  }
  const size_t share = ((size_t)seq * p.c.heads + head) * p.split;  // of this KV head in the workspace
  float* const lses = p.partial + (size_t)p.batch * p.c.heads * p.split * p.rows_pad * D;

  // lane (r, g) holds channels (D/4) g .. of row r: four times D / 16 consecutive ones
  if (!TOKENS) {
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
      const int row = wave_row + nr * 16 + r;
      if (row >= rows) continue;
      float x[D / 4];
#pragma unroll
      for (int c = 0; c < D / 4; ++c) x[c] = s.o[nr][c % (D / 16)][c / (D / 16)];
      if (slices == 1) {
        const int i = row / p.group;
#pragma unroll
        for (int c = 0; c < D / 4; c += 4) write_out<TYPE>(p, q0 + i, head * p.group + row - i * p.group, g * (D / 4) + c, x + c);
      } else {
        float* to = p.partial + ((share + slice) * p.rows_pad + row) * D + g * (D / 4);
#pragma unroll
        for (int c = 0; c < D / 4; c += 2) hand_in(to + c, x[c], x[c + 1]);
        if (g == 0) __hip_atomic_store(lses + (share + slice) * p.rows_pad + row, lse[nr], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    }
    if (slices == 1) return;
  } else {
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
      float* to = part + ((size_t)wave * ROWS + nr * 16 + r) * PITCH + g * (D / 4);
#pragma unroll
      for (int c = 0; c < D / 4; c += 4) {
        f4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = s.o[nr][(c + e) % (D / 16)][(c + e) / (D / 16)];
        *reinterpret_cast<f4*>(to + c) = x;
      }
      if (g == 0) part_lse[wave * ROWS + nr * 16 + r] = lse[nr];
    }
    __syncthreads();
    // the waves' results, weighted by their sums
    for (int at = (int)threadIdx.x; at < (last_row - row0 + 1) * (D / 4); at += 64 * WAVES) {
      const int local = at / (D / 4), c = at % (D / 4) * 4, row = row0 + local;
      float top = -__builtin_inff();
#pragma unroll
      for (int w = 0; w < WAVES; ++w) top = fmaxf(top, part_lse[w * ROWS + local]);
      const float base = top == -__builtin_inff() ? 0.0f : top;
      float total = 0.0f;
      f4 x = (f4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const float e = __builtin_amdgcn_exp2f(part_lse[w * ROWS + local] - base);
        total += e;
        const f4 y = *reinterpret_cast<const f4*>(part + ((size_t)w * ROWS + local) * PITCH + c);
        x += e * y;
      }
      x *= total == 0.0f ? 0.0f : 1.0f / total;
      if (slices == 1) {
        const int i = row / p.group;
        write_out<TYPE>(p, q0 + i, head * p.group + row - i * p.group, c, reinterpret_cast<const float*>(&x));
      } else {
        float* to = p.partial + ((share + slice) * p.rows_pad + row) * D + c;
        hand_in(to, x[0], x[1]);
        hand_in(to + 2, x[2], x[3]);
        if (c == 0)
          __hip_atomic_store(lses + (share + slice) * p.rows_pad + row, base + __builtin_amdgcn_logf(total), __ATOMIC_RELAXED,
                             __HIP_MEMORY_SCOPE_AGENT);
      }
    }
    if (slices == 1) return;
  }

  // ---- keys split over workgroups: the last one to arrive adds the shares, in their order
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the stores above have been acknowledged
  __syncthreads();
  int* const counter = p.counters + ((size_t)seq * p.c.heads + head) * p.row_blocks + rb;
  if (threadIdx.x == 0) ticket_s = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (ticket_s != slices - 1) return;
  if (threadIdx.x == 0) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // ready for the next call
  for (int at = (int)threadIdx.x; at < (last_row - row0 + 1) * (D / 4); at += 64 * WAVES) {
    const int local = at / (D / 4), c = at % (D / 4) * 4, row = row0 + local;
    float top = -__builtin_inff();
    for (int t = 0; t < slices; ++t)
      top = fmaxf(top, __hip_atomic_load(lses + (share + t) * p.rows_pad + row, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    const float base = top == -__builtin_inff() ? 0.0f : top;
    float total = 0.0f;
    f4 x = (f4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int t = 0; t < slices; ++t) {
      const float e = __builtin_amdgcn_exp2f(
          __hip_atomic_load(lses + (share + t) * p.rows_pad + row, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) - base);
      const u64* from = reinterpret_cast<const u64*>(p.partial + ((share + t) * p.rows_pad + row) * D + c);
      const u64 u = __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      const u64 v = __hip_atomic_load(from + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      total += e;
      x[0] += e * __builtin_bit_cast(float, (unsigned)u);
      x[1] += e * __builtin_bit_cast(float, (unsigned)(u >> 32));
      x[2] += e * __builtin_bit_cast(float, (unsigned)v);
      x[3] += e * __builtin_bit_cast(float, (unsigned)(v >> 32));
    }
    x *= total == 0.0f ? 0.0f : 1.0f / total;
    const int i = row / p.group;
    write_out<TYPE>(p, q0 + i, head * p.group + row - i * p.group, c, reinterpret_cast<const float*>(&x));
  }
}

template <int D, int DIG, int TYPE, int NR, bool TOKENS>
void go(qg_kv4_attention_args a, int rows, hipStream_t s) {
  constexpr int ROWS = 16 * NR * (TOKENS ? 1 : WAVES);
  a.row_blocks = (rows + ROWS - 1) / ROWS;
  const long long units = (long long)a.batch * a.c.heads * a.split;
  const dim3 grid((unsigned)((units + 7) / 8 * 8 * a.row_blocks));
  if (a.c.lgp == 4)
    hipLaunchKernelGGL((qg_kv4_attention_kernel<D, DIG, TYPE, NR, TOKENS, true>), grid, dim3(64 * WAVES), 0, s, a);
  else
    hipLaunchKernelGGL((qg_kv4_attention_kernel<D, DIG, TYPE, NR, TOKENS, false>), grid, dim3(64 * WAVES), 0, s, a);
}

template <int D, int TYPE>
void by_rows(const qg_kv4_attention_args& a, int rows, hipStream_t s) {
  constexpr int DIG = TYPE == QG_F32 ? 2 : 1;
  if (rows <= 16)
    go<D, DIG, TYPE, 1, true>(a, rows, s);
  else
    go<D, DIG, TYPE, 1, false>(a, rows, s);
}

template <int D>
void by_type(const qg_kv4_attention_args& a, int dtype, int rows, hipStream_t s) {
  switch (dtype) {
    case QG_F32: by_rows<D, QG_F32>(a, rows, s); break;
    case QG_BF16: by_rows<D, QG_BF16>(a, rows, s); break;
    default: by_rows<D, QG_F16>(a, rows, s);
  }
}

}  // namespace

hipError_t qg_launch_kv4_attention(const qg_kv4_attention_args& a, int head_dim, int dtype, int rows, hipStream_t s) {
  switch (head_dim) {
    case 64: by_type<64>(a, dtype, rows, s); break;
    case 128: by_type<128>(a, dtype, rows, s); break;
    default: by_type<256>(a, dtype, rows, s);
  }
  return hipGetLastError();
}
