// What the two kernels of the attention over the 4-bit cache share: codes into operands of the matrix cores, scores into weights,
// queries, and the joining of results.  Not part of the public interface.
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
// against a reference of their own row, the largest such product that it has met, so that they lie below 2^12 and keep 11 bits
// down to 2^-18 of that.  One such number is enough for a bf16 result (1.68e-3 off, 1.67e-3 with exact weights: the result's own rounding).
// An fp16 result shows it (2.9e-4 off, 2.1e-4 with two), so fp16 and fp32 results take two: 131072 keys of 8 heads 34.4 -> 36.1 us, 512 rows
// of four sequences 146 -> 178.
// Scores, maxima, sums and outputs are fp32.
//
// References.  With alpha the value scale and S a power of two that all rows of a wave share, a row holds
//   l = sum 2^(score - m),  o = sum 2^(score - m) alpha / S (code - theta)
// where m + log2 S is the largest score + log2 alpha of the keys that it sees: what a row does not see, or gives no weight, takes
// nothing from its products however large its values are.  One exponential serves both sums; S only keeps 2^(score - m) within fp32
// and near 1, where the exponent itself is rounded least (values 2^60 apart: 2^-18 of a probability, below 2^-20 within 2^12).
// Scores from 2^24 on are whole numbers in fp32, up to 32 apart: a reference cannot take up the value scale there and is the largest
// score, S the largest value scale, and the exponent the difference of the rounded scores.  (The exact one, up to 16 on either side
// of 0 for the largest score itself, passes fp16's range.)  Every tile is then weighed twice.
#pragma once

#include "qg_kv4.h"
#include "qg_pages.h"

namespace {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef unsigned u2 __attribute__((ext_vector_type(2)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

constexpr int TILE = 32;         // tokens of a wave's step
constexpr int BOOST = 4;             // weights (probability times value scale) are held times 2^BOOST under their largest ...
constexpr float MOST = 0x1p12f;      // ... and the reference moves when one would pass this
constexpr int LAG = 16;              // a value scale may pass the common reference by 2^LAG before that moves
constexpr float SPREAD = 80.0f;      // exponents pass the row's scores by this at most ...
constexpr float SUMS = 0x1p96f;      // ... and their sum this
constexpr float FINE = 0x1p24f;      // fp32 numbers below this take up whole ones

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
__device__ inline f4 product(const frag& a, const frag& b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v, b.v, c, 0, 0, 0); }

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

// theta and its neighbour's in two forms for spread_less(), a pair from one or two tokens
struct zero_pair {
  unsigned low, high;
  __device__ inline explicit zero_pair(unsigned pair) : low(pair + 0xE400E400u), high((pair << 4) + 0xD400D400u) {}
};

// For the values of a row's 8 tokens, words in lanes 8 .. 15: tokens 2 i and 2 i + 1
struct zero_points {
  h2 low[4], high[4];
  __device__ inline explicit zero_points(unsigned word) {
    const unsigned theta = word & 15u;
    const unsigned next = (unsigned)__builtin_amdgcn_mov_dpp((int)theta, 0x101, 0xf, 0xf, true);  // row_shl:1
    const zero_pair z(theta | next << 16);
    low[0] = as_h2(row_lane<8>(z.low));
    low[1] = as_h2(row_lane<10>(z.low));
    low[2] = as_h2(row_lane<12>(z.low));
    low[3] = as_h2(row_lane<14>(z.low));
    high[0] = as_h2(row_lane<8>(z.high));
    high[1] = as_h2(row_lane<10>(z.high));
    high[2] = as_h2(row_lane<12>(z.high));
    high[3] = as_h2(row_lane<14>(z.high));
  }
};

// Four channels of 8 tokens (a dword: two tokens) as the first operands of four products
__device__ inline void spread_values(const u4& x, const masks& m, const zero_points& z, frag* out) {
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    unsigned y[4];
    spread_less(x[t], m, z.low[t], z.high[t], y);
#pragma unroll
    for (int c = 0; c < 4; ++c) out[c].u[t] = y[c];
  }
}

// Where a lane's bytes lie.  Keys: of a token's D/2 bytes lane group g takes KEY_BYTES in each of KEY_LOADS pieces.  Values: of
// 8 tokens lane r takes 16 bytes, four channels, in each of D/64 pieces.
template <int D>
struct lay {
  static constexpr int KEY_BYTES = D == 64 ? 8 : 16, KEY_LOADS = D / 8 / KEY_BYTES, KEY_WORDS = KEY_BYTES / 4, VALUE_LOADS = D / 64;
  // first channel of a lane's dword f of keys; of its outputs 4 i .. 4 i + 3 (16 consecutive ones in all)
  static __device__ constexpr int key_channel(int f, int g) { return f / KEY_WORDS * (8 * KEY_BYTES) + g * (2 * KEY_BYTES) + f % KEY_WORDS * 8; }
  static __device__ constexpr int out_channel(int i, int g) { return 64 * i + 16 * g; }
};

// The pages of a sequence.  An entry that is no page of the cache reads as page 0.
struct page_reader {
  uint8_t* data;
  const int32_t* table;
  int entries, n_pages, lgp;
  size_t page_bytes, head_bytes;
  int head;
  template <int D>
  __device__ inline void init(const qg_kv4_attention_args& p, int seq, int keys, int kv_head) {
    data = p.c.data;
    table = p.pages + (int64_t)seq * p.pages_stride;
    // (alike in all lanes, and said so: as a vector it made the page's address one, and 512 rows of four sequences 152 us instead of 149)
    entries = __builtin_amdgcn_readfirstlane(qg_page_entries(keys, p.c.lgp));
    n_pages = p.c.n_pages;
    lgp = p.c.lgp;
    head_bytes = (size_t)(D + 8) << lgp;
    page_bytes = head_bytes * p.c.heads;
    head = kv_head;
  }
  __device__ inline unsigned page(int t0, int half) const { return (unsigned)table[qg_page_entry(t0, half, lgp, entries)]; }
  __device__ inline const uint8_t* block(unsigned page) const {
    page = page < (unsigned)n_pages ? page : 0u;
    return data + page * page_bytes + head * head_bytes;
  }
};

// Where a lane finds its part of a tile of 32 tokens.  SMALL: pages of 16 tokens, two to a tile; otherwise a tile lies in one page,
// whose address is the same for all lanes.
struct page_ids {
  unsigned first, second;
};
struct spots {
  const uint8_t *keys, *values, *words;
};
template <int D, bool SMALL>
struct reader : page_reader {
  typedef lay<D> L;
  unsigned key_lane, value_lane, word_lane;  // this lane's bytes past the tile's
  bool key_half, value_half;                 // SMALL: the lane's run of 8 tokens lies in the tile's second page

  __device__ inline reader(const qg_kv4_attention_args& p, int seq, int keys, int head, int r, int g) {
    init<D>(p, seq, keys, head);
    const int key_run = r >> 2, key_at = SMALL ? key_run & 1 : key_run, value_at = SMALL ? g & 1 : g;
    key_lane = (unsigned)((8 * key_at + (r & 3)) * (D / 2) + g * L::KEY_BYTES);
    value_lane = (unsigned)(value_at * (4 * D) + r * 16);
    word_lane = (unsigned)(value_at * 64 + r * 4);
    key_half = key_run >= 2;
    value_half = g >= 2;
  }
  __device__ inline page_ids pages(int t0) const {
    if (SMALL) return {page(t0, 0), page(t0, 1)};
    return {page(t0, 0), 0u};
  }
  __device__ inline spots at(int t0, page_ids ids) const {
    spots s;
    if (SMALL) {
      const uint8_t *first = block(ids.first), *second = block(ids.second);
      s.keys = key_half ? second : first;
      s.values = (value_half ? second : first) + 16 * (D / 2);
      s.words = s.values + 16 * (D / 2);
    } else {
      const uint8_t* page = block(ids.first);
      const int P = 1 << lgp, at = t0 & (P - 1);
      s.keys = page + at * (D / 2);
      s.values = page + (P + at) * (D / 2);
      s.words = page + P * D + at * 8;
    }
    return s;
  }
  // tile a of 16 tokens: row r is token 8 (r / 4) + 4 a + r % 4
  __device__ inline void load_keys(const spots& s, int a, int i, unsigned* out) const {
    const uint8_t* from = s.keys + key_lane + a * 4 * (D / 2) + i * 64;
    if (D == 64) {
      const u2 x = *reinterpret_cast<const u2*>(from);
      out[0] = x[0];
      out[1] = x[1];
    } else {
      const u4 x = *reinterpret_cast<const u4*>(from);
#pragma unroll
      for (int j = 0; j < 4; ++j) out[j] = x[j];
    }
  }
  __device__ inline u4 load_values(const spots& s, int i) const { return *reinterpret_cast<const u4*>(s.values + value_lane + i * 256); }
  __device__ inline unsigned load_word(const spots& s) const { return *reinterpret_cast<const unsigned*>(s.words + word_lane); }
};
// theta, twice, of the token that this lane holds as first operand of tile a
__device__ inline unsigned key_zero(unsigned theta, int a, int r) {
  return (unsigned)__builtin_amdgcn_ds_bpermute((16 * (r >> 2) + 4 * a + (r & 3)) * 4, (int)theta) * 0x10001u;
}

// What a wave keeps of its NR tiles of 16 rows
template <int D, int DIG, int NR>
struct state {
  f4 o[NR][D / 16];
  float m[NR], l[NR];              // reference of the exponents (log2, a whole number), sum of 2^(log2 score - m) (this lane's tokens)
  float factor[NR], factor_lo[NR]; // log2 score of a product and a key's scale, in two parts (the second: DIG 2)
  int limit[NR];                   // last token that the row sees
  int vref;                        // biased exponent of the value scales' reference
  bool huge;                       // some score was beyond FINE
  __device__ inline void start() {
    vref = 1;
    huge = false;
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      m[n] = -__builtin_inff();  // (before the first key every exponent is +infinity, and the reference moves)
      l[n] = 0.0f;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) o[n][c] = (f4){0.0f, 0.0f, 0.0f, 0.0f};
    }
  }
};

// Over the four lanes of a row of queries: every lane gets the result, by swaps between the rows of 16 (no trip through the LDS)
template <typename F>
__device__ inline float across(float x, F f) {
  const auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  const unsigned a0 = a[0], a1 = a[1];
  x = f(__builtin_bit_cast(float, a0), __builtin_bit_cast(float, a1));
  const auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  const unsigned b0 = b[0], b1 = b[1];
  return f(__builtin_bit_cast(float, b0), __builtin_bit_cast(float, b1));
}
__device__ inline float across_max(float x) {
  return across(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ inline float across_sum(float x) {
  return across(x, [](float a, float b) { return a + b; });
}
// The largest over all lanes
__device__ inline float wave_max(float x) {
  x = fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x128, 0xf, 0xf, true)));  // row_ror:8, 4, 2, 1
  x = fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x124, 0xf, 0xf, true)));
  x = fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x122, 0xf, 0xf, true)));
  x = fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x121, 0xf, 0xf, true)));
  return across_max(x);
}

// z factor + base, where base is a whole number near -z factor: the sum is small and loses nothing of it.  DIG 2: the factor's own
// rounding (2^-25 of every score) is more than the rest of an fp32 result's error.
template <int DIG>
__device__ inline float exponent(float z, float factor, float factor_lo, float base) {
  const float y = __builtin_fmaf(z, factor, base);
  return DIG == 2 ? __builtin_fmaf(z, factor_lo, y) : y;
}

// Products of a tile's 8 tokens (z[n][a][i]: token 8g + 4a + i) into weights x, probability times value scale, against the running
// references, which move rarely.  MASKED: tokens from `end` on are not there (`word` is 0 for them), and a row may end inside the tile.
template <int D, int DIG, int NR, bool MASKED>
__device__ inline void weigh(state<D, DIG, NR>& s, f4 (*z)[2], unsigned word, int t0, int end, int r, int g, float (*x)[8]) {
  const float scale = __builtin_bit_cast(float, word & ~15u);
  int limit[NR];  // the last of the lane's 8 tokens that the row sees
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    limit[n] = MASKED ? min(s.limit[n], end - 1) - t0 - 8 * g : 7;
    const float ks[8] = {row_lane<0>(scale), row_lane<1>(scale), row_lane<2>(scale), row_lane<3>(scale),
                         row_lane<4>(scale), row_lane<5>(scale), row_lane<6>(scale), row_lane<7>(scale)};
#pragma unroll
    for (int j = 0; j < 8; ++j) z[n][j >> 2][j & 3] *= ks[j];
  }
  float sum[NR], top[NR];
  auto all = [&](const float* factor, const float* factor_lo) {
    const float scaled = __builtin_ldexpf(scale, 127 + BOOST - s.vref);
    const float vs[8] = {row_lane<8>(scaled),  row_lane<9>(scaled),  row_lane<10>(scaled), row_lane<11>(scaled),
                         row_lane<12>(scaled), row_lane<13>(scaled), row_lane<14>(scaled), row_lane<15>(scaled)};
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      sum[n] = 0.0f;
      top[n] = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float y = exponent<DIG>(z[n][j >> 2][j & 3], factor[n], factor_lo[n], -s.m[n]);
        if (MASKED) y = j > limit[n] ? -__builtin_inff() : y;
        const float e = __builtin_amdgcn_exp2f(y);
        sum[n] += e;
        x[n][j] = e * vs[j];
        if (MASKED) x[n][j] = j > limit[n] ? 0.0f : x[n][j];  // (a masked value may be NaN)
        top[n] = fmaxf(top[n], x[n][j]);
      }
    }
  };
  all(s.factor, s.factor_lo);
  bool move[NR], any = false;
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    move[n] = top[n] > MOST || s.l[n] + sum[n] > SUMS || s.huge;
    any |= move[n];
  }
  if (__builtin_expect(__ballot(any) != 0ull, 0)) {
    float far = 0.0f;
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      float most = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) most = fmaxf(most, __builtin_fabsf(z[n][j >> 2][j & 3]));
      far = fmaxf(far, most * __builtin_fabsf(s.factor[n]));
    }
    const bool huge = s.huge || __ballot(far >= FINE) != 0ull;
    s.huge = huge;
    float factor[NR], factor_lo[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const float now = huge ? s.factor[n] : 1.0f;  // (then z becomes the rounded score itself)
      factor[n] = huge ? 1.0f : s.factor[n];
      factor_lo[n] = huge ? 0.0f : s.factor_lo[n];
#pragma unroll
      for (int j = 0; j < 8; ++j) z[n][j >> 2][j & 3] *= now;
    }
    const int e = (word & 0x7f800000u) != 0x7f800000u && r >= 8 ? (int)(word >> 23 & 255u) : 0;  // (zero and NaN: 0)
    const int most = (int)wave_max((float)e), vref = most > s.vref + (huge ? 0 : LAG) ? most : s.vref;
    const float ve = e > 0 ? (float)e : -__builtin_inff();
    const float ves[8] = {row_lane<8>(ve),  row_lane<9>(ve),  row_lane<10>(ve), row_lane<11>(ve),
                          row_lane<12>(ve), row_lane<13>(ve), row_lane<14>(ve), row_lane<15>(ve)};
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      float score = -__builtin_inff(), weight = -__builtin_inff();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float y = z[n][j >> 2][j & 3] * factor[n];
        if (!MASKED || j <= limit[n]) {
          score = fmaxf(score, y);
          weight = fmaxf(weight, y + ves[j]);
        }
      }
      score = rintf(across_max(score));  // (whole: references differ by powers of two)
      weight = rintf(across_max(weight)) - (float)vref;
      u64 rows = __ballot(move[n]);  // (a row's four lanes move together, and no other row moves with it)
      rows |= rows >> 32;
      rows |= rows >> 16;
      const int held = __builtin_amdgcn_frexp_expf(across_sum(s.l[n]));
      float m = s.m[n] + (float)(s.vref - vref);
      if (huge || (rows >> r & 1)) m = fmaxf(m, weight);
      m = fmaxf(m, fmaxf(score, s.m[n] + (float)held) - SPREAD);
      score = fmaxf(score, s.m[n]);
      if (__builtin_fabsf(score) >= FINE) m = score;
      const float by = m == s.m[n] ? 0.0f : fminf(fmaxf(s.m[n] - m, -300.0f), 300.0f);  // (both -infinity: no key yet)
      s.m[n] = m;
      s.l[n] = __builtin_ldexpf(s.l[n], (int)by);
      const float f = __builtin_ldexpf(1.0f, (int)by + s.vref - vref);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) s.o[n][i] *= f;
    }
    s.vref = vref;
    all(factor, factor_lo);
  }
#pragma unroll
  for (int n = 0; n < NR; ++n) s.l[n] += sum[n];
}

// ... and those as second operands of the other product, in PARTS fp16 numbers
template <int NR, int PARTS>
__device__ inline void halves(const float (*x)[8], frag (*p)[PARTS]) {
#pragma unroll
  for (int n = 0; n < NR; ++n)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float w = x[n][j];
      // The product as 32 bits: left to itself the compiler rounds it to fp16 twice, once from the exact product and once from
      // this one, and where the two differ the second part makes up for the wrong first part (one token in some thousands; an
      // fp32 result then loses half its digits).
      if (PARTS == 2) asm("" : "+v"(w));
      const _Float16 hi = (_Float16)w;
      p[n][0].v[j] = hi;
      if (PARTS == 2) p[n][PARTS - 1].v[j] = (_Float16)(w - (float)hi);
    }
}

// The channels of a query that a lane needs, as they lie in memory
template <int D, int TYPE>
struct raw_query {
  typename qg_elem<TYPE>::t x[D / 4];
  __device__ inline void load(const typename qg_elem<TYPE>::t* q, bool there, int g) {
    typedef typename qg_elem<TYPE>::t t;
    typedef lay<D> L;
    constexpr int W = 16 / sizeof(t), RUN = 2 * L::KEY_BYTES;
    typedef t vec __attribute__((ext_vector_type(W)));
    typedef vec vec_any __attribute__((aligned(sizeof(t))));
#pragma unroll
    for (int i = 0; i < D / 4; ++i) x[i] = (t)0.0f;
    if (!there) return;
#pragma unroll
    for (int i = 0; i < D / 4; i += W) {
      const vec v = *reinterpret_cast<const vec_any*>(q + L::key_channel(i / RUN * L::KEY_WORDS, g) + i % RUN);
#pragma unroll
      for (int j = 0; j < W; ++j) x[i + j] = v[j];
    }
  }
};

// ... as fp16 scaled by a power of two; returns the power
template <int D, int DIG, int TYPE>
__device__ inline int split_query(const raw_query<D, TYPE>& raw, frag (*q)[D / 32]) {
  float x[D / 4];
  unsigned top = 0u;
#pragma unroll
  for (int i = 0; i < D / 4; ++i) {
    x[i] = qg_elem<TYPE>::up(raw.x[i]);
    top = max(top, __builtin_bit_cast(unsigned, x[i]) & 0x7fffffffu);
  }
  top = max(top, (unsigned)__shfl_xor((int)top, 16));
  top = max(top, (unsigned)__shfl_xor((int)top, 32));
  const int shift = top == 0u ? 0 : 14 + 127 - max((int)(top >> 23), 1);
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = 8 * i + (j >> 1) + 4 * (j & 1);  // the order in which the codes of a dword are spread
      // (an infinity or NaN: the row's scores become NaN)
      const float y = top < 0x7f800000u ? __builtin_ldexpf(x[c], shift) : __builtin_nanf("");
      const _Float16 hi = (_Float16)y;
      q[0][i].v[j] = hi;
      if (DIG == 2) q[DIG - 1][i].v[j] = (_Float16)(y - (float)hi);
    }
  return shift;
}

// Running sums over the lanes of a wave (lane 63: of all)
__device__ inline int running(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // row_shr:1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15, :31
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}

// Which rows, keys and workgroups a workgroup deals with
struct job {
  int head, seq, slice, slices;
  int q0, n, keys;           // the sequence's first query, its queries, its keys
  int rows, row0, last_row;  // of the KV head; this workgroup's first and last
  int lo, hi;                // its tokens
  int first, units, blocks, block;  // units of a (sequence, KV head, share of the keys) numbered together, `blocks` workgroups each, from `first` on
  int unit0, unit_step;             // those of this one's first share, from share to share
  __device__ inline void look(const qg_kv4_attention_args& p, int b) {
    q0 = b;
    n = 1;
    if (p.q_starts != nullptr) {
      q0 = min(max(p.q_starts[b], 0), p.tokens);
      n = min(max(p.q_starts[b + 1], q0), p.tokens) - q0;
    }
    keys = min(max(p.kv_lens[b], 0), p.max_kv_len);
    rows = min(n, p.max_q_len) * p.group;
  }
  // A unit's workgroups, which differ in their rows, read the same keys: ids that differ by eight share an L2.  The first
  // units / 8 * 8 units go by eights, what is left spreads.
  __device__ inline int id_of(int share) const {
    const int unit = unit0 + share * unit_step, whole = units & ~7;
    return first + (unit < whole ? (unit >> 3) * 8 * blocks + block * 8 + (unit & 7) : whole * blocks + block * (units - whole) + unit - whole);
  }
  template <int ROWS, bool MANY>
  __device__ inline bool init(const qg_kv4_attention_args& p) {
    const int id = (int)blockIdx.x;
    int unit, piece = p.piece;
    if (!MANY || p.shares == 0) {  // heads first: shares that only long sequences have would fall to the same few XCDs otherwise
      units = p.batch * p.c.heads * p.split;
      blocks = p.row_blocks;
      first = 0;
    } else {
      // Every wave deals the keys for itself: shares of at most `chosen` stages of 64 tokens, of one length within a sequence.  Three ways:
      // the fewest stages that make no more workgroups than there are CUs, or than run at once, or half of what each of those would have
      // on average.  A round costs its stages and about four (queries in, results out; four fifths of it for a workgroup that has a CU to
      // itself), the join one a share; the cheapest way is taken.  The prices are fitted.  Each way forced in turn over 43 calls of all head
      // sizes and types, 1 to 42 sequences, 24 to 512 queries: the choice is within 2 % of the best way in 37, at worst 10 % off (8 x 128
      // queries, 8192 keys: 79 us for 72), where a fixed way loses up to 100 % (CUs), 30 % (once: two even sequences of 64 heads over 8 take
      // 184 us, 141 in two rounds) or 90 % (two rounds).
      const int lane = (int)threadIdx.x & 63, longest = (p.max_kv_len + 63) / 64;
      int all, wide;  // of the lane's sequence: stages, workgroups of a share
      auto measure = [&](int b0) {
        look(p, min(b0 + lane, p.batch - 1));
        all = (keys + 63) / 64;
        wide = b0 + lane < p.batch ? (rows + ROWS - 1) / ROWS * p.c.heads : 0;
      };
      measure(0);
      int work = 0;
      for (int b0 = 0; b0 < p.batch; b0 += 64) {
        if (b0 > 0) measure(b0);
        work += __builtin_amdgcn_readlane(running(all * wide), 63);
      }
      auto fit = [&](int workgroups) {  // (a share more or less does no harm: the quotients need not be exact)
        int x = max(p.least, (work + workgroups - 1) / workgroups);
        for (; x < longest; x += max(x >> 3, 1)) {
          const float inv = __builtin_amdgcn_rcpf((float)x);
          int n = 0;
          for (int b0 = 0; b0 < p.batch; b0 += 64) {
            if (p.batch > 64) measure(b0);
            n += __builtin_amdgcn_readlane(running(max((int)__builtin_ceilf((float)all * inv), 1) * wide), 63);
          }
          if (n <= workgroups) break;
        }
        return min(x, longest);
      };
      const int alone = fit(min(p.shares, 256)), once = fit(p.shares), twice = max(p.least, (work + 2 * p.shares - 1) / (2 * p.shares));
      const float cost_alone = 0.8f * (float)(alone + 4) + (float)longest / (float)alone;
      const float cost_once = (float)(once + 4) + (float)longest / (float)once;
      const float cost_twice = 2.0f * (float)(twice + 4) + (float)longest / (float)twice;
      const int chosen = cost_twice < fminf(cost_alone, cost_once) ? twice : cost_alone < cost_once ? alone : once;
      first = 0;
      bool found = false;
      for (int b0 = 0; b0 < p.batch && !found; b0 += 64) {
        if (p.batch > 64) measure(b0);
        const int about = max((all + chosen - 1) / chosen, 1), mine = max((all + about - 1) / about, 1);
        const int n_shares = max((all + mine - 1) / mine, 1);
        const int upto = first + running(n_shares * wide);
        const unsigned long long here = __ballot(id < upto);
        found = here != 0ull;
        const int l = found ? __builtin_ctzll(here) : 63;
        first = __builtin_amdgcn_readlane(upto - (found ? n_shares * wide : 0), l);
        seq = b0 + l;
        units = __builtin_amdgcn_readlane(n_shares, l) * p.c.heads;
        blocks = __builtin_amdgcn_readlane(wide, l) / p.c.heads;
        piece = __builtin_amdgcn_readlane(mine, l) * 64;
      }
      if (!found) return false;
    }
    const int local = id - first, whole = units & ~7, rest = units - whole;
    if (local < whole * blocks) {
      unit = local / (8 * blocks) * 8 + (local & 7);
      block = local / 8 % blocks;
    } else {
      unit = whole + (local - whole * blocks) % rest;
      block = (local - whole * blocks) / rest;
    }
    head = unit % p.c.heads;
    slice = unit / p.c.heads;
    unit_step = p.c.heads;
    if (!MANY || p.shares == 0) {
      seq = slice % p.batch;
      slice /= p.batch;
      unit_step *= p.batch;
    }
    unit0 = unit - slice * unit_step;
    look(p, seq);  // (again where the kernel dealt: broadcasting the lane's figures instead cost registers, and 64 channels 12 us of 62)
    row0 = (blocks - 1 - block) * ROWS;  // (the rows that see the most keys first)
    if (row0 >= rows) return false;
    last_row = min(row0 + ROWS, rows) - 1;
    const int seen = p.causal ? min(max(keys - n + last_row / p.group + 1, 0), keys) : keys;  // keys that some row sees
    slices = max((seen + piece - 1) / piece, 1);
    lo = slice * piece;
    hi = min(lo + piece, seen);
    return slice < slices;
  }
  // keys that all rows from `row` on see
  __device__ inline int seen_by(const qg_kv4_attention_args& p, int row) const {
    return min(hi, p.causal ? keys - n + row / p.group + 1 : keys);
  }
  __device__ inline int limit(const qg_kv4_attention_args& p, int row) const {
    return row >= rows ? 0x7fffffff : p.causal ? keys - n + row / p.group : keys - 1;
  }
  template <int TYPE>
  __device__ inline const typename qg_elem<TYPE>::t* query(const qg_kv4_attention_args& p, int row) const {
    const int i = row / p.group;
    return static_cast<const typename qg_elem<TYPE>::t*>(p.q) +
           (row < rows ? (int64_t)(q0 + i) * p.q_token + (int64_t)(head * p.group + row - i * p.group) * p.q_head : 0);
  }
  // consecutive channels of a finished row
  template <int TYPE, int N>
  __device__ inline void write(const qg_kv4_attention_args& p, int row, int c, const float* x) const {
    typedef typename qg_elem<TYPE>::t t;
    const int i = row / p.group;
    qg_store<TYPE, N>(static_cast<t*>(p.out) + (int64_t)(q0 + i) * p.o_token + (int64_t)(head * p.group + row - i * p.group) * p.o_head + c, x);
  }
};

// A wave's rows divided by their sums, and those: what a part of the keys weighs is sum 2^m, kept as the two numbers (a logarithm of
// a large sum would lose what an fp32 result shows), the sum below 1 where m is small enough to take up its exponent exactly, so that
// parts compare by m.  No key: sum 0, m -infinity.
template <int D, int DIG, int NR>
__device__ inline void finish(state<D, DIG, NR>& s, float* sum) {
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const float l = across_sum(s.l[n]);
    const int e = __builtin_fabsf(s.m[n]) < 0.5f * FINE ? __builtin_amdgcn_frexp_expf(l) : 0;
    sum[n] = __builtin_ldexpf(l, -e);
    s.m[n] += (float)e;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) s.o[n][c][i] = __builtin_ldexpf(s.o[n][c][i] * inv, s.vref - 127 - BOOST);
  }
}
// Weights relative to the largest reference `top` among the parts
__device__ inline float weight(float m, float sum, float top) { return sum * __builtin_amdgcn_exp2f(m - (top == -__builtin_inff() ? 0.0f : top)); }

// Between the four lanes of a row of queries: block k of lane g becomes block g of lane k
__device__ inline void transpose(float* x) {
  auto swap16 = [](float& a, float& b) {
    const auto v = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    const unsigned first = v[0], second = v[1];
    a = __builtin_bit_cast(float, first);
    b = __builtin_bit_cast(float, second);
  };
  auto swap32 = [](float& a, float& b) {
    const auto v = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    const unsigned first = v[0], second = v[1];
    a = __builtin_bit_cast(float, first);
    b = __builtin_bit_cast(float, second);
  };
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    swap32(x[c], x[8 + c]);
    swap32(x[4 + c], x[12 + c]);
    swap16(x[c], x[4 + c]);
    swap16(x[8 + c], x[12 + c]);
  }
}
// The 16 output channels of a lane's run i
template <int D, int DIG, int NR>
__device__ inline void run_of(const state<D, DIG, NR>& s, int n, int i, float* x) {
#pragma unroll
  for (int c = 0; c < 16; ++c) x[c] = s.o[n][4 * i + c % 4][c / 4];
}

// Results of a share of the keys, past the caches that other workgroups do not share: a workgroup's rows under its number
template <int ROWS>
struct shares {
  float *data, *sums;  // rows of D; (m, sum) of each
  const job& j;
  __device__ inline shares(const qg_kv4_attention_args& p, const job& j) : data(p.partial), sums(p.sums), j(j) {}
  __device__ inline size_t at(int slice, int row) const { return (size_t)j.id_of(slice) * ROWS + (row - j.row0); }
};
__device__ inline void hand_in(float* to, f4 x) {  // 16 bytes at once (their registers may not be written to in the next cycle)
  asm volatile("global_store_dwordx4 %0, %1, off sc1\n\ts_nop 1" ::"v"(to), "v"(x) : "memory");
}
__device__ inline void hand_in(float* to, float a, float b) {
  __hip_atomic_store(reinterpret_cast<u64*>(to), (u64)__builtin_bit_cast(unsigned, a) | (u64)__builtin_bit_cast(unsigned, b) << 32,
                     __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline float low(u64 x) { return __builtin_bit_cast(float, (unsigned)x); }
__device__ inline float high(u64 x) { return __builtin_bit_cast(float, (unsigned)(x >> 32)); }
__device__ inline u64 fetch(const float* from) {
  return __hip_atomic_load(reinterpret_cast<const u64*>(from), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Keys split over workgroups: the last one to arrive adds the shares, in their order.  THREADS of the workgroup.  An item is four
// channels of a row; a thread requests BATCH shares of ITEMS items together, since a request past the caches takes more than a
// microsecond.  scratch: 8 floats a thread, or NULL; with it, where there are fewer items than threads, groups of threads take every
// groups-th batch of shares and meet there.
template <int D, int TYPE, int THREADS, int ITEMS, int BATCH, int ROWS>
__device__ inline void join(const qg_kv4_attention_args& p, const job& j, const shares<ROWS>& w, float* scratch, int* ticket) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // what this wave handed in has been acknowledged
  __syncthreads();
  int* const counter = p.counters + j.id_of(0);
  if (threadIdx.x == 0) *ticket = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (*ticket != j.slices - 1) return;
  if (threadIdx.x == 0) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // ready for the next call
  const int items = (j.last_row - j.row0 + 1) * (D / 4);
  const int groups = scratch != nullptr && items * 2 <= THREADS ? THREADS / items : 1;
  for (int at = (int)threadIdx.x; at < items * groups; at += THREADS * ITEMS) {
    const int mine = groups > 1 ? at / items : 0;
    int item[ITEMS];
    float top[ITEMS], total[ITEMS];
    f4 x[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      item[k] = min(at - mine * items + k * THREADS, items - 1);  // (past the end: the last one again, not written)
      top[k] = -__builtin_inff();
      total[k] = 0.0f;
      x[k] = (f4){0.0f, 0.0f, 0.0f, 0.0f};
    }
    for (int t0 = mine * BATCH; t0 < j.slices; t0 += groups * BATCH) {
      u64 ms[ITEMS][BATCH], u[ITEMS][BATCH], v[ITEMS][BATCH];
#pragma unroll
      for (int k = 0; k < ITEMS; ++k)
#pragma unroll
        for (int t = 0; t < BATCH; ++t) {
          const size_t from = w.at(min(t0 + t, j.slices - 1), j.row0 + item[k] / (D / 4));
          ms[k][t] = fetch(w.sums + 2 * from);
          const float* data = w.data + from * D + item[k] % (D / 4) * 4;
          u[k][t] = fetch(data);
          v[k][t] = fetch(data + 2);
        }
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        float most = top[k];
#pragma unroll
        for (int t = 0; t < BATCH; ++t) most = fmaxf(most, low(ms[k][t]));
        const float f = weight(top[k], 1.0f, most);
        top[k] = most;
        total[k] *= f;
        x[k] *= f;
#pragma unroll
        for (int t = 0; t < BATCH; ++t) {
          const float e = t0 + t < j.slices ? weight(low(ms[k][t]), high(ms[k][t]), most) : 0.0f;
          total[k] += e;
          x[k][0] += e * low(u[k][t]);
          x[k][1] += e * high(u[k][t]);
          x[k][2] += e * low(v[k][t]);
          x[k][3] += e * high(v[k][t]);
        }
      }
    }
    if (ITEMS == 1 && groups > 1) {  // (every thread comes here once)
      float* to = scratch + at * 8;
      *reinterpret_cast<f4*>(to) = x[0];
      to[4] = top[0];
      to[5] = total[0];
    } else {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        if (at + k * THREADS >= items) break;
        x[k] *= total[k] == 0.0f ? 0.0f : 1.0f / total[k];
        j.write<TYPE, 4>(p, j.row0 + item[k] / (D / 4), item[k] % (D / 4) * 4, reinterpret_cast<const float*>(&x[k]));
      }
    }
  }
  if (ITEMS > 1 || groups == 1) return;
  __syncthreads();
  const int item = (int)threadIdx.x;
  if (item >= items) return;
  float top = -__builtin_inff(), total = 0.0f;
  for (int k = 0; k < groups; ++k) top = fmaxf(top, scratch[(k * items + item) * 8 + 4]);
  f4 x = (f4){0.0f, 0.0f, 0.0f, 0.0f};
  for (int k = 0; k < groups; ++k) {
    const float* from = scratch + (k * items + item) * 8;
    const float e = weight(from[4], 1.0f, top);
    total += e * from[5];
    x += e * *reinterpret_cast<const f4*>(from);
  }
  x *= total == 0.0f ? 0.0f : 1.0f / total;
  j.write<TYPE, 4>(p, j.row0 + item / (D / 4), item % (D / 4) * 4, reinterpret_cast<const float*>(&x));
}

}  // namespace
