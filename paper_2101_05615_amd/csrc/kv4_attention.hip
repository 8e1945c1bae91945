// Attention over the 4-bit cache for few query rows (a KV head's query heads times the queries of a sequence are at most 32): one
// generated token, or a handful of drafted ones.
//
// Bound by the cache's bytes, so each is read once, straight into the registers of the wave that needs it: the waves of a workgroup
// have the same rows and split its tokens, tile by tile, with one tile on its way while one is worked on; sums meet in LDS.  Long
// sequences in small batches are split over workgroups too.
#include "qg_kv4_tile.h"

namespace {

constexpr int WAVES = 4;  // of a workgroup; eight (64 KiB of LDS, one workgroup a CU) measured the same or a few per cent more

template <int D>
struct tile_bits {
  unsigned k[2][D / 32];  // tile a of 16 tokens: D / 4 channels of one token
  u4 v[D / 64];           // four channels of 8 tokens each
  unsigned w;             // a word of the row's 8 tokens: keys 0 .. 7, then values
};

// A lane's share of the tile at t0
template <int D, bool SMALL>
__device__ inline void load_tile(const reader<D, SMALL>& in, int t0, page_ids ids, tile_bits<D>& b) {
  typedef lay<D> L;
  const spots at = in.at(t0, ids);
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int i = 0; i < L::KEY_LOADS; ++i) in.load_keys(at, a, i, b.k[a] + i * L::KEY_WORDS);
#pragma unroll
  for (int i = 0; i < L::VALUE_LOADS; ++i) b.v[i] = in.load_values(at, i);
  b.w = in.load_word(at);
}

template <int D, int DIG, int NR>
struct rows_of_wave : state<D, DIG, NR> {
  frag q[NR][DIG][D / 32];
  float q_sum[NR];  // DIG 1: less the sum of the queries, times 2^-20
};

template <int D, int DIG, int NR, int PARTS, bool MASKED>
__device__ inline void step(rows_of_wave<D, DIG, NR>& s, const tile_bits<D>& b, int t0, int end, int r, int g) {
  unsigned word = b.w;
  if (MASKED && t0 + 8 * g + (r & 7) >= end) word = 0u;
  const unsigned theta = word & 15u;
  const masks m;

  f4 z[NR][2];
#pragma unroll
  for (int n = 0; n < NR; ++n) z[n][0] = z[n][1] = (f4){0.0f, 0.0f, 0.0f, 0.0f};
  unsigned zero[2];
  if (DIG == 2) {
#pragma unroll
    for (int a = 0; a < 2; ++a) zero[a] = key_zero(theta, a, r);
  }
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      frag k;
      if (DIG == 2) {
        const zero_pair zp(zero[a]);
        spread_less(b.k[a][i], m, as_h2(zp.low), as_h2(zp.high), k.u);
      } else {
        spread(b.k[a][i], k.u);
      }
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int d = 0; d < DIG; ++d) z[n][a] = product(k, s.q[n][d][i], z[n][a]);
    }
  }
  if (DIG == 1) {
    const float t = (float)theta;
    const float zp[8] = {row_lane<0>(t), row_lane<1>(t), row_lane<2>(t), row_lane<3>(t),
                         row_lane<4>(t), row_lane<5>(t), row_lane<6>(t), row_lane<7>(t)};
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int j = 0; j < 8; ++j) z[n][j >> 2][j & 3] = __builtin_fmaf(zp[j], s.q_sum[n], z[n][j >> 2][j & 3]);
  }

  frag p[NR][PARTS];
  float x[NR][8];
  weigh<D, DIG, NR, MASKED>(s, z, word, t0, end, r, g, x);
  halves<NR, PARTS>(x, p);

  const zero_points zp(word);
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    frag v[4];
    spread_values(b.v[i], m, zp, v);
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int d = 0; d < PARTS; ++d) s.o[n][4 * i + c] = product(v[c], p[n][d], s.o[n][4 * i + c]);
  }
}

constexpr int waves_per_simd(int D, int NR) { return NR == 2 || D == 256 ? 2 : 3; }

template <int D, int DIG, int TYPE, int NR, bool SMALL>
__global__ __launch_bounds__(64 * WAVES, waves_per_simd(D, NR)) void qg_kv4_attention_kernel(qg_kv4_attention_args p) {
  constexpr int ROWS = 16 * NR, PITCH = D + 4, STRIDE = TILE * WAVES, PARTS = TYPE == QG_BF16 ? 1 : 2;
  __shared__ float part[WAVES * ROWS * PITCH];
  __shared__ float part_m[WAVES * ROWS], part_sum[WAVES * ROWS];
  __shared__ int ticket;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  job j;
  if (!j.init<ROWS, false>(p)) return;
  const reader<D, SMALL> in(p, j.seq, j.keys, j.head, r, g);
  int t0 = j.lo + wave * TILE;
  page_ids next = {0u, 0u};
  if (t0 < j.hi) next = in.pages(t0);

  raw_query<D, TYPE> raw[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int row = j.row0 + n * 16 + r;
    raw[n].load(j.query<TYPE>(p, row), row < j.rows, g);
  }
  // two tiles in turn, each requested while the other one is worked on (past the end: the last one again), its page one tile before
  const int last = t0 < j.hi ? t0 + (j.hi - 1 - t0) / STRIDE * STRIDE : 0;
  tile_bits<D> a, b;
  if (t0 < j.hi) {
    load_tile(in, t0, next, a);
    next = in.pages(min(t0 + STRIDE, last));
  }
  rows_of_wave<D, DIG, NR> s;
  s.start();
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int shift = split_query<D, DIG, TYPE>(raw[n], s.q[n]);
    if (DIG == 1) {
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += (float)s.q[n][0][i].v[k];
      s.q_sum[n] = across_sum(sum) * -0x1p-20f;
    }
    s.factor[n] = __builtin_ldexpf(p.scale_log2e, (DIG == 1 ? 20 : 0) - shift);
    s.factor_lo[n] = __builtin_ldexpf(p.scale_log2e_lo, -shift);
    s.limit[n] = j.limit(p, j.row0 + n * 16 + r);
  }

  if (t0 < j.hi) {
    const int whole = j.seen_by(p, j.row0);
    while (t0 + STRIDE + TILE <= whole) {
      load_tile(in, min(t0 + STRIDE, last), next, b);
      next = in.pages(min(t0 + 2 * STRIDE, last));
      step<D, DIG, NR, PARTS, false>(s, a, t0, j.hi, r, g);
      t0 += STRIDE;
      load_tile(in, min(t0 + STRIDE, last), next, a);
      next = in.pages(min(t0 + 2 * STRIDE, last));
      step<D, DIG, NR, PARTS, false>(s, b, t0, j.hi, r, g);
      t0 += STRIDE;
    }
    for (; t0 < j.hi; t0 += STRIDE) {
      load_tile(in, min(t0 + STRIDE, last), next, b);
      next = in.pages(min(t0 + 2 * STRIDE, last));
      step<D, DIG, NR, PARTS, true>(s, a, t0, j.hi, r, g);
      a = b;
    }
  }

  // ---- the waves' results meet in LDS, weighted by their sums
  float sum[NR];
  finish(s, sum);
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    float* to = part + (wave * ROWS + n * 16 + r) * PITCH;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      float x[16];
      run_of(s, n, i, x);
#pragma unroll
      for (int c = 0; c < 16; c += 4) *reinterpret_cast<f4*>(to + lay<D>::out_channel(i, g) + c) = (f4){x[c], x[c + 1], x[c + 2], x[c + 3]};
    }
    if (g == 0) {
      part_m[wave * ROWS + n * 16 + r] = s.m[n];
      part_sum[wave * ROWS + n * 16 + r] = sum[n];
    }
  }
  __syncthreads();
  const shares<ROWS> w(p, j);
  for (int at = (int)threadIdx.x; at < (j.last_row - j.row0 + 1) * (D / 4); at += 64 * WAVES) {
    const int local = at / (D / 4), c = at % (D / 4) * 4, row = j.row0 + local;
    float top = -__builtin_inff();
#pragma unroll
    for (int k = 0; k < WAVES; ++k) top = fmaxf(top, part_m[k * ROWS + local]);
    float total = 0.0f;
    f4 x = (f4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < WAVES; ++k) {
      const float e = weight(part_m[k * ROWS + local], part_sum[k * ROWS + local], top);
      total += e;
      x += e * *reinterpret_cast<const f4*>(part + (k * ROWS + local) * PITCH + c);
    }
    x *= total == 0.0f ? 0.0f : 1.0f / total;
    if (j.slices == 1) {
      j.write<TYPE, 4>(p, row, c, reinterpret_cast<const float*>(&x));
    } else {
      hand_in(w.data + w.at(j.slice, row) * D + c, x);
      if (c == 0) hand_in(w.sums + 2 * w.at(j.slice, row), top, total);
    }
  }
  if (j.slices == 1) return;
  // More than two items a thread: four at once, so that their requests overlap (20 rows of 256 channels 25.6 us, one after the other
  // 29.1; 32 rows of 128 channels over 32768 keys 68, 74; four sequences of 20 such rows 18.8, 17.9).  Fewer: 16 shares of one item at
  // once (eight: 32768 keys of one KV head 24.8 -> 26.5, of 16 rows 41.5 -> 44.6; the four shares of 777 keys alone gain, 9.2 -> 8.6).
  if (ROWS * (D / 4) > 2 * 64 * WAVES && (j.last_row - j.row0 + 1) * (D / 4) > 2 * 64 * WAVES)
    join<D, TYPE, 64 * WAVES, 4, 4>(p, j, w, nullptr, &ticket);
  else
    join<D, TYPE, 64 * WAVES, 1, 16>(p, j, w, part, &ticket);
}

template <int D, int TYPE, int NR>
void go(qg_kv4_attention_args a, int rows, hipStream_t s) {
  constexpr int DIG = TYPE == QG_F32 ? 2 : 1;
  a.row_blocks = (rows + 16 * NR - 1) / (16 * NR);
  const dim3 grid((unsigned)(a.batch * a.c.heads * a.split * a.row_blocks));
  if (a.c.lgp == 4)
    hipLaunchKernelGGL((qg_kv4_attention_kernel<D, DIG, TYPE, NR, true>), grid, dim3(64 * WAVES), 0, s, a);
  else
    hipLaunchKernelGGL((qg_kv4_attention_kernel<D, DIG, TYPE, NR, false>), grid, dim3(64 * WAVES), 0, s, a);
}

template <int D, int TYPE>
void by_rows(const qg_kv4_attention_args& a, int rows, hipStream_t s) {
  // (two tiles of 16 rows of 256 channels would leave the registers; two workgroups read the same keys instead)
  if constexpr (D != 256) {
    if (rows > 16) return go<D, TYPE, 2>(a, rows, s);
  }
  go<D, TYPE, 1>(a, rows, s);
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

hipError_t qg_launch_kv4_attention_few(const qg_kv4_attention_args& a, int head_dim, int dtype, int rows, hipStream_t s) {
  switch (head_dim) {
    case 64: by_type<64>(a, dtype, rows, s); break;
    case 128: by_type<128>(a, dtype, rows, s); break;
    default: by_type<256>(a, dtype, rows, s);
  }
  return hipGetLastError();
}
