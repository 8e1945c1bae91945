// Attention over the 4-bit cache for many query rows: a prompt read in pieces, or drafted tokens of many shared heads.
//
// Bound by the vector instructions around the products, so what does not depend on the row is done once: the waves of a workgroup have
// rows of their own (16 NR each) and unpack STAGE tokens together, a part each, into LDS, as first operands in the order in which the
// matrix cores take them (1 KiB per operand, lane after lane: no bank conflicts either way).  Two stages alternate, so that one
// barrier per stage is enough; codes are requested a whole stage before they are unpacked.
#include "qg_kv4_tile.h"

namespace {

constexpr int STAGE = 64;

// Waves of a workgroup.  Eight share the unpacking better, but wait for each other (chunk of 512 queries, 128 channels, keys not
// split: 291 us where four took 240); with 256 channels two workgroups of four do not fit the LDS.
constexpr int waves_of(int D) { return D == 256 ? 8 : 4; }
// Waves of a SIMD that have registers: as many workgroups as the LDS takes (64 channels on two: 512 queries of four sequences, 62 -> 76 us)
constexpr int waves_per_simd(int D) { return D == 64 ? 3 : 2; }

template <int D, int DIG, int NR>
struct rows_of_wave : state<D, DIG, NR> {
  frag q[NR][DIG][D / 32];
};

// The operands of a stage
template <int D>
struct stage_lds {
  frag keys[4][D / 32][64];         // tile of 16 tokens, dword of keys
  frag values[2][D / 16][64];       // step of 32 tokens, output 4 i + c
};

// A part of a stage is 16 tokens' dwords of one load of keys, or 32 tokens' dwords of one load of values
template <int D>
struct parts {
  static constexpr int WAVES = waves_of(D);
  static constexpr int KEYS = 4 * lay<D>::KEY_LOADS, VALUES = 2 * lay<D>::VALUE_LOADS, MINE = (KEYS + VALUES + WAVES - 1) / WAVES;
  u4 bits[MINE];
  unsigned word[2];  // of both steps
};

template <int D, bool SMALL>
__device__ inline void request(const reader<D, SMALL>& in, int t0, const page_ids* ids, int wave, parts<D>& b) {
  typedef parts<D> P;
  const spots at[2] = {in.at(t0, ids[0]), in.at(t0 + TILE, ids[1])};
#pragma unroll
  for (int k = 0; k < P::MINE; ++k) {
    const int u = wave + k * P::WAVES;
    if (u < P::KEYS) {
      unsigned x[4] = {};
      in.load_keys((u >> 1) & 1 ? at[1] : at[0], u & 1, u >> 2, x);
      b.bits[k] = (u4){x[0], x[1], x[2], x[3]};
    } else if (u < P::KEYS + P::VALUES) {
      b.bits[k] = in.load_values((u - P::KEYS) & 1 ? at[1] : at[0], (u - P::KEYS) >> 1);
    }
  }
  b.word[0] = in.load_word(at[0]);
  b.word[1] = in.load_word(at[1]);
}

template <int D>
__device__ inline void unpack(const parts<D>& b, int wave, int lane, stage_lds<D>& to) {
  typedef parts<D> P;
  typedef lay<D> L;
  const masks m;
#pragma unroll
  for (int k = 0; k < P::MINE; ++k) {
    const int u = wave + k * P::WAVES;
    if (u < P::KEYS) {
      const int tile = u & 3, i = u >> 2;
      const zero_pair z(key_zero((tile & 2 ? b.word[1] : b.word[0]) & 15u, tile & 1, lane & 15));
#pragma unroll
      for (int f = 0; f < L::KEY_WORDS; ++f) {
        frag x;
        spread_less(b.bits[k][f], m, as_h2(z.low), as_h2(z.high), x.u);
        to.keys[tile][i * L::KEY_WORDS + f][lane] = x;
      }
    } else if (u < P::KEYS + P::VALUES) {
      const int s = (u - P::KEYS) & 1, i = (u - P::KEYS) >> 1;
      const zero_points z(s ? b.word[1] : b.word[0]);
      frag x[4];
      spread_values(b.bits[k], m, z, x);
#pragma unroll
      for (int c = 0; c < 4; ++c) to.values[s][4 * i + c][lane] = x[c];
    }
  }
}

// Step `which` of a stage: products of queries and keys; of weights and values
template <int D, int DIG, int NR>
__device__ inline void scores(const rows_of_wave<D, DIG, NR>& s, const stage_lds<D>& in, int which, int lane, f4 (*z)[2]) {
#pragma unroll
  for (int a = 0; a < 2; ++a) {
#pragma unroll
    for (int n = 0; n < NR; ++n) z[n][a] = (f4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const frag k = in.keys[2 * which + a][i][lane];
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int d = 0; d < DIG; ++d) z[n][a] = product(k, s.q[n][d][i], z[n][a]);
    }
  }
}
template <int D, int DIG, int NR, int PARTS>
__device__ inline void outputs(rows_of_wave<D, DIG, NR>& s, const stage_lds<D>& in, int which, int lane, const frag (*p)[PARTS]) {
#pragma unroll
  for (int c = 0; c < D / 16; ++c) {
    const frag v = in.values[which][c][lane];
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int d = 0; d < PARTS; ++d) s.o[n][c] = product(v, p[n][d], s.o[n][c]);
  }
}

// A stage.  The second step's scores stand beside the first one's weights, and the first one's outputs beside the second one's
// weights, so that the matrix cores have work while the vector unit has; `between` is what the first scores cover.  (The second scores
// behind the test that the first weights end in: 149 us where this order takes 147.)
template <int D, int DIG, int NR, int PARTS, bool MASKED, typename F>
__device__ inline void stage(rows_of_wave<D, DIG, NR>& s, const stage_lds<D>& in, const unsigned* word, int t0, int end, int lane, F between) {
  const int r = lane & 15, g = lane >> 4;
  unsigned w[2] = {word[0], word[1]};
  if (MASKED) {
    if (t0 + 8 * g + (r & 7) >= end) w[0] = 0u;
    if (t0 + TILE + 8 * g + (r & 7) >= end) w[1] = 0u;
  }
  f4 z[2][NR][2];
  float x[NR][8];
  frag p[NR][PARTS];
  scores(s, in, 0, lane, z[0]);
  between();
  scores(s, in, 1, lane, z[1]);
  weigh<D, DIG, NR, MASKED>(s, z[0], w[0], t0, end, r, g, x);
  halves<NR, PARTS>(x, p);
  outputs(s, in, 0, lane, p);
  weigh<D, DIG, NR, MASKED>(s, z[1], w[1], t0 + TILE, end, r, g, x);
  halves<NR, PARTS>(x, p);
  outputs(s, in, 1, lane, p);
}

template <int D, int DIG, int TYPE, int NR, bool SMALL>
__global__ __launch_bounds__(64 * waves_of(D), waves_per_simd(D)) void qg_kv4_attention_rows_kernel(qg_kv4_attention_args p) {
  constexpr int WAVES = waves_of(D), ROWS = 16 * NR * WAVES, PARTS = TYPE == QG_BF16 ? 1 : 2;
  __shared__ stage_lds<D> lds[2];
  __shared__ int ticket;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  job j;
  if (!j.init<ROWS, true>(p)) return;
  const reader<D, SMALL> in(p, j.seq, j.keys, j.head, r, g);
  const int wave_row = j.row0 + wave * 16 * NR;

  raw_query<D, TYPE> raw[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int row = wave_row + n * 16 + r;
    raw[n].load(j.query<TYPE>(p, row), row < j.rows, g);
  }
  const int last = j.hi > j.lo ? j.lo + (j.hi - 1 - j.lo) / STAGE * STAGE : j.lo;
  auto ids_of = [&](int t, page_ids* ids) {
    ids[0] = in.pages(t);
    ids[1] = in.pages(t + TILE);
  };
  parts<D> next;
  page_ids ids[2];
  if (j.lo < j.hi) {
    ids_of(j.lo, ids);
    request(in, j.lo, ids, wave, next);
    ids_of(min(j.lo + STAGE, last), ids);
  }
  rows_of_wave<D, DIG, NR> s;
  s.start();
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int shift = split_query<D, DIG, TYPE>(raw[n], s.q[n]);
    s.factor[n] = __builtin_ldexpf(p.scale_log2e, -shift);
    s.factor_lo[n] = __builtin_ldexpf(p.scale_log2e_lo, -shift);
    s.limit[n] = j.limit(p, wave_row + n * 16 + r);
  }
  if (j.lo < j.hi) {
    // Keys that all rows of the workgroup see, and that some row of the wave sees.  (Two loops, not a choice in one: with both
    // forms of a step in one loop the outputs are moved about, or leave the registers.)
    const int whole = j.seen_by(p, j.row0);
    const int mine = wave_row < j.rows ? j.seen_by(p, min(wave_row + 16 * NR, j.rows) - 1) : 0;
    unsigned word[2] = {next.word[0], next.word[1]};
    unpack(next, wave, lane, lds[0]);
    request(in, min(j.lo + STAGE, last), ids, wave, next);
    ids_of(min(j.lo + 2 * STAGE, last), ids);
    __syncthreads();
    int which = 0, t0 = j.lo;
    auto prepare = [&]() {  // the stage after t0's into the other half (past the end: the last one again), the one after that on its way
      unpack(next, wave, lane, lds[which ^ 1]);
      word[0] = next.word[0];
      word[1] = next.word[1];
      request(in, min(t0 + 2 * STAGE, last), ids, wave, next);
      ids_of(min(t0 + 3 * STAGE, last), ids);
    };
    for (; t0 + STAGE <= whole; t0 += STAGE) {
      const unsigned now[2] = {word[0], word[1]};
      stage<D, DIG, NR, PARTS, false>(s, lds[which], now, t0, j.hi, lane, prepare);
      which ^= 1;
      __syncthreads();
    }
    for (; t0 < j.hi; t0 += STAGE) {
      const unsigned now[2] = {word[0], word[1]};
      if (t0 < mine)
        stage<D, DIG, NR, PARTS, true>(s, lds[which], now, t0, j.hi, lane, prepare);
      else
        prepare();
      which ^= 1;
      __syncthreads();
    }
  }

  float sum[NR];
  finish(s, sum);
  const shares<ROWS> w(p, j);
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int row = wave_row + n * 16 + r;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      float x[16];
      run_of(s, n, i, x);
      if (j.slices == 1) {
        if (row < j.rows) j.write<TYPE, 16>(p, row, lay<D>::out_channel(i, g), x);
      } else {
        transpose(x);  // (the lanes of a row then write 64 bytes side by side)
        float* to = w.data + w.at(j.slice, row) * D + 64 * i + 4 * g;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (row < j.rows) hand_in(to + 16 * k, (f4){x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]});
      }
    }
    if (j.slices > 1 && g == 0 && row < j.rows) hand_in(w.sums + 2 * w.at(j.slice, row), s.m[n], sum[n]);
  }
  if (j.slices > 1) join<D, TYPE, 64 * WAVES, 4, 4>(p, j, w, nullptr, &ticket);
}

template <int D, int TYPE>
void go(qg_kv4_attention_args a, int rows, hipStream_t s) {
  constexpr int DIG = TYPE == QG_F32 ? 2 : 1, NR = D == 256 || DIG == 2 ? 1 : 2, WAVES = waves_of(D), ROWS = 16 * NR * WAVES;
  a.row_blocks = (rows + ROWS - 1) / ROWS;
  const long long units = (long long)a.batch * a.c.heads * a.row_blocks;
  const dim3 grid((unsigned)(a.shares == 0 ? units : qg_kv4_dealt(units, a.shares, a.max_kv_len, a.least)));
  if (a.c.lgp == 4)
    hipLaunchKernelGGL((qg_kv4_attention_rows_kernel<D, DIG, TYPE, NR, true>), grid, dim3(64 * WAVES), 0, s, a);
  else
    hipLaunchKernelGGL((qg_kv4_attention_rows_kernel<D, DIG, TYPE, NR, false>), grid, dim3(64 * WAVES), 0, s, a);
}

template <int D>
void by_type(const qg_kv4_attention_args& a, int dtype, int rows, hipStream_t s) {
  switch (dtype) {
    case QG_F32: go<D, QG_F32>(a, rows, s); break;
    case QG_BF16: go<D, QG_BF16>(a, rows, s); break;
    default: go<D, QG_F16>(a, rows, s);
  }
}

}  // namespace

hipError_t qg_launch_kv4_attention_many(const qg_kv4_attention_args& a, int head_dim, int dtype, int rows, hipStream_t s) {
  switch (head_dim) {
    case 64: by_type<64>(a, dtype, rows, s); break;
    case 128: by_type<128>(a, dtype, rows, s); break;
    default: by_type<256>(a, dtype, rows, s);
  }
  return hipGetLastError();
}
