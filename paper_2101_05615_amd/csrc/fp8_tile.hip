// Products of 8-bit floats, many rows: plain, the gated block's forward pass, and its backward pass.
//
// Bound by the matrix cores.  A workgroup of four waves has 16 * MF rows and 256 slots of the weights; a wave has all the rows and 64 of
// the slots, as 4 * MF tiles of 16 x 16 in fp32.  The rows' codes go into LDS without passing registers, two blocks of K ahead, and
// every wave reads them all; the weights, which no two waves share, go from memory to registers in the order they are packed in, one
// block of K ahead.  The scales, one for a row's block and one for a fragment's, are operands of the matrix instruction.
#include "qg_fp8.h"

namespace {

constexpr int SLOTS = 256, STAGES = 3;

__device__ inline void request_rows(unsigned lds, unsigned offset, const uint8_t* base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory");
}

struct piece {  // a wave's weights of one block of K
  u4 x[4][2];
  __device__ inline void load(const uint8_t* from, int lane) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) x[j][h] = *reinterpret_cast<const u4*>(from + j * 2048 + h * 1024 + lane * 16);
  }
  __device__ inline void arrived() {  // (in registers from here on: the compiler waits in front of this)
#pragma unroll
    for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(x[j][0]), "+v"(x[j][1]));
  }
};

template <int TYPE, int N>
__device__ inline void get(const qg_fp8_rows& from, int row, int column, int columns, float* v) {
  typedef typename qg_elem<TYPE>::t T;
  const T* in = static_cast<const T*>(from.data) + row * from.stride + column;
  if (column + N <= columns) {
    qg_load<TYPE, N>(in, v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = column + i < columns ? qg_elem<TYPE>::up(in[i]) : 0.0f;
  }
}

__device__ inline void put_codes(const qg_fp8_held& to, int row, int column, const float* v, float power) {
  const u2 w = {codes_of(v[0], v[1], v[2], v[3], power), codes_of(v[4], v[5], v[6], v[7], power)};
  *reinterpret_cast<u2*>(to.codes + (size_t)row * to.pitch + column) = w;
}
__device__ inline unsigned top_of(const float* v) {
  unsigned top = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = umax(top, size_bits(v[i]));
  return max_over_quads(top);
}

// WIDE: sums by the bf16 instructions
template <int MF, int END, bool WIDE>
__global__ __launch_bounds__(256, MF >= 8 ? 1 : 2) void qg_fp8_tile_kernel(qg_fp8_product_args p, int row_tiles, int column_tiles) {
  constexpr int ROWS = 16 * MF, STAGE = ROWS * 128, REQUESTS = MF >= 2 ? MF / 2 : 1;
  __shared__ __align__(1024) uint8_t rows_lds[STAGES * STAGE];
  __shared__ int ticket;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int m = lane & 15, g = lane >> 4;

  // Workgroups go round-robin over the 8 XCDs: each gets a run of tiles, eight rows of tiles at a time, so that those that run at once
  // on an XCD share rows and columns in its L2
  const int tiles = row_tiles * column_tiles, per = (tiles + 7) / 8;
  const int id = (int)blockIdx.x % (per * 8), slice = (int)blockIdx.x / (per * 8);
  const int at = id % 8 * per + id / 8;
  if (at >= tiles || id / 8 >= per) return;
  const int panel = at / (8 * column_tiles), in_panel = at - panel * 8 * column_tiles;
  const int panel_rows = min(8, row_tiles - panel * 8);
  const int row_tile = panel * 8 + in_panel % panel_rows, column_tile = in_panel / panel_rows;
  const int row0 = row_tile * ROWS, last_row = p.tokens - 1;
  const int group = column_tile * 4 + wave;
  const int k0 = slice * p.slice_kb, k1 = min(k0 + p.slice_kb, p.w.kb);

  // requests of 1 KiB: eight rows; within a row's 128 bytes chunk c lies at place c ^ (row >> 1 & 7), so that the reads of 16 rows of one
  // chunk go through all banks
  unsigned offset[REQUESTS];
#pragma unroll
  for (int r = 0; r < REQUESTS; ++r) {
    const int row = 8 * (wave + 4 * r) + lane / 8;
    offset[r] = (unsigned)(min(row0 + row, last_row) - row0) * (unsigned)p.x8.pitch + (unsigned)((lane % 8 ^ (row >> 1 & 7)) * 16);
  }
  const uint8_t* const codes = p.x8.codes + (size_t)row0 * p.x8.pitch;
  const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) uint8_t*)rows_lds;
  auto request = [&](int kb) {
    if (wave * 8 >= ROWS) return;
    const unsigned to = lds0 + (unsigned)((kb - k0) % STAGES) * STAGE + (unsigned)wave * 1024u;
#pragma unroll
    for (int r = 0; r < REQUESTS; ++r) request_rows(to + r * 4096u, offset[r], codes + (size_t)kb * 128);
  };
  const uint8_t* const pieces = p.w.pieces + (size_t)group * p.w.kb * QG_FP8_PIECE;
  const uint32_t* const weight_scales = p.w.scales + (size_t)group * p.w.kb4;
  const uint8_t* row_scales[MF];
#pragma unroll
  for (int i = 0; i < MF; ++i) row_scales[i] = p.x8.scales + (size_t)min(row0 + 16 * i + m, last_row) * p.x8.scale_pitch;

  f4 c[MF][4];
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) c[i][j] = (f4){0.0f, 0.0f, 0.0f, 0.0f};

  const unsigned read0 = (unsigned)(m * 128 + ((g ^ (m >> 1)) * 16));
  unsigned scale[MF], next_scale[MF];
  piece now, next;
  request(k0);
  if (k0 + 1 < k1) request(k0 + 1);
  next.load(pieces + (size_t)k0 * QG_FP8_PIECE, lane);
#pragma unroll
  for (int i = 0; i < MF; ++i) next_scale[i] = *reinterpret_cast<const uint32_t*>(row_scales[i] + k0);
  for (int kb = k0; kb < k1; ++kb) {
    next.arrived();
#pragma unroll
    for (int i = 0; i < MF; ++i) asm volatile("" : "+v"(next_scale[i]));
    now = next;
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();  // the rows of this block are there, and nobody reads the last one's any more
    asm volatile("" ::: "memory");
    if (kb % 4 == 0) {
#pragma unroll
      for (int i = 0; i < MF; ++i) scale[i] = next_scale[i];
    } else {
#pragma unroll
      for (int i = 0; i < MF; ++i) scale[i] >>= 8;
    }
    if (kb + 2 < k1) request(kb + 2);
    if (kb + 1 < k1) next.load(pieces + (size_t)(kb + 1) * QG_FP8_PIECE, lane);
    if (kb % 4 == 3 && kb + 1 < k1) {
#pragma unroll
      for (int i = 0; i < MF; ++i) next_scale[i] = *reinterpret_cast<const uint32_t*>(row_scales[i] + kb + 1);
    }
    const unsigned ws = weight_scales[kb];
    const uint8_t* stage = rows_lds + (kb - k0) % STAGES * STAGE;
    if constexpr (WIDE) {
      wide w[4] = {wide(now.x[0][0], now.x[0][1], scale_of(ws & 255u)), wide(now.x[1][0], now.x[1][1], scale_of(ws >> 8 & 255u)),
                   wide(now.x[2][0], now.x[2][1], scale_of(ws >> 16 & 255u)), wide(now.x[3][0], now.x[3][1], scale_of(ws >> 24))};
#pragma unroll
      for (int i = 0; i < MF; ++i) {
        const wide x(*reinterpret_cast<const u4*>(stage + i * 2048 + read0), *reinterpret_cast<const u4*>(stage + i * 2048 + (read0 ^ 64u)),
                     scale_of(scale[i] & 255u));
#pragma unroll
        for (int j = 0; j < 4; ++j) c[i][j] = wide_product(w[j], x, c[i][j]);
      }
      continue;
    }
#pragma unroll
    for (int i = 0; i < MF; ++i) {
      const i8v x = both(*reinterpret_cast<const u4*>(stage + i * 2048 + read0), *reinterpret_cast<const u4*>(stage + i * 2048 + (read0 ^ 64u)));
#pragma unroll
      for (int j = 0; j < 4; ++j) c[i][j] = matrix_product(both(now.x[j][0], now.x[j][1]), x, c[i][j], j, ws, scale[i]);
    }
  }

  if (p.slices > 1) {  // sums of the slices through memory, past the L2s that the XCDs do not share; the last one to arrive adds them in order
    const int tile = row_tile * column_tiles + column_tile;
    float* const mine = p.partial + ((size_t)tile * p.slices * (SLOTS / 64) + wave) * (size_t)(ROWS * 64) + lane * 4;
    const size_t step = (size_t)(SLOTS / 64) * (ROWS * 64);
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        asm volatile("global_store_dwordx4 %0, %1, off sc1\n\ts_nop 1" ::"v"(mine + slice * step + (i * 4 + j) * 256), "v"(c[i][j]) : "memory");
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) ticket = __hip_atomic_fetch_add(p.counters + tile, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (ticket != p.slices - 1) return;
    if (threadIdx.x == 0) __hip_atomic_store(p.counters + tile, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // ready for the next call
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) c[i][j] = (f4){0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = 0; s < p.slices; ++s) {
      const float* theirs = mine + s * step;
#pragma unroll
      for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const unsigned long long* from = reinterpret_cast<const unsigned long long*>(theirs + (i * 4 + j) * 256);
          const unsigned long long a = __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          const unsigned long long b = __hip_atomic_load(from + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          c[i][j][0] += __builtin_bit_cast(float, (unsigned)a);
          c[i][j][1] += __builtin_bit_cast(float, (unsigned)(a >> 32));
          c[i][j][2] += __builtin_bit_cast(float, (unsigned)b);
          c[i][j][3] += __builtin_bit_cast(float, (unsigned)(b >> 32));
        }
    }
  }

  if constexpr (END == QG_FP8_PLAIN) {
    const int column = group * 64 + 16 * g;
    if (column >= p.channels) return;
    float bias[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) bias[i] = p.bias && column + i < p.channels ? p.bias[column + i] : 0.0f;
#pragma unroll
    for (int i = 0; i < MF; ++i) {
      const int row = row0 + 16 * i + m;
      if (row > last_row) continue;
      float v[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = c[i][j / 4][j % 4] + bias[j];
      put<16>(p.out_type, p.out, row, column, p.channels, v);
    }
  } else {
    // 32 columns of the inner size a wave, 8 a lane
    const int column = group * 32 + 8 * g, block = column_tile, padded = column_tiles * 128;
    constexpr int BATCH = MF < 4 ? MF : 4;   // row fragments whose largest values meet at once
    float* const tops_f = reinterpret_cast<float*>(rows_lds);
    unsigned* const tops = reinterpret_cast<unsigned*>(tops_f);  // [3][4 waves][16 * BATCH]
    const bool held = END == QG_FP8_GATED_BACK || p.out.data == nullptr;
    for (int b0 = 0; b0 < MF; b0 += BATCH) {
      float h[BATCH][8], dg[BATCH][8], du[BATCH][8];
      (void)dg;
      (void)du;
      __syncthreads();
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        const int i = b0 + b, row = row0 + 16 * i + m;
        float dh[8];
        if (END == QG_FP8_GATED_BACK) {
          const int from = min(row, last_row);
          if (p.dh_type == QG_F32) get<QG_F32, 8>(p.dh, from, column, p.channels, dh);
          if (p.dh_type == QG_BF16) get<QG_BF16, 8>(p.dh, from, column, p.channels, dh);
          if (p.dh_type == QG_F16) get<QG_F16, 8>(p.dh, from, column, p.channels, dh);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          f4 gs = c[0][0], us = c[0][0];
#pragma unroll
          for (int f = 0; f < MF; ++f)
            if (f == i) gs = c[f][j / 4 * 2], us = c[f][j / 4 * 2 + 1];
          const float gate = gs[j % 4], up = us[j % 4];
          float slope = 0.0f;
          const float a = activate<END == QG_FP8_GATED_BACK>(p.activation, gate, &slope);
          h[b][j] = a * up;
          if (END == QG_FP8_GATED_BACK) {
            dg[b][j] = dh[j] * up * slope;
            du[b][j] = dh[j] * a;
          }
        }
        if (!held) {
          if (row <= last_row && column < p.channels) put<8>(p.out_type, p.out, row, column, p.channels, h[b]);
          continue;
        }
        const unsigned top_h = top_of(h[b]);
        if (g == 0) tops[wave * 16 * BATCH + 16 * b + m] = top_h;
        if (END == QG_FP8_GATED_BACK) {
          const unsigned top_g = top_of(dg[b]), top_u = top_of(du[b]);
          if (g == 0) tops[(4 + wave) * 16 * BATCH + 16 * b + m] = top_g;
          if (g == 0) tops[(8 + wave) * 16 * BATCH + 16 * b + m] = top_u;
        }
      }
      if (!held) continue;
      __syncthreads();
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        const int row = row0 + 16 * (b0 + b) + m;
        unsigned byte[3];
#pragma unroll
        for (int s = 0; s < (END == QG_FP8_GATED_BACK ? 3 : 1); ++s) {
          const unsigned* of = tops + s * 64 * BATCH + 16 * b + m;
          byte[s] = scale_byte(umax(umax(of[0], of[16 * BATCH]), umax(of[32 * BATCH], of[48 * BATCH])));
        }
        if (row > last_row) continue;
        put_codes(p.out8, row, column, h[b], scale_of(byte[0]));
        if (wave == 0 && g == 0) p.out8.scales[(size_t)row * p.out8.scale_pitch + block] = (uint8_t)byte[0];
        if (END == QG_FP8_GATED_BACK) {
          put_codes(p.dgu8, row, column, dg[b], scale_of(byte[1]));
          put_codes(p.dgu8, row, padded + column, du[b], scale_of(byte[2]));
          if (wave == 0 && g == 0) {
            uint8_t* scales = p.dgu8.scales + (size_t)row * p.dgu8.scale_pitch;
            scales[block] = (uint8_t)byte[1];
            scales[column_tiles + block] = (uint8_t)byte[2];
          }
          __bf16* to = p.dgu + (size_t)row * 2 * padded + column;
          qg_store<QG_BF16, 8>(to, dg[b]);
          qg_store<QG_BF16, 8>(to + padded, du[b]);
        }
      }
    }
  }
}

template <int MF, int END, bool WIDE>
hipError_t launch(const qg_fp8_product_args& a, hipStream_t s) {
  const int rows = (a.tokens + 16 * MF - 1) / (16 * MF), columns = a.w.groups / 4;
  const unsigned per = (unsigned)(((long long)rows * columns + 7) / 8);
  hipLaunchKernelGGL((qg_fp8_tile_kernel<MF, END, WIDE>), dim3(per * 8 * (unsigned)a.slices), dim3(256), 0, s, a, rows, columns);
  return hipGetLastError();
}
template <int END, bool WIDE>
hipError_t launch(const qg_fp8_product_args& a, int row_fragments, hipStream_t s) {
  if (row_fragments == 2) return launch<2, END, WIDE>(a, s);
  if (row_fragments == 4) return launch<4, END, WIDE>(a, s);
  return launch<8, END, WIDE>(a, s);
}

}  // namespace

hipError_t qg_launch_fp8_tile(const qg_fp8_product_args& a, int end, int row_fragments, int wide_sums, hipStream_t s) {
  if (end == QG_FP8_GATED_BACK) return launch<QG_FP8_GATED_BACK, false>(a, row_fragments, s);
  if (wide_sums) return end == QG_FP8_PLAIN ? launch<QG_FP8_PLAIN, true>(a, row_fragments, s) : launch<QG_FP8_GATED, true>(a, row_fragments, s);
  return end == QG_FP8_PLAIN ? launch<QG_FP8_PLAIN, false>(a, row_fragments, s) : launch<QG_FP8_GATED, false>(a, row_fragments, s);
}
