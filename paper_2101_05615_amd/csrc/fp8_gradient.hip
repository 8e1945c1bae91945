// The gradient of a weight matrix from activations kept in 8 bits: out[k][n] = sum over tokens of x[t][k] dy[t][n].
//
// The scales of x change along the sum, so its codes are widened: e4m3 times a power of two is exact in bf16.  dy is one bf16 number, or a
// sum of two (fp16) or three (fp32), which hold all its bits; products go through the bf16 matrix instructions, whose rate bounds the
// kernel, and sums are fp32.  Both operands have the summed index as the slow one in memory while the matrix instructions want eight
// tokens of a column in a lane: a thread requests eight tokens of a few neighbouring columns, pairs the tokens' halves of a dword up
// (one instruction per two numbers), and writes whole operands to LDS, one stage ahead of the waves that read them.
#include "qg_fp8.h"

namespace {

typedef float f16v __attribute__((ext_vector_type(16)));

constexpr int TILE_K = 16;  // tokens of a matrix instruction

__device__ inline unsigned pair_low(unsigned a, unsigned b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }   // low halves
__device__ inline unsigned pair_high(unsigned a, unsigned b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }  // high halves

__device__ inline unsigned bf16_pair(float a, float b) {
  const b2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(unsigned, v);
}
__device__ inline float bf16_up(unsigned half) { return __builtin_bit_cast(float, half << 16); }

// CW neighbouring columns of a token as dwords of two bf16, PARTS numbers each
template <int TYPE, int PARTS, int CW>
struct dy_line {
  static constexpr int BYTES = CW * (int)sizeof(typename qg_elem<TYPE>::t);
  unsigned raw[BYTES / 4];
  __device__ inline void load(const void* base, long long at, int left) {
    typedef typename qg_elem<TYPE>::t T;
    const T* from = static_cast<const T*>(base) + at;
    if (left >= CW) {
      typedef unsigned vec __attribute__((ext_vector_type(BYTES / 4 < 4 ? BYTES / 4 : 4)));
      typedef vec vec_any __attribute__((aligned(sizeof(T))));
      constexpr int W = BYTES / 4 < 4 ? BYTES / 4 : 4;
#pragma unroll
      for (int i = 0; i < BYTES / 4; i += W) {
        const vec v = *reinterpret_cast<const vec_any*>(reinterpret_cast<const uint8_t*>(from) + 4 * i);
#pragma unroll
        for (int j = 0; j < W; ++j) raw[i + j] = v[j];
      }
    } else {
      T v[CW];
#pragma unroll
      for (int i = 0; i < CW; ++i) v[i] = i < left ? from[i] : (T)0.0f;
      __builtin_memcpy(raw, v, BYTES);
    }
  }
  __device__ inline void split(unsigned (*out)[CW / 2]) const {  // [PARTS][CW / 2]
    if constexpr (TYPE == QG_BF16) {
#pragma unroll
      for (int i = 0; i < CW / 2; ++i) out[0][i] = raw[i];
    } else {
      typename qg_elem<TYPE>::t v[CW];
      __builtin_memcpy(v, raw, BYTES);
#pragma unroll
      for (int i = 0; i < CW / 2; ++i) {
        float a = qg_elem<TYPE>::up(v[2 * i]), b = qg_elem<TYPE>::up(v[2 * i + 1]);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          out[p][i] = bf16_pair(a, b);
          const float ra = bf16_up(out[p][i] & 0xffffu), rb = bf16_up(out[p][i] >> 16);
          // (what does not fit: exact; of an infinity nothing, it would become NaN)
          a = __builtin_isfinite(ra) ? a - ra : 0.0f;
          b = __builtin_isfinite(rb) ? b - rb : 0.0f;
        }
      }
    }
  }
};

// TS tokens of a stage; CW columns a thread: 256 threads cover TILE columns x TS tokens in blocks of CW x 8
template <int TILE, int TYPE, int PARTS>
__global__ __launch_bounds__(256, PARTS == 1 ? 2 : 1) void qg_fp8_gradient_kernel(qg_fp8_gradient_args p, int row_tiles, int column_tiles) {
  constexpr int CW = TILE == 256 && PARTS == 1 ? 8 : 4, TS = 256 * 8 * CW / TILE, WT = TILE / 2, F = WT / 32;
  constexpr int PLANE = TILE * TS * 2, STAGE = PLANE * (1 + PARTS);
  static_assert(2 * STAGE <= 160 * 1024 - 64, "two stages");
  __shared__ __align__(1024) uint8_t lds[2 * STAGE];
  __shared__ int ticket;
  const int t = (int)threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int tiles = row_tiles * column_tiles, per = (tiles + 7) / 8;
  const int id = (int)blockIdx.x % (per * 8), slice = (int)blockIdx.x / (per * 8);
  const int at = id % 8 * per + id / 8;
  if (at >= tiles) return;
  const int panel = at / (4 * column_tiles), in_panel = at - panel * 4 * column_tiles;
  const int panel_rows = min(4, row_tiles - panel * 4);
  const int row_tile = panel * 4 + in_panel % panel_rows, column_tile = in_panel / panel_rows;
  const int t0 = slice * p.slice_tokens, t1 = min(t0 + p.slice_tokens, p.tokens);

  // what this thread fetches: columns c0 .. of both operands, tokens 8 * tb .. of a stage
  const int chunks = TILE / CW, c0 = t % chunks * CW, tb = t / chunks;
  const int xc = row_tile * TILE + c0, yc = column_tile * TILE + c0;
  const bool x_there = xc < p.x8.pitch;
  const int y_left = p.n - yc;
  unsigned xraw[8][CW / 4], xs[8];
  dy_line<TYPE, PARTS, CW> y[8];
  auto fetch = [&](int from) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int token = from + 8 * tb + i;
      if (token < t1) {
        if (x_there) {
          const uint8_t* src = p.x8.codes + (size_t)token * p.x8.pitch + xc;
          if constexpr (CW == 8) {
            const u2 v = *reinterpret_cast<const u2*>(src);
            xraw[i][0] = v[0];
            xraw[i][1] = v[1];
          } else {
            xraw[i][0] = *reinterpret_cast<const unsigned*>(src);
          }
          xs[i] = p.x8.scales[(size_t)token * p.x8.scale_pitch + xc / QG_FP8_BLOCK];
        } else {
#pragma unroll
          for (int d = 0; d < CW / 4; ++d) xraw[i][d] = 0u;
          xs[i] = 0u;
        }
        y[i].load(p.dy.data, token * p.dy.stride + yc, y_left);
      } else {
#pragma unroll
        for (int d = 0; d < CW / 4; ++d) xraw[i][d] = 0u;
        xs[i] = 0u;
#pragma unroll
        for (int d = 0; d < (int)(sizeof(y[i].raw) / 4); ++d) y[i].raw[d] = 0u;
      }
    }
  };
  // a stage's planes: [32 columns][TS / 16 steps][2 halves of 8 tokens][32 columns, turned by the number of the 32][8 tokens]
  auto place = [&](int column) {
    const int f = column / 32;
    return (unsigned)((f * (TS / TILE_K) + tb / 2) * 1024 + (tb & 1) * 512 + ((column % 32) ^ (f & 7)) * 16);
  };
  auto put_plane = [&](uint8_t* plane, const unsigned (*line)[CW / 2]) {  // line[token][column pair]
#pragma unroll
    for (int j = 0; j < CW; ++j) {
      u4 v;
#pragma unroll
      for (int d = 0; d < 4; ++d) v[d] = j & 1 ? pair_high(line[2 * d][j / 2], line[2 * d + 1][j / 2]) : pair_low(line[2 * d][j / 2], line[2 * d + 1][j / 2]);
      *reinterpret_cast<u4*>(plane + place(c0 + j)) = v;
    }
  };
  auto store = [&](uint8_t* stage) {
    unsigned line[8][CW / 2];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float s = scale_of(xs[i]);
#pragma unroll
      for (int d = 0; d < CW / 4; ++d) {
        line[i][2 * d] = widened(xraw[i][d], s, false);
        line[i][2 * d + 1] = widened(xraw[i][d], s, true);
      }
    }
    put_plane(stage, line);
    unsigned parts[8][PARTS][CW / 2];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i].split(parts[i]);
#pragma unroll
    for (int q = 0; q < PARTS; ++q) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int d = 0; d < CW / 2; ++d) line[i][d] = parts[i][q][d];
      put_plane(stage + (1 + q) * PLANE, line);
    }
  };

  f16v c[F][F];
#pragma unroll
  for (int i = 0; i < F; ++i)
#pragma unroll
    for (int j = 0; j < F; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) c[i][j][e] = 0.0f;
  const int wr = wave >> 1, wc = wave & 1;
  auto operand = [&](const uint8_t* plane, int f, int step) {
    return *reinterpret_cast<const b8*>(plane + (f * (TS / TILE_K) + step) * 1024 + (lane >> 5) * 512 + ((lane & 31) ^ (f & 7)) * 16);
  };
  if (t0 < t1) {
    fetch(t0);
    store(lds);
    int now = 0;
    for (int from = t0; from < t1; from += TS, now ^= 1) {
      const bool more = from + TS < t1;
      if (more) fetch(from + TS);
      __syncthreads();
      const uint8_t* stage = lds + now * STAGE;
#pragma unroll
      for (int s = 0; s < TS / TILE_K; ++s) {
        b8 x[F];
#pragma unroll
        for (int i = 0; i < F; ++i) x[i] = operand(stage, wr * F + i, s);
#pragma unroll
        for (int j = 0; j < F; ++j)
#pragma unroll
          for (int q = 0; q < PARTS; ++q) {
            const b8 g = operand(stage + (1 + q) * PLANE, wc * F + j, s);
#pragma unroll
            for (int i = 0; i < F; ++i) c[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(g, x[i], c[i][j], 0, 0, 0);
          }
      }
      if (more) store(lds + (now ^ 1) * STAGE);
    }
  }
  // a lane has, of fragment (i, j), row 32 i + lane % 32 and the columns 32 j + 8 (e / 4) + 4 (lane / 32) + e % 4
  if (p.slices > 1) {  // sums of the slices through memory; the last one to arrive adds them in order
    const int tile = row_tile * column_tiles + column_tile;
    const size_t step = (size_t)TILE * TILE;
    float* const mine = p.partial + (size_t)tile * p.slices * step + (size_t)wave * (F * F * 1024) + lane * 4;
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
      for (int j = 0; j < F; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f4 v = {c[i][j][4 * e], c[i][j][4 * e + 1], c[i][j][4 * e + 2], c[i][j][4 * e + 3]};
          asm volatile("global_store_dwordx4 %0, %1, off sc1\n\ts_nop 1" ::"v"(mine + slice * step + ((i * F + j) * 4 + e) * 256), "v"(v) : "memory");
        }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (t == 0) ticket = __hip_atomic_fetch_add(p.counters + tile, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (ticket != p.slices - 1) return;
    if (t == 0) __hip_atomic_store(p.counters + tile, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // ready for the next call
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
      for (int j = 0; j < F; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) c[i][j][e] = 0.0f;
    for (int s = 0; s < p.slices; ++s)
#pragma unroll
      for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const unsigned long long* from = reinterpret_cast<const unsigned long long*>(mine + s * step + ((i * F + j) * 4 + e) * 256);
            const unsigned long long a = __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            const unsigned long long b = __hip_atomic_load(from + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            c[i][j][4 * e] += __builtin_bit_cast(float, (unsigned)a);
            c[i][j][4 * e + 1] += __builtin_bit_cast(float, (unsigned)(a >> 32));
            c[i][j][4 * e + 2] += __builtin_bit_cast(float, (unsigned)b);
            c[i][j][4 * e + 3] += __builtin_bit_cast(float, (unsigned)(b >> 32));
          }
  }
#pragma unroll
  for (int i = 0; i < F; ++i) {
    const int row = row_tile * TILE + (wr * F + i) * 32 + (lane & 31);
    if (row >= p.k) continue;
#pragma unroll
    for (int j = 0; j < F; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int column = column_tile * TILE + (wc * F + j) * 32 + 8 * e + 4 * (lane >> 5);
        const float v[4] = {c[i][j][4 * e], c[i][j][4 * e + 1], c[i][j][4 * e + 2], c[i][j][4 * e + 3]};
        if (column < p.n) put<4>(p.out_type, p.out, row, column, p.n, v);
      }
  }
}

template <int TILE, int TYPE, int PARTS>
hipError_t launch(const qg_fp8_gradient_args& a, hipStream_t s) {
  const int rows = (a.k + TILE - 1) / TILE, columns = (a.n + TILE - 1) / TILE;
  const unsigned per = (unsigned)(((long long)rows * columns + 7) / 8);
  hipLaunchKernelGGL((qg_fp8_gradient_kernel<TILE, TYPE, PARTS>), dim3(per * 8 * (unsigned)a.slices), dim3(256), 0, s, a, rows, columns);
  return hipGetLastError();
}
template <int TILE>
hipError_t launch(const qg_fp8_gradient_args& a, hipStream_t s) {
  return a.dy_type == QG_F32    ? launch<TILE, QG_F32, 3>(a, s)
         : a.dy_type == QG_BF16 ? launch<TILE, QG_BF16, 1>(a, s)
                                : launch<TILE, QG_F16, 2>(a, s);
}

}  // namespace

hipError_t qg_launch_fp8_gradient(const qg_fp8_gradient_args& a, hipStream_t s) {
  return launch<128>(a, s);
}
