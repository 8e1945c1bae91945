// Products of 8-bit floats, few rows: plain, and the gated block's forward pass.
//
// Bound by the bytes of the weights, so each is read once, straight into the registers of the wave that needs it.  A workgroup has NF
// fragments of 16 slots and all rows; its waves split K block by block, each with a batch of blocks on its way while one is worked on, and
// their sums meet in LDS.  Where even then there are few workgroups, K is split over workgroups too.  Up to 16 rows that are not in 8
// bits yet become so in the registers of the wave that multiplies them.  The matrix cores have time to spare: sums by the bf16 instructions.
// Weights from HBM: 16 x 8192 x 8192 14.3 us (4.7 TB/s, where a large copy reaches 5.1), 1 x 4096 x 4096 6.4 (2.6: launch, codes of the first block,
// one batch a wave, the sums in LDS), 4 rows through a pair of 4096 x 10240 17.7 (4.7) and 10240 x 4096 11.8 (3.6).
#include "qg_fp8.h"

namespace {

constexpr int HELD = 3;  // of X: the rows are in 8 bits

template <int X>
struct raw_half {  // 16 channels of a token as they are
  static constexpr int N = X == QG_F32 ? 16 : 8;
  unsigned d[N];
  __device__ inline void load(const qg_fp8_rows& x, int row, int channels, int first) {
    typedef typename qg_elem<X>::t T;
    const T* from = static_cast<const T*>(x.data) + row * x.stride + (first < channels ? first : 0);  // (channels: a multiple of 16)
    typedef u4 any __attribute__((aligned(2)));
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const u4 v = reinterpret_cast<const any*>(from)[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) d[4 * i + j] = v[j];
    }
  }
  __device__ inline void cut(bool there) {
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] = there ? d[i] : 0u;
  }
  // the bits in fp32 of the largest size
  __device__ inline unsigned top() const {
    unsigned t = 0u;
    if constexpr (X == QG_F32) {
#pragma unroll
      for (int i = 0; i < N; ++i) t = umax(t, d[i] & 0x7fffffffu);
      return t;
    } else {
      typedef unsigned short us2 __attribute__((ext_vector_type(2)));
      us2 m = {0, 0};
#pragma unroll
      for (int i = 0; i < N; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(us2, d[i] & 0x7fff7fffu));
      const unsigned short most = m[0] > m[1] ? m[0] : m[1];
      return X == QG_BF16 ? (unsigned)most << 16 : size_bits((float)__builtin_bit_cast(_Float16, most));
    }
  }
  __device__ inline u4 codes(float scale) const {
    u4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (X == QG_F32) {
        w[i] = codes_of(__builtin_bit_cast(float, d[4 * i]), __builtin_bit_cast(float, d[4 * i + 1]), __builtin_bit_cast(float, d[4 * i + 2]),
                        __builtin_bit_cast(float, d[4 * i + 3]), scale);
      } else {
        w[i] = codes_of_pairs<X>(d[2 * i], d[2 * i + 1], scale);
      }
    }
    return w;
  }
};
template <>
struct raw_half<HELD> {};

template <int RF, int NF, int U, int X>
struct batch {
  u4 w[U][NF][2];
  unsigned ws[U];
  u4 x[U][RF][2];
  unsigned xs[U][RF];
  raw_half<X> raw[X == HELD ? 1 : U][2];
};

template <int RF, int NF, int WAVES, int X, bool GATED>
__global__ __launch_bounds__(64 * WAVES) void qg_fp8_stream_kernel(qg_fp8_product_args p) {
  constexpr int U = RF > 1 || NF == 4 ? 1 : 2;  // blocks of a batch
  constexpr int SETS = 4 / NF;
  __shared__ f4 sums[WAVES][RF * NF][64];
  __shared__ int ticket;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int m = lane & 15, g = lane >> 4;
  const int sets = p.w.groups * SETS, set = (int)blockIdx.x % sets, rest = (int)blockIdx.x / sets;
  const int blocks = (p.tokens + 16 * RF - 1) / (16 * RF), row0 = rest % blocks * (16 * RF), slice = rest / blocks;
  const int group = set / SETS, first = set % SETS * NF;
  const int k0 = slice * p.slice_kb, k1 = min(k0 + p.slice_kb, p.w.kb);
  const uint8_t* const pieces = p.w.pieces + (size_t)group * p.w.kb * QG_FP8_PIECE + first * 2048 + lane * 16;
  const uint32_t* const weight_scales = p.w.scales + (size_t)group * p.w.kb4;

  f4 c[RF][NF];
#pragma unroll
  for (int i = 0; i < RF; ++i)
#pragma unroll
    for (int j = 0; j < NF; ++j) c[i][j] = (f4){0.0f, 0.0f, 0.0f, 0.0f};

  auto load = [&](int kb, batch<RF, NF, U, X>& b) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = min(kb + u * WAVES, k1 - 1);  // (past the end: the last block again, not used)
#pragma unroll
      for (int j = 0; j < NF; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) b.w[u][j][h] = *reinterpret_cast<const u4*>(pieces + (size_t)at * QG_FP8_PIECE + j * 2048 + h * 1024);
      b.ws[u] = weight_scales[at] >> (8 * first);
#pragma unroll
      for (int i = 0; i < RF; ++i) {
        const int row = min(row0 + 16 * i + m, p.tokens - 1);   // (rows behind the last: that one again, not written)
        if constexpr (X == HELD) {
          const uint8_t* from = p.x8.codes + (size_t)row * p.x8.pitch + (size_t)at * 128 + g * 16;
#pragma unroll
          for (int h = 0; h < 2; ++h) b.x[u][i][h] = *reinterpret_cast<const u4*>(from + 64 * h);
          b.xs[u][i] = p.x8.scales[(size_t)row * p.x8.scale_pitch + at];
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h) b.raw[u][h].load(p.x, row, p.w.k, at * 128 + 64 * h + 16 * g);
        }
      }
    }
  };
  auto multiply = [&](int kb, batch<RF, NF, U, X>& b) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (kb + u * WAVES >= k1) break;
      if constexpr (X != HELD) {
        const int at = kb + u * WAVES;
        if ((at + 1) * 128 > p.w.k) {
#pragma unroll
          for (int h = 0; h < 2; ++h) b.raw[u][h].cut(at * 128 + 64 * h + 16 * g < p.w.k);
        }
        b.xs[u][0] = scale_byte(max_over_quads(umax(b.raw[u][0].top(), b.raw[u][1].top())));
#pragma unroll
        for (int h = 0; h < 2; ++h) b.x[u][0][h] = b.raw[u][h].codes(scale_of(b.xs[u][0]));
      }
      wide x[RF];
#pragma unroll
      for (int i = 0; i < RF; ++i) x[i] = wide(b.x[u][i][0], b.x[u][i][1], scale_of(b.xs[u][i]));
#pragma unroll
      for (int j = 0; j < NF; ++j) {
        const wide w(b.w[u][j][0], b.w[u][j][1], scale_of(b.ws[u] >> (8 * j) & 255u));
#pragma unroll
        for (int i = 0; i < RF; ++i) c[i][j] = wide_product(w, x[i], c[i][j]);
      }
    }
  };
  constexpr int STEP = WAVES * U;
  if (k0 + wave < k1) {
    batch<RF, NF, U, X> now, next;
    int kb = k0 + wave;
    load(kb, now);
    for (; kb + STEP < k1; kb += STEP) {
      load(kb + STEP, next);
      multiply(kb, now);
      now = next;
    }
    multiply(kb, now);
  }
#pragma unroll
  for (int i = 0; i < RF; ++i)
#pragma unroll
    for (int j = 0; j < NF; ++j) sums[wave][i * NF + j][lane] = c[i][j];
  __syncthreads();

  // a result's four columns (gated: of both matrices) a thread
  constexpr int PER = GATED ? 2 : 1, ITEMS = RF * NF / PER * 64;
  constexpr int TURNS = (ITEMS + 64 * WAVES - 1) / (64 * WAVES);
  f4 s[TURNS][PER];
#pragma unroll
  for (int t = 0; t < TURNS; ++t) {
    const int item = (int)threadIdx.x + t * 64 * WAVES;
    if (item >= ITEMS) break;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      s[t][e] = sums[0][item / 64 * PER + e][item % 64];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) s[t][e] += sums[w][item / 64 * PER + e][item % 64];
    }
  }
  if (p.slices > 1) {  // through memory, past the L2s that the XCDs do not share; the last one to arrive adds them in order
    const int part = set * blocks + rest % blocks;
    float* const mine = p.partial + (size_t)part * p.slices * (ITEMS * PER * 4);
#pragma unroll
    for (int t = 0; t < TURNS; ++t) {
      const int item = (int)threadIdx.x + t * 64 * WAVES;
      if (item >= ITEMS) break;
#pragma unroll
      for (int e = 0; e < PER; ++e)
        asm volatile("global_store_dwordx4 %0, %1, off sc1\n\ts_nop 1" ::"v"(mine + ((size_t)slice * ITEMS * PER + e * ITEMS + item) * 4), "v"(s[t][e]) : "memory");
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) ticket = __hip_atomic_fetch_add(p.counters + part, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (ticket != p.slices - 1) return;
    if (threadIdx.x == 0) __hip_atomic_store(p.counters + part, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // ready for the next call
#pragma unroll
    for (int t = 0; t < TURNS; ++t) {
      const int item = (int)threadIdx.x + t * 64 * WAVES;
      if (item >= ITEMS) break;
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        f4 sum = (f4){0.0f, 0.0f, 0.0f, 0.0f};
        for (int k = 0; k < p.slices; ++k) {
          const unsigned long long* from = reinterpret_cast<const unsigned long long*>(mine + ((size_t)k * ITEMS * PER + e * ITEMS + item) * 4);
          const unsigned long long a = __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          const unsigned long long b = __hip_atomic_load(from + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          sum[0] += __builtin_bit_cast(float, (unsigned)a);
          sum[1] += __builtin_bit_cast(float, (unsigned)(a >> 32));
          sum[2] += __builtin_bit_cast(float, (unsigned)b);
          sum[3] += __builtin_bit_cast(float, (unsigned)(b >> 32));
        }
        s[t][e] = sum;
      }
    }
  }
  const activation act(p.activation);
#pragma unroll
  for (int t = 0; t < TURNS; ++t) {
    const int item = (int)threadIdx.x + t * 64 * WAVES;
    if (item >= ITEMS) break;
    const int part = item / 64, of = item % 64, i = part / (NF / PER), j = part % (NF / PER);
    const int row = row0 + 16 * i + (of & 15);
    const int column = GATED ? group * 32 + 8 * (of >> 4) + 4 * (first / 2 + j) : group * 64 + 16 * (of >> 4) + 4 * (first + j);
    if (row >= p.tokens || column >= p.channels) continue;
    float v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (GATED) {
        v[r] = act.operator()<false>(s[t][0][r], nullptr) * s[t][PER - 1][r];
      } else {
        v[r] = s[t][0][r] + (p.bias && column + r < p.channels ? p.bias[column + r] : 0.0f);
      }
    }
    put<4>(p.out_type, p.out, row, column, p.channels, v);
  }
}

template <int RF, int NF, int WAVES, int X, bool GATED>
hipError_t launch(const qg_fp8_product_args& a, hipStream_t s) {
  const unsigned sets = (unsigned)(a.w.groups * (4 / NF)), blocks = (unsigned)((a.tokens + 16 * RF - 1) / (16 * RF));
  hipLaunchKernelGGL((qg_fp8_stream_kernel<RF, NF, WAVES, X, GATED>), dim3(sets * blocks * (unsigned)a.slices), dim3(64 * WAVES), 0, s, a);
  return hipGetLastError();
}

template <int RF, int NF, int WAVES, int X>
hipError_t launch(const qg_fp8_product_args& a, int gated, hipStream_t s) {
  return gated ? launch<RF, NF, WAVES, X, true>(a, s) : launch<RF, NF, WAVES, X, false>(a, s);
}
template <int NF, int WAVES>
hipError_t launch_few(const qg_fp8_product_args& a, int gated, hipStream_t s) {
  if (!a.x.data) return launch<1, NF, WAVES, HELD>(a, gated, s);
  return a.x_type == QG_F32    ? launch<1, NF, WAVES, QG_F32>(a, gated, s)
         : a.x_type == QG_BF16 ? launch<1, NF, WAVES, QG_BF16>(a, gated, s)
                               : launch<1, NF, WAVES, QG_F16>(a, gated, s);
}

}  // namespace

hipError_t qg_launch_fp8_stream(const qg_fp8_product_args& a, int gated, const qg_fp8_stream_form& f, hipStream_t s) {
  if (f.rows == 2) return f.fragments == 4 ? launch<2, 4, 8, HELD>(a, gated, s) : launch<2, 2, 8, HELD>(a, gated, s);
  if (f.fragments == 4) return f.waves == 4 ? launch_few<4, 4>(a, gated, s) : launch_few<4, 8>(a, gated, s);
  return f.waves == 4 ? launch_few<2, 4>(a, gated, s) : launch_few<2, 8>(a, gated, s);
}
