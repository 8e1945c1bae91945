// Activations and weights into 8-bit floats with a scale per block of 128, and activations back.
#include "qg_fp8.h"

namespace {

template <int N>
__device__ inline unsigned turned(unsigned x) {  // from the lane N further within 16
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + N, 0xf, 0xf, false);
}
__device__ inline unsigned max_of_16(unsigned x) {
  x = umax(x, turned<8>(x));
  x = umax(x, turned<4>(x));
  x = umax(x, turned<2>(x));
  return umax(x, turned<1>(x));
}

// Bound by memory.  A wave takes four blocks of a token, 16 lanes a block, 8 channels a lane: one request of 16 bytes (two of fp32), the
// block's largest over a DPP row, eight codes, and the four scales beside each other.  8192 x 8192 bf16: 39 us into 8 bits, 31 back, 5.2 and 6.5 TB/s
// read and written, the codes from the memory-side cache.
template <int TYPE>
__global__ __launch_bounds__(256) void qg_fp8_quantize_kernel(qg_fp8_rows x, qg_fp8_held to, int tokens, int channels) {
  typedef typename qg_elem<TYPE>::t T;
  const int lane = (int)threadIdx.x & 63, quads = to.scale_pitch / 4;
  const unsigned unit = blockIdx.x * 4u + (threadIdx.x >> 6);
  const int token = (int)(unit / (unsigned)quads), quad = (int)(unit % (unsigned)quads), at = quad * 512 + lane * 8;
  if (token >= tokens) return;
  const T* from = static_cast<const T*>(x.data) + token * x.stride + at;
  float v[8];
  if (at + 8 <= channels) {
    qg_load<TYPE, 8>(from, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = at + i < channels ? qg_elem<TYPE>::up(from[i]) : 0.0f;
  }
  unsigned top = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = umax(top, size_bits(v[i]));
  const unsigned scale = scale_byte(max_of_16(top));
  const float power = scale_of(scale);
  if (at < to.pitch) {
    const u2 w = {codes_of(v[0], v[1], v[2], v[3], power), codes_of(v[4], v[5], v[6], v[7], power)};
    *reinterpret_cast<u2*>(to.codes + (size_t)token * to.pitch + at) = w;
  }
  if ((lane & 15) == 0) to.scales[(size_t)token * to.scale_pitch + quad * 4 + lane / 16] = (uint8_t)scale;
}

template <int TYPE>
__global__ __launch_bounds__(256) void qg_fp8_dequantize_kernel(qg_fp8_held x, qg_fp8_rows to, int tokens, int channels) {
  typedef typename qg_elem<TYPE>::t T;
  const int lane = (int)threadIdx.x & 63, quads = x.scale_pitch / 4;
  const unsigned unit = blockIdx.x * 4u + (threadIdx.x >> 6);
  const int token = (int)(unit / (unsigned)quads), quad = (int)(unit % (unsigned)quads), at = quad * 512 + lane * 8;
  if (token >= tokens || at >= channels) return;
  const u2 w = *reinterpret_cast<const u2*>(x.codes + (size_t)token * x.pitch + at);
  const unsigned scale = x.scales[(size_t)token * x.scale_pitch + at / QG_FP8_BLOCK];
  const float power = scale_of(scale);
  float v[8];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 low = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], power, false), high = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], power, true);
    v[4 * i] = low[0], v[4 * i + 1] = low[1], v[4 * i + 2] = high[0], v[4 * i + 3] = high[1];
  }
  T* out = static_cast<T*>(to.data) + token * to.stride + at;
  if (at + 8 <= channels) {
    qg_store<TYPE, 8>(out, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (at + i < channels) out[i] = qg_elem<TYPE>::down(v[i]);
  }
}

// A block of 128 x 128 per workgroup: read once, kept in registers until its largest is known, codes through LDS into the order of the
// pieces -- of the matrix, of its transpose, or both, which have the same codes and scales.  A pair of 4096 x 10240 bf16 62 us, with the transpose
// 67 (252 MB and 336 MB, 4.1 and 5.0 TB/s); 10240 x 4096 32.
constexpr int PITCH = 144;  // bytes between rows of codes

template <int TYPE>
__global__ __launch_bounds__(256) void qg_fp8_pack_kernel(qg_fp8_pack_args p) {
  typedef typename qg_elem<TYPE>::t T;
  __shared__ __align__(16) uint8_t code[128 * PITCH];
  __shared__ unsigned tops[4];
  const int t = (int)threadIdx.x, nb = (int)blockIdx.x, kb = (int)blockIdx.y, which = (int)blockIdx.z;
  const qg_fp8_matrix_args& m = which ? p.up : p.b;
  const T* base = static_cast<const T*>(m.data);
  const bool down = m.row_stride == 1 && m.column_stride != 1;  // neighbours in memory lie along K
  // eight neighbours of eight lines a thread
  float v[8][8];
  unsigned top = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int line = t / 16 + 16 * i, first = t % 16 * 8;
    const int k0 = kb * 128 + (down ? first : line), n0 = nb * 128 + (down ? line : first);
    const long long step = down ? m.row_stride : m.column_stride;
    const int left = down ? (n0 < p.n ? p.k - k0 : 0) : (k0 < p.k ? p.n - n0 : 0);
    const T* from = base + k0 * m.row_stride + n0 * m.column_stride;
    if (left >= 8 && step == 1) {
      qg_load<TYPE, 8>(from, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = j < left ? qg_elem<TYPE>::up(from[j * step]) : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) top = umax(top, size_bits(v[i][j]));
  }
  top = max_over_quads(max_of_16(top));
  if ((t & 63) == 0) tops[t >> 6] = top;
  __syncthreads();
  const unsigned scale = scale_byte(umax(umax(tops[0], tops[1]), umax(tops[2], tops[3])));
  const float power = scale_of(scale);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int line = t / 16 + 16 * i, first = t % 16 * 8;
    const u2 w = {codes_of(v[i][0], v[i][1], v[i][2], v[i][3], power), codes_of(v[i][4], v[i][5], v[i][6], v[i][7], power)};
    if (!down) {
      *reinterpret_cast<u2*>(code + line * PITCH + first) = w;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) code[(first + j) * PITCH + line] = (uint8_t)(w[j / 4] >> (8 * (j % 4)));
    }
  }
  __syncthreads();
  if (p.pieces && kb < p.kb) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = t + 256 * i, lane = c % 64, half = c / 64 % 2, q = lane % 16 / 4, r = lane % 4;
      const int k = 64 * half + 16 * (lane / 16);
      int group, fragment, n;
      if (p.gated) {
        const int j2 = c / 128 % 2;
        n = c / 256 * 32 + 8 * q + 4 * j2 + r;
        fragment = 2 * j2 + which;
        group = nb * 4 + c / 256;
      } else {
        fragment = c / 128 % 4;
        n = c / 512 * 64 + 16 * q + 4 * fragment + r;
        group = nb * 2 + c / 512;
      }
      u4 w;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        unsigned x = 0u;
#pragma unroll
        for (int b = 0; b < 4; ++b) x |= (unsigned)code[(k + 4 * d + b) * PITCH + n] << (8 * b);
        w[d] = x;
      }
      *reinterpret_cast<u4*>(p.pieces + ((size_t)group * p.kb + kb) * QG_FP8_PIECE + fragment * 2048 + half * 1024 + lane * 16) = w;
    }
    if (p.gated) {
      if (t < 8)
        reinterpret_cast<uint8_t*>(p.scales)[((size_t)(nb * 4 + t / 2) * p.kb4 + kb) * 4 + t % 2 * 2 + which] = (uint8_t)scale;
    } else if (t < 2) {
      p.scales[(size_t)(nb * 2 + t) * p.kb4 + kb] = scale * 0x01010101u;
    }
  }
  const int t_kb = which * (p.t_kb / 2) + nb;  // (of a gated pair the transposes lie below each other)
  if (p.t_pieces && t_kb < p.t_kb) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = t + 256 * i, lane = c % 64, half = c / 64 % 2, fragment = c / 128 % 4, group = c / 512;
      const int k = group * 64 + 16 * (lane % 16 / 4) + 4 * fragment + lane % 4, n = 64 * half + 16 * (lane / 16);
      *reinterpret_cast<u4*>(p.t_pieces + ((size_t)(kb * 2 + group) * p.t_kb + t_kb) * QG_FP8_PIECE + fragment * 2048 + half * 1024 + lane * 16) =
          *reinterpret_cast<const u4*>(code + k * PITCH + n);
    }
    if (t < 2) p.t_scales[(size_t)(kb * 2 + t) * p.t_kb4 + t_kb] = scale * 0x01010101u;
  }
}

template <int TYPE>
hipError_t quantize(const qg_fp8_rows& x, int tokens, int channels, const qg_fp8_held& to, hipStream_t s) {
  const long long units = (long long)tokens * (to.scale_pitch / 4);
  hipLaunchKernelGGL(qg_fp8_quantize_kernel<TYPE>, dim3((unsigned)((units + 3) / 4)), dim3(256), 0, s, x, to, tokens, channels);
  return hipGetLastError();
}
template <int TYPE>
hipError_t dequantize(const qg_fp8_held& x, int tokens, int channels, const qg_fp8_rows& to, hipStream_t s) {
  const long long units = (long long)tokens * (x.scale_pitch / 4);
  hipLaunchKernelGGL(qg_fp8_dequantize_kernel<TYPE>, dim3((unsigned)((units + 3) / 4)), dim3(256), 0, s, x, to, tokens, channels);
  return hipGetLastError();
}

}  // namespace

hipError_t qg_launch_fp8_quantize(const qg_fp8_rows& x, int type, int tokens, int channels, const qg_fp8_held& to, hipStream_t s) {
  return type == QG_F32    ? quantize<QG_F32>(x, tokens, channels, to, s)
         : type == QG_BF16 ? quantize<QG_BF16>(x, tokens, channels, to, s)
                           : quantize<QG_F16>(x, tokens, channels, to, s);
}

hipError_t qg_launch_fp8_dequantize(const qg_fp8_held& x, int type, int tokens, int channels, const qg_fp8_rows& to, hipStream_t s) {
  return type == QG_F32    ? dequantize<QG_F32>(x, tokens, channels, to, s)
         : type == QG_BF16 ? dequantize<QG_BF16>(x, tokens, channels, to, s)
                           : dequantize<QG_F16>(x, tokens, channels, to, s);
}

hipError_t qg_launch_fp8_pack(const qg_fp8_pack_args& a, int type, hipStream_t s) {
  // column blocks: all that B's pieces have slots for; row blocks: all that the transpose's have
  const int columns = a.gated ? qg_fp8_up(a.n, 128) / 128 : qg_fp8_up(a.n, 256) / 128;
  const int rows = a.t_pieces ? qg_fp8_up(a.k, 256) / 128 : qg_fp8_up(a.k, 128) / 128;
  const dim3 grid((unsigned)columns, (unsigned)rows, a.gated ? 2u : 1u);
  if (type == QG_F32) hipLaunchKernelGGL(qg_fp8_pack_kernel<QG_F32>, grid, dim3(256), 0, s, a);
  if (type == QG_BF16) hipLaunchKernelGGL(qg_fp8_pack_kernel<QG_BF16>, grid, dim3(256), 0, s, a);
  if (type == QG_F16) hipLaunchKernelGGL(qg_fp8_pack_kernel<QG_F16>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}
