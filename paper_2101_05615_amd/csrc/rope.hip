// Rotary positions: the table of cosines and sines, and the rotation of a tensor of heads.
//
// A pair of channels (x1, x2) at position p turns by the angle p f: y1 = x1 cos - x2 sin, y2 = x2 cos + x1 sin.  The angles come
// from a table made once in 64 bits: p f in fp32 loses the angle's low bits from a few thousand positions on, and the table's row
// (4 bytes per channel) is shared by all heads of a token.
#include "qg_kv4.h"

namespace {

struct freqs {
  double f[128];
};

__global__ __launch_bounds__(256) void qg_rope_table_kernel(freqs w, int pairs, int max_pos, double magnitude, float* __restrict__ table) {
  const size_t total = (size_t)max_pos * pairs;
  for (size_t t = (size_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (size_t)gridDim.x * 256) {
    const size_t p = t / pairs;
    const int i = (int)(t - p * pairs);
    double s, c;
    sincos((double)p * w.f[i], &s, &c);
    table[p * 2 * pairs + i] = (float)(c * magnitude);
    table[p * 2 * pairs + pairs + i] = (float)(s * magnitude);
  }
}

// 16 channels a lane (two runs of eight, see qg_runs): head_dim and rot multiples of 16.  Bound by memory.  Heads of a token follow each
// other in a workgroup, so that rows are read and written in one piece and a row of the table once (8192 x 40 x 128 bf16 out of rows of
// 48, in a graph: 30 us, 5.7 TB/s; with the tokens of a head side by side 38); tokens are numbered in spans that keep the division short.
template <int TYPE>
__global__ void qg_rope_kernel(qg_rope_args p, int span) {
  typedef typename qg_elem<TYPE>::t t;
  const int lanes = p.head_dim / 16;  // of a head
  const int per = (int)blockDim.x / lanes, local = (int)threadIdx.x / lanes, lane = (int)threadIdx.x - local * lanes;
  const unsigned unit = blockIdx.x * per + local, in_span = unit / (unsigned)p.heads;
  const int head = (int)(unit - in_span * p.heads);
  const int64_t token = (int64_t)blockIdx.y * span + in_span;
  if (local >= per || in_span >= (unsigned)span || token >= p.tokens) return;
  const qg_runs r = qg_runs_of(lane, p.rot, p.interleaved);
  const t* x = static_cast<const t*>(p.x) + token * p.x_token + head * p.x_head;
  t* y = static_cast<t*>(p.y) + token * p.y_token + head * p.y_head;
  float a[8], b[8];
  qg_load<TYPE, 8>(x + r.a, a);
  qg_load<TYPE, 8>(x + r.b, b);
  const int pos = p.positions[token];
  qg_turn_runs(a, b, r, (unsigned)pos < (unsigned)p.max_pos ? p.table + (size_t)pos * p.rot : nullptr, p.rot, p.interleaved, p.sign);
  qg_store<TYPE, 8>(y + r.a, a);
  qg_store<TYPE, 8>(y + r.b, b);
}

// Any even extents: a thread takes one pair, or two of the channels that are only copied; a workgroup a head of some tokens.  Bound by
// its requests of one element and a division a pair: 8192 x 32 x 96 of which 24 turn 50 us in bf16, 2.0 TB/s, 68 in fp32 (all 96, by the
// kernel above: 18 and 35); x 80 of which 20 turn 43 and 63.
constexpr int ANY_TOKENS = 8;
template <int TYPE>
__global__ void qg_rope_any_kernel(qg_rope_args p) {
  typedef typename qg_elem<TYPE>::t t;
  const int half = p.rot / 2, pairs = half + (p.head_dim - p.rot + 1) / 2;
  for (long long at = (long long)blockIdx.y * ANY_TOKENS; at < p.tokens; at += (long long)gridDim.y * ANY_TOKENS)
  for (int i = (int)threadIdx.x; i < ANY_TOKENS * pairs; i += (int)blockDim.x) {
    const int local = i / pairs, k = i - local * pairs;
    const long long token = at + local;
    if (token >= p.tokens) break;
    const t* x = static_cast<const t*>(p.x) + token * p.x_token + blockIdx.x * p.x_head;
    t* y = static_cast<t*>(p.y) + token * p.y_token + blockIdx.x * p.y_head;
    if (k >= half) {
      const int c = p.rot + 2 * (k - half);
      y[c] = x[c];
      if (c + 1 < p.head_dim) y[c + 1] = x[c + 1];
      continue;
    }
    const int ca = p.interleaved ? 2 * k : k, cb = p.interleaved ? 2 * k + 1 : k + half;
    float a = qg_elem<TYPE>::up(x[ca]), b = qg_elem<TYPE>::up(x[cb]);
    const int pos = p.positions[token];
    const bool in = (unsigned)pos < (unsigned)p.max_pos;
    const float* row = p.table + (in ? (size_t)pos * p.rot : 0);
    const float cos = in ? row[k] : __builtin_nanf(""), sin = in ? row[half + k] : __builtin_nanf("");
    qg_turn(a, b, cos, p.sign * sin);
    y[ca] = qg_elem<TYPE>::down(a);
    y[cb] = qg_elem<TYPE>::down(b);
  }
}

}  // namespace

hipError_t qg_launch_rope_table(const double* f, int rot, int max_pos, double magnitude, float* table, hipStream_t s) {
  freqs w = {};
  for (int i = 0; i < rot / 2; ++i) w.f[i] = f[i];
  const long long blocks = ((long long)max_pos * (rot / 2) + 255) / 256;
  hipLaunchKernelGGL(qg_rope_table_kernel, dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(256), 0, s, w, rot / 2, max_pos,
                     magnitude, table);
  return hipGetLastError();
}

hipError_t qg_launch_rope(const qg_rope_args& a, int dtype, hipStream_t s) {
  const bool runs = a.head_dim % 16 == 0 && a.rot % 16 == 0;
  const int per_token = runs ? a.head_dim / 16 : a.head_dim / 2;
  // one wave a workgroup while that leaves CUs idle otherwise
  const int block = (long long)a.tokens * a.heads * per_token < 256 * 1024 ? 64 : 256;
  const int units = runs ? block / per_token : 1;  // heads of a token in a workgroup
  const long long most = (1ll << 22) / a.heads, span = a.tokens < most ? a.tokens : most;
  const long long spans = (a.tokens + span - 1) / span, blocks = ((long long)a.tokens + ANY_TOKENS - 1) / ANY_TOKENS;
  if (runs && spans > 65535) return hipErrorInvalidConfiguration;  // (65535 heads: 4 million tokens)
  const dim3 grid = runs ? dim3((unsigned)((span * a.heads + units - 1) / units), (unsigned)spans)
                         : dim3((unsigned)a.heads, (unsigned)(blocks < 65535 ? blocks : 65535));
#define QG_GO(T)                                                                  \
  if (runs)                                                                       \
    hipLaunchKernelGGL(qg_rope_kernel<T>, grid, dim3(block), 0, s, a, (int)span);           \
  else                                                                            \
    hipLaunchKernelGGL(qg_rope_any_kernel<T>, grid, dim3(block), 0, s, a)
  switch (dtype) {
    case QG_F32: QG_GO(QG_F32); break;
    case QG_BF16: QG_GO(QG_BF16); break;
    default: QG_GO(QG_F16);
  }
#undef QG_GO
  return hipGetLastError();
}
