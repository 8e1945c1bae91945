// The 4-bit key/value cache: layout of a page, element types and rotation, shared by the kernels that write, read and attend to it.
// Not part of the public interface.
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "qgemm.h"

// ---------------------------------------------------------------------------
// A page holds, for each KV head, a block of P tokens (P = 16 .. 256, head dimension D):
//   key codes    [P][D/2] bytes                        what a lane of the matrix cores' first operand wants: a token's channels in a row
//   value codes  [P/8][D/4][8 tokens] 16-bit words     the second product sums over tokens, so its operand wants 8 tokens of one
//                                                      channel in a lane: a word is four channels of a token, and a dword four
//                                                      channels of two neighbouring tokens, which unpack into pairs of fp16
//   words        [P/8][key, value][8] 32-bit           bits(alpha) | theta: the 16 words of 8 tokens are the 16 lanes of a DPP row
// ---------------------------------------------------------------------------
struct qg_kv4_layout {
  uint8_t* data;
  int n_pages, heads, lgp;  // lgp = log2(P)
};

template <int D>
static __device__ inline size_t qg_kv4_block(const qg_kv4_layout& c, int page, int head) {
  return ((size_t)page * c.heads + head) * ((size_t)(D + 8) << c.lgp);
}

// ---- element types: fp32 in registers, rounded to the type once (nearest even)
template <int TYPE>
struct qg_elem;
template <>
struct qg_elem<QG_F32> {
  typedef float t;
  static __device__ inline float up(float x) { return x; }
  static __device__ inline float down(float x) { return x; }
};
template <>
struct qg_elem<QG_BF16> {
  typedef __bf16 t;
  static __device__ inline float up(__bf16 x) { return (float)x; }
  static __device__ inline __bf16 down(float x) { return (__bf16)x; }
};
template <>
struct qg_elem<QG_F16> {
  typedef _Float16 t;
  static __device__ inline float up(_Float16 x) { return (float)x; }
  static __device__ inline _Float16 down(float x) { return (_Float16)x; }
};

// N consecutive elements at any address that the element type allows: the hardware takes wide requests at any of them
template <int TYPE, int N>
static __device__ inline void qg_load(const typename qg_elem<TYPE>::t* p, float* out) {
  typedef typename qg_elem<TYPE>::t t;
  constexpr int W = 16 / sizeof(t) < N ? 16 / sizeof(t) : N;
  typedef t vec __attribute__((ext_vector_type(W)));
  typedef vec vec_any __attribute__((aligned(sizeof(t))));
#pragma unroll
  for (int i = 0; i < N; i += W) {
    const vec v = *reinterpret_cast<const vec_any*>(p + i);
#pragma unroll
    for (int j = 0; j < W; ++j) out[i + j] = qg_elem<TYPE>::up(v[j]);
  }
}
template <int TYPE, int N>
static __device__ inline void qg_store(typename qg_elem<TYPE>::t* p, const float* in) {
  typedef typename qg_elem<TYPE>::t t;
  constexpr int W = 16 / sizeof(t) < N ? 16 / sizeof(t) : N;
  typedef t vec __attribute__((ext_vector_type(W)));
  typedef vec vec_any __attribute__((aligned(sizeof(t))));
#pragma unroll
  for (int i = 0; i < N; i += W) {
    vec v;
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = qg_elem<TYPE>::down(in[i + j]);
    *reinterpret_cast<vec_any*>(p + i) = v;
  }
}

// One pair turned: two products and a sum each, every one rounded to fp32 (the library is built without contraction)
static __device__ inline void qg_turn(float& a, float& b, float cos, float sin) {
  const float y = a * cos - b * sin;
  b = b * cos + a * sin;
  a = y;
}

// Which channels a lane of a head takes: two runs of eight, `a` and `b`.  Neighbouring pairs lie inside a run; pairs half the
// rotated part apart lie at the same place of the two runs, so that a lane has all it turns (and may write where it read).
struct qg_runs {
  int a, b;       // first channels
  int cos;        // first pair whose angle is needed (half apart: of 8; neighbours: of 4 in a, 4 in b); -1: not rotated
  int cos_b;      // neighbours: the same for b
};
static __device__ inline qg_runs qg_runs_of(int lane, int rot, int interleaved) {
  qg_runs r;
  if (interleaved) {
    r.a = 16 * lane;
    r.b = r.a + 8;
    r.cos = r.a < rot ? r.a / 2 : -1;
    r.cos_b = r.b < rot ? r.b / 2 : -1;
  } else if (lane < rot / 16) {
    r.a = 8 * lane;
    r.b = r.a + rot / 2;
    r.cos = r.cos_b = r.a;
  } else {
    r.a = rot + 16 * (lane - rot / 16);
    r.b = r.a + 8;
    r.cos = r.cos_b = -1;
  }
  return r;
}

// Turns the 16 channels of a lane; row: the position's row of the table, NULL for a position outside it (NaN)
static __device__ inline void qg_turn_runs(float* a, float* b, const qg_runs& r, const float* row, int rot, int interleaved,
                                           float sign) {
  if (r.cos < 0 && r.cos_b < 0) return;
  float c[8], s[8];
  if (row == nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = s[i] = __builtin_nanf("");
  } else if (interleaved) {
    qg_load<QG_F32, 4>(row + r.cos, c);
    qg_load<QG_F32, 4>(row + rot / 2 + r.cos, s);
    qg_load<QG_F32, 4>(row + r.cos_b, c + 4);   // (rot is a multiple of 16: both runs are rotated or none)
    qg_load<QG_F32, 4>(row + rot / 2 + r.cos_b, s + 4);
  } else {
    qg_load<QG_F32, 8>(row + r.cos, c);
    qg_load<QG_F32, 8>(row + rot / 2 + r.cos, s);
  }
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      qg_turn(a[2 * i], a[2 * i + 1], c[i], sign * s[i]);
      qg_turn(b[2 * i], b[2 * i + 1], c[4 + i], sign * s[4 + i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) qg_turn(a[i], b[i], c[i], sign * s[i]);
  }
}

// Arguments of the kernels (by value)
struct qg_rope_args {
  const void* x;
  void* y;
  const int32_t* positions;
  const float* table;
  int tokens, heads, head_dim, rot, max_pos, interleaved;
  float sign;
  int64_t x_token, x_head, y_token, y_head;
};
struct qg_kv4_append_args {
  const void *k, *v, *q;
  void* q_out;
  const int64_t* slots;
  const int32_t* positions;  // null: no rotation
  const float* table;
  qg_kv4_layout c;
  int tokens, q_heads, rot, max_pos, interleaved;
  int64_t k_token, k_head, v_token, v_head, q_token, q_head, o_token, o_head;
};
struct qg_kv4_read_args {
  void *k, *v;               // null: not wanted
  const int64_t* slots;
  qg_kv4_layout c;
  int tokens;
  int64_t k_token, k_head, v_token, v_head;
};
struct qg_kv4_attention_args {
  const void* q;
  void* out;
  const int32_t* pages;
  const int32_t* kv_lens;
  const int32_t* q_starts;   // null: one query per sequence
  qg_kv4_layout c;
  int tokens, group, batch, pages_stride, max_q_len, max_kv_len, causal;
  float scale_log2e, scale_log2e_lo;  // two parts
  int split, piece;          // workgroups that share a sequence's keys, and tokens each takes (a multiple of 64); or, many rows:
  int shares, least;         // workgroups that run at once, to whom the kernel deals the keys (0: split 1), and stages of 64 tokens each has at least
  int row_blocks;            // workgroups over a KV head's query rows
  int* counters;             // one a workgroup, zero before and after
  float *partial, *sums;     // [workgroup][rows of a workgroup][D]; reference and sum of each row
  int64_t q_token, q_head, o_token, o_head;
};

hipError_t qg_launch_rope_table(const double* freqs, int rot, int max_pos, double magnitude, float* table, hipStream_t s);
hipError_t qg_launch_rope(const qg_rope_args& a, int dtype, hipStream_t s);
hipError_t qg_launch_kv4_append(const qg_kv4_append_args& a, int head_dim, int dtype, hipStream_t s);
hipError_t qg_launch_kv4_read(const qg_kv4_read_args& a, int head_dim, int dtype, hipStream_t s);
// Query rows of a KV head (its query heads times a sequence's queries): up to QG_KV4_FEW a wave has all of them; beyond, the waves
// of a workgroup share unpacked keys and values.
#define QG_KV4_FEW 32
static inline int qg_kv4_rows_per_workgroup(int head_dim, long long rows) {
  if (rows <= QG_KV4_FEW) return head_dim == 256 || rows <= 16 ? 16 : 32;
  return 128;  // (fp32 with 128 channels and less: 64; the split of the keys is the same for all types)
}
// Workgroups of a dealt launch at most: `units` (sequence, head, block of rows), of which each has one share more than it fills, in two
// rounds of `at_once`; shares have `least` stages of 64 tokens
static inline long long qg_kv4_dealt(long long units, int at_once, int max_kv_len, int least) {
  const long long rounds = 2ll * at_once + units, pieces = units * (((max_kv_len + 63) / 64 + least - 1) / least);
  return rounds < pieces ? rounds : pieces;
}
hipError_t qg_launch_kv4_attention_few(const qg_kv4_attention_args& a, int head_dim, int dtype, int rows, hipStream_t s);
hipError_t qg_launch_kv4_attention_many(const qg_kv4_attention_args& a, int head_dim, int dtype, int rows, hipStream_t s);
