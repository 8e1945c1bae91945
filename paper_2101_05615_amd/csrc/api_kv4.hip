// Host side of the positions, the 4-bit cache and its attention (qgemm.h): argument checks, the rotation's frequencies, and how a
// sequence's keys are split over workgroups.  As in the rest of the library nothing is allocated, created or waited for here.
#include <math.h>

#include "qg_kv4.h"

namespace {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

constexpr size_t ELEM[3] = {4, 2, 2};

bool known(int dtype) { return dtype == QG_F32 || dtype == QG_BF16 || dtype == QG_F16; }

int check_heads(const qg_heads& h, int dtype) {
  if (!h.data) return QG_ENULL;
  return aligned(h.data, ELEM[dtype]) ? QG_OK : QG_EALIGN;
}

// A launch's threads along one axis; the kernels over tokens number them so
bool too_many(long long tokens, long long heads, int head_dim) { return tokens * heads * (head_dim / 16) > 0x7fff0000ll; }

int lg_of_page(int page_tokens) {
  for (int l = 4; l <= 8; ++l)
    if (page_tokens == 1 << l) return l;
  return -1;
}

int check_cache(const qg_kv4_cache* c, qg_kv4_layout* out) {
  if (!c) return QG_ENULL;
  if (qg_kv4_bytes(c->n_pages, c->kv_heads, c->head_dim, c->page_tokens) == 0) return QG_EINVAL;
  if (!c->data) return QG_ENULL;
  if (!aligned(c->data, 64)) return QG_EALIGN;
  out->data = static_cast<uint8_t*>(c->data);
  out->n_pages = c->n_pages;
  out->heads = c->kv_heads;
  out->lgp = lg_of_page(c->page_tokens);
  return QG_OK;
}

// A table is needed wherever positions are
int check_rotation(const float* table, int max_pos, int rot, int interleaved, int head_dim) {
  if (!table) return QG_ENULL;
  if (max_pos < 1 || rot < 2 || rot % 2 != 0 || rot > head_dim || (interleaved != 0 && interleaved != 1)) return QG_EINVAL;
  return aligned(table, 16) ? QG_OK : QG_EALIGN;
}

// ---- keys over workgroups
// With few sequences a workgroup per (sequence, KV head, rows) leaves most of the 256 CUs idle, and with long ones that differ in
// length the longest ends alone.  A share is at least what a workgroup's start and end cost, and keys are not dealt at all up to
// twice that (777 keys of 8 KV heads: 9.0 us in four shares, 9.1 whole).
//   Few rows: shares of equal length, so many that every CU has a workgroup if all sequences are as long as the longest may be.  More
//   would cost more than it evens out: every share is written, and read by the last one to arrive (131072 keys of 8 KV heads, 8 rows:
//   34 us in 256 shares, 40 in 512, 49 in 1024), and so would shares by the lengths there are, as below (64 sequences of up to 8192
//   keys: 69.3 us for 69.0; 16 of up to 4096, 5 queries: 27.9 for 25.4).
//   Many rows: workgroups run for long, so the kernel deals the keys by the lengths that it finds, in one or two rounds of the
//   workgroups that run at once (three a CU with 64 channels, two with 128, one with 256).  512 queries of four sequences of 8192,
//   1981, 1766 and 1310 keys, 32 heads over 8 of 128 channels: 149 us (equal shares 164, whole 240); four of 4096 keys: 169, as whole
//   (two rounds 197); one of 8192, 8 heads over one: 58 (in as many shares as run at once 65).
constexpr int FEW_SHARES = 256;
constexpr size_t COUNTERS = QG_KV4_COUNTER_BYTES / 4;  // a fixed part of every workspace, so that calls of other extents find it zero
constexpr int LEAST_FEW = 256, LEAST_MANY = 512;       // tokens of a share; up to twice that keys are not split

struct share {
  int split, piece, shares, least;
  long long rows;  // of results in the workspace; 0: keys not split
};

int at_once_of(int head_dim) { return head_dim == 64 ? 768 : head_dim == 128 ? 512 : 256; }

// Workgroups that the kernel deals keys to at most, for so many (sequence, head, block of rows): what two rounds take and one more for
// each, and no more than shares of the least length make
long long dealt_most(long long units, int at_once, int max_kv_len) { return qg_kv4_dealt(units, at_once, max_kv_len, LEAST_MANY / 64); }

share share_of(const qg_kv4_cache* c, int q_heads, int batch, int max_q_len, int max_kv_len) {
  const long long rows = (long long)max_q_len * (q_heads / c->kv_heads), per = qg_kv4_rows_per_workgroup(c->head_dim, rows);
  const long long heads = (long long)batch * c->kv_heads, blocks = (rows + per - 1) / per;
  const long long most = heads * ((rows + 15) / 16);  // workgroups have 16 rows at least
  const bool few = rows <= QG_KV4_FEW;
  const int least = few ? LEAST_FEW : LEAST_MANY;
  share s = {1, 0x40000000, 0, 0, 0};
  if (max_kv_len <= 2 * least) return s;
  if (few) {
    const long long piece = ((long long)max_kv_len * heads * blocks / FEW_SHARES + 63) / 64 * 64;
    if (piece >= max_kv_len || most + 16 > (long long)COUNTERS) return s;
    s.piece = (int)(piece < least ? least : piece);
    s.split = (max_kv_len + s.piece - 1) / s.piece;
    s.rows = heads * blocks * s.split * per;
  } else {
    const int at_once = at_once_of(c->head_dim);
    // (more than two rounds even out by themselves; the kernel adds up workgroups, and the stages of all, in 32 bits)
    if (heads * blocks > 2 * at_once || most + 16 > (long long)COUNTERS || most * ((max_kv_len + 63) / 64) > 0x7fff0000ll) return s;
    s.shares = at_once;
    s.least = least / 64;
    s.rows = dealt_most(heads * blocks, at_once, max_kv_len) * per;  // (blocks of 64 rows: at most twice the heads * blocks, half the rows each)
  }
  return s;
}

// Rows of results that calls with at most these extents may want.  More sequences, queries or keys can mean fewer shares, so this
// is no call's own figure: few rows, `split` is at most FEW_SHARES / units + 1 and at most the keys' number of least pieces, and units
// number less than FEW_SHARES; many rows as in share_of.
long long most_rows_of(const qg_kv4_cache* c, int q_heads, int batch, int max_q_len, int max_kv_len) {
  const long long rows = (long long)max_q_len * (q_heads / c->kv_heads), heads = (long long)batch * c->kv_heads;
  long long most = 0;
  if (max_kv_len > 2 * LEAST_FEW) {
    const long long some = rows < QG_KV4_FEW ? rows : QG_KV4_FEW, per = qg_kv4_rows_per_workgroup(c->head_dim, some);
    long long units = heads * ((some + per - 1) / per);
    if (units >= FEW_SHARES) units = FEW_SHARES - 1;
    const long long pieces = units * ((max_kv_len + LEAST_FEW - 1) / LEAST_FEW);
    most = (pieces < FEW_SHARES + units ? pieces : FEW_SHARES + units) * per;
  }
  if (rows > QG_KV4_FEW && max_kv_len > 2 * LEAST_MANY) {
    const long long per = qg_kv4_rows_per_workgroup(c->head_dim, rows), at_once = at_once_of(c->head_dim);
    long long units = heads * ((rows + per - 1) / per);
    if (units > 2 * at_once) units = 2 * at_once;
    const long long here = dealt_most(units, (int)at_once, max_kv_len) * per;
    if (here > most) most = here;
  }
  return most;
}

size_t share_bytes(long long rows, int head_dim) { return rows == 0 ? 0 : COUNTERS * 4 + (size_t)rows * (head_dim + 2) * 4; }

bool extents_ok(const qg_kv4_cache* c, int q_heads, int batch, int max_q_len, int max_kv_len) {
  if (q_heads < 1 || q_heads % c->kv_heads != 0 || batch < 0 || max_q_len < 0 || max_kv_len < 0) return false;
  if (max_kv_len > 1 << 30) return false;
  return (long long)max_q_len * (q_heads / c->kv_heads) <= 1 << 28;
}

}  // namespace

extern "C" {

int qg_rope_table(const qg_rope_params* p, float* table_dev, void* stream) {
  if (!p || !table_dev) return QG_ENULL;
  if (p->rot < 2 || p->rot % 2 != 0 || p->rot > 256 || p->max_pos < 1) return QG_EINVAL;
  if (!(p->base > 1.0) || !isfinite(p->base) || !(p->magnitude > 0.0) || !isfinite(p->magnitude)) return QG_EINVAL;
  if (p->scaling < QG_ROPE_PLAIN || p->scaling > QG_ROPE_BY_TURNS) return QG_EINVAL;
  const bool scaled = p->scaling != QG_ROPE_PLAIN, by_band = p->scaling == QG_ROPE_BY_INDEX || p->scaling == QG_ROPE_BY_TURNS;
  if (scaled && (!(p->factor >= 1.0) || !isfinite(p->factor))) return QG_EINVAL;
  if (by_band && (!(p->low > 0.0) || !(p->high > p->low) || !isfinite(p->high) || !(p->context > 0.0) || !isfinite(p->context)))
    return QG_EINVAL;
  if (!aligned(table_dev, 16)) return QG_EALIGN;
  const double two_pi = 6.283185307179586476925286766559;
  // the (fractional) pair that makes `turns` turns in `context` positions: context * base^(-2 i / rot) = 2 pi turns
  auto pair_of = [&](double turns) { return p->rot * log(p->context / (two_pi * turns)) / (2.0 * log(p->base)); };
  const int pairs = p->rot / 2;
  double from = 0.0, to = 1.0;
  if (p->scaling == QG_ROPE_BY_INDEX) {  // (the far end may lie behind the last pair: then no pair is interpolated in full)
    from = floor(pair_of(p->high));
    to = ceil(pair_of(p->low));
    from = from < 0.0 ? 0.0 : from;
    to = to < 0.0 ? 0.0 : to > p->rot - 1 ? p->rot - 1 : to;
    if (to <= from) to = from + 0.001;
  }
  double f[128];
  for (int i = 0; i < pairs; ++i) {
    f[i] = pow(p->base, -2.0 * i / p->rot);
    double w = 0.0;
    if (p->scaling == QG_ROPE_LINEAR) w = 1.0;
    if (p->scaling == QG_ROPE_BY_INDEX) w = (i - from) / (to - from);
    if (p->scaling == QG_ROPE_BY_TURNS) w = (p->high - p->context * f[i] / two_pi) / (p->high - p->low);
    w = w < 0.0 ? 0.0 : w > 1.0 ? 1.0 : w;
    f[i] = f[i] * (1.0 - w) + (scaled ? f[i] / p->factor * w : 0.0);
  }
  return qg_launch_rope_table(f, p->rot, p->max_pos, p->magnitude, table_dev, static_cast<hipStream_t>(stream)) == hipSuccess
             ? QG_OK
             : QG_ELAUNCH;
}

int qg_rope(const qg_heads* x, int dtype, int tokens, int heads, int head_dim, const int32_t* positions, const float* table_dev,
            int max_pos, int rot, int interleaved, int inverse, const qg_heads* y, void* stream) {
  if (!x || !y) return QG_ENULL;
  if (!known(dtype) || tokens < 0 || heads < 1 || heads > 65535 || head_dim < 2 || head_dim > 1024) return QG_EINVAL;
  if (inverse != 0 && inverse != 1) return QG_EINVAL;
  int rc = check_rotation(table_dev, max_pos, rot, interleaved, head_dim);
  if (rc != QG_OK) return rc;
  if (tokens == 0) return QG_OK;
  if (!positions) return QG_ENULL;
  if ((rc = check_heads(*x, dtype)) != QG_OK || (rc = check_heads(*y, dtype)) != QG_OK) return rc;
  if (!aligned(positions, 4)) return QG_EALIGN;
  if (x->data == y->data && (x->token_stride != y->token_stride || x->head_stride != y->head_stride)) return QG_EINVAL;
  qg_rope_args a = {};
  a.x = x->data;
  a.y = y->data;
  a.positions = positions;
  a.table = table_dev;
  a.tokens = tokens;
  a.heads = heads;
  a.head_dim = head_dim;
  a.rot = rot;
  a.max_pos = max_pos;
  a.interleaved = interleaved;
  a.sign = inverse ? -1.0f : 1.0f;
  a.x_token = x->token_stride;
  a.x_head = x->head_stride;
  a.y_token = y->token_stride;
  a.y_head = y->head_stride;
  return qg_launch_rope(a, dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? QG_OK : QG_ELAUNCH;
}

size_t qg_kv4_bytes(int n_pages, int kv_heads, int head_dim, int page_tokens) {
  if (n_pages < 1 || kv_heads < 1 || kv_heads > 32767 || lg_of_page(page_tokens) < 0) return 0;
  if (head_dim != 64 && head_dim != 128 && head_dim != 256) return 0;
  return (size_t)n_pages * kv_heads * page_tokens * (head_dim + 8);
}

int qg_kv4_append(const qg_kv4_cache* c, const qg_kv4_append_params* p, void* stream) {
  if (!p) return QG_ENULL;
  qg_kv4_append_args a = {};
  int rc = check_cache(c, &a.c);
  if (rc != QG_OK) return rc;
  if (!known(p->dtype) || p->tokens < 0 || p->q_heads < 0 || p->q_heads + 2 * c->kv_heads > 65535) return QG_EINVAL;
  if (p->tokens > QG_KV4_MAX_TOKENS) return QG_EINVAL;
  if (p->positions) {
    if ((rc = check_rotation(p->table, p->max_pos, p->rot, p->interleaved, c->head_dim)) != QG_OK) return rc;
    if (p->rot % 16 != 0) return QG_EUNSUPPORTED;
    if (!aligned(p->positions, 4)) return QG_EALIGN;
  }
  if (too_many(p->tokens, 2 * c->kv_heads + p->q_heads, c->head_dim)) return QG_EUNSUPPORTED;
  if (p->tokens == 0) return QG_OK;
  if (!p->slots) return QG_ENULL;
  if (!aligned(p->slots, 8)) return QG_EALIGN;
  if ((rc = check_heads(p->k, p->dtype)) != QG_OK || (rc = check_heads(p->v, p->dtype)) != QG_OK) return rc;
  if (p->q_heads > 0) {
    if ((rc = check_heads(p->q, p->dtype)) != QG_OK || (rc = check_heads(p->q_out, p->dtype)) != QG_OK) return rc;
    if (p->q.data == p->q_out.data && (p->q.token_stride != p->q_out.token_stride || p->q.head_stride != p->q_out.head_stride))
      return QG_EINVAL;
  }
  a.k = p->k.data;
  a.v = p->v.data;
  a.q = p->q.data;
  a.q_out = p->q_out.data;
  a.slots = p->slots;
  a.positions = p->positions;
  a.table = p->table;
  a.tokens = p->tokens;
  a.q_heads = p->q_heads;
  a.rot = p->rot;
  a.max_pos = p->max_pos;
  a.interleaved = p->interleaved;
  a.k_token = p->k.token_stride;
  a.k_head = p->k.head_stride;
  a.v_token = p->v.token_stride;
  a.v_head = p->v.head_stride;
  a.q_token = p->q.token_stride;
  a.q_head = p->q.head_stride;
  a.o_token = p->q_out.token_stride;
  a.o_head = p->q_out.head_stride;
  return qg_launch_kv4_append(a, c->head_dim, p->dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? QG_OK : QG_ELAUNCH;
}

int qg_kv4_read(const qg_kv4_cache* c, const int64_t* slots, int tokens, int dtype, const qg_heads* k, const qg_heads* v,
                void* stream) {
  if (!k || !v) return QG_ENULL;
  qg_kv4_read_args a = {};
  int rc = check_cache(c, &a.c);
  if (rc != QG_OK) return rc;
  if (!known(dtype) || tokens < 0 || tokens > QG_KV4_MAX_TOKENS) return QG_EINVAL;
  if (too_many(tokens, 2 * c->kv_heads, c->head_dim)) return QG_EUNSUPPORTED;
  if (tokens == 0) return QG_OK;
  if (!slots) return QG_ENULL;
  if (!aligned(slots, 8)) return QG_EALIGN;
  if (k->data && (rc = check_heads(*k, dtype)) != QG_OK) return rc;
  if (v->data && (rc = check_heads(*v, dtype)) != QG_OK) return rc;
  a.k = k->data;
  a.v = v->data;
  a.slots = slots;
  a.tokens = tokens;
  a.k_token = k->token_stride;
  a.k_head = k->head_stride;
  a.v_token = v->token_stride;
  a.v_head = v->head_stride;
  return qg_launch_kv4_read(a, c->head_dim, dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? QG_OK : QG_ELAUNCH;
}

size_t qg_kv4_attention_workspace_bytes(const qg_kv4_cache* c, int q_heads, int batch, int max_q_len, int max_kv_len) {
  if (!c || qg_kv4_bytes(c->n_pages, c->kv_heads, c->head_dim, c->page_tokens) == 0) return 0;
  if (!extents_ok(c, q_heads, batch, max_q_len, max_kv_len) || batch == 0 || max_q_len == 0 || max_kv_len == 0) return 0;
  return share_bytes(most_rows_of(c, q_heads, batch, max_q_len, max_kv_len), c->head_dim);
}

int qg_kv4_attention(const qg_kv4_cache* c, const qg_kv4_attention_params* p, void* stream) {
  if (!p) return QG_ENULL;
  qg_kv4_attention_args a = {};
  int rc = check_cache(c, &a.c);
  if (rc != QG_OK) return rc;
  if (!known(p->dtype) || p->tokens < 0 || !extents_ok(c, p->q_heads, p->batch, p->max_q_len, p->max_kv_len)) return QG_EINVAL;
  if (!isfinite(p->scale) || (p->causal != 0 && p->causal != 1) || p->pages_stride < 0) return QG_EINVAL;
  if (p->max_kv_len > (long long)p->pages_stride * c->page_tokens) return QG_EINVAL;
  if (!p->q_starts && p->batch != p->tokens) return QG_EINVAL;
  if (p->tokens == 0 || p->batch == 0 || p->max_q_len == 0) return QG_OK;
  if (!p->kv_lens || (!p->pages && p->max_kv_len > 0)) return QG_ENULL;
  if (!aligned(p->kv_lens, 4) || !aligned(p->pages, 4) || !aligned(p->q_starts, 4)) return QG_EALIGN;
  if ((rc = check_heads(p->q, p->dtype)) != QG_OK || (rc = check_heads(p->out, p->dtype)) != QG_OK) return rc;
  const int max_q = p->q_starts ? p->max_q_len : 1;
  share s = share_of(c, p->q_heads, p->batch, max_q, p->max_kv_len);
  if (!p->workspace) s = {1, 0x40000000, 0, 0, 0};
  if (s.rows > 0) {
    if (p->workspace_bytes < share_bytes(s.rows, c->head_dim)) return QG_EWORKSPACE;
    if (!aligned(p->workspace, 16)) return QG_EALIGN;
  }
  const long long rows = (long long)max_q * (p->q_heads / c->kv_heads);
  if ((long long)p->batch * c->kv_heads * s.split * ((rows + 15) / 16) > 0x7fffffffll / 512) return QG_EUNSUPPORTED;
  a.q = p->q.data;
  a.out = p->out.data;
  a.pages = p->pages;
  a.kv_lens = p->kv_lens;
  a.q_starts = p->q_starts;
  a.tokens = p->tokens;
  a.group = p->q_heads / c->kv_heads;
  a.batch = p->batch;
  a.pages_stride = p->pages_stride;
  a.max_q_len = max_q;
  a.max_kv_len = p->max_kv_len;
  a.causal = p->causal;
  const double to_log2 = (double)p->scale * 1.4426950408889634074;
  a.scale_log2e = (float)to_log2;
  a.scale_log2e_lo = (float)(to_log2 - (double)a.scale_log2e);
  a.split = s.split;
  a.piece = s.piece;
  a.shares = s.shares;
  a.least = s.least;
  if (s.rows > 0) {
    a.counters = static_cast<int*>(p->workspace);
    a.partial = reinterpret_cast<float*>(a.counters + COUNTERS);
    a.sums = a.partial + (size_t)s.rows * c->head_dim;
  }
  a.q_token = p->q.token_stride;
  a.q_head = p->q.head_stride;
  a.o_token = p->out.token_stride;
  a.o_head = p->out.head_stride;
  const auto launch = rows <= QG_KV4_FEW ? qg_launch_kv4_attention_few : qg_launch_kv4_attention_many;
  return launch(a, c->head_dim, p->dtype, (int)rows, static_cast<hipStream_t>(stream)) == hipSuccess ? QG_OK : QG_ELAUNCH;
}

}  // extern "C"
