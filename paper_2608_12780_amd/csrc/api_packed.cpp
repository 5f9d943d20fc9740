// C ABI of rotary positions and of attention over packed sequences: argument
// validation before any HIP call, then the launches.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <initializer_list>

#include "../../include/scope.h"
#include "kernels.h"

namespace {

constexpr int kMaxRows = 1 << 24;
constexpr int64_t kMaxStride = 1LL << 40;  // elements: products with heads stay in 64 bits
constexpr int64_t kMaxRun = 1LL << 60;     // elements from the first row to the last

// Elements from a tensor's first to past its last, or -1 where the strides are not
// usable.  out: its rows must not overlap one another.
int64_t extent(const scope_strides *t, int64_t heads, int64_t rows, int64_t d, bool out) {
  if (t->row < 0 || t->head < 0 || t->row > kMaxStride || t->head > kMaxStride) return -1;
  if (heads < 1 || rows < 1) return 0;
  if (rows > 1 && t->row > kMaxRun / (rows - 1)) return -1;
  if (out) {
    if ((rows > 1 && t->row < d) || (heads > 1 && t->head < d)) return -1;
    const int64_t by_rows = (rows - 1) * t->row + d, by_heads = (heads - 1) * t->head + d;
    if (rows > 1 && heads > 1 && t->head < by_rows && t->row < by_heads) return -1;
  }
  return (rows - 1) * t->row + (heads - 1) * t->head + d;
}

scope_strides dense_or(const scope_strides *t, int64_t rows, int64_t d) {
  return t ? *t : scope_strides{d, rows * d};
}

bool overlap(const void *a, int64_t a_bytes, const void *b, int64_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + b_bytes && y < x + a_bytes;
}

struct Tensor {
  const void *p;
  const scope_strides *strides;
  int heads, rows;
  bool out;
};

// A tensor of the packed calls: its strides in bytes.  The rows of a tile, up to 66 of one
// key head or of the heads that share it, are addressed with 32-bit byte offsets.
int32_t check_rows(const Tensor &t, int d, int el, int shared, scope::PackRows *rows) {
  const scope_strides s = dense_or(t.strides, t.rows, d);
  const int64_t all = extent(&s, t.heads, t.rows, d, t.out);
  if (all < 0) return SCOPE_ERR_INVALID_ARGUMENT;
  if (!t.p && t.rows) return SCOPE_ERR_INVALID_ARGUMENT;
  // rows are read and written as 16-byte vectors
  if (reinterpret_cast<uintptr_t>(t.p) % 16 || s.row * el % 16 || s.head * el % 16) return SCOPE_ERR_INVALID_ARGUMENT;
  const int64_t near = t.rows < 66 ? t.rows : 66;
  if (t.rows && ((near - 1) * s.row + (shared - 1) * s.head + d) * el >= (1LL << 32)) return SCOPE_ERR_UNSUPPORTED;
  rows->base = static_cast<char *>(const_cast<void *>(t.p));
  rows->row = s.row * el;
  rows->head = s.head * el;
  return SCOPE_OK;
}

int32_t check_pack(const scope_pack *p) {
  if (!p || p->heads < 1 || p->kv_heads < 1 || p->heads % p->kv_heads || p->rows_q < 0 || p->rows_k < 0 || p->sequences < 1)
    return SCOPE_ERR_INVALID_ARGUMENT;
  if (p->dtype != SCOPE_F32 && p->dtype != SCOPE_BF16) return SCOPE_ERR_UNSUPPORTED;
  if (p->d != 64 && p->d != 128) return SCOPE_ERR_UNSUPPORTED;
  if (p->heads > 65535 || p->rows_q > kMaxRows || p->rows_k > kMaxRows || p->sequences > 65536) return SCOPE_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(p->heads) * p->rows_q >= (1LL << 31) || static_cast<int64_t>(p->kv_heads) * p->rows_k >= (1LL << 31))
    return SCOPE_ERR_UNSUPPORTED;
  // costs of 32 bits, and as many bytes of a key head's row statistics
  if (static_cast<int64_t>(p->heads / p->kv_heads) * p->rows_q >= (1LL << 30)) return SCOPE_ERR_UNSUPPORTED;
  if (!scope::packed_launchable(p)) return SCOPE_ERR_UNSUPPORTED;
  return SCOPE_OK;
}

int32_t check_int32(std::initializer_list<const void *> needed, std::initializer_list<const void *> optional) {
  for (const void *p : needed)
    if (!p || reinterpret_cast<uintptr_t>(p) % 4) return SCOPE_ERR_INVALID_ARGUMENT;
  for (const void *p : optional)
    if (reinterpret_cast<uintptr_t>(p) % 4) return SCOPE_ERR_INVALID_ARGUMENT;
  return SCOPE_OK;
}

// Outputs that are the same memory as an input or another output: refused where both
// are one block of memory (rows of one projection may interleave those of another).
int32_t check_apart(const Tensor *t, int count, int d, int el) {
  auto whole = [&](const Tensor &x, int64_t *bytes) {
    const scope_strides s = dense_or(x.strides, x.rows, d);
    *bytes = extent(&s, x.heads, x.rows, d, false) * el;
    return *bytes == static_cast<int64_t>(x.heads) * x.rows * d * el;
  };
  for (int i = 0; i < count; ++i) {
    if (!t[i].out || !t[i].rows) continue;
    for (int j = 0; j < count; ++j) {
      if (i == j || !t[j].rows) continue;
      int64_t a, b;
      const bool dense = whole(t[i], &a) && whole(t[j], &b);
      if (t[i].p == t[j].p || (dense && overlap(t[i].p, a, t[j].p, b))) return SCOPE_ERR_INVALID_ARGUMENT;
    }
  }
  return SCOPE_OK;
}

void set_pack(const scope_pack *p, const int32_t *offsets_q, const int32_t *offsets_k, const int32_t *lengths_k, float scale,
              void *workspace, int32_t *status, scope::PackArgs *a, scope::PackCall *c) {
  a->kv_heads = p->kv_heads;
  a->group = p->heads / p->kv_heads;
  a->rows_q = p->rows_q;
  a->rows_k = p->rows_k;
  a->sequences = p->sequences;
  a->causal = p->causal != 0;
  a->clear = p->clear != 0;
  a->offsets_q = offsets_q;
  a->offsets_k = offsets_k;
  a->lengths_k = lengths_k;
  a->scale = scale > 0.0f ? scale : static_cast<float>(1.0 / sqrt(static_cast<double>(p->d)));
  a->scale_log2 = a->scale * 1.4426950408889634f;
  c->d = p->d;
  c->bf16 = p->dtype == SCOPE_BF16;
  a->status = status;
  scope::packed_workspace(p, workspace, a, c);
}

int32_t check_workspace(const scope_pack *p, void *ws, size_t bytes) {
  if (!ws || bytes < scope::packed_workspace(p, nullptr, nullptr, nullptr) || reinterpret_cast<uintptr_t>(ws) % 256)
    return SCOPE_ERR_WORKSPACE;
  return SCOPE_OK;
}

}  // namespace

extern "C" {

int32_t scope_rotary(const scope_rotation *r, const int32_t *positions, const uint64_t *turns, const void *x,
                     const scope_strides *x_strides, void *y, const scope_strides *y_strides, const void *x2,
                     const scope_strides *x2_strides, void *y2, const scope_strides *y2_strides, void *stream) {
  if (!r || r->rows < 0 || r->heads[0] < 1 || r->heads[1] < 0 || r->d < 2 || r->d % 2) return SCOPE_ERR_INVALID_ARGUMENT;
  if (r->dtype != SCOPE_F32 && r->dtype != SCOPE_BF16) return SCOPE_ERR_UNSUPPORTED;
  if (r->d > 1024 || static_cast<int64_t>(r->heads[0]) + r->heads[1] > 65535) return SCOPE_ERR_UNSUPPORTED;
  if (r->axes < 1 || r->axes > 3 || (r->layout != SCOPE_PAIRS && r->layout != SCOPE_HALVES)) return SCOPE_ERR_INVALID_ARGUMENT;
  if (!(r->factor - r->factor == 0.0f)) return SCOPE_ERR_INVALID_ARGUMENT;
  scope::RotaryArgs a{};
  a.rows = r->rows;
  a.axes = r->axes;
  a.inverse = r->inverse != 0;
  a.factor = r->factor;
  a.positions = positions;
  a.turns = turns;
  const bool pairs = r->layout == SCOPE_PAIRS;
  const int el = r->dtype == SCOPE_BF16 ? 2 : 4;
  const int w = 16 / el;  // elements of a vector
  bool vectors = r->d % w == 0;
  for (int i = 0; i < r->axes; ++i) {
    const int o = r->range_off[i], n = r->range_len[i];
    if (o < 0 || n < 2 || n % 2 || n > r->d || o > r->d - n || (pairs && o % 2)) return SCOPE_ERR_INVALID_ARGUMENT;
    int at = i;
    for (int j = 0; j < i; ++j) {
      if (o < r->range_off[j] + r->range_len[j] && r->range_off[j] < o + n) return SCOPE_ERR_INVALID_ARGUMENT;
      if (o < r->range_off[j]) --at;
    }
    for (int j = i; j > at; --j) a.by_off[j] = a.by_off[j - 1];
    a.by_off[at] = i;
    a.off[i] = o;
    a.len[i] = n;
    if (!pairs) vectors = vectors && o % w == 0 && n % (2 * w) == 0;
  }
  if ((r->rows && !positions) || !turns || reinterpret_cast<uintptr_t>(positions) % 4 || reinterpret_cast<uintptr_t>(turns) % 8)
    return SCOPE_ERR_INVALID_ARGUMENT;
  const void *xs[2] = {x, x2};
  void *ys[2] = {y, y2};
  const scope_strides *sx[2] = {x_strides, x2_strides}, *sy[2] = {y_strides, y2_strides};
  int64_t x_bytes[2] = {0, 0}, y_bytes[2] = {0, 0};  // of tensors that are one block of memory
  for (int i = 0; i < 2; ++i) {
    const int heads = a.heads[i] = r->heads[i];
    if (!heads) continue;
    if (r->rows && (!xs[i] || !ys[i])) return SCOPE_ERR_INVALID_ARGUMENT;
    a.xs[i] = dense_or(sx[i], r->rows, r->d);
    a.ys[i] = dense_or(sy[i], r->rows, r->d);
    const int64_t ex = extent(&a.xs[i], heads, r->rows, r->d, false), ey = extent(&a.ys[i], heads, r->rows, r->d, true);
    if (ex < 0 || ey < 0) return SCOPE_ERR_INVALID_ARGUMENT;
    for (const void *p : {xs[i], static_cast<const void *>(ys[i])}) {
      if (reinterpret_cast<uintptr_t>(p) % el) return SCOPE_ERR_INVALID_ARGUMENT;
      vectors = vectors && reinterpret_cast<uintptr_t>(p) % 16 == 0;
    }
    for (int64_t s : {a.xs[i].row, a.xs[i].head, a.ys[i].row, a.ys[i].head}) vectors = vectors && s * el % 16 == 0;
    a.x[i] = xs[i];
    a.y[i] = ys[i];
    // in place with other strides, or over a part of itself
    const int64_t whole = static_cast<int64_t>(heads) * r->rows * r->d;
    if (r->rows && xs[i] == ys[i] && (a.xs[i].row != a.ys[i].row || a.xs[i].head != a.ys[i].head) && whole > r->d)
      return SCOPE_ERR_INVALID_ARGUMENT;
    x_bytes[i] = ex == whole ? ex * el : 0;
    y_bytes[i] = ey == whole ? ey * el : 0;
  }
  // the same memory, or blocks of it that overlap (rows of one projection may interleave)
  auto meet = [](const void *p, int64_t p_bytes, const void *q, int64_t q_bytes) {
    return p == q || (p_bytes && q_bytes && overlap(p, p_bytes, q, q_bytes));
  };
  for (int i = 0; i < 2 && r->rows; ++i) {
    if (!a.heads[i]) continue;
    if (xs[i] != ys[i] && meet(xs[i], x_bytes[i], ys[i], y_bytes[i])) return SCOPE_ERR_INVALID_ARGUMENT;
    // a thread stores heads of one tensor before it, or another, has loaded the other's
    if (a.heads[1 - i] && meet(ys[i], y_bytes[i], xs[1 - i], x_bytes[1 - i])) return SCOPE_ERR_INVALID_ARGUMENT;
  }
  if (r->rows && r->heads[1] && meet(y, y_bytes[0], y2, y_bytes[1])) return SCOPE_ERR_INVALID_ARGUMENT;
  if (static_cast<int64_t>(r->rows) * r->d >= (1LL << 32) - 256) return SCOPE_ERR_UNSUPPORTED;  // threads of a launch
  if (!r->rows) return SCOPE_OK;
  return scope::rotary_run(a, r->dtype == SCOPE_BF16, pairs, vectors, r->d, static_cast<hipStream_t>(stream)) == hipSuccess
             ? SCOPE_OK
             : SCOPE_ERR_HIP;
}

int32_t scope_packed_workspace_size(const scope_pack *pack, size_t *bytes) {
  const int32_t st = check_pack(pack);
  if (st) return st;
  if (!bytes) return SCOPE_ERR_INVALID_ARGUMENT;
  *bytes = scope::packed_workspace(pack, nullptr, nullptr, nullptr);
  return SCOPE_OK;
}

int32_t scope_packed_attention(const scope_pack *pack, const void *q, const scope_strides *q_strides, const void *k,
                               const scope_strides *k_strides, const void *v, const scope_strides *v_strides,
                               const int32_t *offsets_q, const int32_t *offsets_k, const int32_t *lengths_k, float scale, void *o,
                               const scope_strides *o_strides, float *lse, void *workspace, size_t ws_bytes, int32_t *dev_status,
                               void *stream) {
  int32_t st = check_pack(pack);
  if (st) return st;
  scope::PackArgs a{};
  scope::PackCall c{};
  const int el = pack->dtype == SCOPE_BF16 ? 2 : 4, group = pack->heads / pack->kv_heads;
  const Tensor t[] = {{q, q_strides, pack->heads, pack->rows_q, false},
                      {k, k_strides, pack->kv_heads, pack->rows_k, false},
                      {v, v_strides, pack->kv_heads, pack->rows_k, false},
                      {o, o_strides, pack->heads, pack->rows_q, true}};
  scope::PackRows *const rows[] = {&a.q, &a.k, &a.v, &c.o};
  for (int i = 0; i < 4; ++i)
    if ((st = check_rows(t[i], pack->d, el, t[i].heads == pack->heads && (i == 0 || i == 3) ? group : 1, rows[i]))) return st;
  if ((st = check_apart(t, 4, pack->d, el))) return st;
  if ((st = check_int32({offsets_q, offsets_k}, {lengths_k, dev_status, lse}))) return st;
  if (!lse && pack->rows_q) return SCOPE_ERR_INVALID_ARGUMENT;
  if (!(scale == scale) || isinf(scale)) return SCOPE_ERR_INVALID_ARGUMENT;
  if ((st = check_workspace(pack, workspace, ws_bytes))) return st;
  set_pack(pack, offsets_q, offsets_k, lengths_k, scale, workspace, dev_status, &a, &c);
  a.lse = lse;
  return scope::packed_forward(a, c, static_cast<hipStream_t>(stream)) == hipSuccess ? SCOPE_OK : SCOPE_ERR_HIP;
}

int32_t scope_packed_attention_backward(const scope_pack *pack, const void *q, const scope_strides *q_strides, const void *k,
                                        const scope_strides *k_strides, const void *v, const scope_strides *v_strides, const void *o,
                                        const scope_strides *o_strides, const float *lse, const void *d_o,
                                        const scope_strides *d_o_strides, const int32_t *offsets_q, const int32_t *offsets_k,
                                        float scale, void *dq, const scope_strides *dq_strides, void *dk,
                                        const scope_strides *dk_strides, void *dv, const scope_strides *dv_strides, void *workspace,
                                        size_t ws_bytes, int32_t *dev_status, void *stream) {
  int32_t st = check_pack(pack);
  if (st) return st;
  scope::PackArgs a{};
  scope::PackCall c{};
  const int el = pack->dtype == SCOPE_BF16 ? 2 : 4, group = pack->heads / pack->kv_heads;
  const int H = pack->heads, G = pack->kv_heads, nq = pack->rows_q, nk = pack->rows_k;
  const Tensor t[] = {{q, q_strides, H, nq, false},   {o, o_strides, H, nq, false},   {d_o, d_o_strides, H, nq, false},
                      {dq, dq_strides, H, nq, true},  {k, k_strides, G, nk, false},   {v, v_strides, G, nk, false},
                      {dk, dk_strides, G, nk, true},  {dv, dv_strides, G, nk, true}};
  scope::PackRows *const rows[] = {&a.q, &a.o, &a.d_o, &c.dq, &a.k, &a.v, &c.dk, &c.dv};
  for (int i = 0; i < 8; ++i)
    if ((st = check_rows(t[i], pack->d, el, i < 4 ? group : 1, rows[i]))) return st;
  if ((st = check_apart(t, 8, pack->d, el))) return st;
  if ((st = check_int32({offsets_q, offsets_k}, {dev_status, lse}))) return st;
  if (!lse && nq) return SCOPE_ERR_INVALID_ARGUMENT;
  if (!(scale == scale) || isinf(scale)) return SCOPE_ERR_INVALID_ARGUMENT;
  if ((st = check_workspace(pack, workspace, ws_bytes))) return st;
  set_pack(pack, offsets_q, offsets_k, nullptr, scale, workspace, dev_status, &a, &c);
  a.lse = const_cast<float *>(lse);
  return scope::packed_backward(a, c, static_cast<hipStream_t>(stream)) == hipSuccess ? SCOPE_OK : SCOPE_ERR_HIP;
}

}  // extern "C"
