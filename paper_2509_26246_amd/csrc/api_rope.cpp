// Entry points slimattn_rope_*: argument checks and launches.  No device allocation and no synchronisation happens here.
#include "internal.h"

namespace slimattn {
int& last_hip_error();
}  // namespace slimattn

using namespace slimattn;

namespace {

bool aligned(const void* p, unsigned to) { return p && (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int hip_rc(int e) {
  if (e == 0) return SLIMATTN_OK;
  last_hip_error() = e;
  return SLIMATTN_EHIP;
}

// A tensor side: T rows of `width` bytes, `stride` bytes apart.
struct Rows { const void* p; int64_t stride, width; };

bool strides_ok(int64_t stride, int64_t row, int64_t elem) {
  return stride == 0 || (stride >= row && stride * elem % 16 == 0 && stride <= (int64_t(1) << 31));
}

// Whether writing `out` could change what is read of (or written to) `x` elsewhere: any shared byte, unless the two are the same rows and
// `same_ok`.  Rows of equal stride are compared column by column (two column ranges of one buffer do not touch); others by their whole span.
bool clash(const Rows& out, const Rows& x, int64_t T, bool same_ok) {
  if (!out.width || !x.width) return false;
  const int64_t a = (int64_t)reinterpret_cast<uintptr_t>(out.p), b = (int64_t)reinterpret_cast<uintptr_t>(x.p);
  const int64_t a_end = a + (T - 1) * out.stride + out.width, b_end = b + (T - 1) * x.stride + x.width;
  if (a_end <= b || b_end <= a) return false;
  if (same_ok && a == b && (out.stride == x.stride || T == 1)) return false;
  if (out.stride != x.stride) return true;
  int64_t d = (b - a) % out.stride;
  if (d < 0) d += out.stride;
  return d < out.width || d + x.width > out.stride;
}

// A span of bytes, and whether rows (T of them) or another span share any of them.
struct Span { const void* p; int64_t bytes; };

bool touches(const Rows& x, int64_t T, const Span& s) {
  if (!x.width || !s.p || s.bytes <= 0) return false;
  const int64_t at = (int64_t)reinterpret_cast<uintptr_t>(s.p) - (int64_t)reinterpret_cast<uintptr_t>(x.p);
  if (at + s.bytes <= 0 || at >= (T - 1) * x.stride + x.width) return false;
  return at < 0 || at % x.stride < x.width || at % x.stride + s.bytes > x.stride;
}

bool touches(const Span& a, const Span& b) { return a.p && a.bytes > 0 && touches(Rows{a.p, a.bytes, a.bytes}, 1, b); }

int check(const slimattn_rope_params* p) {
  if (!p || (p->dtype != SLIMATTN_F32 && p->dtype != SLIMATTN_BF16)) return SLIMATTN_EINVAL;
  const int d = p->head_dim;
  if (d != 16 && d != 32 && d != 64 && d != 128) return SLIMATTN_EINVAL;
  if (p->total_tokens < 0 || p->total_tokens > (1 << 27)) return SLIMATTN_EINVAL;   // 16 threads a token, 2^32 a launch; strides times tokens in 64 bits
  if (p->n_q_heads < 0 || p->n_kv_heads < 0 || p->n_q_heads + (int64_t)p->n_kv_heads < 1) return SLIMATTN_EINVAL;
  if (p->n_q_heads > 65535 || p->n_kv_heads > 65535) return SLIMATTN_EINVAL;
  if (p->flags & ~(SLIMATTN_ROPE_NORM | SLIMATTN_ROPE_ADJACENT | SLIMATTN_ROPE_DEALT)) return SLIMATTN_EINVAL;
  const bool norm = p->flags & SLIMATTN_ROPE_NORM;
  if (p->rotary_dim < 0 || p->rotary_dim > d || p->rotary_dim % 8 != 0 || (p->rotary_dim == 0 && !norm)) return SLIMATTN_EINVAL;
  if (p->rotary_dim > 0) {
    if (p->n_axes < 1 || p->n_axes > 4) return SLIMATTN_EINVAL;
    int64_t sum = 0;
    for (int i = 0; i < p->n_axes; ++i) {
      if (p->sections[i] < 0) return SLIMATTN_EINVAL;
      sum += p->sections[i];
    }
    if (sum != p->rotary_dim / 2) return SLIMATTN_EINVAL;
  }
  if (norm && !(p->eps >= 0x1p-100f && p->eps <= 0x1p100f)) return SLIMATTN_EINVAL;
  const int64_t e = p->dtype == SLIMATTN_F32 ? 4 : 2, q_row = (int64_t)p->n_q_heads * d, k_row = (int64_t)p->n_kv_heads * d;
  if (!strides_ok(p->q_stride, q_row, e) || !strides_ok(p->dq_stride, q_row, e) || !strides_ok(p->k_stride, k_row, e) ||
      !strides_ok(p->dk_stride, k_row, e))
    return SLIMATTN_EINVAL;
  return SLIMATTN_OK;
}

Rows rows(const slimattn_rope_params* p, const void* x, int heads, int64_t stride) {
  const int64_t e = p->dtype == SLIMATTN_F32 ? 4 : 2, w = heads * (int64_t)p->head_dim * e;
  return {x, stride ? stride * e : w, w};
}

bool small_inputs_ok(const slimattn_rope_params* p, const float* qw, const float* kw, const int32_t* pos, const float* freq) {
  if (p->rotary_dim > 0 && (!aligned(pos, 4) || !aligned(freq, 4))) return false;
  return (!qw || aligned(qw, 4)) && (!kw || aligned(kw, 4));
}

// The arrays beside the tensors that a call reads.
struct SmallInputs { Span s[4]; };
SmallInputs small_inputs(const slimattn_rope_params* p, const float* qw, const float* kw, const int32_t* pos, const float* freq) {
  const bool norm = p->flags & SLIMATTN_ROPE_NORM, turn = p->rotary_dim > 0;
  const int64_t w = norm ? 4 * p->head_dim : 0;
  return {{{qw, w}, {kw, w}, {pos, turn ? 4 * (int64_t)p->n_axes * p->total_tokens : 0}, {freq, turn ? 2 * p->rotary_dim : 0}}};
}

}  // namespace

extern "C" {

int slimattn_rope_fwd(const slimattn_rope_params* p, const void* q, const void* k, const float* q_weight, const float* k_weight,
                      const int32_t* positions, const float* inv_freq, void* q_out, void* k_out, void* stream) {
  const int rc = check(p);
  if (rc != SLIMATTN_OK) return rc;
  const int64_t T = p->total_tokens;
  if (T == 0) return SLIMATTN_OK;
  if (p->n_q_heads && (!aligned(q, 16) || !aligned(q_out, 16))) return SLIMATTN_EINVAL;
  if (p->n_kv_heads && (!aligned(k, 16) || !aligned(k_out, 16))) return SLIMATTN_EINVAL;
  if (!small_inputs_ok(p, q_weight, k_weight, positions, inv_freq)) return SLIMATTN_EINVAL;
  const Rows rq = rows(p, q, p->n_q_heads, p->q_stride), rk = rows(p, k, p->n_kv_heads, p->k_stride);
  const Rows oq = rows(p, q_out, p->n_q_heads, 0), ok = rows(p, k_out, p->n_kv_heads, 0);
  if (clash(oq, rq, T, true) || clash(oq, rk, T, false) || clash(ok, rk, T, true) || clash(ok, rq, T, false) || clash(oq, ok, T, false))
    return SLIMATTN_EINVAL;
  for (const Span& s : small_inputs(p, q_weight, k_weight, positions, inv_freq).s)
    if (touches(oq, T, s) || touches(ok, T, s)) return SLIMATTN_EINVAL;
  return hip_rc(launch_rope_fwd(*p, q, k, q_weight, k_weight, positions, inv_freq, q_out, k_out, stream));
}

size_t slimattn_rope_bwd_workspace_bytes(const slimattn_rope_params* p) {
  return check(p) == SLIMATTN_OK && (p->flags & SLIMATTN_ROPE_NORM) ? rope_partial_bytes(*p) : 0;
}

int slimattn_rope_bwd(const slimattn_rope_params* p, const void* q, const void* k, const float* q_weight, const float* k_weight,
                      const int32_t* positions, const float* inv_freq, const void* dq_out, const void* dk_out, void* dq, void* dk,
                      float* dq_weight, float* dk_weight, void* workspace, void* stream) {
  const int rc = check(p);
  if (rc != SLIMATTN_OK) return rc;
  const int64_t T = p->total_tokens;
  const bool norm = p->flags & SLIMATTN_ROPE_NORM;
  if ((dq_weight && !aligned(dq_weight, 4)) || (dk_weight && !aligned(dk_weight, 4))) return SLIMATTN_EINVAL;
  // what is written beside the tensors (nothing of it without a norm)
  const int64_t w = norm ? 4 * p->head_dim : 0;
  const Span dqw{dq_weight, w}, dkw{dk_weight, w}, ws{workspace, dq_weight || dk_weight ? (int64_t)slimattn_rope_bwd_workspace_bytes(p) : 0};
  if (touches(dqw, dkw) || touches(dqw, ws) || touches(dkw, ws)) return SLIMATTN_EINVAL;
  if (T > 0) {
    if (p->n_q_heads && (!aligned(dq_out, 16) || !aligned(dq, 16) || (norm && !aligned(q, 16)))) return SLIMATTN_EINVAL;
    if (p->n_kv_heads && (!aligned(dk_out, 16) || !aligned(dk, 16) || (norm && !aligned(k, 16)))) return SLIMATTN_EINVAL;
    if (!small_inputs_ok(p, q_weight, k_weight, positions, inv_freq)) return SLIMATTN_EINVAL;
    if (norm && (dq_weight || dk_weight) && !aligned(workspace, 16)) return SLIMATTN_EINVAL;
    const Rows gq = rows(p, dq_out, p->n_q_heads, 0), gk = rows(p, dk_out, p->n_kv_heads, 0);
    const Rows oq = rows(p, dq, p->n_q_heads, p->dq_stride), ok = rows(p, dk, p->n_kv_heads, p->dk_stride);
    const Rows xq = rows(p, q, norm ? p->n_q_heads : 0, p->q_stride), xk = rows(p, k, norm ? p->n_kv_heads : 0, p->k_stride);
    if (clash(oq, gq, T, true) || clash(oq, gk, T, false) || clash(ok, gk, T, true) || clash(ok, gq, T, false) || clash(oq, xq, T, true) ||
        clash(oq, xk, T, false) || clash(ok, xk, T, true) || clash(ok, xq, T, false) || clash(oq, ok, T, false))
      return SLIMATTN_EINVAL;
    for (const Span& s : small_inputs(p, q_weight, k_weight, positions, inv_freq).s)
      if (touches(oq, T, s) || touches(ok, T, s) || touches(dqw, s) || touches(dkw, s) || touches(ws, s)) return SLIMATTN_EINVAL;
    for (const Span& s : {dqw, dkw, ws})
      for (const Rows& x : {oq, ok, gq, gk, xq, xk})
        if (touches(x, T, s)) return SLIMATTN_EINVAL;
  }
  return hip_rc(launch_rope_bwd(*p, q, k, q_weight, k_weight, positions, inv_freq, dq_out, dk_out, dq, dk, dq_weight, dk_weight, workspace,
                                stream));
}

}  // extern "C"
