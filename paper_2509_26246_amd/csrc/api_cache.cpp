// Entry points slimattn_cache_*: argument checks and launches.  No device allocation and no synchronisation happens here.
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

bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return na > 0 && nb > 0 && x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

// Whether a call writes `out` over the arrays that it reads beside the tensors.
bool over_arrays(const slimattn_cache_params* p, const void* out, int64_t n, const int32_t* row_ptr, const int32_t* lens, const int32_t* table) {
  return overlap(out, n, lens, 4 * (int64_t)p->n_seqs) || overlap(out, n, table, 4 * (int64_t)p->n_seqs * p->max_pages) ||
         overlap(out, n, row_ptr, row_ptr ? 4 * ((int64_t)p->n_seqs + 1) : 0);
}

bool geometry_ok(int32_t n_pages, int32_t page_size, int32_t n_kv_heads, int32_t d) {
  if (n_pages < 1 || n_kv_heads < 1 || n_kv_heads > 65535 || (d != 64 && d != 128)) return false;
  return page_size == 16 || page_size == 32 || page_size == 64 || page_size == 128 || page_size == 256;
}

int check(const slimattn_cache_params* p) {
  if (!p || (p->dtype != SLIMATTN_F32 && p->dtype != SLIMATTN_BF16)) return SLIMATTN_EINVAL;
  if (!geometry_ok(p->n_pages, p->page_size, p->n_kv_heads, p->head_dim)) return SLIMATTN_EINVAL;
  if (p->n_seqs < 0 || p->n_seqs > 65536 || p->max_pages < 1) return SLIMATTN_EINVAL;
  if (p->n_rows < 0 || p->n_rows > (1 << 25)) return SLIMATTN_EINVAL;            // a wave a row, 2^32 threads a launch; strides times rows in 64 bits
  if ((int64_t)p->max_pages * p->page_size > (1 << 30)) return SLIMATTN_EINVAL;   // positions and the steps behind them in 32 bits
  return SLIMATTN_OK;
}

int check_arrays(const slimattn_cache_params* p, const int32_t* row_ptr, const int32_t* lens, const int32_t* table) {
  if (row_ptr ? !aligned(row_ptr, 4) : p->n_rows != p->n_seqs) return SLIMATTN_EINVAL;
  return aligned(lens, 4) && aligned(table, 4) ? SLIMATTN_OK : SLIMATTN_EINVAL;
}

int64_t elem(const slimattn_cache_params* p) { return p->dtype == SLIMATTN_F32 ? 4 : 2; }

bool heads_ok(const slimattn_cache_params* p, int32_t n_q_heads) {
  return n_q_heads >= 1 && n_q_heads <= 65535 && n_q_heads % p->n_kv_heads == 0;
}

}  // namespace

extern "C" {

size_t slimattn_cache_bytes(int32_t n_pages, int32_t page_size, int32_t n_kv_heads, int32_t head_dim) {
  if (!geometry_ok(n_pages, page_size, n_kv_heads, head_dim)) return 0;
  return (size_t)n_pages * page_size * n_kv_heads * (head_dim + head_dim / 8);
}

int slimattn_cache_write(const slimattn_cache_params* p, const void* k, const void* v, int64_t k_stride, int64_t v_stride,
                         const int32_t* row_ptr, const int32_t* lens, const int32_t* page_table, void* cache, void* stream) {
  int rc = check(p);
  if (rc != SLIMATTN_OK) return rc;
  const int64_t row = (int64_t)p->n_kv_heads * p->head_dim, e = elem(p);
  auto stride_ok = [&](int64_t s) { return s == 0 || (s >= row && s * e % 16 == 0 && s <= (int64_t(1) << 31)); };
  if (!stride_ok(k_stride) || !stride_ok(v_stride)) return SLIMATTN_EINVAL;
  if (p->n_rows == 0 || p->n_seqs == 0) return SLIMATTN_OK;
  rc = check_arrays(p, row_ptr, lens, page_table);
  if (rc != SLIMATTN_OK) return rc;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(cache, 16)) return SLIMATTN_EINVAL;
  const int64_t ks = k_stride ? k_stride : row, vs = v_stride ? v_stride : row;
  const int64_t bytes = (int64_t)slimattn_cache_bytes(p->n_pages, p->page_size, p->n_kv_heads, p->head_dim);
  if (overlap(cache, bytes, k, ((p->n_rows - 1) * ks + row) * e) || overlap(cache, bytes, v, ((p->n_rows - 1) * vs + row) * e) ||
      over_arrays(p, cache, bytes, row_ptr, lens, page_table))
    return SLIMATTN_EINVAL;
  return hip_rc(launch_cache_write(*p, k, v, ks, vs, row_ptr, lens, page_table, cache, stream));
}

int slimattn_cache_read(const slimattn_cache_params* p, const void* cache, const int32_t* row_ptr, const int32_t* lens,
                        const int32_t* page_table, void* k, void* v, void* stream) {
  int rc = check(p);
  if (rc != SLIMATTN_OK) return rc;
  if (p->n_rows == 0 || p->n_seqs == 0) return SLIMATTN_OK;
  rc = check_arrays(p, row_ptr, lens, page_table);
  if (rc != SLIMATTN_OK) return rc;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(cache, 16)) return SLIMATTN_EINVAL;
  const int64_t n = (int64_t)p->n_rows * p->n_kv_heads * p->head_dim * elem(p);
  const int64_t bytes = (int64_t)slimattn_cache_bytes(p->n_pages, p->page_size, p->n_kv_heads, p->head_dim);
  if (overlap(k, n, v, n) || overlap(k, n, cache, bytes) || overlap(v, n, cache, bytes) || over_arrays(p, k, n, row_ptr, lens, page_table) ||
      over_arrays(p, v, n, row_ptr, lens, page_table))
    return SLIMATTN_EINVAL;
  return hip_rc(launch_cache_read(*p, cache, row_ptr, lens, page_table, k, v, stream));
}

size_t slimattn_cache_attn_workspace_bytes(const slimattn_cache_params* p, int32_t n_q_heads) {
  return check(p) == SLIMATTN_OK && heads_ok(p, n_q_heads) ? cache_attn_bytes(*p, n_q_heads) : 0;
}

int slimattn_cache_attn(const slimattn_cache_params* p, int32_t n_q_heads, float scale, const void* q, const int32_t* row_ptr,
                        const int32_t* lens, const int32_t* page_table, const void* cache, void* o, float* lse, void* workspace,
                        void* stream) {
  int rc = check(p);
  if (rc != SLIMATTN_OK) return rc;
  if (!heads_ok(p, n_q_heads) || !(scale >= -0x1p127f && scale <= 0x1p127f)) return SLIMATTN_EINVAL;   // times log2 e it is finite
  if (p->n_rows == 0 || p->n_seqs == 0) return SLIMATTN_OK;
  rc = check_arrays(p, row_ptr, lens, page_table);
  if (rc != SLIMATTN_OK) return rc;
  if (!aligned(q, 16) || !aligned(o, 16) || !aligned(cache, 16) || !aligned(workspace, 16) || (lse && !aligned(lse, 4))) return SLIMATTN_EINVAL;
  const int64_t n = (int64_t)p->n_rows * n_q_heads * p->head_dim * elem(p);
  const struct { const void* p; int64_t n; } out[] = {{o, n}, {lse, lse ? 4 * (int64_t)p->n_rows * n_q_heads : 0}, {workspace, (int64_t)cache_attn_bytes(*p, n_q_heads)}};
  const int64_t bytes = (int64_t)slimattn_cache_bytes(p->n_pages, p->page_size, p->n_kv_heads, p->head_dim);
  for (int i = 0; i < 3; ++i) {
    if (overlap(out[i].p, out[i].n, q, n) || overlap(out[i].p, out[i].n, cache, bytes) || over_arrays(p, out[i].p, out[i].n, row_ptr, lens, page_table))
      return SLIMATTN_EINVAL;
    for (int j = 0; j < i; ++j)
      if (overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return SLIMATTN_EINVAL;
  }
  return hip_rc(launch_cache_attn(*p, n_q_heads, scale, q, row_ptr, lens, page_table, cache, o, lse, workspace, stream));
}

}  // extern "C"
