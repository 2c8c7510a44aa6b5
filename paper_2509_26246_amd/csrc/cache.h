// A key/value cache in 4 bits: its layout in memory, and what the kernels that write and read it share (gfx950).
//
// A value is scale * code.  32 neighbouring channels of one token's head share a scale; a code is a 4-bit float (sign, 2 exponent bits, 1
// mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6), which the hardware converts two at a time in either direction.  The scale has six significant
// bits and is kept as bf16: scale * code then needs at most eight bits, so every value of the cache is exactly a bf16 number.
//
// A page holds page_size tokens of all KV heads, one piece per head (D = head dim, P = page_size, bytes):
//   [P][D/2] key codes | [P][D/2] value codes | [P][D/32] key scales (bf16) | [P][D/32] value scales (bf16).
// A token's value codes lie in channel order, two a byte, the lower channel in the lower half.  Its key codes lie as the score product's
// A operand (16x16x32: lane group h of four holds k = 8h .. 8h+7) takes them: the 32-bit word h * (D/32) + g holds channels
// 32g + 8h .. +7, so a lane's codes for all D/32 products are one load.
#pragma once
#include <hip/hip_runtime.h>

#include "internal.h"
#include "mfma_utils.h"

namespace slimattn {

constexpr int kCacheGroup = 32;   // channels that share a scale
constexpr int kCacheChunk = 16;   // keys that always lie in one page one behind the other (the smallest page)

struct CacheView {
  int n_pages, page_shift, n_kv_heads, n_seqs, max_pages, n_rows;
  int max_len;                    // max_pages * page_size
  const int32_t* row_ptr;         // NULL: one row per sequence
  const int32_t* lens;
  const int32_t* table;
};

template <int D> __device__ __forceinline__ long long head_bytes(const CacheView& c) { return (long long)(D + D / 8) << c.page_shift; }
template <int D> __device__ __forceinline__ long long page_bytes(const CacheView& c) { return head_bytes<D>(c) * c.n_kv_heads; }
// Offsets inside a head's piece; t: token in the page.
template <int D> __device__ __forceinline__ int key_codes(int t) { return t * (D / 2); }
template <int D> __device__ __forceinline__ int value_codes(const CacheView& c, int t) { return ((D / 2) << c.page_shift) + t * (D / 2); }
template <int D> __device__ __forceinline__ int scales(const CacheView& c, int value, int t) {
  return (D << c.page_shift) + value * ((D / 16) << c.page_shift) + t * (D / 16);
}

__device__ __forceinline__ int seq_len(const CacheView& c, int b) { return min(max(c.lens[b], 0), c.max_len); }

// A page of sequence b's table, -1 where the table names none.  The table is data: what it holds is checked before it becomes an address.
__device__ __forceinline__ int page_at(const CacheView& c, int b, int pos) {
  const int p = c.table[(size_t)b * c.max_pages + (pos >> c.page_shift)];
  return (unsigned)p < (unsigned)c.n_pages ? p : -1;
}

// The sequence a row belongs to, for a whole wave (row: uniform): 64 starts are looked at together, so up to 4096 sequences take two
// rounds of loads.  The last one whose first row is not behind `row`; with row_ptr in no order some sequence.
__device__ __forceinline__ int wave_find_seq(const CacheView& c, int row) {
  if (!c.row_ptr) return row;
  int lo = 0, n = c.n_seqs;
  while (n > 1) {
    const int step = (n + 63) >> 6, at = (int)(threadIdx.x & 63) * step;
    const bool before = at < n && c.row_ptr[lo + at] <= row;
    const int k = max(__popcll(__ballot(before)), 1) - 1;
    lo += k * step;
    n = min(step, n - k * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Position of a row in its sequence (uniform): negative where the sequence is shorter than its rows, or where the row is nobody's.  A sequence's rows end
// with the tensors', wherever row_ptr does (as in seq_rows of the attention).
__device__ __forceinline__ int row_position(const CacheView& c, int row, int b) {
  if (!c.row_ptr) return seq_len(c, b) - 1;
  const int r0 = c.row_ptr[b], r1 = min(c.row_ptr[b + 1], c.n_rows);
  return row < r0 || row >= r1 ? INT32_MIN : seq_len(c, b) - (r1 - row);
}

// Eight codes (one word, ascending channels or keys from the low bits) as bf16.
__device__ __forceinline__ bf16x8 codes_to_bf16(unsigned w) {
  typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
  union { bf2 p[4]; bf16x8 v; } u;
  u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 0);
  u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 1);
  u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 2);
  u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 3);
  return u.v;
}

// The halves of a word of two bf16 as floats.
__device__ __forceinline__ float lo_bf16(unsigned w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float hi_bf16(unsigned w) { return __builtin_bit_cast(float, w & 0xffff0000u); }

}  // namespace slimattn
